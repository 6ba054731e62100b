"""A paged cache of keys and values: appending with norm and rotation, attention over it, keeping accepted drafts; against oracle/cache.py and oracle/rotary.py in 64 bits.

Tolerances.  u = 2^-24 and h = half a step of the type (bf16 2^-8, fp32 2^-24), relative to the value rounded.
Attention: products of bf16 values are exact in fp32, so a score is off by at most (D + 8) u times the sum of its products' sizes (their sum, the scale, the exponent's argument), in fp32 by (2 D + 12) u, with
a cap by 2^-21 of it more, with a bias by 4 u of it; call the largest of a row delta.  Weights and their sum are off by 2 delta and, for n keys, (n + 64) u (sums, rescaled up to once a step, and the exponential);
bf16 weights are rounded as operands (w = 2^-8; fp32: 0), results once more.  So |error| <= sum p |v| (w + 2 delta + (n + 64) u) (1 + 2^-7) + h |result|, and the log-sum-exp is off by
delta + (n + 64) u + 8 u (1 + |lse|).
Appending: a norm's sum of D squares and its root are off by (D + 8) u, a rotated value by 4 u of both of its terms; rounded once: |error| <= h |y| + (D + 16) u (|a| + |b|) with the terms a, b."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2508_12969_amd as ca
from oracle import cache as OC
from oracle import rotary as OR
from paper_2508_12969_amd import cache as C
from paper_2508_12969_amd import rotary as R

DEV = "cuda:0"
U = 2.0 ** -24
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}

# ---------------------------------------------------------------- refusals (no tensor is touched)

P = [0x10000000000 * (i + 1) for i in range(16)]   # addresses that are never read


def _status(call):
    lib = ca.load_library()
    return call(lib), lib.compact_attn_last_error().decode()


def _raw_cache(**how):
    base = dict(k=P[0], v=P[1], num_pages=8, page_tokens=64, kv_heads=2, head_dim=128, dtype=1, sequences=3, table_width=4, table=P[2], lengths=P[3], starts=P[4], origins=None,
                tokens=5, frame_height=1, frame_width=1)
    base.update(how)
    return C.ca_cache(**base)


BAD_CACHES = [(dict(k=None), -1, "null"), (dict(table=None), -1, "null"), (dict(lengths=None), -1, "null"), (dict(starts=None), -1, "null"), (dict(dtype=2), -1, "dtype"),
              (dict(num_pages=0), -1, "positive"), (dict(num_pages=2 ** 31), -1, "2^31"), (dict(kv_heads=0), -1, "positive"), (dict(sequences=0), -1, "positive"),
              (dict(table_width=0), -1, "positive"), (dict(tokens=-1), -1, "positive"), (dict(page_tokens=24), -1, "multiple of 16"), (dict(page_tokens=0), -1, "multiple of 16"),
              (dict(page_tokens=65536 + 16), -1, "multiple of 16"), (dict(page_tokens=65536, table_width=16385), -1, "2^30"), (dict(frame_height=0), -1, "frame"),
              (dict(frame_height=65536, frame_width=65536), -1, "frame"), (dict(head_dim=12), -1, "16 bytes"), (dict(head_dim=520), -2, "520"), (dict(head_dim=260, dtype=0), -2, "260"),
              (dict(kv_heads=65536), -2, "heads"), (dict(sequences=2 ** 20 + 1), -2, "sequences"), (dict(num_pages=2 ** 31 - 1, kv_heads=60000), -1, "2^46"),
              (dict(k=P[0] + 8), -1, "16-byte"), (dict(table=P[2] + 2), -1, "4-byte"), (dict(origins=P[5] + 1), -1, "4-byte")]


def _append_call(cache=None, **how):
    base = dict(q=P[6], k=P[7], v=P[8], q_out=P[9], heads=4, normed=1, eps=1e-6)
    base.update(how)
    a = C.ca_append(**base)
    return _status(lambda lib: lib.compact_attn_cache_append(a, cache or _raw_cache(), None))


def _attend_call(cache=None, q=P[6], strides=None, heads=4, out=P[9], lse=P[10], workspace=P[11], size=1 << 40, **how):
    reach = C.ca_reach(**how)
    return _status(lambda lib: lib.compact_attn_cache_attend(q, strides, heads, cache or _raw_cache(), reach, out, lse, workspace, size, None))


def _keep_call(cache=None, kept=P[6], width=8, counts=P[7]):
    return _status(lambda lib: lib.compact_attn_cache_keep(cache or _raw_cache(), kept, width, counts, None))


@pytest.mark.parametrize("how,status,text", BAD_CACHES)
def test_malformed_caches_are_refused_by_every_call(how, status, text):
    bad = _raw_cache(**how)
    for call in (_append_call, _attend_call, _keep_call, lambda c: _status(lambda lib: lib.compact_attn_cache_workspace(c, 4, ctypes.c_int64()))):
        st, message = call(bad)
        assert st == status and text in message, (how, st, message)


def test_append_refusals():
    rotary = ca.compact_attn_build_rotary((32, 48, 56), (9, 9, 9))
    table = ca.compact_attn_build_rotary((64, 0, 0), (9, 9, 9))
    late = ctypes.pointer(R.ca_where((ctypes.c_int32 * 3)(-1, 0, 0), None))
    odd = ctypes.pointer(R.ca_where((ctypes.c_int32 * 3)(0, 0, 0), P[12] + 2))
    step = lambda token, head: ctypes.pointer(R.ca_strides(0, head, token))
    for bad, text in ((dict(k=None), "null"), (dict(v=None), "null"), (dict(q=None), "both"), (dict(q_out=None), "both"), (dict(heads=0), "heads"), (dict(heads=65533), "heads"),
                      (dict(k=P[7] + 8), "16-byte"), (dict(k_weight=P[12] + 4), "16-byte"), (dict(normed=2), "normed"), (dict(normed=0, k_weight=P[12]), "norm"),
                      (dict(q=None, q_out=None, q_weight=P[12]), "without q"), (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"), (dict(eps=float("inf")), "eps"),
                      (dict(rotary=rotary.handle), "rotated"), (dict(rotary=table.handle, where=late), "negative"), (dict(rotary=table.handle, where=odd), "4-byte"),
                      (dict(k_strides=step(256, 100)), "16 bytes"), (dict(v_strides=step(-256, 128)), "negative"), (dict(q_strides=step(2 ** 41, 128)), "2^40"),
                      (dict(q_out=P[6]), "overlap the inputs"), (dict(q_out=P[0]), "each other"), (dict(q_out=P[3]), "arrays"), (dict(k=P[0] + 4096), "overlap the inputs")):
        st, message = _append_call(**bad)
        assert st == -1 and text in message, (bad, st, message)
    assert _append_call(_raw_cache(tokens=1 << 26))[0] == -2
    assert _append_call(_raw_cache(v=P[0]))[0] == -1 and _append_call(_raw_cache(kv_heads=33000))[0] == -2
    assert _append_call(_raw_cache(tokens=0), k=None, v=None, q=None, q_out=None)[0] == 0   # nothing to do


def test_attend_refusals():
    step = lambda token, head: R.ca_strides(0, head, token)
    for bad, text in ((dict(q=None), "null"), (dict(out=None), "null"), (dict(lse=None), "null"), (dict(out=P[9] + 8), "16-byte"), (dict(lse=P[10] + 2), "4-byte"), (dict(heads=3), "multiple"),
                      (dict(heads=0), "multiple"), (dict(cap=-1.0), "cap"), (dict(cap=5000.0), "cap"), (dict(cap=float("nan")), "cap"), (dict(scale=float("nan")), "scale"),
                      (dict(scale=float("inf")), "scale"), (dict(scale=1e-38), "scale"), (dict(scale=2.0 ** 101), "scale"), (dict(causal=2), "causal"), (dict(window=-1), "window"), (dict(slopes=P[12] + 2), "4-byte"), (dict(tree=P[12] + 4), "8-byte"),
                      (dict(strides=step(512, 4)), "16 bytes"), (dict(out=P[6]), "overlap"), (dict(out=P[1]), "overlap"), (dict(lse=P[9]), "each other"), (dict(lse=P[4]), "arrays"),
                      (dict(tree=P[9]), "overlap"), (dict(slopes=P[10]), "overlap")):
        st, message = _attend_call(**bad)
        assert st == -1 and text in message, (bad, st, message)
    lib = ca.load_library()
    assert lib.compact_attn_cache_attend(P[6], None, 4, _raw_cache(), None, P[9], P[10], P[11], 1 << 40, None) == -1
    assert _attend_call(_raw_cache(head_dim=96))[0] == -2 and _attend_call(_raw_cache(head_dim=32, dtype=0))[0] == -2
    assert _attend_call(_raw_cache(tokens=2 ** 31 - 1, kv_heads=1), heads=64)[0] == -2
    assert _attend_call(_raw_cache(tokens=0), q=None, out=None, lse=None)[0] == 0
    size = ctypes.c_int64()
    assert lib.compact_attn_cache_workspace(_raw_cache(), 4, None) == -1 and lib.compact_attn_cache_workspace(_raw_cache(), 3, size) == -1
    assert lib.compact_attn_cache_workspace(_raw_cache(), 4, size) == 0 and size.value >= 0


def test_keep_refusals():
    for bad, text in ((dict(width=65), "width"), (dict(width=-1), "width"), (dict(counts=None), "null"), (dict(kept=None), "null"), (dict(kept=P[6] + 2), "4-byte"),
                      (dict(counts=P[0] + 64), "overlap")):
        st, message = _keep_call(**bad)
        assert st == -1 and text in message, (bad, st, message)
    assert _keep_call(_raw_cache(v=P[0]))[0] == -1
    assert _keep_call(width=0, kept=None)[0] == 0


def test_host_tensors_are_refused():
    k = torch.zeros(2, 1, 16, 64, dtype=torch.bfloat16)
    ints = lambda *shape: torch.zeros(shape, dtype=torch.int32)
    with pytest.raises(ValueError):
        ca.Cache(k, k.clone(), ints(1, 2), ints(1), ints(2))


# ---------------------------------------------------------------- a cache on both sides

class Paged:
    """Sequences of (tokens, new tokens), their keys and values in 64 bits, and the pages that hold them; the rest of the pages is NaN."""

    def __init__(self, sequences, kv_heads, D, page, dtype="bf16", origins=None, frame=(1, 1), seed=0, spare=2, behind=0, extra_width=1):
        rng = np.random.default_rng(seed)
        self.sequences, self.kv, self.D, self.page, self.dtype, self.frame, self.rng = sequences, kv_heads, D, page, dtype, frame, rng
        self.origins = origins
        self.rows = sum(m for _, m in sequences)
        self.tokens = self.rows + behind
        used = [-(-n // page) for n, _ in sequences]
        self.num_pages = sum(used) + spare
        order = rng.permutation(self.num_pages)
        self.table = np.full((len(sequences), max(used) + extra_width), -1, np.int32)
        for s, count in enumerate(used):
            self.table[s, :count], order = order[:count], order[count:]
        nan = torch.full((self.num_pages, kv_heads, page, D), math.nan, dtype=DTYPES[dtype])
        self.pages = [nan.clone(), nan.clone()]
        for t in self.pages:
            for s, (n, _) in enumerate(sequences):
                for j in range(0, n, page):
                    count = min(page, n - j)
                    t[int(self.table[s, j // page]), :, :count] = self.randn(kv_heads, count, D)
        self.upload()

    def randn(self, *shape):
        return torch.from_numpy(self.rng.normal(size=shape).astype(np.float32)).to(DTYPES[self.dtype])

    def upload(self):
        dev = lambda x: torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(DEV)
        self.k, self.v = (t.to(DEV) for t in self.pages)
        self.dev_table, self.lengths = dev(self.table), dev([n for n, _ in self.sequences])
        self.starts = dev(np.cumsum([0] + [m for _, m in self.sequences]))
        self.dev_origins = None if self.origins is None else dev(self.origins)
        self.cache = ca.Cache(self.k, self.v, self.dev_table, self.lengths, self.starts, origins=self.dev_origins, frame=self.frame)

    def host(self, s, which):
        """float64 [length, kv_heads, D], bool [length]: a sequence's keys (0) or values (1), and which are there."""
        n = self.sequences[s][0]
        out, there = np.zeros((n, self.kv, self.D)), np.zeros(n, bool)
        for j in range(0, n, self.page):
            place = OC.place_of(self.table, s, j, self.page, self.num_pages)
            if place is not None:
                count = min(self.page, n - j)
                out[j:j + count] = self.pages[which][place[0], :, :count].double().numpy().transpose(1, 0, 2)
                there[j:j + count] = True
        return out, there


def _origin(p, s):
    return 0 if p.origins is None else min(p.origins[s], p.sequences[s][0])


def check_attend(p, q, got, scale=0.0, cap=0.0, slopes=None, causal=True, window=0, words=None, finite=True):
    """Every row of every sequence against the oracle, within the bounds that the head of this file derives."""
    out, lse = got[0].double().cpu().numpy(), got[1].double().cpu().numpy()
    qh, heads = q.double().cpu().numpy(), q.shape[1]
    group, scale = heads // p.kv, scale or 1 / math.sqrt(p.D)
    row, worst = 0, 0.0
    for s, (n, m) in enumerate(p.sequences):
        (k, there), (v, _) = p.host(s, 0), p.host(s, 1)
        seen, row_frame, token_frame = OC.seen_by(n, m, _origin(p, s), p.frame[0] * p.frame[1], causal, window, None if words is None else words[row:row + m])
        seen &= there[None, :]
        for h in range(heads):
            slope = None if slopes is None else float(slopes[h])
            want, want_lse, weights, size = OC.attend(qh[row:row + m, h], k[:, h // group], v[:, h // group], seen, scale, cap, slope, row_frame, token_frame)
            some = seen.any(1)
            delta = np.max(np.where(seen, size, 0), axis=1, initial=0) * (p.D + 8 if p.dtype == "bf16" else 2 * p.D + 12) * U + cap * 2.0 ** -21
            if slope is not None:
                delta = delta + 4 * U * slope * np.max(np.abs(row_frame[:, None] - token_frame[None, :]) * seen, axis=1, initial=0)
            lost = (n + 64) * U
            bound = (weights @ np.abs(np.where(seen.any(0)[:, None], v[:, h // group], 0))) * ((2.0 ** -8 if p.dtype == "bf16" else 0) + 2 * delta + lost)[:, None] * (1 + 2.0 ** -7) + HALF[p.dtype] * np.abs(want)
            o, l = out[row:row + m, h], lse[row:row + m, h]
            assert np.all(o[~some] == 0) and np.all(l[~some] == -math.inf), (s, h)
            if some.any():
                err = np.abs(o - want)[some] / (bound[some] + 1e-30)
                lse_err = np.abs(l[some] - want_lse[some]) / (delta[some] + lost + 8 * U * (1 + np.abs(want_lse[some])))
                assert np.all(np.isfinite(o)) and err.max() <= 1, (s, h, err.max())
                assert lse_err.max() <= 1, (s, h, lse_err.max())
                worst = max(worst, err.max())
        row += m
    return worst


def chain_words(rng, m):
    """A random tree: parents come before their children."""
    words = []
    for i in range(m):
        parent = rng.integers(0, i) if i and rng.random() < 0.6 else i - 1
        words.append((words[parent] if i else 0) | (1 << i if i < 64 else 0))
    return words


def to_words(words):
    return torch.from_numpy(np.array(words, dtype=np.uint64).view(np.int64)).to(DEV)


ATTEND = {
    # sequences (tokens, new), key heads, group, D, page, and what is seen
    "one-token": dict(sequences=[(1, 1)], kv=1, group=1, D=64, page=16),
    "one-token-128": dict(sequences=[(1, 1), (2, 1), (33, 1)], kv=2, group=1, D=128, page=16),
    "ragged": dict(sequences=[(1, 1), (31, 1), (32, 1), (33, 1), (64, 1), (65, 1), (300, 1), (1000, 1)], kv=3, group=1, D=64, page=16),
    "ragged-grouped": dict(sequences=[(97, 1), (5, 1), (511, 1), (512, 1), (513, 1)], kv=2, group=4, D=128, page=48),
    "some-without": dict(sequences=[(40, 0), (70, 3), (0, 0), (90, 1), (12, 0)], kv=2, group=2, D=64, page=32),
    "prompt-only": dict(sequences=[(77, 77), (130, 130)], kv=2, group=1, D=128, page=32),
    "prompts-grouped": dict(sequences=[(77, 77), (200, 129), (3, 3)], kv=1, group=5, D=64, page=16),
    "wide-group": dict(sequences=[(150, 2), (20, 1)], kv=1, group=40, D=128, page=64),
    "odd-group": dict(sequences=[(150, 9), (20, 7)], kv=3, group=7, D=64, page=256),
    "all-seen": dict(sequences=[(150, 40), (64, 64)], kv=2, group=1, D=64, page=16, causal=False),
    "frames": dict(sequences=[(150, 35), (64, 64), (35, 1)], kv=2, group=2, D=64, page=16, frame=(5, 7)),
    "frames-prompt": dict(sequences=[(160, 35), (64, 64), (12, 12), (9, 1)], kv=2, group=1, D=128, page=48, frame=(5, 7), origins=[17, 20, 40, 9]),
    "prompt-all-seen": dict(sequences=[(160, 150)], kv=1, group=1, D=64, page=48, frame=(5, 7), origins=[17], causal=False),
    "window": dict(sequences=[(700, 1), (701, 50), (20, 20)], kv=2, group=2, D=64, page=16, window=100),
    "window-one": dict(sequences=[(100, 100), (33, 1)], kv=1, group=1, D=128, page=16, window=1),
    "window-frames": dict(sequences=[(700, 70), (64, 64)], kv=2, group=1, D=128, page=64, frame=(5, 7), origins=[40, 33], window=3),
    "window-all-seen": dict(sequences=[(700, 70)], kv=2, group=1, D=64, page=64, frame=(5, 7), origins=[40], window=3, causal=False),
    "cap": dict(sequences=[(333, 1), (128, 128)], kv=2, group=2, D=128, page=32, cap=15.0),
    "bias": dict(sequences=[(333, 1), (128, 128)], kv=2, group=2, D=64, page=32, slopes=True),
    "bias-frames-cap": dict(sequences=[(333, 30), (128, 128)], kv=2, group=2, D=128, page=32, frame=(2, 11), origins=[50, 3], slopes=True, cap=20.0),
    "scale": dict(sequences=[(100, 3)], kv=2, group=2, D=64, page=32, scale=0.31),
    "scale-least": dict(sequences=[(100, 3), (90, 90)], kv=2, group=2, D=64, page=32, scale=2.0 ** -100),
    "scale-least-cap": dict(sequences=[(100, 3), (90, 90)], kv=1, group=2, D=128, page=32, scale=2.0 ** -100, cap=4096.0),
    "cap-least": dict(sequences=[(100, 3), (90, 90)], kv=1, group=2, D=64, page=32, scale=2.0 ** 100, cap=2.0 ** -16),
    "tree": dict(sequences=[(100, 64), (64, 64), (1, 1), (500, 37), (33, 2)], kv=2, group=2, D=128, page=16, tree=True),
    "tree-window-bias": dict(sequences=[(100, 40), (47, 33), (200, 9)], kv=1, group=3, D=64, page=48, tree=True, window=20, slopes=True),
    "tree-frames": dict(sequences=[(100, 40), (47, 33), (30, 20)], kv=1, group=3, D=64, page=48, tree=True, frame=(2, 3), origins=[31, 47, 29], window=2, slopes=True),
    "tree-past-64": dict(sequences=[(100, 70), (80, 80)], kv=1, group=2, D=64, page=16, tree=True),
    "long": dict(sequences=[(20011, 1), (9, 1)], kv=1, group=2, D=128, page=128),
    "long-64": dict(sequences=[(30000, 2)], kv=1, group=1, D=64, page=256),
    "rows-cut": dict(sequences=[(6000, 60), (1200, 200), (40, 40)], kv=1, group=2, D=128, page=48),
    "rows-cut-64": dict(sequences=[(9000, 35), (2, 2)], kv=2, group=2, D=64, page=16, window=3000, cap=20.0),
    "rows-cut-frames": dict(sequences=[(4000, 140), (70, 70)], kv=2, group=1, D=128, page=256, frame=(7, 10), origins=[333, 5], window=30, slopes=True),
    "rows-cut-tree": dict(sequences=[(5000, 64), (300, 33)], kv=1, group=4, D=64, page=64, tree=True),
    "few-cut-tree": dict(sequences=[(5000, 9), (300, 5), (0, 0), (777, 8)], kv=3, group=3, D=128, page=64, tree=True, slopes=True),
    "many-sequences": dict(sequences=[((i * 53) % 40 + 20, 20 if i % 4 else 0) for i in range(530)], kv=1, group=3, D=64, page=32),
    "side-by-side": dict(sequences=[(3000, 600)], kv=2, group=1, D=128, page=64),
    "side-by-side-64": dict(sequences=[(2600, 700)], kv=1, group=2, D=64, page=48, frame=(7, 10), origins=[77], cap=20.0, slopes=True),
    "side-by-side-window": dict(sequences=[(5000, 600)], kv=2, group=1, D=64, page=64, window=300),
    "side-by-side-ragged": dict(sequences=[(900, 400), (3, 1), (700, 700), (0, 0), (650, 650)], kv=40, group=3, D=64, page=128),
    "side-by-side-cap": dict(sequences=[(5000, 600)], kv=2, group=1, D=128, page=64, cap=20.0),
    "rows-cut-cap": dict(sequences=[(9000, 35), (300, 33), (4100, 40)], kv=2, group=2, D=64, page=64, cap=20.0),
    "tiles-cap": dict(sequences=[((i * 53) % 40 + 20, 20) for i in range(530)] + [(4500, 20)], kv=1, group=3, D=64, page=64, cap=20.0),
    "more-new-than-tokens": dict(sequences=[(20, 30), (40, 10)], kv=1, group=2, D=64, page=16),
    "many": dict(sequences=[((i * 37) % 90 + 1, (i * 37) % 90 % 2 + (i % 3 > 0)) if (i * 37) % 90 > 3 else (3, 0) for i in range(700)], kv=1, group=1, D=64, page=16),
}


def attend_case(name, seed=3, dtype="bf16"):
    c = dict(dict(causal=True, window=0, cap=0.0, scale=0.0, slopes=None, tree=False, frame=(1, 1), origins=None), **ATTEND[name])
    p = Paged(c["sequences"], c["kv"], c["D"], c["page"], dtype=dtype, origins=c["origins"], frame=c["frame"], seed=seed)
    heads = c["kv"] * c["group"]
    q = p.randn(p.rows, heads, c["D"]).mul(2).to(DEV)
    slopes = np.linspace(0.02, 0.3, heads).astype(np.float32) if c["slopes"] else None
    words = [w for _, m in c["sequences"] for w in chain_words(p.rng, m)] if c["tree"] else None
    how = dict(scale=c["scale"], cap=c["cap"], causal=c["causal"], window=c["window"])
    return p, q, slopes, words, how


def run_attend(p, q, slopes, words, how, **more):
    return ca.compact_attn_cache_attend(q, p.cache, slopes=None if slopes is None else torch.from_numpy(slopes).to(DEV), tree=None if words is None else to_words(words), **how, **more)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", list(ATTEND))
def test_attend(name, dtype):
    print("attend", name, dtype, flush=True)
    p, q, slopes, words, how = attend_case(name, dtype=dtype)
    got = run_attend(p, q, slopes, words, how)
    again = run_attend(p, q, slopes, words, how)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])
    print("worst", check_attend(p, q, got, slopes=slopes, words=words, **how))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kv,group", [(2, 2), (1, 40)])   # few rows a sequence, many
@pytest.mark.parametrize("tokens", [1, 5])
def test_small_capped_scores_are_precise(tokens, kv, group, dtype):
    """Inputs are multiples of 1/8 whose products' sums are exact.  Then a score s is off by the roundings of scale / cap (2 u), of z (2 u), of the polynomial (it and its last terms, 8 u) and of the way
    back (4 u): 16 u |s|.  Of one token the log-sum-exp is the score; of n the weights' sum (n + 8) u and the logarithm 4 u (1 + |lse|) join it."""
    p = Paged([(tokens, 1)] * 50, kv, 64, 16, dtype=dtype, seed=8)
    p.pages[0] = (p.pages[0].float() * 4).round().div(4).to(DTYPES[dtype])
    p.upload()
    q = p.randn(p.rows, kv * group, 64).float().round().div(8).to(DTYPES[dtype]).to(DEV)
    lse = ca.compact_attn_cache_attend(q, p.cache, scale=0.125, cap=30.0)[1].double().cpu().numpy()
    for s in range(50):
        k, _ = p.host(s, 0)
        for h in range(kv * group):
            x = 30.0 * np.tanh(k[:, h // group] @ q[s, h].double().cpu().numpy() * 0.125 / 30.0)
            assert np.abs(x).max() < 15
            want = np.log(np.exp(x).sum())
            bound = 16 * U * np.abs(x).max() + (0 if tokens == 1 else (tokens + 8) * U + 4 * U * (1 + abs(want)))
            assert abs(lse[s, h] - want) <= bound, (s, h, lse[s, h], want)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,frame,tree", [(64, (1, 1), False), (128, (3, 5), False), (128, (1, 1), True)])
def test_pages_that_are_not_there(D, frame, tree, dtype):
    """Entries below 0 and past the pages: their tokens are seen by none, and nothing is read there; a sequence without any page has empty rows."""
    p = Paged([(200, 30), (300, 1), (50, 2), (90, 40)], 2, D, 16, dtype=dtype, frame=frame, seed=8)
    p.table[0, 1], p.table[0, 2], p.table[0, 7] = -1, p.num_pages, 2 ** 31 - 1
    p.table[1, 0:9], p.table[1, 18] = -2 ** 31, -5
    p.table[2, :] = -1
    p.table[3, 5] = p.num_pages + 7   # holds the last tokens, new ones among them
    p.upload()
    q = p.randn(p.rows, 4, D).to(DEV)
    words = [w for _, m in p.sequences for w in chain_words(p.rng, m)] if tree else None
    check_attend(p, q, run_attend(p, q, None, words, {}), words=words)


@pytest.mark.gpu
def test_sequences_may_share_pages():
    p = Paged([(200, 1), (210, 1), (96, 1)], 2, 64, 32, seed=9)
    p.table[1, :6] = p.table[0, :6]
    p.table[2, :3] = p.table[0, 0]   # the same page three times
    p.upload()
    q = p.randn(p.rows, 2, 64).to(DEV)
    check_attend(p, q, run_attend(p, q, None, None, {}))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_infinities_and_nan_stay_in_their_sequence(bad, dtype):
    """A key or value that is not finite reaches the rows of its sequence that see it, and no other sequence's."""
    p = Paged([(100, 1), (120, 1), (64, 1)], 2, 128, 32, dtype=dtype, seed=10)
    for t in p.pages:
        t[int(p.table[1, 2]), 1, 3, 5] = bad
    p.upload()
    q = p.randn(p.rows, 4, 128).to(DEV)
    out, lse = run_attend(p, q, None, None, {})
    hit = torch.zeros(3, 4, dtype=torch.bool, device=DEV)
    hit[1, 2:] = True
    assert torch.isfinite(out[~hit]).all() and torch.isfinite(lse[~hit]).all()
    assert not torch.isfinite(out[hit]).all()
    p.pages = [torch.where(torch.isfinite(t), t, torch.full_like(t, math.nan)) for t in p.pages]
    keep = [s for s in range(3) if s != 1]
    rows = torch.tensor(keep, device=DEV)
    some = Paged([p.sequences[s] for s in keep], 2, 128, 32, dtype=dtype, seed=10)
    some.table, some.pages, some.num_pages = p.table[keep], p.pages, p.num_pages
    some.upload()
    check_attend(some, q[rows], (out[rows], lse[rows]))


@pytest.mark.gpu
def test_arrays_out_of_range_are_cut_off():
    """Lengths, starts and origins that no program should write: cut to the tensors; rows of no sequence are left as they were."""
    p = Paged([(64, 4), (64, 4), (64, 4)], 1, 64, 16, seed=11, extra_width=0)
    q = p.randn(20, 2, 64).to(DEV)
    for lengths, starts, origins in (([64, 2 ** 31 - 1, -5], [0, 4, 8, 12], None), ([64, 64, 64], [-3, 4, 2 ** 31 - 1, 7], None), ([64, 64, 64], [5, 3, 9, 2], [-1, 2 ** 31 - 1, 70]),
                                     ([0, 0, 0], [0, 0, 0, 0], [-2 ** 31] * 3)):
        p.lengths.copy_(torch.tensor(lengths, dtype=torch.int32))
        p.starts.copy_(torch.tensor(starts, dtype=torch.int32))
        o = None if origins is None else torch.tensor(origins, dtype=torch.int32, device=DEV)
        cache = ca.Cache(p.k, p.v, p.dev_table, p.lengths, p.starts, origins=o)
        out, lse = torch.full_like(q, 7.0), torch.full((20, 2), 7.0, device=DEV)
        ca.compact_attn_cache_attend(q, cache, out=(out, lse))
        covered = set()
        for a, b in zip(starts, starts[1:]):
            covered |= set(range(max(0, a), max(0, min(b, 20))))
        rest = [r for r in range(20) if r not in covered]
        assert (out[rest] == 7).all() and (lse[rest] == 7).all()
        rows = sorted(covered)
        assert not (out[rows] == 7).any()
    p.lengths.copy_(torch.tensor([64, 64, 64], dtype=torch.int32))
    p.starts.copy_(torch.tensor([0, 4, 8, 12], dtype=torch.int32))
    check_attend(p, q[:12], [t[:12] for t in ca.compact_attn_cache_attend(q, p.cache)])


@pytest.mark.gpu
def test_rows_behind_the_last_sequence_and_strides():
    """A padded batch: q cut out of a fused projection, results in tensors of the caller's; rows behind the last sequence keep what they held."""
    p = Paged([(70, 3), (33, 1)], 2, 128, 16, seed=12, behind=9)
    fused = p.randn(p.tokens, 4 + 2 + 2, 128).to(DEV)
    for q in (fused[:, 2:6], fused[:, :8:2], p.randn(4, p.tokens, 128).to(DEV).transpose(0, 1)):
        out, lse = torch.full((p.tokens, 4, 128), 5.0, dtype=torch.bfloat16, device=DEV), torch.full((p.tokens, 4), 5.0, device=DEV)
        got = ca.compact_attn_cache_attend(q, p.cache, out=(out, lse))
        assert got[0] is out and got[1] is lse
        assert (out[p.rows:] == 5).all() and (lse[p.rows:] == 5).all()
        check_attend(p, q[:p.rows], (out[:p.rows], lse[:p.rows]))


@pytest.mark.gpu
def test_no_tokens_at_all():
    p = Paged([(30, 0), (5, 0)], 1, 64, 16, seed=13)
    out, lse = ca.compact_attn_cache_attend(torch.empty(0, 2, 64, dtype=torch.bfloat16, device=DEV), p.cache)
    assert out.shape == (0, 2, 64) and lse.shape == (0, 2)
    empty = torch.empty(0, 1, 64, dtype=torch.bfloat16, device=DEV)
    assert ca.compact_attn_cache_append(empty, empty, p.cache) is None
    behind = torch.full((6, 2, 64), 3.0, dtype=torch.bfloat16, device=DEV)   # rows, of no sequence
    before = p.k.clone(), p.v.clone()
    q = ca.compact_attn_cache_append(behind[:, :1], behind[:, 1:], p.cache, q=behind, out=torch.full_like(behind, 9.0))
    assert (q == 9).all() and all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(before, (p.k, p.v)))


@pytest.mark.gpu
def test_bindings_refuse_what_does_not_fit():
    p = Paged([(30, 2)], 2, 64, 16, seed=14)
    q = p.randn(2, 4, 64).to(DEV)
    for bad in (q.float(), q[:, :, :32], q[:, :3], q.permute(2, 1, 0).contiguous().permute(2, 1, 0), q.cpu(), q[0]):
        with pytest.raises((ValueError, ca.CompactAttnError)):
            ca.compact_attn_cache_attend(bad, p.cache)
    with pytest.raises(ValueError):
        ca.compact_attn_cache_attend(q, p.cache, slopes=torch.ones(3, device=DEV))
    with pytest.raises(ValueError):
        ca.compact_attn_cache_attend(q, p.cache, tree=torch.ones(2, dtype=torch.int32, device=DEV))
    with pytest.raises(ValueError):
        ca.compact_attn_cache_attend(q, p.cache, out=(q.new_empty(2, 3, 64), torch.empty(2, 4, device=DEV)))
    k = p.randn(2, 2, 64).to(DEV)
    for kwargs in (dict(q=q[:1]), dict(out=q), dict(k_weight=k[0, 0].float()), dict(norm=False, k_weight=k[0, 0].contiguous()), dict(positions=torch.zeros(2, 3, device=DEV))):
        with pytest.raises((ValueError, ca.CompactAttnError)):
            ca.compact_attn_cache_append(k, k, p.cache, **kwargs)
    with pytest.raises(ValueError):
        ca.Cache(p.k, p.v, p.dev_table, p.lengths, p.lengths)
    with pytest.raises(ValueError):
        ca.compact_attn_cache_keep(p.cache, torch.zeros(2, 3, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV))


# ---------------------------------------------------------------- appending

APPEND = {
    "plain": dict(sequences=[(40, 3), (9, 9), (17, 0), (64, 1)], kv=2, heads=4, D=64, page=16, norm=False),
    "norm": dict(sequences=[(40, 3), (9, 9)], kv=2, heads=4, D=128, page=32, weights=True),
    "rotated": dict(sequences=[(40, 3), (300, 9)], kv=2, heads=4, D=128, page=48, weights=True, channels=(128, 0, 0), pairing="half"),
    "rotated-part": dict(sequences=[(40, 3), (300, 9)], kv=2, heads=6, D=96, page=48, norm=False, channels=(64, 0, 0), pairing="interleaved"),
    "frames": dict(sequences=[(160, 160), (37, 36)], kv=3, heads=3, D=128, page=64, weights=True, channels=(32, 48, 48), pairing="half", frame=(5, 7), origins=[12, 4]),
    "frames-origin": dict(sequences=[(80, 40)], kv=1, heads=2, D=64, page=16, channels=(16, 24, 24), pairing="interleaved", frame=(5, 7), origins=[3], origin=(4, 1, 2)),
    "apart": dict(sequences=[(50, 11)], kv=2, heads=2, D=80, page=16, weights=True, channels=(30, 0, 0), pairing="half"),
    "no-queries": dict(sequences=[(50, 11), (70, 70)], kv=5, heads=0, D=64, page=16, weights=True, channels=(64, 0, 0), pairing="half"),
    "positions": dict(sequences=[(50, 11), (70, 20)], kv=2, heads=4, D=64, page=16, weights=True, channels=(16, 24, 24), pairing="half", positions=True, frame=(3, 3)),
    "wide-heads": dict(sequences=[(20, 5)], kv=2, heads=2, D=256, page=16, weights=True, channels=(256, 0, 0), pairing="half"),
    "narrow-heads": dict(sequences=[(200, 77)], kv=2, heads=2, D=8, page=16, channels=(8, 0, 0), pairing="interleaved"),
    "many": dict(sequences=[(i % 50 + 2, i % 3) for i in range(900)], kv=1, heads=2, D=64, page=16, channels=(64, 0, 0), pairing="half"),
}


def append_case(name, dtype, fused, seed=21):
    c = dict(dict(norm=True, weights=False, channels=None, pairing="half", frame=(1, 1), origins=None, origin=(0, 0, 0), positions=False), **APPEND[name])
    p = Paged(c["sequences"], c["kv"], c["D"], c["page"], dtype=dtype, origins=c["origins"], frame=c["frame"], seed=seed, behind=3)
    h, kv, D = c["heads"], c["kv"], c["D"]
    if fused:
        both = p.randn(p.tokens, h + 2 * kv, D)
        q, k, v = both[:, :h], both[:, h:h + kv], both[:, h + kv:]
        dev = both.to(DEV)
        on = dev[:, :h], dev[:, h:h + kv], dev[:, h + kv:]
    else:
        q, k, v = p.randn(p.tokens, h, D), p.randn(p.tokens, kv, D), p.randn(p.tokens, kv, D)
        on = tuple(t.to(DEV) for t in (q, k, v))
    w = [(1 + 0.2 * p.randn(D).float()).to(DTYPES[dtype]) for _ in range(2)] if c["weights"] else [None, None]
    rotary = None if c["channels"] is None else ca.compact_attn_build_rotary(c["channels"], (400, 12, 12), pairing=c["pairing"])
    positions = np.random.default_rng(seed).integers(-1, 12, size=(p.tokens, 3)).astype(np.int32) if c["positions"] else None
    return c, p, (q, k, v), on, w, rotary, positions


def run_append(c, p, on, w, rotary, positions, **more):
    q, k, v = on
    return ca.compact_attn_cache_append(k, v, p.cache, q=q if c["heads"] else None, norm=c["norm"], q_weight=None if w[0] is None or not c["heads"] else w[0].to(DEV),
                                        k_weight=None if w[1] is None else w[1].to(DEV), rotary=rotary, origin=c["origin"],
                                        positions=None if positions is None else torch.from_numpy(positions).to(DEV), **more)


def want_rows(c, p, x, weight, row0, s, rotary, positions):
    """Rows of a sequence's new tokens in 64 bits, and the bound's sum of sizes |a| + |b|."""
    n, m = p.sequences[s]
    x = x[row0:row0 + m].double().numpy()
    y = np.stack([OR.norm(x[:, h], np.ones(p.D) if weight is None else weight.double().numpy(), 1e-6) if c["norm"] else x[:, h] for h in range(x.shape[1])], axis=1) if m else x
    size = np.abs(y)
    if c["channels"] is None:
        return y, size
    if positions is not None:
        at = positions[row0:row0 + m]
    else:
        behind = np.arange(n - m, n) - _origin(p, s)
        H, W = p.frame
        at = np.stack([behind // (H * W), behind // W % H, behind % W], axis=1) + np.array(c["origin"])
        at[behind < 0] = -1
    angle = OR.angles(at, [OR.frequencies(ch) for ch in c["channels"]])
    out = np.stack([OR.rotate(y[:, h], angle, c["pairing"]) for h in range(y.shape[1])], axis=1) if m else y
    half = angle.shape[1]
    a, b = (size[..., :half], size[..., half:2 * half]) if c["pairing"] == "half" else (size[..., 0:2 * half:2], size[..., 1:2 * half:2])
    both = a + b
    size = size.copy()
    if c["pairing"] == "half":
        size[..., :half] = size[..., half:2 * half] = both
    else:
        size[..., 0:2 * half:2] = size[..., 1:2 * half:2] = both
    return out, size


def bits(t):
    return t.contiguous().view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", list(APPEND))
def test_append(name, dtype):
    print("append", name, dtype, flush=True)
    for fused in (False, True):
        c, p, host, on, w, rotary, positions = append_case(name, dtype, fused)
        before = [t.clone() for t in p.pages]
        out = None if not c["heads"] else torch.full((p.tokens, c["heads"], p.D), 6.0, dtype=DTYPES[dtype], device=DEV)
        q = run_append(c, p, on, w, rotary, positions, out=out)
        assert q is out
        got_k, got_v = p.k.cpu(), p.v.cpu()
        row, half = 0, HALF[dtype]
        for s, (n, m) in enumerate(p.sequences):
            want_k, size_k = want_rows(c, p, host[1], w[1], row, s, rotary, positions)
            if c["heads"]:
                want_q, size_q = want_rows(c, p, host[0], w[0], row, s, rotary, positions)
                err = np.abs(q[row:row + m].double().cpu().numpy() - want_q)
                assert np.all(err <= half * np.abs(want_q) + (p.D + 16) * U * size_q), (s, err.max(initial=0))
            for i in range(m):
                page, slot = OC.place_of(p.table, s, n - m + i, p.page, p.num_pages)
                err = np.abs(got_k[page, :, slot].double().numpy() - want_k[i])
                assert np.all(err <= half * np.abs(want_k[i]) + (p.D + 16) * U * size_k[i]), (s, i, err.max())
                assert torch.equal(bits(got_v[page, :, slot]), bits(host[2][row + i]))
                before[0][page, :, slot], before[1][page, :, slot] = got_k[page, :, slot], got_v[page, :, slot]
            row += m
        # nothing else has changed: other slots, rows behind the last sequence
        assert torch.equal(bits(before[0]), bits(got_k)) and torch.equal(bits(before[1]), bits(got_v))
        if c["heads"]:
            assert (q[p.rows:] == 6).all()


@pytest.mark.gpu
def test_append_where_there_is_no_page():
    """New tokens whose page is not there, or whose number is below 0 or past the table, are not stored; their queries are written."""
    p = Paged([(64, 20), (10, 30), (48, 2)], 1, 64, 16, seed=30, extra_width=0)
    p.table[0, 3], p.table[2, 2] = -1, p.num_pages
    p.upload()
    p.lengths.copy_(torch.tensor([64, 10, 70], dtype=torch.int32))   # the last one is past its table: cut to 64, past its two last pages
    x = p.randn(52, 3, 64).to(DEV)
    before = p.k.cpu(), p.v.cpu()
    q = ca.compact_attn_cache_append(x[:, :1], x[:, 1:2], p.cache, q=x[:, 2:], norm=False)
    assert torch.equal(q, x[:, 2:])
    stored = {(int(p.table[0, 2]), t - 32): t - 44 for t in range(44, 48)} | {(int(p.table[1, 0]), t): 20 + 20 + t for t in range(10)}
    for pages, old, new in ((p.k.cpu(), before[0], x[:, 0].cpu()), (p.v.cpu(), before[1], x[:, 1].cpu())):
        for (page, slot), row in stored.items():
            old[page, 0, slot] = new[row]
        assert torch.equal(bits(pages), bits(old))


@pytest.mark.gpu
def test_append_positions_past_the_table_are_nan():
    p = Paged([(30, 30)], 1, 64, 16, seed=31)
    rotary = ca.compact_attn_build_rotary((32, 0, 0), (20, 1, 1), pairing="half")
    x = p.randn(30, 1, 64).to(DEV)
    q = ca.compact_attn_cache_append(x, x, p.cache, q=x, norm=False, rotary=rotary)
    assert torch.isfinite(q[:20]).all() and torch.isnan(q[20:, :, :32]).all() and torch.equal(q[20:, :, 32:], x[20:, :, 32:])
    q = ca.compact_attn_cache_append(x, x, p.cache, q=x, norm=False, rotary=rotary, origin=(2 ** 31 - 1, 0, 0))   # (a sum past 32 bits is past the table as well)
    assert torch.isnan(q[:, :, :32]).all()


# ---------------------------------------------------------------- keeping drafts

@pytest.mark.gpu
@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("bf16", 128), ("f32", 128), ("bf16", 512), ("f32", 256), ("bf16", 8)])
def test_keep(dtype, D):
    sequences = [(100, 64), (64, 64), (37, 5), (200, 40), (12, 0), (90, 1), (500, 33), (30, 40)]
    p = Paged(sequences, 2, D, 16, dtype=dtype, seed=40)
    p.table[6, 30] = -1   # the page of tokens 480 .. 495 is not there
    p.upload()
    paths = [list(range(64))[::-1], [0, 3, 9, 60], [4, 4, 4], [0, 7, 7, 39, 40, -1, 2], [0, 1], [0], [0, 20, 21, 32, 14], [10, 12, 39]]
    width = 64
    kept = np.full((len(sequences), width), -1, np.int32)
    for s, path in enumerate(paths):
        kept[s, :len(path)] = path
    counts = [len(path) for path in paths]
    counts[5] = -3
    host = [(p.host(s, 0), p.host(s, 1)) for s in range(len(sequences))]
    old = [t.clone() for t in p.pages]
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(DEV)
    ca.compact_attn_cache_keep(p.cache, dev(kept), dev(counts))
    for which, got in enumerate((p.k.cpu(), p.v.cpu())):
        for s, (n, m) in enumerate(sequences):
            base, path = n - m, paths[s][:max(0, counts[s])]
            for j, i in enumerate(path):
                if not (0 <= i < m and j < m) or base + i < 0 or base + j < 0:
                    continue
                a, b = (OC.place_of(p.table, s, base + x, p.page, p.num_pages) for x in (i, j))
                if a is not None and b is not None:
                    old[which][b[0], :, b[1]] = p.pages[which][a[0], :, a[1]]
        assert torch.equal(bits(got), bits(old[which]))
    del host


# ---------------------------------------------------------------- offsets, streams, graphs

@pytest.mark.gpu
def test_offsets_past_32_bits():
    """Pages of 5 GB: tokens in the last ones."""
    pages, kv, page, D = 1250, 8, 2048, 128   # 4 MB a page
    k, v = (torch.zeros(pages, kv, page, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    sequences = [(3000, 1), (2049, 3)]
    p = Paged(sequences, kv, D, page, seed=50)
    table = np.array([[1249, 1247], [1246, 1248]], dtype=np.int32)
    for s in range(2):
        for i in range(2):
            k[table[s, i]], v[table[s, i]] = p.k[p.table[s, i]], p.v[p.table[s, i]]
    cache = ca.Cache(k, v, torch.from_numpy(table).to(DEV), p.lengths, p.starts)
    x = p.randn(p.rows, kv * 4, D).to(DEV)
    q = ca.compact_attn_cache_append(x[:, :kv], x[:, kv:2 * kv], cache, q=x[:, 2 * kv:], norm=False)
    row = 0
    for s, (n, m) in enumerate(sequences):
        for i in range(m):
            t = n - m + i
            assert torch.equal(k[table[s, t // page], :, t % page], x[row + i, :kv]) and torch.equal(v[table[s, t // page], :, t % page], x[row + i, kv:2 * kv])
            p.pages[0][p.table[s, t // page], :, t % page], p.pages[1][p.table[s, t // page], :, t % page] = x[row + i, :kv].cpu(), x[row + i, kv:2 * kv].cpu()
        row += m
    check_attend(p, q, ca.compact_attn_cache_attend(q, cache))
    kept, counts = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in ([[0, -1], [2, 1]], [1, 1]))
    ca.compact_attn_cache_keep(cache, kept, counts)
    assert torch.equal(k[1246, :, 2046], k[1248, :, 0])


@pytest.mark.gpu
def test_calls_on_other_streams():
    """Two streams at once, each with a cache of its own, against the calls one after the other."""
    cases = [attend_case("ragged-grouped", seed=60), attend_case("long", seed=61)]
    want = [run_attend(*c) for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    got = [[], []]
    for _ in range(4):
        for i, (c, stream) in enumerate(zip(cases, streams)):
            got[i].append(run_attend(*c, stream=stream))
    torch.cuda.synchronize()
    for i, w in enumerate(want):
        for g in got[i]:
            assert torch.equal(g[0], w[0]) and torch.equal(g[1], w[1])


class Stream:
    """A program that makes tokens: appends to its cache, attends, keeps drafts; everything it changes lies on the device."""

    def __init__(self, D, kv, group, frame, origins, start, seed, dtype="bf16"):
        self.D, self.kv, self.group, self.frame, self.origins = D, kv, group, frame, origins
        self.rng = np.random.default_rng(seed)
        self.history = [[] for _ in start]   # per sequence: (k, v) rows in 64 bits, as stored
        n, page = len(start), 16
        width = 40
        self.table = self.rng.permutation(n * width).reshape(n, width).astype(np.int32)
        self.k, self.v = (torch.full((n * width, kv, page, D), math.nan, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        dev = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
        self.lengths, self.starts = dev([0] * n), dev([0] * (n + 1))
        self.cache = ca.Cache(self.k, self.v, torch.from_numpy(self.table).to(DEV), self.lengths, self.starts, origins=None if origins is None else dev(origins), frame=frame)
        self.channels = (D // 4 * 2, D // 4, D // 4)
        self.rotary = ca.compact_attn_build_rotary(self.channels, (700, 16, 16), pairing="half")
        self.weights = [(1 + 0.2 * torch.from_numpy(self.rng.normal(size=D).astype(np.float32))).to(torch.bfloat16).to(DEV) for _ in range(2)]
        self.tokens = [0] * n

    def inputs(self, new):
        m = sum(new)
        x = torch.from_numpy(self.rng.normal(size=(m, self.kv * (self.group + 2), self.D)).astype(np.float32)).to(torch.bfloat16)
        return x

    def announce(self, new):
        self.tokens = [n + m for n, m in zip(self.tokens, new)]
        self.lengths.copy_(torch.tensor(self.tokens, dtype=torch.int32))
        self.starts.copy_(torch.tensor(np.cumsum([0] + list(new)), dtype=torch.int32))

    def step(self, x, tree=None, **how):
        h = self.kv * self.group
        q, k, v = x[:, :h], x[:, h:h + self.kv], x[:, h + self.kv:]
        q = ca.compact_attn_cache_append(k, v, self.cache, q=q, q_weight=self.weights[0], k_weight=self.weights[1], rotary=self.rotary)
        return q, *ca.compact_attn_cache_attend(q, self.cache, tree=tree, **how)


@pytest.mark.gpu
@pytest.mark.parametrize("cap,window", [(0.0, 0), (20.0, 2)])
def test_frames_one_after_the_other_are_a_clip(cap, window):
    """The use that the cache is for: a prompt, then frames one by one, give what one call over the whole clip gives, and what the oracle gives for the clip."""
    H, W, frames, prompt = 3, 5, 6, 7
    new_by_step = [[prompt]] + [[H * W]] * frames
    whole = Stream(64, 2, 2, (H, W), [prompt], [0], 70)
    x = whole.inputs([prompt + frames * H * W]).to(DEV)
    whole.announce([prompt + frames * H * W])
    want = whole.step(x, cap=cap, window=window)
    parts = Stream(64, 2, 2, (H, W), [prompt], [0], 70)
    got, row = [], 0
    for new in new_by_step:
        parts.announce(new)
        got.append(parts.step(x[row:row + new[0]], cap=cap, window=window))
        row += new[0]
    q, out, lse = (torch.cat(t) for t in zip(*got))
    for page in range(prompt + frames * H * W):   # the pages hold the same tokens
        a, b = (t.k[t.table[0, page // 16], :, page % 16] for t in (whole, parts))
        assert torch.equal(a, b)
    assert torch.equal(q, want[0])
    p = Paged([(prompt + frames * H * W, prompt + frames * H * W)], 2, 64, 16, origins=[prompt], frame=(H, W), seed=1)
    p.table, p.pages, p.num_pages = whole.table, [whole.k.cpu(), whole.v.cpu()], whole.k.shape[0]
    for result in ((out, lse), want[1:]):
        check_attend(p, q, result, cap=cap, window=window)


@pytest.mark.gpu
def test_accepted_drafts_are_a_sequence_without_the_others():
    """Drafts are appended with the positions of their places, verified, and the accepted ones kept: the cache then holds what appending those alone gives."""
    with_drafts, plain = (Stream(128, 2, 2, (1, 1), None, [0, 0], 80) for _ in range(2))
    x = with_drafts.inputs([50, 33]).to(DEV)
    for t in (with_drafts, plain):
        t.announce([50, 33])
        t.step(x)
    trees = [chain_words(np.random.default_rng(s), m) for s, m in ((1, 20), (2, 11))]
    path = []
    for words in trees:   # the path to the last draft
        path.append([i for i in range(len(words)) if words[-1] >> i & 1])
    drafts = with_drafts.inputs([20, 11]).to(DEV)
    with_drafts.announce([20, 11])
    at = np.array([base + bin(w).count("1") - 1 for base, words in zip((50, 33), trees) for w in words], dtype=np.int32)
    positions = torch.from_numpy(np.stack([at, at * 0, at * 0], axis=1)).to(DEV)
    h = 4
    q = ca.compact_attn_cache_append(drafts[:, h:h + 2], drafts[:, h + 2:], with_drafts.cache, q=drafts[:, :h], q_weight=with_drafts.weights[0], k_weight=with_drafts.weights[1],
                                     rotary=with_drafts.rotary, positions=positions)
    out, lse = ca.compact_attn_cache_attend(q, with_drafts.cache, tree=to_words(trees[0] + trees[1]))
    width = max(map(len, path))
    kept = torch.tensor([p + [-1] * (width - len(p)) for p in path], dtype=torch.int32, device=DEV)
    counts = torch.tensor([len(p) for p in path], dtype=torch.int32, device=DEV)
    ca.compact_attn_cache_keep(with_drafts.cache, kept, counts)
    rows = torch.tensor(path[0] + [20 + i for i in path[1]], device=DEV)
    plain.announce([len(p) for p in path])
    q2 = ca.compact_attn_cache_append(drafts[rows, h:h + 2], drafts[rows, h + 2:], plain.cache, q=drafts[rows, :h], q_weight=plain.weights[0], k_weight=plain.weights[1],
                                      rotary=plain.rotary, positions=positions[rows])
    assert torch.equal(q2, q[rows])
    for s, n in enumerate((50 + len(path[0]), 33 + len(path[1]))):
        for t in range(n):
            for a, b in ((with_drafts.k, plain.k), (with_drafts.v, plain.v)):
                assert torch.equal(a[with_drafts.table[s, t // 16], :, t % 16], b[plain.table[s, t // 16], :, t % 16])
    p = Paged([(50 + len(path[0]), len(path[0])), (33 + len(path[1]), len(path[1]))], 2, 128, 16, seed=1)
    p.table, p.pages, p.num_pages = plain.table, [plain.k.cpu(), plain.v.cpu()], plain.k.shape[0]
    check_attend(p, q2, (out[rows], lse[rows]))
    check_attend(p, q2, ca.compact_attn_cache_attend(q2, plain.cache))


@pytest.mark.gpu
@pytest.mark.parametrize("kv,group", [(2, 2), (1, 17)])   # few rows a sequence, many
def test_a_captured_step_goes_by_what_lies_in_the_arrays(kv, group):
    """Append, attend and keep in one graph, replayed with other lengths, rows and drafts, with eager work in between: every replay gives what eager calls give."""
    eager, graph = (Stream(64, kv, group, (1, 1), None, [0, 0, 0], 90) for _ in range(2))
    rows = 12
    x, words = torch.zeros(rows, kv * (group + 2), 64, dtype=torch.bfloat16, device=DEV), torch.zeros(rows, dtype=torch.int64, device=DEV)
    kept, counts = torch.zeros(3, 4, dtype=torch.int32, device=DEV), torch.zeros(3, dtype=torch.int32, device=DEV)
    ca.compact_attn_rotary_upload(eager.rotary)
    ca.compact_attn_rotary_upload(graph.rotary)

    def all_of(t, x, words, kept, counts):
        results = t.step(x, tree=words)
        ca.compact_attn_cache_keep(t.cache, kept, counts)
        return results

    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        results = all_of(graph, x, words, kept, counts)
    rng = np.random.default_rng(5)
    for turn in range(6):
        new = [(4, 4, 4), (1, 7, 4), (12, 0, 0), (0, 3, 2), (5, 5, 2), (1, 1, 1)][turn]
        n = sum(new)
        fresh = eager.inputs([rows]).to(DEV)
        tree = [w for m in new for w in chain_words(rng, m)] + [0] * (rows - n)
        for t in (eager, graph):
            t.announce(new)
        x.copy_(fresh)
        words.copy_(to_words(tree))
        kept.copy_(torch.from_numpy(rng.integers(0, 5, size=(3, 4)).astype(np.int32)))
        counts.copy_(torch.from_numpy(rng.integers(0, 5, size=3).astype(np.int32)))
        g.replay()
        torch.cuda.synchronize()
        want = all_of(eager, fresh, words, kept, counts)
        torch.randn(1000, device=DEV).sum().item()
        for a, b in zip(results, want):
            assert torch.equal(a[:n], b[:n]), turn
        assert torch.equal(bits(graph.k), bits(eager.k)) and torch.equal(bits(graph.v), bits(eager.v)), turn
        assert torch.isfinite(want[1][:n]).all()
