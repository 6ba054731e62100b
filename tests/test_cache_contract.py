"""What the paged cache promises beside its formulas: how precise capped scores are wherever a row's tokens lie, which attributes of a Cache may change, workspaces that do not fit, and runs long
enough that the kernels look up where pages lie more than once."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2508_12969_amd as ca
from test_cache import DEV, DTYPES, U, P, Paged, _append_call, _attend_call, _raw_cache, chain_words, check_attend, run_attend

# ---------------------------------------------------------------- capped scores


def _exact_products(sequences, kv, D, page, dtype, seed, **more):
    """A cache whose keys, and queries to go with them, are multiples of 1/8 and 1/4: sums of their products are exact in fp32."""
    p = Paged(sequences, kv, D, page, dtype=dtype, seed=seed, **more)
    p.pages[0] = (p.pages[0].float() * 4).round().div(4).to(DTYPES[dtype])
    p.upload()
    return p


def _wider(p, tokens):
    """The same cache with a table that has room for so many tokens a sequence."""
    table = np.full((p.table.shape[0], tokens // p.page), -1, np.int32)
    table[:, :p.table.shape[1]] = p.table
    return ca.Cache(p.k, p.v, torch.from_numpy(table).to(DEV), p.lengths, p.starts, origins=p.dev_origins, frame=p.frame)


def _capped(p, q, s, h, group, scale, cap):
    """Scores of all new tokens and all tokens of a sequence in 64 bits."""
    k, _ = p.host(s, 0)
    return cap * np.tanh(k[:, h // group] @ q.double().cpu().numpy().T * scale / cap).T


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("cap", [30.0, 4096.0])
@pytest.mark.parametrize("kind", ["causal", "window", "prompt"])
def test_capped_scores_of_few_tokens_are_precise_in_wide_tables(kind, cap, D, dtype):
    """Rows that see one to five tokens, beside 32 rows and more of their sequence, in tables with room for 100 000 tokens and for few.  Products are exact, so a score s is off by the roundings of
    scale / cap (2 u), of z (2 u), of the polynomial (8 u) and of the way back (4 u): 16 u |s|.  Of one token the log-sum-exp is the score; of n, (n + 8) u of the weights' sum and 4 u (1 + |lse|) of
    the logarithm join it.  (Off by cap 2^-22, a score of 8 at cap 4096 would miss that by a factor of 100.)"""
    print("capped", kind, cap, D, dtype, flush=True)
    how = dict(causal=dict(sequences=[(60, 60), (70, 70)]), window=dict(sequences=[(600, 60), (5000, 70)]),
               prompt=dict(sequences=[(5 + 7000, 7005)], frame=(70, 100), origins=[5]))[kind]
    kv, group = (1, 1) if kind == "prompt" else (2, 2)
    p = _exact_products(how.pop("sequences"), kv, D, 16, dtype, 8, **how)
    q = p.randn(p.rows, kv * group, D).float().round().div(8).to(DTYPES[dtype]).to(DEV)
    for tokens in (7168, 100000):
        lse = ca.compact_attn_cache_attend(q, _wider(p, tokens), scale=0.125, cap=cap, window=3 if kind == "window" else 0)[1].double().cpu().numpy()
        row = 0
        for s, (n, m) in enumerate(p.sequences):
            rows = range(m) if kind == "window" else range(5)
            for h in range(kv * group):
                x = _capped(p, q[row:row + m, h][list(rows)], s, h, group, 0.125, cap)
                for i in rows:
                    seen = x[i, n - m + i - 2:n - m + i + 1] if kind == "window" else x[i, :5] if kind == "prompt" else x[i, :i + 1]
                    assert np.abs(seen).max() < 15
                    want = np.log(np.exp(seen).sum())
                    bound = 16 * U * np.abs(seen).max() + (0 if len(seen) == 1 else (len(seen) + 8) * U + 4 * U * (1 + abs(want)))
                    assert abs(lse[row + i, h] - want) <= bound, (tokens, s, h, i, lse[row + i, h], want, bound)
            row += m


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cap", [30.0, 4096.0])
def test_capped_scores_of_many_tokens(cap, dtype):
    """Rows that see 5000 tokens and more, of which one has all of the weight that counts (its score is 40 above the others' largest), so that the log-sum-exp is that score.  It is off by 16 u |s| as
    above and by u (1 + |s|) from the others (5100 e^-40 is below u); with a cap of at most 64 by cap 2^-22 more."""
    p = _exact_products([(5100, 40)], 2, 64, 16, dtype, 9)
    q = torch.zeros(p.rows, 4, 64, dtype=DTYPES[dtype], device=DEV)
    q[:, :, 0] = 8
    for h in range(2):
        page, slot = int(p.table[0, 700 // 16]), 700 % 16
        p.pages[0][:, h, :, 0] = torch.where(torch.isnan(p.pages[0][:, h, :, 0]), p.pages[0][:, h, :, 0], torch.tensor(-2.0, dtype=DTYPES[dtype]))
        p.pages[0][page, h, slot, 0] = 2.0
    p.upload()
    top, other = (cap * math.tanh(x * 2.0 / cap) for x in (16.0, -16.0))
    assert top - other > 40
    lse = ca.compact_attn_cache_attend(q, p.cache, scale=2.0, cap=cap)[1].double().cpu().numpy()
    bound = 16 * U * abs(top) + U * (1 + abs(top)) + 4 * U * (1 + abs(top)) + (cap * 2.0 ** -22 if cap <= 64 else 0)
    assert np.abs(lse - top).max() <= bound, (np.abs(lse - top).max(), bound)


@pytest.mark.gpu
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kind", ["side-by-side", "shares", "tree"])
def test_capped_tiles_of_both_forms_in_one_launch(kind, D):
    """Prompts whose first tiles see few tokens and whose last see more than 4096, drafts over long and short caches: tiles of both forms, whole and cut, with a distance bias; every row against the oracle."""
    print("both forms", kind, D, flush=True)
    sequences = {"side-by-side": [(6000, 6000)], "shares": [(6000, 6000), (300, 40), (5000, 700), (4100, 33)], "tree": [(6000, 40), (300, 40), (4200, 64), (4100, 33)]}[kind]
    p = Paged(sequences, 1, D, 16, seed=17, origins=[3] * len(sequences))
    q = p.randn(p.rows, 2, D).mul(2).to(DEV)
    slopes, words = np.array([0.02, 0.001], dtype=np.float32), [w for _, m in sequences for w in chain_words(p.rng, m)] if kind == "tree" else None
    how = dict(cap=20.0)
    got = run_attend(p, q, slopes, words, how)
    again = run_attend(p, q, slopes, words, how)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])
    check_attend(p, q, got, slopes=slopes, words=words, **how)


# ---------------------------------------------------------------- what a Cache holds


@pytest.mark.parametrize("name", ["k", "v", "table", "lengths", "starts", "origins", "frame"])
def test_attributes_of_a_cache_cannot_be_replaced(name):
    cache = ca.Cache.__new__(ca.Cache)   # (one that is made needs device tensors)
    with pytest.raises(AttributeError, match=name):
        setattr(cache, name, None)
    with pytest.raises(AttributeError):
        delattr(cache, name)


@pytest.mark.gpu
def test_a_cache_keeps_the_tensors_that_calls_read():
    """What a program may try to go on with: new tensors for old ones.  They are refused, the calls' tensors stay alive and are what the attributes give."""
    p = Paged([(40, 2), (30, 1)], 2, 64, 16, seed=5, origins=[3, 4], frame=(2, 3))
    q = p.randn(p.rows, 4, 64).to(DEV)
    want = ca.compact_attn_cache_attend(q, p.cache)
    own = dict(k=p.k, v=p.v, table=p.dev_table, lengths=p.lengths, starts=p.starts, origins=p.dev_origins, frame=(2, 3))
    for name, value in own.items():
        other = (1, 1) if name == "frame" else value + 1
        with pytest.raises(AttributeError, match=name):
            setattr(p.cache, name, other)
        assert getattr(p.cache, name) is value or name == "frame" and p.cache.frame == value
    got = ca.compact_attn_cache_attend(q, p.cache)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    p.lengths += 1   # in place: the next call goes by it
    p.lengths -= 1
    check_attend(p, q, ca.compact_attn_cache_attend(q, p.cache))


# ---------------------------------------------------------------- sizes and workspaces that do not fit (nothing is launched)


@pytest.mark.parametrize("D,dtype", [(512, 1), (264, 1), (256, 0), (132, 0)])
def test_appending_more_tokens_than_a_launch_takes_is_refused(D, dtype):
    """Rows of more than 512 bytes are four a workgroup, and 2^24 workgroups of 256 threads are past what a launch takes: the three sizes below 2^26 are refused like 2^26 is, before a launch."""
    for tokens in (2 ** 26 - 3, 2 ** 26 - 1, 2 ** 26):
        status, message = _append_call(_raw_cache(head_dim=D, dtype=dtype, tokens=tokens))
        assert status == -2 and "2^26" in message, (tokens, status, message)


NEEDY = {   # calls that need a workspace: few and many rows on a line of shares, one sequence cut into parts, fp32
    "few": dict(table_width=100), "many": dict(table_width=100, tokens=200), "parts": dict(table_width=800, sequences=1, tokens=1000, page_tokens=64), "f32": dict(table_width=100, dtype=0),
}


@pytest.mark.parametrize("name", list(NEEDY))
def test_workspaces_that_do_not_fit_are_refused(name):
    """Too small, absent, not aligned, or over anything that the call reads or writes.  (A table of items is 256 bytes at least, and sums follow it.)"""
    cache, size = _raw_cache(**NEEDY[name]), ctypes.c_int64()
    assert ca.load_library().compact_attn_cache_workspace(cache, 4, size) == 0 and size.value > 256
    need = size.value
    for workspace, given in ((None, need), (None, 1 << 40), (P[11], 0), (P[11], 1), (P[11], 256), (P[11] + 8, need), (P[11] + 4, 1 << 40)):
        status, message = _attend_call(cache, workspace=workspace, size=given)
        assert status == -1 and "workspace of" in message and "bytes" in message, (workspace, given, status, message)
    tree = P[12]
    for over in (P[6], P[0], P[1], P[2], P[3], P[4], P[9], P[10], tree, P[13], P[2] - 256):
        status, message = _attend_call(cache, workspace=over, size=need, tree=tree, slopes=P[13])
        assert status == -1 and "overlap" in message, (over, status, message)


# ---------------------------------------------------------------- long runs

LONG = {
    # Where pages lie is looked up for 32 steps of a wave (bf16, 32 tokens each), 64 (fp32, 16 each) or 128 of a workgroup (many rows, 64 each).  `alike`: so many sequences share one table row, for
    # lines of which every workgroup takes several such runs: few rows 400 steps of 639 for each item (100 a wave) at head dim 128, 197 a wave in fp32; many rows 490 of 629
    "few": dict(tokens=20000, new=1, kv=2, group=2, D=128, alike=80),
    "few-64": dict(tokens=20000, new=3, kv=2, group=1, D=64, alike=160),
    "few-f32": dict(tokens=20000, new=1, kv=2, group=2, D=128, alike=80, dtype="f32"),
    "few-f32-64": dict(tokens=20000, new=20, kv=2, group=1, D=64, alike=80, dtype="f32"),
    "many": dict(tokens=40000, new=40, kv=2, group=1, D=128, alike=200),
    "many-64": dict(tokens=40000, new=20, kv=2, group=2, D=64, alike=200),
    # 505 items of 313 steps, which 512 places take whole; 768 places take 505 items of 625 steps in three parts each
    "items": dict(tokens=20000, new=640, kv=5, group=20, D=128, alike=1),
    "parts": dict(tokens=40000, new=640, kv=5, group=20, D=64, alike=1),
}


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(LONG))
def test_runs_that_look_up_pages_more_than_once(name):
    """Walks so long that the kernels refill what they know of the table; pages lie in random order.  A few sequences and key heads, two query heads of each, against the oracle."""
    print("long", name, flush=True)
    c = dict(dict(dtype="bf16"), **LONG[name])
    p = Paged([(c["tokens"], c["new"])], c["kv"], c["D"], 16, dtype=c["dtype"], seed=70)
    alike, new, group = c["alike"], c["new"], c["group"]
    ints = lambda x: torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(DEV)
    cache = ca.Cache(p.k, p.v, ints(np.repeat(p.table, alike, axis=0)), ints([c["tokens"]] * alike), ints(np.arange(alike + 1) * new))
    q = p.randn(alike * new, c["kv"] * group, c["D"]).mul(2).to(DEV)
    out, lse = ca.compact_attn_cache_attend(q, cache)
    again = ca.compact_attn_cache_attend(q, cache)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
    pages = p.pages
    for s in sorted({0, alike // 3, alike - 1}):
        for key_head in sorted({0, c["kv"] - 1}):
            heads = [key_head * group] if group == 1 else [key_head * group, key_head * group + group - 1]
            p.pages, p.kv = [t[:, key_head:key_head + 1] for t in pages], 1
            rows = slice(s * new, (s + 1) * new)
            check_attend(p, q[rows][:, heads], (out[rows][:, heads], lse[rows][:, heads]))
