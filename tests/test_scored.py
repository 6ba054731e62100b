"""Scored attention (capped, biased and masked scores) and its gradients: refusals, the transposed lists and the oracle's gradients on the CPU, the kernels
against the oracle on the GPU.

Tolerances, per element.  u = 2^-24 and h = 2^-8 are half a step of fp32 and bf16.  A score is a sum of D products of bf16 values in fp32, off by at most
(D + 2) u scale sum |q k|; capping adds 8 u cap, the bias 4 u of itself, the shift to the row's reference and the exponential 4 u (|s| + |lse|) + 4 u:
delta, the relative error of a weight, is at most their sum over the plane.  Weights are rounded to bf16 for the product with V and the result is
rounded: |out| is off by h (sum p |v| + |out|) + 2 delta sum p |v|, the log-sum-exp by delta + 8 u (1 + |lse|).  Backwards: dV as out.  dS is
rounded to bf16; before that it is off by 2 delta |dS| + 16 u p |dp - D| (the slope of the cap) and by p times the errors of dp, D u sum |dO v|,
and of the row's sum of dO O, where O is rounded: sum |dO| (error of out).  dQ and dK are sums of dS times K or Q, rounded."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2508_12969_amd as ca
from oracle import layout as OL
from oracle import permute as OP
from oracle import scored as OS
from oracle.geometry import Geometry
from paper_2508_12969_amd import scored as SC

DEV = "cuda:0"
ABSENT = (-1, -1)
U, HALF = 2.0 ** -24, 2.0 ** -8
P = [0x100000000 * (i + 1) for i in range(16)]   # addresses that are never read


def _layout(T, H, W, tile, n_text, batch, heads, D, dtype="bf16", scale=0.0, csr=None):
    if csr is not None:
        return ca.compact_attn_layout_from_csr(T, H, W, tile, n_text, batch, len(csr), D, dtype, csr, scale)
    return ca.compact_attn_build_layout(T, H, W, tile, n_text, batch, len(heads), D, dtype, heads, scale)


# ---------------------------------------------------------------- host

def _call(fn, *args):
    lib = ca.load_library()
    return getattr(lib, fn)(*args), lib.compact_attn_last_error().decode()


def test_refusals():
    lay = _layout(4, 8, 8, (1, 8, 8), 64, 1, [[(1, (0, 0), ABSENT)]] * 2, 64)
    need = ctypes.c_int64()
    plain = SC.ca_scores(0.0, None, None, None, None)
    full = SC.ca_scores(20.0, P[8], P[9], P[10], P[11])
    assert _call("compact_attn_scored_workspace", lay.handle, plain, 0, need)[0] == 0 and need.value == 0
    assert _call("compact_attn_scored_workspace", lay.handle, SC.ca_scores(1.0, None, P[9], None, None), 0, need)[0] == 0 and need.value == 0
    assert _call("compact_attn_scored_workspace", lay.handle, full, 0, need)[0] == 0 and need.value > 0
    forward_need = need.value
    assert _call("compact_attn_scored_workspace", lay.handle, full, 1, need)[0] == 0 and need.value > forward_need
    backward_need = need.value
    for args in ((None, plain, 0, need), (lay.handle, None, 0, need), (lay.handle, plain, 2, need), (lay.handle, plain, 0, None)):
        assert _call("compact_attn_scored_workspace", *args)[0] == -1

    def forward(q=P[0], k=P[1], v=P[2], s=full, out=P[3], lse=P[4], ws=P[5], size=forward_need):
        return _call("compact_attn_forward_scored", q, k, v, lay.handle, s, out, lse, ws, size, None)

    def backward(do=P[6], q=P[0], k=P[1], v=P[2], o=P[3], lse=P[4], s=full, dq=P[12], dk=P[13], dv=P[14], ws=P[5], size=backward_need):
        return _call("compact_attn_backward_scored", do, q, k, v, o, lse, lay.handle, s, dq, dk, dv, ws, size, None)

    S = SC.ca_scores
    bad_scores = [S(-1.0, None, None, None, None), S(math.nan, None, None, None, None), S(math.inf, None, None, None, None), S(1e-6, None, None, None, None), S(5000.0, None, None, None, None), S(0.0, P[8], None, None, None),
                  S(0.0, None, None, P[10], None), S(0.0, P[8] + 2, P[9], None, None), S(0.0, None, P[9] + 1, None, None), S(0.0, None, P[9], P[10] + 2, None),
                  S(0.0, None, None, None, P[11] + 3)]
    for bad in [dict(q=None), dict(out=None), dict(lse=None), dict(s=None), dict(q=P[0] + 8), dict(out=P[3] + 8), dict(lse=P[4] + 2), dict(ws=None), dict(ws=P[5] + 8),
                dict(size=forward_need - 1), dict(out=P[0]), dict(out=P[2] + 128), dict(lse=P[1] + 64), dict(ws=P[0]), dict(lse=P[3] + 64), dict(ws=P[3]), dict(out=P[9]),
                dict(ws=P[10] + 16)] + [dict(s=s) for s in bad_scores]:
        st, message = forward(**bad)
        assert st == -1 and message, (bad, st, message)
    for bad in [dict(do=None), dict(o=None), dict(dq=None), dict(do=P[6] + 8), dict(lse=P[4] + 1), dict(dv=P[14] + 4), dict(ws=None), dict(size=backward_need - 1), dict(dq=P[0]),
                dict(dk=P[12] + 512), dict(dv=P[6]), dict(ws=P[14]), dict(dq=P[4])] + [dict(s=s) for s in bad_scores]:
        st, message = backward(**bad)
        assert st == -1 and message, (bad, st, message)


@pytest.mark.parametrize("tile,D,dtype", [((1, 4, 4), 64, "bf16"), ((1, 8, 8), 32, "bf16"), ((1, 8, 8), 64, "f32"), ((2, 8, 16), 128, "bf16")])
def test_layouts_that_no_kernel_takes_are_refused(tile, D, dtype):
    lay = _layout(4, 16, 16, tile, 0, 1, [[(1, (0, 0), ABSENT)]], D, dtype)
    need = ctypes.c_int64()
    st, message = _call("compact_attn_scored_workspace", lay.handle, SC.ca_scores(0.0, None, None, None, None), 0, need)
    assert st == -2 and "scored" in message


def test_oracle_gradients_from_differences():
    rng = np.random.default_rng(1)
    n, d = 9, 4
    q, k, v, do = (rng.normal(size=(n, d)) for _ in range(4))
    pos = rng.integers(-3, 6, n)
    lim = pos + rng.integers(-1, 3, n)
    lim[4] = -100   # sees nothing
    doc = rng.integers(-1, 2, n)
    seen = OS.visible(rng.random((n, n)) < 0.8, pos, lim, doc)
    how = dict(cap=1.5, slope=0.3, positions=pos)
    f = lambda q, k, v: (OS.forward(q, k, v, seen, 0.7, **how)[0] * do).sum()
    grads = OS.backward(do, q, k, v, seen, 0.7, **how)[:3]
    for which in range(3):
        for i in range(n):
            for j in range(d):
                args = [q, k, v]
                ends = []
                for sign in (1, -1):
                    args[which] = (q, k, v)[which].copy()
                    args[which][i, j] += sign * 1e-6
                    ends.append(f(*args))
                assert abs((ends[0] - ends[1]) / 2e-6 - grads[which][i, j]) < 1e-8
    assert not seen[4].any() and not grads[0][4].any()


# ---------------------------------------------------------------- kernels

def _random_csr(rng, n, heads, share):
    """Random lists: empty rows and columns among them."""
    out = []
    for _ in range(heads):
        rows = [np.flatnonzero(rng.random(n) < share) if rng.random() > 0.15 else np.zeros(0, int) for _ in range(n)]
        out.append((np.concatenate([[0], np.cumsum([len(r) for r in rows])]), np.concatenate(rows)))
    return out


class Problem:
    def __init__(self, grid, tile, n_text, D, heads=2, batch=1, seed=0, lists="windows", cap=0.0, bias=False, prefix=None, docs=None, gain=1.0, scale=0.0):
        rng = self.rng = np.random.default_rng(seed)
        g = self.geom = Geometry(*grid, *tile, n_text)
        self.batch, self.heads, self.D = batch, heads, D
        n = g.n
        if lists == "windows":
            descriptions = [[(0, (1, 1), ABSENT), (1, (0, 0), ABSENT)], [(g.nT - 1, (g.nH - 1, g.nW - 1), ABSENT)], []]
            groups = [descriptions[h % 3] for h in range(heads)]
            self.layout = _layout(*grid, tile, n_text, batch, groups, D, scale=scale)
        else:
            csr = _random_csr(rng, n, heads, lists)
            self.layout = _layout(*grid, tile, n_text, batch, None, D, scale=scale, csr=csr)
        self.tile_of = g.token_slots() // g.B
        self.keep = []
        for h in range(heads):
            row_ptr, col = ca.compact_attn_layout_csr(self.layout, h)
            m = np.zeros((n, n), bool)
            for r in range(n):
                m[r, col[row_ptr[r]:row_ptr[r + 1]]] = True
            self.keep.append(m[self.tile_of][:, self.tile_of])
        N = g.N_real
        self.scale = scale or D ** -0.5
        self.cap = cap
        tokens = lambda lo, hi: rng.integers(lo, hi, size=(batch, N)).astype(np.int32)
        frame = np.concatenate([np.arange(g.T * g.H * g.W) // (g.H * g.W), np.zeros(n_text, int)]).astype(np.int32)
        frame = np.tile(frame, (batch, 1))
        self.positions = self.limits = self.documents = self.slopes = None
        if prefix == "random":
            self.positions, self.limits = tokens(-5, 40), tokens(-8, 40)
            self.limits[:, ::7] = -100   # sees nothing
        elif prefix is not None:
            self.positions = frame
            self.limits = np.maximum(frame, prefix - 1)
        elif bias:
            self.positions = tokens(-50, 50)
        if bias:
            self.slopes = np.linspace(0.02, 0.4, heads).astype(np.float32)
            self.slopes[-1] = -0.05
        if docs == "random":
            self.documents = tokens(-1, 3)
        elif docs == "frames":
            self.documents = np.minimum(frame // 2, 2).astype(np.int32)
            self.documents[:, N - n_text // 3:] = -7
        elif docs == "none there":
            self.documents = np.full((batch, N), -1, np.int32)
        values = lambda gain: torch.from_numpy((gain * rng.normal(size=(batch, heads, N, D))).astype(np.float32)).to(torch.bfloat16)
        self.q, self.k, self.v, self.do = values(gain), values(1.0), values(1.0), values(1.0)

    def tiled(self, x):
        out = torch.zeros(self.batch, self.heads, self.geom.N_pad, self.D, dtype=x.dtype)
        out[:, :, torch.from_numpy(self.geom.token_slots())] = x
        return out.to(DEV)

    def how(self):
        put = lambda x: None if x is None else torch.from_numpy(x).to(DEV)
        return dict(cap=self.cap, slopes=put(self.slopes), positions=put(self.positions), limits=put(self.limits), documents=put(self.documents))

    def run(self, **kw):
        self.args = [self.tiled(x) for x in (self.q, self.k, self.v)]
        self.dout = self.tiled(self.do)
        self.given = self.how()
        out, lse = ca.compact_attn_forward_scored(*self.args, self.layout, **self.given, **kw)
        grads = ca.compact_attn_backward_scored(self.dout, *self.args, out, lse, self.layout, **self.given, **kw)
        return out, lse, *grads

    def check(self, out, lse, dq, dk, dv):
        real = OP.slot_valid(self.geom)
        worst = {}

        def close(name, got, want, bound):
            got = got.double().cpu().numpy()
            assert np.isfinite(got).all(), name
            assert not got[~real].any(), f"{name}: padding rows"
            ratio = (np.abs(OP.unpermute(self.geom, got) - want) / (bound + 1e-30)).max()
            worst[name] = max(worst.get(name, 0.0), ratio)

        for b in range(self.batch):
            for h in range(self.heads):
                q, k, v, do = (x[b, h].double().numpy() for x in (self.q, self.k, self.v, self.do))
                at = lambda x: None if x is None else x[b].astype(np.int64)
                pos = at(self.positions)
                seen = OS.visible(self.keep[h], pos, at(self.limits), at(self.documents))
                slope = None if self.slopes is None else float(self.slopes[h])
                rule = dict(cap=self.cap, slope=slope, positions=pos)
                want, want_lse, p = OS.forward(q, k, v, seen, self.scale, **rule)
                wdq, wdk, wdv, ds, _ = OS.backward(do, q, k, v, seen, self.scale, **rule)
                there = np.isfinite(want_lse)
                s, _ = OS.scores(q, k, self.scale, **rule)
                raw = (np.abs(q) @ np.abs(k).T) * self.scale
                far = np.abs(slope) * np.abs(pos[:, None] - pos[None, :]) if slope is not None else 0.0
                span = np.abs(s) + np.abs(np.where(there, want_lse, 0.0))[:, None]
                delta = np.where(seen, (self.D + 2) * U * raw + 8 * U * self.cap + 4 * U * far + 4 * U * span + 4 * U, 0.0).max()
                pv = p @ np.abs(v)
                out_bound = HALF * (pv + np.abs(want)) * (1 + HALF) + 2 * delta * pv
                close("out", out[b, h], want, out_bound)
                got_lse = lse[b, h].double().cpu().numpy()
                assert (got_lse[~real] == -math.inf).all()
                got_lse = OP.unpermute(self.geom, got_lse[:, None])[:, 0]
                assert np.array_equal(np.isfinite(got_lse), there) and (got_lse[~there] == -math.inf).all()
                if there.any():
                    worst["lse"] = max(worst.get("lse", 0.0), (np.abs(got_lse - want_lse)[there] / (delta + 8 * U * (1 + np.abs(want_lse[there])))).max())
                close("dv", dv[b, h], wdv, HALF * (p.T @ np.abs(do) + np.abs(wdv)) * (1 + HALF) + 2 * delta * (p.T @ np.abs(do)))
                dp = do @ v.T
                row = (do * want).sum(1, keepdims=True)
                ds_bound = HALF * np.abs(ds) + (2 * delta + HALF * delta) * np.abs(ds) + 16 * U * p * np.abs(dp - row)
                ds_bound += p * ((self.D + 2) * U * (np.abs(do) @ np.abs(v).T) + (np.abs(do) * out_bound).sum(1, keepdims=True))
                close("dq", dq[b, h], wdq, self.scale * ds_bound @ np.abs(k) + HALF * (np.abs(wdq) + self.scale * ds_bound @ np.abs(k)))
                close("dk", dk[b, h], wdk, self.scale * ds_bound.T @ np.abs(q) + HALF * (np.abs(wdk) + self.scale * ds_bound.T @ np.abs(q)))
        print({n: round(float(r), 3) for n, r in worst.items()}, flush=True)
        assert all(r <= 1 for r in worst.values()), worst


SHAPES = [((3, 13, 20), (1, 8, 8), 64, 64), ((3, 9, 17), (1, 8, 8), 64, 128), ((5, 13, 12), (2, 8, 8), 128, 64), ((3, 13, 20), (2, 8, 8), 128, 128)]
RULES = {"plain": dict(), "cap": dict(cap=2.0, gain=4.0), "bias": dict(bias=True), "causal": dict(prefix=0), "prefix": dict(prefix=2), "clips": dict(docs="frames"),
         "all": dict(cap=5.0, gain=3.0, bias=True, prefix="random", docs="random", batch=2), "nothing there": dict(docs="none there"),
         "random lists": dict(lists=0.4, docs="frames", prefix=1, heads=3), "random lists, plain": dict(lists=0.4, heads=3, batch=2, scale=0.2)}


@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"B{math.prod(s[1])}-D{s[3]}")
@pytest.mark.parametrize("rule", RULES)
def test_forward_and_gradients(shape, rule):
    print("scored", shape, rule, flush=True)
    pb = Problem(*shape, seed=5, **RULES[rule])
    results = pb.run()
    again = pb.run()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(results, again))
    pb.check(*results)


@pytest.mark.gpu
@pytest.mark.parametrize("grid,tile,n_text,D", [((1, 1, 1), (1, 8, 8), 0, 64), ((1, 1, 1), (2, 8, 8), 0, 128), ((1, 1, 3), (4, 4, 8), 128, 64), ((7, 1, 1), (1, 8, 8), 0, 128),
                                                ((2, 3, 5), (1, 8, 16), 0, 128)], ids=str)
@pytest.mark.parametrize("rule", ["plain", "all"])
def test_few_tokens(grid, tile, n_text, D, rule):
    print("scored", grid, tile, rule, flush=True)
    pb = Problem(grid, tile, n_text, D, seed=6, **RULES[rule])
    pb.check(*pb.run())

@pytest.mark.gpu
def test_peaked_and_flat_rows():
    """Scores that a cap bends hard, and rows whose weight lies on one key."""
    for kw in (dict(cap=1.0, gain=30.0), dict(cap=50.0, gain=20.0), dict(gain=20.0), dict(cap=0.5, gain=0.0), dict(cap=2.0 ** -16, gain=1.0), dict(cap=4096.0, gain=2.0)):
        print("scored", kw, flush=True)
        pb = Problem((2, 9, 17), (1, 8, 8), 0, 64, seed=7, **kw)
        pb.check(*pb.run())


@pytest.mark.gpu
@pytest.mark.parametrize("cap", [34.0, 60.0])
@pytest.mark.parametrize("D", [64, 128])
def test_all_scores_at_an_end_of_the_cap(cap, D):
    """Rows whose scores are all near minus the cap, all near the cap, and half each: weights as small as exp(-2 cap)."""
    pb = Problem((2, 9, 17), (1, 8, 8), 64, D, seed=13, cap=cap, docs="frames")
    pb.q[:, :, 0::3], pb.q[:, :, 1::3] = 8.0, -8.0
    pb.k[:], pb.k[:, :, 5::7] = -8.0, 8.0
    pb.check(*pb.run())


@pytest.mark.gpu
def test_lowest_and_highest_limits_and_far_positions():
    pb = Problem((3, 9, 17), (1, 8, 8), 64, 64, seed=8, prefix="random", bias=True)
    pb.positions[:] = pb.rng.integers(-2 ** 24, 2 ** 24, pb.positions.shape)
    pb.slopes[:] = 1e-7
    pb.limits[:, 0::3], pb.limits[:, 1::3] = 2 ** 31 - 1, -2 ** 31
    pb.limits[:, 2::3] = pb.positions[:, 2::3]
    pb.check(*pb.run())


@pytest.mark.gpu
def test_agrees_with_the_sparse_forward():
    """Without arrays and cap it is compact_attn_forward: both are within the bound of the oracle."""
    pb = Problem(*SHAPES[3], seed=9)
    out, lse, *grads = pb.run()
    other = ca.compact_attn_forward(*pb.args, pb.layout)
    pb.check(other, lse, *grads)


@pytest.mark.gpu
def test_lists_longer_than_a_cut():
    """More than 512 key tiles a row, and (transposed) query tiles a column."""
    grid, tile, D = (9, 61, 64), (1, 8, 8), 64
    n = 9 * 8 * 8
    lay = _layout(*grid, tile, 0, 1, [[(8, (7, 7), ABSENT)]], D)
    assert lay.n_tiles == n > 512
    gen = torch.Generator(device=DEV)
    gen.manual_seed(3)
    q, k, v, do = (torch.randn(1, 1, lay.n_tokens_real, D, generator=gen, device=DEV).to(torch.bfloat16) for _ in range(4))
    frames = (torch.arange(lay.n_tokens_real, device=DEV) // (61 * 64)).to(torch.int32)[None]
    for how in (dict(), dict(positions=frames, limits=frames.clamp(min=3), documents=torch.zeros_like(frames))):
        tiled = [ca.compact_attn_permute(x, lay) for x in (q, k, v, do)]
        out, lse = ca.compact_attn_forward_scored(*tiled[:3], lay, **how)
        grads = ca.compact_attn_backward_scored(tiled[3], *tiled[:3], out, lse, lay, **how)
        got = [ca.compact_attn_permute(x, lay, inverse=True)[0, 0].double() for x in (out, *grads)]
        qd, kd, vd, dod = (x[0, 0].double() for x in (q, k, v, do))
        want = [torch.zeros_like(qd) for _ in range(4)]
        for lo in range(0, lay.n_tokens_real, 4096):
            at = slice(lo, lo + 4096)
            s = qd[at] @ kd.t() / 8
            if how:
                s = s.masked_fill(frames[0][None, :] > how["limits"][0][at, None], -math.inf)
            p = torch.softmax(s, dim=1)
            want[0][at] = p @ vd
            dp = dod[at] @ vd.t()
            ds = p * (dp - (p * dp).sum(1, keepdim=True)) / 8
            want[1][at] = ds @ kd
            want[2] += ds.t() @ qd[at]
            want[3] += p.t() @ dod[at]
        # 35136 weights, each rounded with an independent error of at most 2^-8 (rms 2^-9 / sqrt 3 ... 2^-8 / sqrt 3), and a rounded result: relative error in norm
        # below 2 * 2^-8 / sqrt 3 < 5e-3; twice that where dS is rounded and its row sum comes from a rounded result
        for name, a, b, most in zip(("out", "dq", "dk", "dv"), got, want, (5e-3, 1e-2, 1e-2, 5e-3)):
            off = float((a - b).norm() / b.norm())
            print(name, off, flush=True)
            assert off <= most, (name, off)


@pytest.mark.gpu
def test_planes_past_4_gib():
    """Offsets past 32 bits: the last of 40 heads, 5 GiB into every tensor, gives what it gives alone."""
    grid, tile, heads, D = (64, 64, 128), (1, 8, 8), 40, 128
    group = [(0, (0, 0), ABSENT)]
    many, one = (_layout(*grid, tile, 0, 1, [group] * n, D) for n in (heads, 1))
    N = many.shape(True)[2]
    assert (heads - 1) * N * D * 2 > 2 ** 32
    gen = torch.Generator(device=DEV)
    gen.manual_seed(4)
    last = [torch.randn(1, 1, N, D, generator=gen, device=DEV).to(torch.bfloat16) for _ in range(4)]
    wide = []
    for x in last:
        t = torch.zeros(1, heads, N, D, dtype=torch.bfloat16, device=DEV)
        t[:, -1:] = x
        wide.append(t)
    documents = (torch.arange(N, device=DEV) // 96 % 5).to(torch.int32)[None]
    for how in (dict(), dict(cap=20.0, documents=documents)):
        results = []
        for lay, (q, k, v, do) in ((many, wide), (one, last)):
            out, lse = ca.compact_attn_forward_scored(q, k, v, lay, **how)
            results.append((out, lse, *ca.compact_attn_backward_scored(do, q, k, v, out, lse, lay, **how)))
        for a, b in zip(*results):
            assert torch.equal(a[:, -1:], b) and bool(torch.isfinite(a[:, -1]).any())
        del results


@pytest.mark.gpu
def test_side_stream_and_graph():
    """A stream of its own and a captured training step; replays read the arrays that lie there then."""
    pb = Problem(*SHAPES[2], seed=10, **RULES["all"])
    want = pb.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = pb.run(stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    q, k, v = pb.args
    how = pb.given

    def step():
        out, lse = ca.compact_attn_forward_scored(q, k, v, pb.layout, **how)
        return out, lse, *ca.compact_attn_backward_scored(pb.dout, q, k, v, out, lse, pb.layout, **how)

    graphs = []
    for _ in range(2):   # two graphs of the same layout: each has a workspace of its own
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            captured = step()
        graphs.append((graph, captured))
    for replay in range(3):
        q.mul_(-0.5 if replay % 2 else -2)
        how["documents"].copy_(how["documents"].flip(1))
        want = step()
        for graph, captured in graphs:
            for t in captured:
                t.zero_()
            graph.replay()
        torch.cuda.synchronize()
        for _, captured in graphs:
            assert all(torch.equal(a, b) for a, b in zip(want, captured)), replay


@pytest.mark.gpu
def test_backward_lists_must_be_on_the_device_before_a_capture():
    pb = Problem(*SHAPES[0], seed=11)
    q, k, v = (pb.tiled(x) for x in (pb.q, pb.k, pb.v))
    dout = pb.tiled(pb.do)
    out, lse = ca.compact_attn_forward_scored(q, k, v, pb.layout)
    grads = [torch.zeros_like(q) for _ in range(3)]
    graph, refused = torch.cuda.CUDAGraph(), None
    with torch.cuda.graph(graph):
        out.add_(0)
        try:
            ca.compact_attn_backward_scored(dout, q, k, v, out, lse, pb.layout, grads=grads)
        except ca.CompactAttnError as e:
            refused = e
    assert refused is not None and refused.status == -1 and "upload_scored" in str(refused)
    ca.compact_attn_layout_upload_scored(pb.layout)
    with torch.cuda.graph(torch.cuda.CUDAGraph()):
        ca.compact_attn_backward_scored(dout, q, k, v, out, lse, pb.layout, grads=grads)


@pytest.mark.gpu
def test_binding_refusals():
    pb = Problem(*SHAPES[0], seed=12)
    q, k, v = (pb.tiled(x) for x in (pb.q, pb.k, pb.v))
    tokens = torch.zeros(1, pb.geom.N_real, dtype=torch.int32, device=DEV)
    run = lambda *t, **kw: ca.compact_attn_forward_scored(*(t or (q, k, v)), pb.layout, **kw)
    for bad in (lambda: run(q.cpu(), k, v), lambda: run(q.float(), k, v), lambda: run(q[:, :, :-1], k, v), lambda: run(documents=tokens[0]), lambda: run(documents=tokens.long()),
                lambda: run(positions=tokens, slopes=torch.zeros(3, device=DEV)), lambda: run(documents=tokens.cpu()), lambda: run(out=(q, k)),
                lambda: ca.compact_attn_backward_scored(q, q, k, v, q, q, pb.layout)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: run(limits=tokens), lambda: run(slopes=torch.zeros(2, device=DEV)), lambda: run(cap=-1.0),
                lambda: run(out=(q, torch.empty(q.shape[:3], device=DEV)))):
        with pytest.raises(ca.CompactAttnError):
            bad()
