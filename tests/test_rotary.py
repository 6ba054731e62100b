"""Rotary positions and norms of queries and keys with the rotation: the table, the refusals and the oracle's gradient on the
CPU, the kernels against the oracle on the GPU.

Tolerances.  A result is rounded once: half a step of its type, `finfo.eps / 2` relative.  Before that, in fp32: sine and cosine are rounded to
2^-24, the two products and their sum to 2^-24 each, so a rotation is off by at most 4 * 2^-24 of |c x| + |s x'|; a norm's sum of D <= 512 squares is added up
in at most 8 + 6 steps, its root and the products with the weight add 6 more: 32 * 2^-24 covers all of it.  Weight gradients are sums over
tokens whose longest chain of additions in these tests is below 400: 400 * 2^-24 of the sum of magnitudes."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2508_12969_amd as ca
from oracle import permute as OP
from oracle import rotary as OR
from oracle.geometry import Geometry
from paper_2508_12969_amd import rotary as R

DEV = "cuda:0"
ABSENT = (-1, -1)
U32 = 2.0 ** -24
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}


def _layout(T, H, W, tile, n_text, batch, heads, D, dtype):
    return ca.compact_attn_build_layout(T, H, W, tile, n_text, batch, heads, D, dtype, [[(0, (0, 0), ABSENT)]] * heads)


# ---------------------------------------------------------------- table (host)

@pytest.mark.parametrize("method,stretch", [("linear", 1.0), ("linear", 4.0), ("base", 4.0), ("bands", 4.0)])
def test_table_holds_the_angles(method, stretch):
    channels, lengths, base = (16, 24, 2), (70000, 33, 5), (10000.0, 500.0, 10000.0)
    rotary = ca.compact_attn_build_rotary(channels, lengths, base=base, method=method, stretch=stretch, trained=(4096.0, 8.0, 5.0), turns=(1.0, 4.0), magnitude=1.25)
    for axis in range(3):
        f = OR.frequencies(channels[axis], base[axis], stretch, method, (4096.0, 8.0, 5.0)[axis], (1.0, 4.0))
        angle = np.arange(lengths[axis])[:, None] * f
        got = ca.compact_attn_rotary_angles(rotary, axis)
        want = 1.25 * np.stack([np.cos(angle), np.sin(angle)], axis=-1)
        # the frequency itself is exact to a few 2^-53, which a position of 70000 makes 2^-53 * 70000 * 8 < 1e-10 of the angle
        assert np.abs(got - want).max() <= 1.25 * U32 + 1e-10


def test_table_axis_without_channels():
    rotary = ca.compact_attn_build_rotary((0, 8, 0), (7, 5, 7))
    assert ca.compact_attn_rotary_angles(rotary, 0) is None
    assert ca.compact_attn_rotary_angles(rotary, 1).shape == (5, 4, 2)
    rotary.free()
    rotary.free()


@pytest.mark.parametrize("kwargs", [
    dict(channels=(3, 0, 0), lengths=(4, 4, 4)), dict(channels=(-2, 4, 0), lengths=(4, 4, 4)), dict(channels=(0, 0, 0), lengths=(4, 4, 4)),
    dict(channels=(4, 4, 4), lengths=(4, 0, 4)), dict(channels=(4, 4, 4), lengths=(4, 4, 4), base=0.0), dict(channels=(4, 4, 4), lengths=(4, 4, 4), stretch=-1.0),
    dict(channels=(4, 4, 4), lengths=(4, 4, 4), base=float("inf")), dict(channels=(4, 4, 4), lengths=(4, 4, 4), method="bands"),
    dict(channels=(4, 4, 4), lengths=(4, 4, 4), method="bands", trained=4.0, turns=(2.0, 2.0)), dict(channels=(4, 4, 4), lengths=(4, 4, 4), magnitude=float("nan")),
    dict(channels=(1024, 0, 0), lengths=(1 << 30, 1, 1)),
])
def test_malformed_tables_are_refused(kwargs):
    with pytest.raises(ca.CompactAttnError) as e:
        ca.compact_attn_build_rotary(**kwargs)
    assert e.value.status == -1


def test_unknown_names_are_refused():
    with pytest.raises(ValueError):
        ca.compact_attn_build_rotary((4, 4, 4), (4, 4, 4), pairing="both")
    with pytest.raises(ValueError):
        ca.compact_attn_build_rotary((4, 4, 4), (4, 4, 4), method="none")
    with pytest.raises(ValueError):
        ca.compact_attn_build_rotary((4, 4), (4, 4, 4))


# ---------------------------------------------------------------- refusals of the C entry points (no tensor is touched)

P = [0x100000000 * (i + 1) for i in range(12)]   # addresses that are never read


def _status(call):
    lib = ca.load_library()
    return call(lib), lib.compact_attn_last_error().decode()


def test_rotate_refusals():
    lay = _layout(4, 8, 8, (1, 4, 4), 16, 1, 2, 64, "f32")
    rotary = ca.compact_attn_build_rotary((8, 28, 28), (4, 8, 8))
    wide = ca.compact_attn_build_rotary((8, 32, 32), (4, 8, 8))
    dense = R.ca_strides(2 * 272 * 64, 64, 128)

    def call(src=P[0], ss=None, dst=P[1], ds=None, table=rotary, where=None, tiled=1, transpose=0):
        return _status(lambda lib: lib.compact_attn_rotate(src, ss, dst, ds, lay.handle, table.handle if table else None, where, tiled, transpose, None))

    where = R.ca_where((ctypes.c_int32 * 3)(0, 0, 0), None)
    late = R.ca_where((ctypes.c_int32 * 3)(1, 0, 0), None)
    odd = R.ca_where((ctypes.c_int32 * 3)(0, 0, 0), P[3] + 2)
    for bad, text in ((dict(src=None), "null"), (dict(dst=None), "null"), (dict(table=None), "null"), (dict(src=P[0] + 4), "aligned"), (dict(dst=P[1] + 8), "aligned"),
                      (dict(tiled=2), "tiled"), (dict(transpose=2), "transpose"), (dict(ds=dense), "tile order"), (dict(ss=dense, transpose=1), "tile order"),
                      (dict(ss=R.ca_strides(0, 64, 6)), "16 bytes"), (dict(ss=R.ca_strides(0, -64, 64)), "negative"), (dict(dst=P[0] + 64), "overlap"),
                      (dict(ds=R.ca_strides(0, 64, 64), tiled=0), "share memory"), (dict(table=wide), "more rotated channels"), (dict(where=late), "outside"),
                      (dict(where=odd), "4-byte")):
        st, message = call(**bad)
        assert st == -1 and text in message, (bad, st, message)
    st, message = call(where=where)   # nothing to refuse: the next thing asked for is a device
    assert st == -4 or torch.cuda.is_available(), (st, message)


@pytest.mark.parametrize("dtype,D", [("bf16", 520), ("f32", 260)])
def test_head_dim_beyond_the_kernels_is_refused(dtype, D):
    lay = _layout(2, 4, 4, (1, 4, 4), 0, 1, 1, D, dtype)
    rotary = ca.compact_attn_build_rotary((8, 8, 8), (2, 4, 4))
    st, message = _status(lambda lib: lib.compact_attn_rotate(P[0], None, P[1], None, lay.handle, rotary.handle, None, 1, 0, None))
    assert st == -2 and str(D) in message
    need = ctypes.c_int64()
    assert _status(lambda lib: lib.compact_attn_norm_workspace(lay.handle, need))[0] == -2


def test_norm_refusals():
    lay = _layout(4, 8, 8, (1, 4, 4), 16, 1, 2, 64, "f32")
    need = ctypes.c_int64()
    assert _status(lambda lib: lib.compact_attn_norm_workspace(lay.handle, need))[0] == 0 and need.value > 0

    def norm(q=P[0], k=P[1], qs=None, ks=None, wq=P[2], wk=P[3], eps=1e-6, tiled=1):
        return R.ca_norm(q, k, None if qs is None else ctypes.pointer(qs), None if ks is None else ctypes.pointer(ks), wq, wk, None, None, eps, tiled)

    def forward(q_out=P[4], k_out=P[5], **kw):
        return _status(lambda lib: lib.compact_attn_norm_rotate(norm(**kw), q_out, k_out, lay.handle, None))

    def backward(dqo=P[4], dko=P[5], dq=P[6], dqs=None, dk=P[7], dks=None, dwq=P[8], dwk=P[9], ws=P[10], size=need.value, **kw):
        return _status(lambda lib: lib.compact_attn_norm_rotate_backward(norm(**kw), dqo, dko, dq, dqs, dk, dks, dwq, dwk, lay.handle, ws, size, None))

    nan = float("nan")
    for bad in (dict(q=None), dict(k=None), dict(q_out=None), dict(q=P[0] + 8), dict(wq=P[2] + 4), dict(q_out=P[4] + 8), dict(eps=-1.0), dict(eps=nan), dict(eps=float("inf")),
                dict(tiled=3), dict(qs=R.ca_strides(0, 0, 2)), dict(q_out=P[0]), dict(k_out=P[0] + 64), dict(k_out=P[4] + 1024)):
        st, message = forward(**bad)
        assert st == -1 and message, (bad, st, message)
    for bad in (dict(q=None), dict(dqo=None), dict(dk=None), dict(dq=P[6] + 8), dict(dwq=None), dict(ws=None), dict(ws=P[10] + 8), dict(size=need.value - 1), dict(dk=P[6]),
                dict(dq=P[4]), dict(dq=P[0] + 16), dict(dqs=R.ca_strides(64, 64, 64)), dict(dks=R.ca_strides(0, 64, 4)), dict(dwk=P[8]), dict(dwq=P[10] + 16), dict(ws=P[7]),
                dict(dwq=P[8] + 2)):
        st, message = backward(**bad)
        assert st == -1 and message, (bad, st, message)


def test_strides_and_overlaps_beyond_the_tensors_are_refused():
    lay = _layout(4, 8, 8, (1, 4, 4), 16, 1, 2, 64, "f32")
    tokens = lay.n_tokens_real
    rotary = ca.compact_attn_build_rotary((8, 28, 28), (4, 8, 8))
    rotate = lambda ss=None, where=None: _status(lambda lib: lib.compact_attn_rotate(P[0], ss, P[1], None, lay.handle, rotary.handle, where, 1, 0, None))
    st, message = rotate(R.ca_strides(0, 64, (1 << 40) // (tokens - 1) // 4 * 4 + 4))
    assert st == -1 and "2^40" in message
    st, message = rotate(R.ca_strides(0, (1 << 62), 64))
    assert st == -1 and "2^40" in message
    st, message = rotate(where=R.ca_where((ctypes.c_int32 * 3)(0, 0, 0), P[1] + 64))
    assert st == -1 and "positions" in message
    norm = R.ca_norm(P[0], P[1], None, None, P[2], P[3], rotary.handle, ctypes.pointer(R.ca_where((ctypes.c_int32 * 3)(0, 0, 0), P[4])), 1e-6, 1)
    for outs in ((P[2], P[5]), (P[5], P[3] + 16), (P[4], P[5])):
        st, message = _status(lambda lib: lib.compact_attn_norm_rotate(norm, *outs, lay.handle, None))
        assert st == -1 and "overlap" in message, outs
    for dq, dwq in ((P[2], P[9]), (P[7], P[3]), (P[7], P[4] + 64)):
        st, message = _status(lambda lib: lib.compact_attn_norm_rotate_backward(norm, P[5], P[6], dq, None, P[8], None, dwq, P[10], lay.handle, P[11], 1 << 30, None))
        assert st == -1 and "overlap" in message, (dq, dwq)


def test_freed_tables_and_short_origins_are_refused():
    lay = _layout(4, 8, 8, (1, 4, 4), 16, 1, 2, 64, "f32")
    rotary = ca.compact_attn_build_rotary((8, 28, 28), (4, 8, 8))
    with pytest.raises(ValueError):
        R._where(lay, (1, 2), None)
    assert R._where(lay, [0, 0, 0], None) is None and R._table(None) is None and R._table(rotary) is rotary.handle
    rotary.free()
    with pytest.raises(ValueError):   # not a call without a rotation
        R._table(rotary)


# ---------------------------------------------------------------- the oracle's gradient, from differences

@pytest.mark.parametrize("pairing", ["half", "interleaved"])
def test_oracle_gradient_from_differences(pairing):
    rng = np.random.default_rng(3)
    x, w, dy = rng.normal(size=(5, 12)), 1 + 0.2 * rng.normal(size=12), rng.normal(size=(5, 12))
    angle = rng.normal(size=(5, 4))
    f = lambda x, w: (OR.rotate(OR.norm(x, w, 1e-3), angle, pairing, 1.1) * dy).sum()
    dx, dw = OR.norm_gradient(x, w, 1e-3, OR.rotate(dy, angle, pairing, 1.1, transpose=True))
    h = 1e-6
    for i in range(5):
        for j in range(12):
            e = np.zeros_like(x)
            e[i, j] = h
            assert abs((f(x + e, w) - f(x - e, w)) / (2 * h) - dx[i, j]) < 1e-7
    for j in range(12):
        e = np.zeros_like(w)
        e[j] = h
        assert abs((f(x, w + e) - f(x, w - e)) / (2 * h) - dw[j]) < 1e-7


# ---------------------------------------------------------------- kernels

# grid, tile, text, batch, heads, D, dtype, channels per axis, pairing
CASES = [
    ((1, 1, 1), (1, 4, 4), 0, 1, 1, 64, "bf16", (8, 28, 28), "interleaved"),       # a single token
    ((4, 8, 8), (1, 4, 4), 0, 1, 2, 64, "f32", (8, 28, 28), "half"),
    ((5, 13, 20), (2, 8, 8), 128, 2, 3, 128, "bf16", (16, 56, 56), "interleaved"),  # padded on two faces, text, batch
    ((3, 7, 11), (3, 5, 7), 105, 1, 5, 80, "bf16", (4, 18, 18), "half"),            # halves of 20 channels: not a whole number of chunks
    ((3, 7, 11), (2, 4, 8), 64, 2, 1, 80, "f32", (6, 20, 10), "half"),              # halves of 18 channels in chunks of 4
    ((2, 5, 9), (1, 6, 10), 60, 1, 9, 72, "bf16", (0, 10, 0), "half"),              # one axis, halves of 5 channels
    ((2, 5, 9), (1, 6, 10), 0, 1, 2, 36, "f32", (2, 6, 4), "interleaved"),          # 9 chunks of 4
    ((7, 1, 1), (4, 1, 1), 4, 2, 17, 8, "bf16", (8, 0, 0), "interleaved"),          # one chunk a row, a line of tokens
    ((2, 3, 5), (1, 2, 2), 4, 1, 2, 512, "bf16", (64, 192, 256), "half"),           # a wave for a row
    ((2, 3, 5), (1, 2, 2), 0, 1, 2, 256, "f32", (64, 64, 64), "interleaved"),
]


def _id(case):
    return f"{'x'.join(map(str, case[0]))}-D{case[5]}-{case[6]}-{case[8]}"


class Problem:
    def __init__(self, case, seed=0, token_major=False, explicit=False, magnitude=1.0):
        (T, H, W), tile, n_text, self.batch, self.heads, self.D, self.dtype, channels, self.pairing = case
        self.geom = Geometry(T, H, W, *tile, n_text)
        self.layout = _layout(T, H, W, tile, n_text, self.batch, self.heads, self.D, self.dtype)
        self.lengths = (T + 3, H + 2, W + 1)
        self.magnitude = magnitude
        self.rotary = ca.compact_attn_build_rotary(channels, self.lengths, pairing=self.pairing, stretch=2.0, magnitude=magnitude)
        self.freqs = [OR.frequencies(c, stretch=2.0) for c in channels]
        self.rng = np.random.default_rng(seed)
        self.token_major = token_major
        self.origin = (3, 1, 0)
        self.positions = None
        if explicit:
            at = np.stack([self.rng.integers(-1, n, size=(self.batch, self.geom.N_real)) for n in self.lengths], axis=-1)
            self.positions = torch.from_numpy(at.astype(np.int32)).to(DEV)
        self.how = dict(positions=self.positions) if explicit else dict(origin=self.origin)

    def tensor(self, token_major=None):
        shape = (self.batch, self.heads, self.geom.N_real, self.D)
        x = torch.from_numpy(self.rng.normal(size=shape).astype(np.float32)).to(TORCH[self.dtype])
        if self.token_major if token_major is None else token_major:
            return x.transpose(1, 2).contiguous().to(DEV).transpose(1, 2)
        return x.to(DEV)

    def weight(self):
        return torch.from_numpy((1 + 0.3 * self.rng.normal(size=self.D)).astype(np.float32)).to(TORCH[self.dtype]).to(DEV)

    def turn(self, x, b, transpose=False):
        at = OR.grid_positions(self.geom, self.origin) if self.positions is None else self.positions[b].cpu().numpy()
        angle = OR.angles(at, self.freqs)
        turned = np.concatenate([np.repeat(at[:, i:i + 1] >= 0, len(f), axis=1) for i, f in enumerate(self.freqs)], axis=1)
        return OR.rotate(x, angle, self.pairing, np.where(turned, self.magnitude, 1.0), transpose)

    def scale(self, x):
        """|c x| + |s x'| per element is at most this."""
        half = self.rotated // 2
        part = np.abs(x)
        out = part.copy()
        if self.pairing == "half":
            out[:, :half] += part[:, half:2 * half]
            out[:, half:2 * half] += part[:, :half]
        else:
            out[:, 0:2 * half:2] += part[:, 1:2 * half:2]
            out[:, 1:2 * half:2] += part[:, 0:2 * half:2]
        return out * max(1.0, self.magnitude)

    @property
    def rotated(self):
        return 2 * sum(len(f) for f in self.freqs)


def f64(t):
    return t.detach().cpu().double().numpy()


def check(got, want, slack, dtype, what):
    """Off by at most half a step of its type, and slack before the rounding."""
    err, bound = np.abs(got - want), HALF_STEP[dtype] * (np.abs(want) + slack) + slack + (1e-40 if dtype == "f32" else 1e-38)
    assert np.isfinite(got).all(), what
    assert (err <= bound).all(), f"{what}: {(err / bound).max():.2f} times the bound"


@pytest.mark.gpu
@pytest.mark.parametrize("case", CASES, ids=_id)
@pytest.mark.parametrize("tiled,token_major,explicit", [(True, False, False), (False, True, False), (True, True, True), (False, False, True)])
def test_rotate_and_transpose(case, tiled, token_major, explicit):
    print("rotate", _id(case), tiled, token_major, explicit, flush=True)
    pb = Problem(case, 1, token_major, explicit, magnitude=1.25)
    x = pb.tensor()
    y = ca.compact_attn_rotate(x, pb.layout, pb.rotary, tiled=tiled, **pb.how)
    g = pb.tensor(False)
    g_in = ca.compact_attn_permute(g, pb.layout) if tiled else g
    back = ca.compact_attn_rotate(g_in, pb.layout, pb.rotary, tiled=tiled, transpose=True, **pb.how)
    # into memory with strides of its own
    wide = torch.full((pb.batch, pb.geom.N_real, 2, pb.heads, pb.D), 7.0, dtype=x.dtype, device=DEV)
    spread = wide[:, :, 1].transpose(1, 2)
    ca.compact_attn_rotate(g_in, pb.layout, pb.rotary, tiled=tiled, transpose=True, out=spread, **pb.how)
    torch.cuda.synchronize()
    assert torch.equal(spread, back) and bool((wide[:, :, 0] == 7.0).all())
    assert y.shape == pb.layout.shape(tiled) and back.shape == x.shape
    for b in range(pb.batch):
        for h in range(pb.heads):
            xs, gs = f64(x[b, h]), f64(g[b, h])
            got = f64(y[b, h])
            if tiled:
                assert not got[~OP.slot_valid(pb.geom)].any()
                got = OP.unpermute(pb.geom, got)
            check(got, pb.turn(xs, b), 4 * U32 * pb.scale(xs), pb.dtype, "rotated")
            check(f64(back[b, h]), pb.turn(gs, b, True), 4 * U32 * pb.scale(gs), pb.dtype, "turned back")


@pytest.mark.gpu
@pytest.mark.parametrize("case", CASES, ids=_id)
@pytest.mark.parametrize("tiled,token_major,explicit", [(True, False, False), (False, True, True), (True, True, False)])
def test_norm_rotate_and_gradients(case, tiled, token_major, explicit):
    print("norm", _id(case), tiled, token_major, explicit, flush=True)
    pb = Problem(case, 2, token_major, explicit)
    eps = 1e-3
    q, k, wq, wk = pb.tensor(), 0.01 * pb.tensor(), pb.weight(), pb.weight()
    args = (q, k, wq, wk, pb.layout, pb.rotary, eps)
    outs = ca.compact_attn_norm_rotate(*args, tiled=tiled, **pb.how)
    grads = [pb.tensor(False) for _ in range(2)]
    dys = [ca.compact_attn_permute(g, pb.layout) if tiled else g for g in grads]
    *dxs, dwq, dwk = ca.compact_attn_norm_rotate_backward(*dys, *args, tiled=tiled, **pb.how)
    again = ca.compact_attn_norm_rotate_backward(*dys, *args, tiled=tiled, **pb.how)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((*dxs, dwq, dwk), again))
    for x, w, y, g, dx, dw in ((q, wq, outs[0], grads[0], dxs[0], dwq), (k, wk, outs[1], grads[1], dxs[1], dwk)):
        assert dx.stride() == x.stride() or 1 in x.shape
        w64, sum_dw, sum_abs = f64(w), np.zeros(pb.D), np.zeros(pb.D)
        for b in range(pb.batch):
            for h in range(pb.heads):
                xs, gs = f64(x[b, h]), f64(g[b, h])
                n = OR.norm(xs, w64, eps)
                got = f64(y[b, h])
                if tiled:
                    assert not got[~OP.slot_valid(pb.geom)].any()
                    got = OP.unpermute(pb.geom, got)
                check(got, pb.turn(n, b), 32 * U32 * pb.scale(n), pb.dtype, "normed")
                du = pb.turn(gs, b, True)
                dx64, dw64 = OR.norm_gradient(xs, w64, eps, du)
                r = 1 / np.sqrt((xs * xs).mean(axis=1, keepdims=True) + eps)
                lean = np.abs(xs) * r ** 3 * (pb.scale(gs) * np.abs(w64) * np.abs(xs)).mean(axis=1, keepdims=True)
                check(f64(dx[b, h]), dx64, 48 * U32 * (r * pb.scale(gs) * np.abs(w64) + lean), pb.dtype, "gradient")
                sum_dw += dw64
                sum_abs += (pb.scale(gs) * np.abs(xs) * r).sum(axis=0)
        assert (np.abs(f64(dw) - sum_dw) <= 400 * U32 * sum_abs + 1e-30).all()


@pytest.mark.gpu
def test_norm_without_weights_or_rotation():
    pb = Problem(CASES[2], 4)
    q, k = pb.tensor(), pb.tensor()
    outs = ca.compact_attn_norm_rotate(q, k, None, None, pb.layout, None, 0.0, tiled=False)
    dq, dk, dwq, dwk = ca.compact_attn_norm_rotate_backward(k, q, q, k, None, None, pb.layout, None, 0.0, tiled=False)
    wq = pb.weight()
    only = ca.compact_attn_norm_rotate_backward(k, q, q, k, wq, None, pb.layout, None, 0.0, tiled=False)
    torch.cuda.synchronize()
    assert dwq is None and dwk is None and only[2] is not None and only[3] is None
    assert torch.equal(only[1], dk)
    for x, y in ((q, outs[0]), (k, outs[1])):
        want = OR.norm(f64(x).reshape(-1, pb.D), 1.0, 0.0)
        check(f64(y).reshape(-1, pb.D), want, 32 * U32 * np.abs(want), "bf16", "normed")


@pytest.mark.gpu
def test_unrotated_positions_are_the_permutation_bit_for_bit():
    pb = Problem(CASES[2], 5, magnitude=3.0)
    x = pb.tensor()
    nowhere = torch.full((pb.batch, pb.geom.N_real, 3), -1, dtype=torch.int32, device=DEV)
    got = ca.compact_attn_rotate(x, pb.layout, pb.rotary, positions=nowhere)
    assert torch.equal(got, ca.compact_attn_permute(x, pb.layout))


@pytest.mark.gpu
def test_positions_past_the_table_are_nan_and_nothing_else():
    pb = Problem(CASES[3], 6)
    x = pb.tensor()
    at = torch.zeros((pb.batch, pb.geom.N_real, 3), dtype=torch.int32, device=DEV)
    want = ca.compact_attn_rotate(x, pb.layout, pb.rotary, positions=at, tiled=False)
    at[0, 5, 1] = pb.lengths[1]
    at[0, 7, 0] = 2 ** 31 - 1
    got = ca.compact_attn_rotate(x, pb.layout, pb.rotary, positions=at, tiled=False)
    torch.cuda.synchronize()
    nan = torch.isnan(got)
    assert not torch.isnan(want).any() and torch.equal(got[~nan], want[~nan])
    channel = torch.arange(pb.D, device=DEV)
    pair = torch.where(channel < 40, channel % 20, torch.full_like(channel, -1))
    expected = torch.zeros_like(nan)
    expected[0, :, 5] = (pair >= 2) & (pair < 11)
    expected[0, :, 7] = (pair >= 0) & (pair < 2)
    assert torch.equal(nan, expected)


@pytest.mark.gpu
def test_side_stream_and_graph():
    """On a stream of its own, and captured: every replay gives the eager results for the inputs that lie there then."""
    pb = Problem(CASES[2], 7)
    q, k, wq, wk = pb.tensor(), pb.tensor(), pb.weight(), pb.weight()
    dyq, dyk = (ca.compact_attn_permute(pb.tensor(False), pb.layout) for _ in range(2))

    def step(stream=None):
        args = (q, k, wq, wk, pb.layout, pb.rotary)
        return (*ca.compact_attn_norm_rotate(*args, stream=stream), *ca.compact_attn_norm_rotate_backward(dyq, dyk, *args, stream=stream),
                ca.compact_attn_rotate(dyq, pb.layout, pb.rotary, transpose=True, stream=stream))

    want = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = step(side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for replay in range(3):
        q.copy_(pb.tensor())
        dyk.mul_(-1)
        want = step()
        for t in captured:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, captured)), replay


@pytest.mark.gpu
def test_table_must_be_on_the_device_before_a_capture():
    pb = Problem(CASES[1], 8)
    x = pb.tensor()
    out = torch.empty_like(x)
    graph, refused = torch.cuda.CUDAGraph(), None
    with torch.cuda.graph(graph):
        x.add_(0)
        try:
            ca.compact_attn_rotate(x, pb.layout, pb.rotary, origin=pb.origin, tiled=False, out=out)
        except ca.CompactAttnError as e:
            refused = e
    assert refused is not None and refused.status == -1 and "compact_attn_rotary_upload" in str(refused)
    ca.compact_attn_rotary_upload(pb.rotary)
    ca.compact_attn_rotate(x, pb.layout, pb.rotary, origin=pb.origin, tiled=False, out=out)


@pytest.mark.gpu
def test_binding_refusals():
    pb = Problem(CASES[2], 9)
    x, w = pb.tensor(), pb.weight()
    rot = lambda src=x, **kw: ca.compact_attn_rotate(src, pb.layout, pb.rotary, **kw)
    for bad in (lambda: rot(x.cpu()), lambda: rot(x.float()), lambda: rot(x[:, :2]), lambda: rot(x.transpose(2, 3).contiguous().transpose(2, 3)), lambda: rot(transpose=True),
                lambda: rot(out=torch.empty_like(x)), lambda: rot(positions=torch.zeros(pb.batch, pb.geom.N_real, 3, device=DEV)),
                lambda: ca.compact_attn_norm_rotate(x, x, w[:-8], w, pb.layout, pb.rotary), lambda: ca.compact_attn_norm_rotate(x, x, w.float(), w, pb.layout, pb.rotary),
                lambda: ca.compact_attn_norm_rotate_backward(x, x, x, x, w, w, pb.layout, pb.rotary)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: rot(origin=(9, 0, 0)), lambda: rot(origin=(-1, 0, 0))):
        with pytest.raises(ca.CompactAttnError):
            bad()


@pytest.mark.gpu
def test_a_head_that_is_shared_is_read_in_place():
    """Expanded keys (stride 0 over the heads): results and gradients are those of a copy, a gradient for every head."""
    pb = Problem(CASES[2], 11)
    q, wq, wk = pb.tensor(), pb.weight(), pb.weight()
    k = pb.tensor()[:, :1].expand(q.shape)
    dyq, dyk = (ca.compact_attn_permute(pb.tensor(False), pb.layout) for _ in range(2))
    step = lambda k: (*ca.compact_attn_norm_rotate(q, k, wq, wk, pb.layout, pb.rotary),
                      *ca.compact_attn_norm_rotate_backward(dyq, dyk, q, k, wq, wk, pb.layout, pb.rotary))
    for a, b in zip(step(k), step(k.contiguous())):
        assert torch.equal(a, b)


@pytest.mark.gpu
def test_rows_past_4_gib():
    """Token strides that lead past 32 bits, of the tensor that is read and of the one that is written."""
    pb = Problem(((4, 8, 8), (1, 4, 4), 0, 1, 2, 64, "bf16", (16, 24, 24), "half"), 12)
    gap = 1 << 24   # elements from token to token: 255 * 2^25 bytes
    source, target = (torch.empty(pb.geom.N_real * gap, dtype=torch.bfloat16, device=DEV).view(1, pb.geom.N_real, gap) for _ in range(2))
    rows = lambda t: t[:, :, :2 * pb.D].view(1, pb.geom.N_real, 2, pb.D).transpose(1, 2)
    x, wq, wk = pb.tensor(False), pb.weight(), pb.weight()
    far = rows(source)
    far.copy_(x)
    assert (pb.geom.N_real - 1) * gap * 2 > 2 ** 32
    assert torch.equal(ca.compact_attn_rotate(far, pb.layout, pb.rotary), ca.compact_attn_rotate(x, pb.layout, pb.rotary))
    dy = ca.compact_attn_permute(pb.tensor(False), pb.layout)
    ca.compact_attn_rotate(dy, pb.layout, pb.rotary, transpose=True, out=rows(target))
    assert torch.equal(rows(target), ca.compact_attn_rotate(dy, pb.layout, pb.rotary, transpose=True))
    near = ca.compact_attn_norm_rotate_backward(dy, dy, x, x, wq, wk, pb.layout, pb.rotary)
    got = ca.compact_attn_norm_rotate_backward(dy, dy, far, far, wq, wk, pb.layout, pb.rotary, out=(rows(target), torch.empty_like(x)))
    assert all(torch.equal(a, b) for a, b in zip(near, got))


@pytest.mark.gpu
def test_long_table_and_far_positions():
    """Positions of 10^6: the angle is as exact as at 0."""
    n, far = 8, 1_000_000
    lay = _layout(n, 1, 1, (1, 1, 1), 0, 1, 1, 32, "f32")
    rotary = ca.compact_attn_build_rotary((32, 0, 0), (far + n, 1, 1))
    x = torch.ones(1, 1, n, 32, device=DEV)
    got = f64(ca.compact_attn_rotate(x, lay, rotary, origin=(far, 0, 0)))[0, 0]
    at = np.zeros((n, 3), dtype=np.int64)
    at[:, 0] = far + np.arange(n)
    want = OR.rotate(np.ones((n, 32)), OR.angles(at, [OR.frequencies(32), np.zeros(0), np.zeros(0)]), "interleaved")
    check(got, want, 8 * U32 + 1e-9, "f32", "far")
