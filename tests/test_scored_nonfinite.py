"""Scored attention beside values that are not finite: infinities and NaN in queries, keys, values and the results' gradients reach what depends on them and nothing else.

What a formula gives for them: a NaN score makes its query's row NaN, forwards and in dQ; a score of plus infinity does the same without a cap (infinity less infinity) and is the
cap with one; a score of minus infinity is no weight without a cap and minus the cap with one; a row all of whose scores are minus infinity is an empty one.  Rows that keep no tile of such a
token, and channels beside an infinite one, hold the same bits as without it."""
import math

import pytest
import torch

import paper_2508_12969_amd as ca

DEV = "cuda:0"
INF, NAN = math.inf, math.nan
KERNELS = [((1, 8, 8), 64), ((1, 8, 8), 128), ((2, 8, 8), 64), ((2, 8, 8), 128)]
ids = lambda k: f"B{math.prod(k[0])}-D{k[1]}"


class Step:
    """Head 0 keeps, of every tile row and column of tiles, its own; head 1 keeps everything."""

    def __init__(self, tile, D, long=False, **how):
        T, H, W = (6, 18, 23) if long else (3, 13, 20)
        self.layout = ca.compact_attn_build_layout(T, H, W, tile, 0, 1, 2, D, "bf16", [[(0, (0, 0), (-1, -1))], [(T, (H, W), (-1, -1))]])
        self.N, self.D, self.how = self.layout.n_tokens_real, D, how
        g = torch.Generator().manual_seed(3)
        self.q, self.k, self.v, self.do = (torch.randn(1, 2, self.N, D, generator=g).to(torch.bfloat16).to(DEV) for _ in range(4))
        t = torch.arange(self.N, device=DEV)
        t, y, x = t // (H * W), t // W % H, t % W
        self.tile = (t // tile[0] * 100 + y // tile[1]) * 100 + x // tile[2]   # a number of its own for every tile

    def run(self, **other):
        """(out, lse, dq, dk, dv) in natural order; q, k, v, do as given or the step's own."""
        q, k, v, do = (ca.compact_attn_permute(other.get(n, getattr(self, n)), self.layout) for n in ("q", "k", "v", "do"))
        out, lse = ca.compact_attn_forward_scored(q, k, v, self.layout, **self.how)
        grads = ca.compact_attn_backward_scored(do, q, k, v, out, lse, self.layout, **self.how)
        back = lambda x: ca.compact_attn_permute(x, self.layout, inverse=True)[0]
        lse = back(lse[..., None].repeat(1, 1, 1, self.D).to(torch.bfloat16))[..., 0]   # (rounded: for finite or not)
        torch.cuda.synchronize()
        return (back(out), lse, *(back(g) for g in grads))

    def changed(self, name, token, value, channel=None):
        x = getattr(self, name).clone()
        x[:, :, token, slice(None) if channel is None else channel] = value
        return x


def _step(kernel, how):
    pb = Step(*kernel, long=how == "shares")
    if how == "arrays":
        frames = (torch.arange(pb.N, device=DEV) // 260).to(torch.int32)[None]
        pb.how = dict(positions=frames, limits=frames + 9, documents=torch.zeros_like(frames), slopes=torch.tensor([0.1, 0.2], device=DEV))
    if how == "cap":
        pb.how = dict(cap=6.0)
    return pb


HOWS = ["plain", "arrays", "cap", "shares"]


@pytest.mark.gpu
@pytest.mark.parametrize("how", HOWS)
@pytest.mark.parametrize("kernel", KERNELS, ids=ids)
def test_a_query_that_is_nan_is_a_row_of_nan(kernel, how):
    print("nan query", kernel, how, flush=True)
    pb = _step(kernel, how)
    token = pb.N // 2 + 1
    want, got = pb.run(), pb.run(q=pb.changed("q", token, NAN))
    others = torch.arange(pb.N, device=DEV) != token
    for name, a, b in zip(("out", "lse", "dq"), want, got):
        assert torch.isnan(b[:, token]).all(), name
        assert torch.equal(a[:, others], b[:, others]), name
    far = pb.tile != pb.tile[token]                # head 0: keys that do not see it
    for name, a, b in zip(("dk", "dv"), want[3:], got[3:]):
        assert torch.equal(a[0, far], b[0, far]) and torch.isnan(b[0, ~far]).all() and torch.isnan(b[1]).all(), name


@pytest.mark.gpu
@pytest.mark.parametrize("how", HOWS)
@pytest.mark.parametrize("kernel", KERNELS, ids=ids)
def test_a_key_that_is_nan_reaches_the_rows_that_see_it(kernel, how):
    print("nan key", kernel, how, flush=True)
    pb = _step(kernel, how)
    token = pb.N // 3
    want, got = pb.run(), pb.run(k=pb.changed("k", token, NAN))
    far = pb.tile != pb.tile[token]
    for name, a, b in zip(("out", "lse", "dq", "dk", "dv"), want, got):
        assert torch.equal(a[0, far], b[0, far]) and torch.isnan(b[0, ~far]).all() and torch.isnan(b[1]).all(), name


@pytest.mark.gpu
@pytest.mark.parametrize("how", HOWS)
@pytest.mark.parametrize("kernel", KERNELS, ids=ids)
def test_infinite_values_and_gradients_keep_to_their_channel(kernel, how):
    """Every weight is positive here, so an infinite channel of a value is infinite in the rows that see it, and one of a result's gradient in dV of the keys that it saw."""
    print("infinite value", kernel, how, flush=True)
    pb = _step(kernel, how)
    token, channel = pb.N - 1, 5                   # the last token, of a tile with padding behind it
    far = pb.tile != pb.tile[token]
    others = torch.arange(pb.D, device=DEV) != channel
    for sign in (INF, -INF):
        want, got = pb.run()[0], pb.run(v=pb.changed("v", token, sign, channel))[0]
        assert torch.equal(want[..., others], got[..., others]) and torch.equal(want[0, far], got[0, far])
        assert (got[0, ~far, channel] == sign).all() and (got[1, :, channel] == sign).all()
        want, got = pb.run()[4], pb.run(do=pb.changed("do", token, sign, channel))[4]
        assert torch.equal(want[..., others], got[..., others]) and torch.equal(want[0, far], got[0, far])
        assert (got[0, ~far, channel] == sign).all() and (got[1, :, channel] == sign).all()


@pytest.mark.gpu
@pytest.mark.parametrize("how", HOWS)
@pytest.mark.parametrize("kernel", KERNELS, ids=ids)
def test_infinite_scores(kernel, how):
    """One channel of a key is infinite and the queries hold 1 or -1 there: minus infinity is a key without weight (minus the cap with one), plus infinity a row of NaN (the cap)."""
    print("infinite score", kernel, how, flush=True)
    pb = _step(kernel, how)
    token = pb.N // 2
    q = pb.q.clone()
    q[..., 0] = -1
    k = pb.changed("k", token, 0, 0)
    gone = pb.changed("k", token, INF, 0)
    got = pb.run(q=q, k=gone)
    if how == "cap":                               # as a key so far down that its score is minus the cap
        far_down = torch.zeros_like(pb.k[:, :, token])
        far_down[..., 0] = 2.0 ** 20
        k[:, :, token] = gone[:, :, token] = far_down
        gone[:, :, token, 0] = INF
        want, got = pb.run(q=q, k=k), pb.run(q=q, k=gone)
        assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1]) and torch.equal(want[4], got[4])
    else:                                          # as without that key: it has no weight, so its value does not count
        assert all(torch.isfinite(x).all() for x in got[:2]) and torch.isfinite(got[4]).all()
        assert (got[4][:, token] == 0).all()
        other = pb.run(q=q, k=gone, v=pb.changed("v", token, 1000.0))
        assert torch.equal(got[0], other[0]) and torch.equal(got[1], other[1])
    token_q = pb.N // 2 + 1
    q[:, :, token_q, 0] = 1
    row = pb.run(q=q, k=gone)
    others = torch.arange(pb.N, device=DEV) != token_q
    assert torch.equal(row[0][:, others], got[0][:, others])
    sees = torch.tensor([bool(pb.tile[token] == pb.tile[token_q]), True], device=DEV)
    if how == "cap":
        assert torch.isfinite(row[0]).all() and torch.isfinite(row[1]).all()
    else:
        assert torch.isnan(row[0][sees, token_q]).all() and torch.isfinite(row[0][~sees, token_q]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("how", ["plain", "arrays", "shares"])
@pytest.mark.parametrize("kernel", KERNELS, ids=ids)
def test_a_row_of_minus_infinite_scores_is_empty(kernel, how):
    print("row of minus infinity", kernel, how, flush=True)
    pb = _step(kernel, how)
    token = pb.N // 2
    q, k = pb.q.clone(), pb.k.clone()
    k[..., 0] = 1
    q[:, :, token] = 0
    q[:, :, token, 0] = -INF
    want, got = pb.run(k=k), pb.run(q=q, k=k)
    others = torch.arange(pb.N, device=DEV) != token
    assert (got[0][:, token] == 0).all() and (got[1][:, token] == -INF).all()
    assert torch.equal(want[0][:, others], got[0][:, others]) and torch.equal(want[1][:, others], got[1][:, others])
    assert torch.isfinite(got[4]).all()            # dV: it has no weight
    far = pb.tile != pb.tile[token]
    assert torch.equal(want[4][0, far], got[4][0, far])


@pytest.mark.gpu
@pytest.mark.parametrize("kernel", KERNELS, ids=ids)
def test_hidden_tokens_may_hold_the_largest_finite_values(kernel):
    """Tokens of no document hold plus or minus 2^100 (products past the range of fp32 among them): results of the others are those beside zeros, and theirs are empty."""
    print("hidden", kernel, flush=True)
    pb = Step(*kernel)
    documents = torch.zeros(1, pb.N, dtype=torch.int32, device=DEV)
    hidden = torch.arange(pb.N, device=DEV) % 5 == 3
    documents[:, hidden] = -4
    for cap in (0.0, 6.0):
        pb.how = dict(documents=documents, cap=cap)
        results = []
        for value in (0.0, 2.0 ** 100, -2.0 ** 100):
            fill = {n: pb.changed(n, hidden, value) for n in ("q", "k", "v")}
            fill["k"][:, :, hidden, 1::2] = -value
            results.append(pb.run(**fill, do=pb.changed("do", hidden, 0.0)))
        for other in results[1:]:
            assert all(torch.equal(a, b) for a, b in zip(results[0], other)), cap
        assert (results[0][0][:, hidden] == 0).all() and (results[0][1][:, hidden] == -INF).all()
        assert all((g[:, hidden] == 0).all() for g in results[0][2:])


@pytest.mark.gpu
@pytest.mark.parametrize("kernel", KERNELS, ids=ids)
def test_an_infinite_key_beside_queries_that_are_not_there(kernel):
    """Queries of no document are zero where a key is infinite: they have no part in its gradients, whether or not pairs of their tile are hidden for another reason."""
    print("infinite key, hidden queries", kernel, flush=True)
    pb = Step(*kernel)
    token = pb.N // 2
    hidden = torch.arange(pb.N, device=DEV) % 5 == (token + 3) % 5
    documents = torch.where(hidden, -4, 0).to(torch.int32)[None]
    q = pb.q.clone()
    q[..., 0] = -1                                 # the key's scores are minus infinity
    q[:, :, hidden] = 0
    frames = (torch.arange(pb.N, device=DEV) // 260).to(torch.int32)[None]
    for how in (dict(documents=documents), dict(documents=documents, positions=frames, limits=frames), dict(documents=documents, cap=6.0)):
        pb.how = how
        out, lse, _, _, dv = pb.run(q=q, k=pb.changed("k", token, INF, 0))
        there = ~hidden
        assert torch.isfinite(out).all() and torch.isfinite(lse[:, there]).all() and torch.isfinite(dv).all()
        if not how.get("cap"):
            assert (dv[:, token] == 0).all()
