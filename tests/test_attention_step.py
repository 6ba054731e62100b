"""The operators of a training step of one attention layer together, as a model runs them: norm and rotation of queries and keys that a projection left behind,
scored attention over the tile lists, and the gradients back to the projection's output and the norm's weights; against torch's derivatives in 64 bits.

Tolerances, in norm.  r = 2^-8 / sqrt(3) is the root mean square of bf16 roundings that are spread evenly over half a step.  Every intermediate tensor that is
rounded adds an independent relative error of at most r to what follows (a score of unit spread moves by r for a rounded q and for a rounded k; the weights,
and with them dS, by as much).  The result: normed q, normed k, weights, the result itself: 4 roundings.  The gradient of v: the same with dO for v.  Gradients of
q and k: normed q and k (scores), k or q as a factor, dS, the attention's result (through its row sums), the rounded gradient, the gradient after the norm: 7.
Gradients of the weights are sums of those over tokens, without the last rounding.  Bounds are twice sqrt(count) r, for correlations between them."""
import math

import numpy as np
import pytest
import torch

import paper_2508_12969_amd as ca
from oracle import scored as OS
from oracle.geometry import Geometry

DEV = "cuda:0"
R = 2.0 ** -8 / math.sqrt(3)
MOST = {"out": 2 * math.sqrt(4) * R, "dv": 2 * math.sqrt(4) * R, "dq": 2 * math.sqrt(7) * R, "dk": 2 * math.sqrt(7) * R, "dwq": 2 * math.sqrt(7) * R,
        "dwk": 2 * math.sqrt(7) * R}


class Layer:
    """A fused projection [batch, tokens, 3, heads, D], the norm's weights, tile lists, and how scores are bent and hidden."""

    def __init__(self, grid, tile, n_text, D, heads, batch, pairing, cap, masked, seed):
        rng = np.random.default_rng(seed)
        self.geom = g = Geometry(*grid, *tile, n_text)
        self.D, self.heads, self.batch, self.cap = D, heads, batch, cap
        groups = [[(0, (1, 1), (-1, -1)), (1, (0, 0), (-1, -1))], [(g.nT - 1, (g.nH - 1, g.nW - 1), (-1, -1))]]
        self.layout = ca.compact_attn_build_layout(*grid, tile, n_text, batch, heads, D, "bf16", [groups[h % 2] for h in range(heads)])
        channels = (D // 4, D // 4, D // 4)
        self.rotary = ca.compact_attn_build_rotary(channels, grid, pairing=pairing)
        self.pairing = pairing
        N = g.N_real
        put = lambda x: torch.from_numpy(x.astype(np.float32)).to(torch.bfloat16).to(DEV)
        self.fused = put(rng.normal(size=(batch, N, 3, heads, D)))
        self.dout = put(rng.normal(size=(batch, heads, N, D)))
        self.weights = [put(1 + 0.2 * rng.normal(size=D)) for _ in range(2)]
        self.how = dict(cap=cap)
        self.frames = np.tile(np.concatenate([np.arange(g.T * g.H * g.W) // (g.H * g.W), np.zeros(n_text, int)]).astype(np.int32), (batch, 1))
        self.documents = self.slopes = None
        if masked:
            self.documents = np.zeros((batch, N), np.int32)
            for b in range(batch):   # a padded prompt in each batch entry, of another length
                self.documents[b, N - n_text // 2 - 5 * b:] = -1
            self.slopes = np.linspace(0.05, 0.2, heads).astype(np.float32)
            dev = lambda x: torch.from_numpy(x).to(DEV)
            self.how |= dict(slopes=dev(self.slopes), positions=dev(self.frames), limits=dev(self.frames), documents=dev(self.documents))

    def step(self):
        """-> result and gradients, all in natural order; the gradient of the projection as it lies in memory."""
        q, k, v = (self.fused[:, :, i].transpose(1, 2) for i in range(3))
        args = (q, k, *self.weights, self.layout, self.rotary)
        qt, kt = ca.compact_attn_norm_rotate(*args)
        vt = ca.compact_attn_permute(v.contiguous(), self.layout)
        ot, lse = ca.compact_attn_forward_scored(qt, kt, vt, self.layout, **self.how)
        out = ca.compact_attn_permute(ot, self.layout, inverse=True)
        dot = ca.compact_attn_permute(self.dout, self.layout)
        dqt, dkt, dvt = ca.compact_attn_backward_scored(dot, qt, kt, vt, ot, lse, self.layout, **self.how)
        dfused = torch.empty_like(self.fused)
        dq, dk, dv = (dfused[:, :, i].transpose(1, 2) for i in range(3))
        _, _, dwq, dwk = ca.compact_attn_norm_rotate_backward(dqt, dkt, *args, out=(dq, dk))
        dv.copy_(ca.compact_attn_permute(dvt, self.layout, inverse=True))
        return out, dfused, dwq, dwk

    def keep(self, head, b):
        n, of = self.geom.n, self.geom.token_slots() // self.geom.B
        row_ptr, col = ca.compact_attn_layout_csr(self.layout, head)
        m = np.zeros((n, n), bool)
        for r in range(n):
            m[r, col[row_ptr[r]:row_ptr[r + 1]]] = True
        m = m[of][:, of]
        return m if self.documents is None else OS.visible(m, self.frames[b].astype(np.int64), self.frames[b].astype(np.int64), self.documents[b].astype(np.int64))

    def plain(self, fused, wq, wk):
        """The same in 64 bits, on the CPU, as torch can derive it."""
        g, D = self.geom, self.D
        turned = D // 4 * 3
        t = torch.arange(g.T * g.H * g.W)
        at = [t // (g.H * g.W), t // g.W % g.H, t % g.W]
        z = []
        for axis in range(3):
            a = torch.from_numpy(ca.compact_attn_rotary_angles(self.rotary, axis)).double()[at[axis]]
            z.append(torch.complex(a[..., 0], a[..., 1]))
        z = torch.cat([torch.cat(z, dim=1), torch.ones(g.n_text, turned // 2, dtype=torch.complex128)])

        def normed(x, w):
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w
            p, half = x[..., :turned], turned // 2
            c = torch.complex(p[..., :half], p[..., half:]) if self.pairing == "half" else torch.complex(p[..., 0::2], p[..., 1::2])
            c = c * z
            p = torch.cat([c.real, c.imag], -1) if self.pairing == "half" else torch.stack([c.real, c.imag], -1).flatten(-2)
            return torch.cat([p, x[..., turned:]], -1)

        outs = []
        for b in range(self.batch):
            for h in range(self.heads):
                q, k, v = (fused[b, :, i, h] for i in range(3))
                s = normed(q, wq) @ normed(k, wk).t() * D ** -0.5
                if self.cap:
                    s = self.cap * torch.tanh(s / self.cap)
                if self.slopes is not None:
                    pos = torch.from_numpy(self.frames[b]).double()
                    s = s - float(self.slopes[h]) * (pos[:, None] - pos[None, :]).abs()
                seen = torch.from_numpy(self.keep(h, b))
                s = s.masked_fill(~seen, -1e300)
                p = torch.softmax(s, -1) * seen
                outs.append(p @ v)
        return torch.stack(outs).reshape(self.batch, self.heads, g.N_real, D)


@pytest.mark.gpu
@pytest.mark.parametrize("pairing,D,tile,cap,masked", [("interleaved", 128, (2, 8, 8), 0.0, False), ("half", 64, (1, 8, 8), 10.0, True),
                                                       ("interleaved", 64, (1, 8, 16), 0.0, True), ("half", 128, (1, 8, 8), 10.0, True)])
def test_training_step(pairing, D, tile, cap, masked):
    print("step", pairing, D, tile, cap, masked, flush=True)
    layer = Layer((3, 11, 13), tile, 128, D, 2, 2, pairing, cap, masked, seed=D)
    first = layer.step()
    leaves = [x.double().cpu().requires_grad_() for x in (layer.fused, *layer.weights)]
    out = layer.plain(*leaves)
    out.backward(layer.dout.double().cpu())
    dfused = first[1].double().cpu()
    got = {"out": first[0].double().cpu(), "dq": dfused[:, :, 0], "dk": dfused[:, :, 1], "dv": dfused[:, :, 2], "dwq": first[2].double().cpu(), "dwk": first[3].double().cpu()}
    want = {"out": out.detach(), "dq": leaves[0].grad[:, :, 0], "dk": leaves[0].grad[:, :, 1], "dv": leaves[0].grad[:, :, 2], "dwq": leaves[1].grad, "dwk": leaves[2].grad}
    off = {name: float((got[name] - want[name]).norm() / want[name].norm()) for name in got}
    print({name: f"{e:.2e} of {MOST[name]:.2e}" for name, e in off.items()}, flush=True)
    for name in got:
        assert torch.isfinite(got[name]).all() and off[name] <= MOST[name], (name, off[name])
    # along the formula's gradient the loss changes by its norm: from differences of the loss in 64 bits, against the kernels' gradient
    at = [x.detach() for x in leaves]
    along = [x.grad / x.grad.norm() for x in leaves]
    loss = lambda t: float((layer.plain(*(x + t * d for x, d in zip(at, along))) * layer.dout.double().cpu()).sum())
    slope = (loss(1e-4) - loss(-1e-4)) / 2e-4
    measured = float((dfused * along[0]).sum() + (got["dwq"] * along[1]).sum() + (got["dwk"] * along[2]).sum())
    assert abs(measured - slope) <= MOST["dq"] * sum(float(x.grad.norm()) for x in leaves)

    # captured twice, replayed with other inputs in the same memory
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            results = layer.step()
        graphs.append((graph, results))
    for replay in range(3):
        layer.fused.mul_(-0.5 if replay % 2 else -2)
        layer.dout.copy_(layer.dout.flip(2))
        again = layer.step()
        for graph, results in graphs:
            for t in results:
                t.zero_()
            graph.replay()
        torch.cuda.synchronize()
        for _, results in graphs:
            assert all(torch.equal(a, b) for a, b in zip(again, results)), replay


@pytest.mark.gpu
def test_two_steps_at_once():
    """Two layers on two streams, each with workspaces of its own: what either gives alone."""
    layers = [Layer((3, 11, 13), (1, 8, 8), 128, 64, 2, 2, "half", 10.0, True, seed=s) for s in (1, 2)]
    alone = [layer.step() for layer in layers]
    streams = [torch.cuda.Stream() for _ in layers]
    for stream in streams:
        stream.wait_stream(torch.cuda.current_stream())
    results = [[], []]
    for _ in range(4):
        for i, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                results[i].append(layers[i].step())
    torch.cuda.synchronize()
    for want, many in zip(alone, results):
        for got in many:
            assert all(torch.equal(a, b) for a, b in zip(want, got))
