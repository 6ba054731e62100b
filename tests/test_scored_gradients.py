"""Scored attention: gradients in norm, where the per-element bounds of test_scored.py cannot see a row's shift.

delta = rowsum(dO O) is made from a rounded O, and dS is rounded as an operand; both move all of a row's dS the same way, and the kernels take that off again with sums of their own (an
extra product for dQ, a corrected delta for dK).  Left out or with the wrong sign it would still lie within bounds that add up magnitudes.

Bound.  Rounding to bf16 is off by at most 2^-8 of the power of two below the value, evenly spread: in the root mean square 2^-8 / sqrt(3) * sqrt(3 / (8 ln 2)) = 1.66e-3 of values
whose mantissas are spread evenly over their logarithm.  A gradient is a sum over tokens of terms that are rounded once, dS (or P, for dV and the result), independently, and is rounded itself:
sqrt(2) * 1.66e-3 = 2.35e-3 of its norm, where the terms do not mostly cancel; a tenth more for the spread of mantissas and sums: 2.6e-3.  The values share a mean here, as
those of a model do, which makes O large beside what of it differs from row to row, and with it what the shift does.  The first test shows on the CPU, in 64 bits with the kernels'
roundings, that this bound holds with the correction and is missed without it, with its sign turned, or with twenty times as much."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2508_12969_amd as ca
from oracle import permute as OP
from oracle import scored as OS
from oracle.geometry import Geometry
from paper_2508_12969_amd import scored as SC

DEV = "cuda:0"
ROUNDING = 2.0 ** -8 / math.sqrt(3) * math.sqrt(3 / (8 * math.log(2)))
MOST = 1.1 * math.sqrt(2) * ROUNDING

# name: grid, tile, head dim, rule, whether runs are shared by several workgroups
CASES = {
    "plain": ((2, 13, 16), (1, 8, 8), 64, dict(), False),
    "plain, 128 channels": ((2, 13, 16), (2, 8, 8), 128, dict(), False),
    "plain, shares": ((4, 22, 24), (1, 8, 8), 64, dict(), True),
    "plain, 128 channels, shares": ((4, 23, 24), (2, 8, 8), 128, dict(), True),
    "cap": ((2, 13, 16), (2, 8, 8), 64, dict(cap=5.0), False),
    "cap, 128 channels, shares": ((4, 22, 24), (1, 8, 8), 128, dict(cap=10.0), True),
    "clips, cap": ((2, 13, 16), (1, 8, 8), 64, dict(cap=5.0, clips=True), False),
    "clips, shares": ((4, 18, 20), (1, 8, 8), 128, dict(clips=True), True),
    "clips, cap, shares": ((4, 18, 20), (2, 8, 8), 64, dict(cap=10.0, clips=True), True),
}


def bf16(x):
    return torch.from_numpy(np.asarray(x, dtype=np.float32)).to(torch.bfloat16).double().numpy()


class Problem:
    """One head that keeps every tile; q, k, v and dO share a mean over the tokens, scores have a spread of about 4."""

    def __init__(self, name):
        grid, tile, D, rule, self.shared = CASES[name]
        rng = np.random.default_rng(sorted(CASES).index(name) + 1)
        self.geom = g = Geometry(*grid, *tile, 0)
        self.D, self.cap, self.scale = D, rule.get("cap", 0.0), D ** -0.5
        self.layout = ca.compact_attn_build_layout(*grid, tile, 0, 1, 1, D, "bf16", [[(g.nT - 1, (g.nH - 1, g.nW - 1), (-1, -1))]])
        N = g.N_real
        values = lambda gain, mean: bf16(gain * rng.normal(size=(N, D)) + mean * rng.normal(size=D))
        self.q, self.k, self.v, self.do = values(4.0, 0.3), values(1.0, 1.0), values(1.0, 4.0), values(1.0, 0.5)
        self.arrays = {}
        if rule.get("clips"):
            frame = np.arange(N) // (g.H * g.W)
            self.arrays = dict(positions=frame, limits=frame, documents=(rng.random(N) < 0.1).astype(int))
        self.seen = OS.visible(np.ones((N, N), bool), *(self.arrays.get(n) for n in ("positions", "limits", "documents")))
        self.out, self.lse, self.p = OS.forward(self.q, self.k, self.v, self.seen, self.scale, cap=self.cap)
        self.grads = OS.backward(self.do, self.q, self.k, self.v, self.seen, self.scale, cap=self.cap)[:3]

    def emulated(self, correction):
        """Relative errors of dQ and dK with the kernels' roundings in otherwise 64 bits, and `correction` times what they take off."""
        p = self.p
        delta = (self.do * bf16(bf16(p) @ self.v)).sum(1, keepdims=True)
        _, steep = OS.scores(self.q, self.k, self.scale, cap=self.cap)
        dp = self.do @ self.v.T
        t = p * (dp - delta)
        lean, ds, weight = t.sum(1, keepdims=True), bf16(t * steep), bf16(p * steep)
        if self.cap:
            sums = weight.sum(1, keepdims=True)
            shift = lean + np.divide((ds - t * steep).sum(1, keepdims=True), sums, out=np.zeros_like(sums), where=sums != 0)
        else:
            shift = lean = ds.sum(1, keepdims=True)
        dq = bf16(self.scale * (ds @ self.k - correction * shift * (weight @ self.k)))
        dk = bf16(self.scale * bf16(p * (dp - delta - correction * lean) * steep).T @ self.q)
        return [off(got, want) for got, want in zip((dq, dk), self.grads)]


def off(got, want):
    return float(np.linalg.norm(got - want) / np.linalg.norm(want))


def _workspace(layout, scores, backward):
    need = ctypes.c_int64()
    assert ca.load_library().compact_attn_scored_workspace(layout.handle, scores, backward, need) == 0
    return need.value


@pytest.mark.parametrize("name", CASES)
def test_the_bound_tells_the_correction_from_its_absence(name):
    pb = Problem(name)
    right = pb.emulated(1)
    others = off(bf16(bf16(pb.p) @ pb.v), pb.out), off(bf16(bf16(pb.p).T @ pb.do), pb.grads[2])   # the result and dV
    print(name, "right", right, others)
    assert max(*right, *others) <= MOST, (right, others)
    for wrong in (0, -1, 20):
        errors = pb.emulated(wrong)
        print("   ", wrong, errors)
        assert min(errors) > 1.1 * MOST, (wrong, errors)
    if not pb.arrays:   # without arrays a workspace of the forward call holds nothing but shares
        assert (_workspace(pb.layout, SC.ca_scores(pb.cap, None, None, None, None), 0) > 0) == pb.shared
    else:               # the device cuts runs of more than eight steps of 64 tokens where the longest is far above an even share, which is below two here
        assert (len(np.unique(pb.geom.token_slots() // 64)) > 8) == pb.shared


@pytest.mark.gpu
@pytest.mark.parametrize("name", CASES)
def test_gradients_in_norm(name):
    print("scored gradients", name, flush=True)
    pb = Problem(name)

    def tiled(x):
        t = torch.zeros(1, 1, pb.geom.N_pad, pb.D, dtype=torch.bfloat16)
        t[0, 0, torch.from_numpy(pb.geom.token_slots())] = torch.from_numpy(x).to(torch.bfloat16)
        return t.to(DEV)

    q, k, v, do = (tiled(x) for x in (pb.q, pb.k, pb.v, pb.do))
    how = dict(cap=pb.cap, **{n: torch.from_numpy(x.astype(np.int32))[None].to(DEV) for n, x in pb.arrays.items()})
    out, lse = ca.compact_attn_forward_scored(q, k, v, pb.layout, **how)
    grads = ca.compact_attn_backward_scored(do, q, k, v, out, lse, pb.layout, **how)
    torch.cuda.synchronize()
    natural = lambda t: OP.unpermute(pb.geom, t[0, 0].double().cpu().numpy())
    errors = {n: off(natural(t), want) for n, t, want in zip(("out", "dq", "dk", "dv"), (out, *grads), (pb.out, *pb.grads))}
    print(errors, flush=True)
    assert max(errors.values()) <= MOST, errors
