"""Rotary positions and norms with the rotation, in 64 bits (oracle side; test infrastructure).

Tokens in natural order, one (batch, head) plane at a time: x is [tokens, D], the angles [tokens, R/2] for the
first R channels.  Pairs of channels are turned as complex numbers.
"""
import math

import numpy as np


def frequencies(channels, base=10000.0, stretch=1.0, method="linear", trained=None, turns=(1.0, 32.0)):
    """Angle per position of every pair of an axis."""
    out = []
    for i in range(channels // 2):
        b = base * stretch ** (channels / (channels - 2)) if method == "base" and channels > 2 else base
        f = b ** (-2.0 * i / channels)
        if method == "linear":
            f /= stretch
        elif method == "bands":
            times = trained * f / (2 * math.pi)
            keep = min(1.0, max(0.0, (times - turns[0]) / (turns[1] - turns[0])))
            f = keep * f + (1 - keep) * f / stretch
        out.append(f)
    return np.array(out)


def angles(positions, per_axis):
    """positions int [tokens, 3], frequencies of the three axes -> [tokens, pairs]; a negative position does not turn."""
    positions = np.asarray(positions)
    return np.concatenate([np.maximum(positions[:, i:i + 1], 0) * f[None, :] for i, f in enumerate(per_axis)], axis=1)


def grid_positions(geom, origin=(0, 0, 0)):
    """int [N_real, 3]: origin + (t, y, x), and -1 for text tokens."""
    video = np.stack(np.meshgrid(*(o + np.arange(n) for o, n in zip(origin, (geom.T, geom.H, geom.W))), indexing="ij"), axis=-1).reshape(-1, 3)
    return np.concatenate([video, np.full((geom.n_text, 3), -1)])


def rotate(x, angle, pairing, magnitude=1.0, transpose=False):
    """x [tokens, D].  magnitude applies to turned pairs only: pass an array [tokens, pairs] where some are not."""
    x = np.asarray(x, dtype=np.float64)
    pairs = angle.shape[1]
    part = x[:, :2 * pairs]
    z = part[:, :pairs] + 1j * part[:, pairs:] if pairing == "half" else part[:, 0::2] + 1j * part[:, 1::2]
    z = z * magnitude * np.exp((-1j if transpose else 1j) * angle)
    out = x.copy()
    if pairing == "half":
        out[:, :pairs], out[:, pairs:2 * pairs] = z.real, z.imag
    else:
        out[:, 0:2 * pairs:2], out[:, 1:2 * pairs:2] = z.real, z.imag
    return out


def norm(x, weight, eps):
    x = np.asarray(x, dtype=np.float64)
    return x / np.sqrt((x * x).mean(axis=1, keepdims=True) + eps) * weight


def norm_gradient(x, weight, eps, du):
    """Gradients of norm for its result's gradient du -> (dx [tokens, D], dweight [D])."""
    x = np.asarray(x, dtype=np.float64)
    rms = np.sqrt((x * x).mean(axis=1, keepdims=True) + eps)
    dn = du * weight
    dx = dn / rms - x * (dn * x).mean(axis=1, keepdims=True) / rms ** 3
    return dx, (du * x / rms).sum(axis=0)
