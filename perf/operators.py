"""Operators around sparse attention, as cases that can be timed and compared: rotary positions, norms of
queries and keys with the rotation in the same pass, and attention whose scores are capped, biased and masked.

Every case works on a T x H x W grid of video tokens plus text tokens.  `op`, what is called:
  rotate       compact_attn_rotate: natural order -> rotated, in tile order (or natural order)
  rotate_back  its transpose: the gradient of a rotated tensor, back to natural order
  norm         compact_attn_norm_rotate on q and k
  norm_step    the same and compact_attn_norm_rotate_backward: gradients of q, k and both weights
  scored       compact_attn_forward_scored
  scored_step  the same and compact_attn_backward_scored: gradients of q, k and v

Layouts and rotary tables are made and uploaded once and kept, as a program does that calls the same layer at
every step; the plain forms are given the same things as index, mask and cosine tensors.
"""
import math
import random

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
ABSENT = (-1, -1)
EPS = 1e-6


def _case(name, op, grid, tile, n_text, heads, head_dim, dtype, batch=1, rotated=0, pairing="interleaved", method="linear", stretch=1.0,
          token_major=False, tiled=True, cap=0.0, bias=False, prefix=-1, docs=0, reach=1.0, mask_seed=0):
    case = dict(zip(("T", "H", "W"), grid)) | dict(zip(("tt", "th", "tw"), tile))
    case |= dict(op=op, n_text=n_text, heads=heads, head_dim=head_dim, dtype=dtype, batch=batch, rotated=rotated, pairing=pairing, method=method,
                 stretch=stretch, token_major=token_major, tiled=tiled, cap=cap, bias=bias, prefix=prefix, docs=docs, reach=reach, mask_seed=mask_seed)
    return dict(name=name, **case) if name else case


def listed():
    return [
        # the smallest call: one tensor of 256 tokens in fp32, as a check of a model in full precision makes; latency is all there is
        _case("rotate-f32-256tok", "rotate", (4, 8, 8), (1, 4, 4), 0, 2, 64, "f32", rotated=64, pairing="half", tiled=False),
        # low-resolution clip of twice the trained length, into tile order, three quarters of the head rotated, text as it is
        _case("rotate-33Ktok", "rotate", (21, 30, 52), (2, 8, 8), 256, 16, 128, "bf16", rotated=96, method="bands", stretch=2.0),
        # the gradient of that on a ragged grid with a head of 80 channels, packed clips with positions of their own
        _case("rotate-back-d80-20Ktok", "rotate_back", (13, 29, 51), (2, 4, 8), 128, 12, 80, "bf16", batch=2, rotated=40, pairing="half", method="base",
              stretch=4.0, docs=3, mask_seed=3),
        # q and k of 16 new frames of a small fp32 model, ragged
        _case("norm-f32-7Ktok", "norm", (7, 30, 33), (1, 8, 8), 64, 8, 128, "f32", rotated=128, pairing="half"),
        # q and k of a 75K-token layer as its projection leaves them (tokens first), into tile order
        _case("norm-75Ktok", "norm", (21, 45, 80), (1, 8, 8), 0, 40, 128, "bf16", rotated=128, token_major=True),
        # a training step of a small model with head dim 64, two clips in a batch
        _case("norm-step-d64-20Ktok", "norm_step", (13, 30, 52), (2, 8, 8), 128, 12, 64, "bf16", batch=2, rotated=64, token_major=True),
        # attention on the smallest clip: latency
        _case("scored-d64-256tok", "scored", (4, 8, 8), (1, 8, 8), 0, 2, 64, "bf16", cap=20.0, mask_seed=7),
        # frames in causal order after two given ones, scores that fall with the frame distance
        _case("scored-causal-d64-8Ktok", "scored", (8, 32, 32), (1, 8, 8), 64, 12, 64, "bf16", bias=True, prefix=2, docs=1, reach=0.9, mask_seed=8),
        # the largest forward: a low-resolution clip, capped scores, a prompt that is padded; one rank's share of the heads
        _case("scored-cap-33Ktok", "scored", (21, 30, 52), (2, 8, 8), 256, 4, 128, "bf16", cap=30.0, docs=1, reach=0.6, mask_seed=9),
        # a training step on three packed clips of a ragged grid, causal, capped and biased
        _case("scored-step-9Ktok", "scored_step", (9, 30, 33), (2, 8, 8), 128, 8, 128, "bf16", cap=30.0, bias=True, prefix=1, docs=3, reach=0.8, mask_seed=10),
        # a training step with head dim 64 and nothing but the sparse layout
        _case("scored-step-d64-8Ktok", "scored_step", (8, 32, 32), (1, 8, 8), 0, 12, 64, "bf16", batch=2, reach=0.5, mask_seed=11),
        # the largest training step: 20K tokens
        _case("scored-step-20Ktok", "scored_step", (13, 30, 52), (1, 8, 8), 128, 6, 128, "bf16", docs=1, reach=0.7, mask_seed=12),
    ]


def draw(rng):
    limits = {}
    for c in listed():
        w = work(c)
        for key in ("flops", "bytes"):
            limits[_family(c), key] = max(limits.get((_family(c), key), 0), w[key])

    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        op = rng.choice(["rotate", "rotate_back", "norm", "norm_step", "scored", "scored", "scored_step", "scored_step"])
        grid = (log_int(1, 32), log_int(1, 60), log_int(4, 104))
        heads, batch, docs = log_int(1, 40), rng.choice([1, 1, 1, 2]), rng.choice([0, 1, 2, 3])
        if op.startswith("scored"):
            tile, head_dim, dtype = rng.choice([(1, 8, 8), (2, 4, 8), (2, 8, 8), (2, 8, 8), (1, 8, 16), (4, 4, 8)]), rng.choice([64, 128]), "bf16"
        else:
            tile = rng.choice([(1, 4, 4), (1, 8, 8), (2, 2, 4), (1, 6, 10), (2, 4, 8), (2, 8, 8), (3, 5, 7)])
            head_dim, dtype = rng.choice([32, 64, 64, 80, 96, 128, 128, 128]), rng.choice(["f32", "bf16", "bf16", "bf16"])
        case = _case(None, op, grid, tile, rng.choice([0, 1, 2, 3]) * tile[0] * tile[1] * tile[2], heads, head_dim, dtype, batch=batch, docs=min(docs, grid[0]),
                     mask_seed=rng.randrange(1 << 30))
        if op.startswith("scored"):
            case |= dict(cap=rng.choice([0.0, 15.0, 30.0, 50.0]), bias=rng.random() < 0.5, prefix=rng.choice([-1, -1, 0, 1, 3]), reach=round(rng.uniform(0.2, 1.0), 2))
            if batch * heads * _tokens(case) ** 2 > (5e9 if op == "scored" else 2.5e9):  # the scores of a plain form have to fit the card
                continue
        else:
            case |= dict(rotated=rng.choice([head_dim, head_dim, head_dim // 2, head_dim // 8 * 6]), pairing=rng.choice(["half", "interleaved"]),
                         method=rng.choice(["linear", "base", "bands"]), stretch=rng.choice([1.0, 2.0, 4.0]), token_major=rng.random() < 0.5, tiled=rng.random() < 0.75)
        w = work(case)
        if any(w[key] > limits[_family(case), key] for key in ("flops", "bytes")) or w["bytes"] < 50_000:
            continue
        return case


def _family(case):
    return case["op"] if case["op"].startswith("scored") else "rows"


# ---- geometry, masks and positions ------------------------------------------------------------------

def _tiles(case):
    return tuple(-(-case[n] // case[t]) for n, t in (("T", "tt"), ("H", "th"), ("W", "tw")))


def _tile_tokens(case):
    return case["tt"] * case["th"] * case["tw"]


def _tokens(case):
    return case["T"] * case["H"] * case["W"] + case["n_text"]


def _padded(case):
    return math.prod(_tiles(case)) * _tile_tokens(case) + case["n_text"]


def _head_groups(case):
    """Per head (max tile-frame distance, window, window) groups: local, cross-shaped and global heads; the row operators read no tile lists."""
    if not case["op"].startswith("scored"):
        return [[(0, (0, 0), ABSENT)]] * case["heads"]
    nT, nH, nW = _tiles(case)
    heads = []
    for h in range(case["heads"]):
        r = random.Random(f"{case['mask_seed']}/{h}")
        kind = r.choice(["local", "cross", "global"])
        windows = {"local": ((2, 2), ABSENT), "cross": ((0, nW - 1), (nH - 1, 0)), "global": ((nH - 1, nW - 1), ABSENT)}[kind]
        far = r.randint(0, max(0, math.ceil(case["reach"] * (nT - 1))))
        heads.append([(far, *windows)] + ([(far + 1, (1, 1), ABSENT)] if far + 1 < nT else []))
    return heads


def _keep(case):
    """bool [heads, n, n]: key tiles that each query tile keeps; text tiles keep and are kept."""
    nT, nH, nW = _tiles(case)
    n_vid = nT * nH * nW
    n = n_vid + case["n_text"] // _tile_tokens(case)
    ids = np.arange(n_vid)
    dist = [np.abs(c[:, None] - c[None, :]) for c in (ids // (nH * nW), ids // nW % nH, ids % nW)]
    keep = np.ones((case["heads"], n, n), dtype=bool)
    for h, groups in enumerate(_head_groups(case)):
        video, last = np.zeros((n_vid, n_vid), dtype=bool), -1
        for max_dt, a, b in groups:
            inside = ((dist[1] <= a[0]) & (dist[2] <= a[1])) | ((dist[1] <= b[0]) & (dist[2] <= b[1]))
            video |= inside & (dist[0] > last) & (dist[0] <= max_dt)
            last = max_dt
        keep[h, :n_vid, :n_vid] = video
    return keep


def _places(case):
    """Position in tile order of every natural-order token."""
    nT, nH, nW = _tiles(case)
    t, y, x = np.meshgrid(np.arange(case["T"]), np.arange(case["H"]), np.arange(case["W"]), indexing="ij")
    tile = ((t // case["tt"]) * nH + y // case["th"]) * nW + x // case["tw"]
    slot = ((t % case["tt"]) * case["th"] + y % case["th"]) * case["tw"] + x % case["tw"]
    return np.concatenate([(tile * _tile_tokens(case) + slot).reshape(-1), nT * nH * nW * _tile_tokens(case) + np.arange(case["n_text"])])


def _clips(case):
    """First frame of each of the clips that share the grid."""
    r = random.Random(f"{case['mask_seed']}/clips")
    return [0] + sorted(r.sample(range(1, case["T"]), max(1, case["docs"]) - 1))


def _line(case):
    """Per frame, then per text token: (document, place, limit).  A clip's prompt stands at its first frame; the last quarter of the text is padding."""
    starts = _clips(case)
    first = np.array([max(s for s in starts if s <= t) for t in range(case["T"])])
    doc = np.array([max(i for i, s in enumerate(starts) if s <= t) for t in range(case["T"])])
    place = np.arange(case["T"])
    limit = np.maximum(place, first + case["prefix"] - 1)
    text = np.arange(case["n_text"])
    text_doc = text * len(starts) // max(1, case["n_text"])
    ends = np.array(starts[1:] + [case["T"]]) - 1
    text_doc_shown = np.where(text >= case["n_text"] - case["n_text"] // 4, -1, text_doc)
    return (np.concatenate([doc, text_doc_shown]), np.concatenate([place, np.array(starts)[text_doc]]),
            np.concatenate([limit, ends[text_doc]]))


def _per_token(case, values):
    """Values per frame and text token -> int32 [batch, tokens]."""
    frames, text = values[:case["T"]], values[case["T"]:]
    return np.tile(np.concatenate([np.repeat(frames, case["H"] * case["W"]), text]), (case["batch"], 1)).astype(np.int32)


def _visible_frames(case):
    """bool [frames + text, frames + text] by documents and limits alone."""
    doc, place, limit = _line(case)
    seen = np.ones((len(doc), len(doc)), dtype=bool)
    if case["docs"]:
        seen &= (doc[:, None] == doc[None, :]) & (doc[:, None] >= 0)
    if case["prefix"] >= 0:
        seen &= place[None, :] <= limit[:, None]
    return seen


def _pairs_within(length, tile, radius):
    """Pairs (i, j) of tokens on an axis whose tiles are at most `radius` apart."""
    sizes = np.array([min(tile, length - i) for i in range(0, length, tile)], dtype=np.int64)
    i = np.arange(len(sizes))
    return int(sizes @ (np.abs(i[:, None] - i[None, :]) <= radius) @ sizes)


def _visible_pairs(case):
    seen = _visible_frames(case).astype(np.int64)
    T, frame = case["T"], case["H"] * case["W"]
    text = int(seen[T:, T:].sum() + frame * (seen[:T, T:].sum() + seen[T:, :T].sum()))
    tile_frame = np.arange(T) // case["tt"]
    dist = np.abs(tile_frame[:, None] - tile_frame[None, :])
    total = 0
    for groups in _head_groups(case):
        last = -1
        for max_dt, a, b in groups:
            area = sum(_pairs_within(case["H"], case["th"], w[0]) * _pairs_within(case["W"], case["tw"], w[1]) for w in (a, b) if w != ABSENT)
            if b != ABSENT:
                area -= _pairs_within(case["H"], case["th"], min(a[0], b[0])) * _pairs_within(case["W"], case["tw"], min(a[1], b[1]))
            total += int(seen[:T, :T][(dist > last) & (dist <= max_dt)].sum()) * area
            last = max_dt
        total += text
    return case["batch"] * total


def work(case):
    """Tensors of real and padding tokens once; products over visible pairs (four per head channel and pair forwards, ten backwards) or a few operations per value."""
    real, padded, rows = _tokens(case), _padded(case), case["batch"] * case["heads"]
    row = case["head_dim"] * (2 if case["dtype"] == "bf16" else 4)
    there = padded if case["tiled"] else real
    op, values = case["op"], rows * real * case["head_dim"]
    if op in ("rotate", "rotate_back"):
        return {"bytes": rows * row * (real + there), "flops": 3 * values}
    if op == "norm":
        return {"bytes": 2 * rows * row * (real + there), "flops": 2 * 7 * values}
    if op == "norm_step":  # q and k, the rotated ones, their gradients, the gradients of q and k
        return {"bytes": 2 * rows * row * (2 * real + 2 * there), "flops": 2 * 20 * values}
    pairs = _visible_pairs(case)
    if op == "scored":
        return {"bytes": rows * padded * (4 * row + 4), "flops": 4 * case["head_dim"] * pairs}
    return {"bytes": rows * padded * (8 * row + 4), "flops": 14 * case["head_dim"] * pairs}  # q, k, v, the result and its gradient, three gradients


# ---- rotary positions -------------------------------------------------------------------------------

def _axes(case):
    """Channels of the frame, row and column axis, and how many positions each has: an eighth of the pairs for frames, the rest shared."""
    pairs = case["rotated"] // 2
    t = max(1, pairs // 8) if case["T"] > 1 or case["H"] == 1 else 0
    x = (pairs - t) // 2
    return (2 * t, 2 * (pairs - t - x), 2 * x), (case["T"], case["H"], case["W"])


def _frequencies(channels, positions, method, stretch):
    """Angle per position of each pair of an axis, in 64 bits; trained positions: as many as there are, divided by the stretch."""
    i = np.arange(channels // 2, dtype=np.float64)
    base = 10000.0
    if method == "base" and channels > 2:
        base = base * stretch ** (channels / (channels - 2))
    turn = base ** (-2 * i / channels) if channels else i
    if method == "linear":
        turn = turn / stretch
    if method == "bands":
        turns = positions / stretch * turn / (2 * math.pi)
        whole = np.clip((turns - 1.0) / (4.0 - 1.0), 0.0, 1.0)
        turn = whole * turn + (1 - whole) * turn / stretch
    return turn


def _positions(case):
    """int32 [batch, tokens, 3] or None: clips that share the grid begin at frame 0 each; a prompt's tokens are not rotated."""
    if not case["docs"]:
        return None
    starts = _clips(case)
    t = np.array([t - max(s for s in starts if s <= t) for t in range(case["T"])])
    grid = np.stack(np.meshgrid(t, np.arange(case["H"]), np.arange(case["W"]), indexing="ij"), axis=-1).reshape(-1, 3)
    return np.tile(np.concatenate([grid, np.full((case["n_text"], 3), -1)]), (case["batch"], 1, 1)).astype(np.int32)


def _angles(case):
    """float64 [batch or 1, tokens, rotated / 2]; zero for tokens that are not rotated."""
    channels, lengths = _axes(case)
    at = _positions(case)
    if at is None:
        grid = np.stack(np.meshgrid(*(np.arange(case[n]) for n in ("T", "H", "W")), indexing="ij"), axis=-1).reshape(-1, 3)
        at = np.concatenate([grid, np.full((case["n_text"], 3), -1)])[None]
    at = torch.from_numpy(at).to(DEVICE)
    parts = []
    for axis in range(3):
        turn = torch.from_numpy(_frequencies(channels[axis], lengths[axis], case["method"], case["stretch"])).to(DEVICE)
        parts.append(at[..., axis, None].clamp(min=0).double() * turn)
    return torch.cat(parts, dim=-1)


# ---- inputs -----------------------------------------------------------------------------------------

def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device=DEVICE)


def _natural(case, gen, gain=1.0, tokens=None, token_major=False):
    """[batch, heads, tokens, head_dim], unit noise times `gain` with a share that all tokens have; tokens first in memory if asked."""
    tokens = _tokens(case) if tokens is None else tokens
    b, h, d = case["batch"], case["heads"], case["head_dim"]
    x = torch.empty((b, tokens, h, d) if token_major else (b, h, tokens, d), dtype=DTYPES[case["dtype"]], device=DEVICE)
    for i in range(b):
        x[i] = gain * (_randn(gen, *x.shape[1:]) + 0.3 * _randn(gen, d))
    return x.transpose(1, 2) if token_major else x


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    op, places = case["op"], torch.from_numpy(_places(case)).to(DEVICE)
    state = {"case": case, "places": places, "padded": _padded(case)}

    def tile_order(x):
        y = x.new_zeros(x.shape[0], x.shape[1], _padded(case), x.shape[3])
        y[:, :, places] = x
        return y

    if op.startswith("scored"):
        state["q"], state["k"], state["v"] = (tile_order(_natural(case, gen, gain)) for gain in (2.0, 1.5, 1.0))
        if op == "scored_step":
            state["dout"] = tile_order(_natural(case, gen))
        doc, place, limit = (torch.from_numpy(_per_token(case, v)).to(DEVICE) for v in _line(case))
        slopes = (torch.arange(case["heads"], device=DEVICE) + 1) * (0.5 / case["heads"])
        state |= {"documents": doc if case["docs"] else None, "limits": limit if case["prefix"] >= 0 else None,
                  "positions": place if case["bias"] or case["prefix"] >= 0 else None, "slopes": slopes if case["bias"] else None}
    else:
        at = _positions(case)
        state["positions"] = None if at is None else torch.from_numpy(at).to(DEVICE)
        count = 1 if op.startswith("rotate") else 4 if op == "norm_step" else 2
        for i, name in enumerate(("q", "k", "dq", "dk")[:count]):
            x = _natural(case, gen, token_major=case["token_major"] and i < 2 and op != "rotate_back")
            state[name] = tile_order(x) if case["tiled"] and (i >= 2 or op == "rotate_back") else x
        if op.startswith("norm"):
            state["wq"], state["wk"] = ((1 + 0.2 * _randn(gen, case["head_dim"])).to(DTYPES[case["dtype"]]) for _ in range(2))
    if own:
        import paper_2508_12969_amd as ca
        state["layout"] = ca.compact_attn_build_layout(case["T"], case["H"], case["W"], (case["tt"], case["th"], case["tw"]), case["n_text"], case["batch"],
                                                       case["heads"], case["head_dim"], case["dtype"], _head_groups(case))
        ca.compact_attn_layout_upload(state["layout"])
        if not op.startswith("scored"):
            channels, lengths = _axes(case)
            state["rotary"] = ca.compact_attn_build_rotary(channels, lengths, pairing=case["pairing"], method=case["method"], stretch=case["stretch"],
                                                           trained=tuple(n / case["stretch"] for n in lengths), turns=(1.0, 4.0))
            ca.compact_attn_rotary_upload(state["rotary"])
    elif op.startswith("scored"):
        state["keep"] = torch.from_numpy(_keep(case)).to(DEVICE)
    else:
        angles = _angles(case)[:, None]
        state["cos"], state["sin"] = angles.cos().float(), angles.sin().float()
    return state


# ---- one pass ---------------------------------------------------------------------------------------

def run(state):
    op = state["case"]["op"]
    if own:
        return _run_own(state)
    if op.startswith("rotate"):
        return _rotate_plain(state)
    return _norm_plain(state) if op.startswith("norm") else _scored_plain(state)


def _run_own(state):
    import paper_2508_12969_amd as ca
    case, layout = state["case"], state["layout"]
    op = case["op"]
    if op.startswith("scored"):
        how = dict(cap=case["cap"], slopes=state["slopes"], positions=state["positions"], limits=state["limits"], documents=state["documents"])
        q, k, v = state["q"], state["k"], state["v"]
        out, lse = ca.compact_attn_forward_scored(q, k, v, layout, **how)
        if op == "scored":
            return out, lse
        return out, lse, *ca.compact_attn_backward_scored(state["dout"], q, k, v, out, lse, layout, **how)
    how = dict(positions=state["positions"], tiled=case["tiled"])
    if op.startswith("rotate"):
        return ca.compact_attn_rotate(state["q"], layout, state["rotary"], transpose=op == "rotate_back", **how)
    inputs = state["q"], state["k"], state["wq"], state["wk"], layout, state["rotary"], EPS
    outputs = ca.compact_attn_norm_rotate(*inputs, **how)
    if op == "norm":
        return outputs
    return *outputs, *ca.compact_attn_norm_rotate_backward(state["dq"], state["dk"], *inputs, **how)


def _into_tiles(state, x):
    if not state["case"]["tiled"]:
        return x
    y = x.new_zeros(*x.shape[:2], state["padded"], x.shape[3])
    y[:, :, state["places"]] = x
    return y


def _out_of_tiles(state, x):
    return x[:, :, state["places"]] if state["case"]["tiled"] else x


def _turn(state, x, sin):
    """Every pair of channels of the rotated part turned by its angle."""
    case, cos = state["case"], state["cos"]
    part, rest = x[..., :case["rotated"]], x[..., case["rotated"]:]
    if case["pairing"] == "half":
        a, b = part.chunk(2, dim=-1)
        return torch.cat([a * cos - b * sin, a * sin + b * cos, rest], dim=-1)
    a, b = part[..., 0::2], part[..., 1::2]
    return torch.cat([torch.stack([a * cos - b * sin, a * sin + b * cos], dim=-1).flatten(-2), rest], dim=-1)


def _rotate_plain(state):
    x = state["q"]
    if state["case"]["op"] == "rotate":
        return _into_tiles(state, _turn(state, x.float(), state["sin"]).to(x.dtype))
    return _turn(state, _out_of_tiles(state, x).float(), -state["sin"]).to(x.dtype)


def _normed(x):
    x = x.float()
    r = torch.rsqrt(x.square().mean(dim=-1, keepdim=True) + EPS)
    return x * r, r


def _norm_gradient(state, x, w, dy):
    n, r = _normed(x)
    du = _turn(state, _out_of_tiles(state, dy).float(), -state["sin"])
    dn = du * w.float()
    dx = r * (dn - n * (dn * n).mean(dim=-1, keepdim=True))
    return dx.to(x.dtype), (du * n).sum(dim=(0, 1, 2))


def _norm_plain(state):
    one = lambda x, w: _into_tiles(state, _turn(state, _normed(x)[0] * w.float(), state["sin"]).to(x.dtype))
    q, k = one(state["q"], state["wq"]), one(state["k"], state["wk"])
    if state["case"]["op"] == "norm":
        return q, k
    dq, dwq = _norm_gradient(state, state["q"], state["wq"], state["dq"])
    dk, dwk = _norm_gradient(state, state["k"], state["wk"], state["dk"])
    return q, k, dq, dk, dwq, dwk


def _scored_plain(state):
    case, places = state["case"], state["places"]
    tile = places // _tile_tokens(case)
    q, k, v = (state[n][:, :, places].float() for n in ("q", "k", "v"))
    scale = case["head_dim"] ** -0.5
    visible = state["keep"][:, tile][:, :, tile][None]
    if state["documents"] is not None:
        doc = state["documents"][:, None]
        visible = visible & (doc[..., :, None] == doc[..., None, :]) & (doc[..., :, None] >= 0)
    if state["limits"] is not None:
        visible = visible & (state["positions"][:, None, None, :] <= state["limits"][:, None, :, None])
    s = torch.matmul(q, k.transpose(-1, -2)).mul_(scale)
    if case["cap"]:
        bent = torch.tanh_(s.div_(case["cap"]))
        s = bent * case["cap"]
    if state["slopes"] is not None:
        at = state["positions"].float()[:, None]
        s -= state["slopes"][:, None, None] * (at[..., :, None] - at[..., None, :]).abs_()
    s.masked_fill_(~visible, -math.inf)
    m = s.amax(dim=-1, keepdim=True).clamp_(min=-1e30)
    p = s.sub_(m).exp_()
    total = p.sum(dim=-1, keepdim=True)
    lse = (m + total.log())[..., 0]
    p *= torch.where(total > 0, 1 / total, torch.zeros_like(total))
    out = torch.matmul(p, v)

    def tile_order(x, empty=0.0):
        y = torch.full((*x.shape[:2], state["padded"], *x.shape[3:]), empty, dtype=x.dtype, device=x.device)
        y[:, :, places] = x
        return y

    results = [tile_order(out.to(state["q"].dtype)), tile_order(lse, -math.inf)]
    if case["op"] == "scored":
        return tuple(results)
    do = state["dout"][:, :, places].float()
    dv = torch.matmul(p.transpose(-1, -2), do)
    ds = torch.matmul(do, v.transpose(-1, -2)).sub_((do * out).sum(dim=-1, keepdim=True)).mul_(p).mul_(scale)
    if case["cap"]:
        ds *= bent.square_().neg_().add_(1)
    dq, dk = torch.matmul(ds, k), torch.matmul(ds.transpose(-1, -2), q)
    return (*results, *(tile_order(x.to(state["q"].dtype)) for x in (dq, dk, dv)))


# ---- the same from the definitions, in 64 bits --------------------------------------------------------

def exact(case, seed):
    if case["op"].startswith("scored"):
        return _scored_exact(case, seed)
    state = prepare(case, seed)
    # a pair as a complex number, turned by exp(i angle)
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEVICE), _angles(case))

    def turned(x, by):
        head, rest = x[..., :case["rotated"]], x[..., case["rotated"]:]
        pairs = head.unflatten(-1, (2, -1)).transpose(-1, -2) if case["pairing"] == "half" else head.unflatten(-1, (-1, 2))
        pairs = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * by)
        return torch.cat([(pairs.transpose(-1, -2) if case["pairing"] == "half" else pairs).flatten(-2), rest], dim=-1)

    places, op = state["places"], case["op"]

    def per_head(count, fn):
        """fn(batch entry, head) -> values of one plane, put together."""
        planes = [[fn(b, h) for h in range(case["heads"])] for b in range(case["batch"])]
        return [torch.stack([torch.stack([plane[i] for plane in row]) for row in planes]) for i in range(count)]

    def there(x):
        if not case["tiled"]:
            return x
        y = x.new_zeros(state["padded"], x.shape[1])
        y[places] = x
        return y

    def back(x):
        return x.double()[places] if case["tiled"] else x.double()

    angle = lambda b: turn[b if turn.shape[0] > 1 else 0]
    if op == "rotate":
        return per_head(1, lambda b, h: [there(turned(state["q"][b, h].double(), angle(b)))])[0]
    if op == "rotate_back":
        return per_head(1, lambda b, h: [turned(back(state["q"][b, h]), angle(b).conj())])[0]
    if case["batch"] * case["heads"] * _tokens(case) * case["head_dim"] * 8 > 1.6e10:  # in 64 bits, several times over: too much
        return None

    def forward(name):
        def one(b, h):
            x = state[name][b, h].double()
            return [there(turned(x / (x.pow(2).sum(-1, keepdim=True) / case["head_dim"] + EPS).sqrt() * state["w" + name].double(), angle(b)))]
        return per_head(1, one)[0]

    def backward(name):
        def one(b, h):
            x, w = state[name][b, h].double(), state["w" + name].double()
            du = turned(back(state["d" + name][b, h]), angle(b).conj())
            rms = (x.pow(2).sum(-1, keepdim=True) / case["head_dim"] + EPS).sqrt()
            dx = du * w / rms - x * (du * w * x).sum(-1, keepdim=True) / (case["head_dim"] * rms.pow(3))
            return [dx, (du * x / rms).sum(0)]
        dx, dw = per_head(2, one)
        return dx, dw.sum(dim=(0, 1))

    if op == "norm":
        return forward("q"), forward("k")
    (dq, dwq), (dk, dwk) = backward("q"), backward("k")
    return forward("q"), forward("k"), dq, dk, dwq, dwk


def _scored_exact(case, seed):
    if (4 if case["op"] == "scored" else 14) * case["batch"] * case["heads"] * _tokens(case) ** 2 * case["head_dim"] > 1e14:
        return None
    state = prepare(case, seed)
    places, scale, step = state["places"], 1 / math.sqrt(case["head_dim"]), case["op"] == "scored_step"
    keep, tile = torch.from_numpy(_keep(case)).to(DEVICE), places // _tile_tokens(case)
    seen = torch.from_numpy(_visible_frames(case)).to(DEVICE)
    line = torch.from_numpy(np.concatenate([np.repeat(np.arange(case["T"]), case["H"] * case["W"]), case["T"] + np.arange(case["n_text"])])).to(DEVICE)
    place = torch.from_numpy(_line(case)[1]).to(DEVICE).double()[line]
    shape = (case["batch"], case["heads"], state["padded"], case["head_dim"])
    out, *grads = (torch.zeros(shape, dtype=torch.float64, device=DEVICE) for _ in range(4 if step else 1))
    lse = torch.full(shape[:3], -math.inf, dtype=torch.float64, device=DEVICE)
    rows = max(1, (1 << 28) // len(line))  # queries at a time
    for b in range(case["batch"]):
        for h in range(case["heads"]):
            q, k, v = (state[n][b, h].double()[places] for n in ("q", "k", "v"))
            dk, dv = torch.zeros_like(k), torch.zeros_like(v)
            for lo in range(0, len(line), rows):
                at = slice(lo, lo + rows)
                s = q[at] @ k.t() * scale
                steep = 1
                if case["cap"]:
                    steep = 1 / torch.cosh(s / case["cap"]) ** 2
                    s = case["cap"] * torch.tanh(s / case["cap"])
                if case["bias"]:
                    s = s - state["slopes"][h].double() * (place[at, None] - place[None, :]).abs()
                s = torch.where(seen[line[at]][:, line] & keep[h][tile[at]][:, tile], s, -math.inf)
                row = torch.logsumexp(s, dim=1)
                p = torch.where(row[:, None] > -math.inf, (s - row[:, None]).exp(), 0.0)
                del s
                out[b, h, places[at]] = p @ v
                lse[b, h, places[at]] = row
                if step:
                    do = state["dout"][b, h].double()[places[at]]
                    dv += p.t() @ do
                    dp = do @ v.t()
                    ds = p * (dp - (p * dp).sum(1, keepdim=True)) * steep * scale
                    del dp, p
                    grads[0][b, h, places[at]] = ds @ k
                    dk += ds.t() @ q[at]
            if step:
                grads[1][b, h, places], grads[2][b, h, places] = dk, dv
    return (out, lse, *grads)
