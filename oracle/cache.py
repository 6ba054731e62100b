"""A paged cache of keys and values from its definitions, in 64 bits (oracle side; test infrastructure).

Sequences are lists of tokens; pages are looked up token by token.
"""
import math

import numpy as np


def place_of(table, s, token, page_tokens, num_pages):
    """(page, slot) of a token, None where it is not there."""
    if token < 0 or token // page_tokens >= table.shape[1]:
        return None
    page = int(table[s, token // page_tokens])
    return (page, token % page_tokens) if 0 <= page < num_pages else None


def frames(places, origin, span):
    places = np.asarray(places)
    return np.where(places >= origin, (places - origin) // span, -1)


def seen_by(length, new, origin, span, causal, window, words=None):
    """bool [new, length], and the frames of the new tokens' rows and of all tokens.  words: bits of a tree's drafts, one a new token."""
    base = length - new
    tokens = np.arange(length)
    own = base + np.arange(new)
    places = tokens.copy()
    if words is not None:
        words = [int(w) & ((1 << min(new, 64)) - 1) for w in words]
        own = np.array([base + max(bin(w).count("1"), 1) - 1 for w in words], dtype=np.int64)
        for i in range(max(0, -base), new):
            places[base + i] = own[i]
    row_frame, token_frame = frames(own, origin, span), frames(places, origin, span)
    seen = np.ones((new, length), dtype=bool)
    if causal:
        seen &= token_frame[None, :] <= row_frame[:, None]
    if window:
        seen &= (token_frame[None, :] > row_frame[:, None] - window) | (tokens[None, :] < origin)
    if words is not None:
        for i in range(new):
            for j in range(max(0, -base), new):
                seen[i, base + j] = j < 64 and bool(words[i] >> j & 1)
    for i in range(new):
        if base + i < 0:
            seen[i] = False
    return seen, row_frame, token_frame


def attend(q, k, v, seen, scale, cap=0.0, slope=None, row_frame=None, token_frame=None):
    """One query head of one sequence: q [new, D], k and v [length, D] -> (out, lse, weights, scores' sizes before they are bent)."""
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))
    k, v = np.where(seen.any(0)[:, None], k, 0.0), np.where(seen.any(0)[:, None], v, 0.0)
    s = q @ k.T * scale
    size = np.abs(q) @ np.abs(k).T * abs(scale)
    if cap:
        s = cap * np.tanh(s / cap)
    if slope is not None:
        s = s - slope * np.abs(row_frame[:, None] - token_frame[None, :])
    s = np.where(seen, s, -math.inf)
    top = np.max(s, axis=1, keepdims=True, initial=-math.inf)
    top = np.where(np.isfinite(top), top, 0.0)
    e = np.exp(s - top)
    total = e.sum(axis=1, keepdims=True)
    p = np.divide(e, total, out=np.zeros_like(e), where=total > 0)
    with np.errstate(divide="ignore"):
        lse = (np.log(total) + top)[:, 0]
    return p @ v, lse, p, size


def keep(rows, path):
    """New tokens of one sequence after an accepted path: rows [new, ...]."""
    out = rows.copy()
    for j, i in enumerate(path):
        if 0 <= i < len(rows) and j < len(rows):
            out[j] = rows[i]
    return out
