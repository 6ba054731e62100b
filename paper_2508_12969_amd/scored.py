"""Scored attention (capped, biased and masked scores) and its gradients: argument marshalling for the entry points of that part of
include/compact_attn.h, as binding.py does it for the others."""
import ctypes

from . import binding
from .binding import CA_ERR_ALLOC, CompactAttnError, _check, _check_tensor, _lend, _stream_ptr, load_library
from .rotary import _on, _on_current_device


class ca_scores(ctypes.Structure):
    _fields_ = [("cap", ctypes.c_float), ("slopes", ctypes.c_void_p), ("positions", ctypes.c_void_p), ("limits", ctypes.c_void_p), ("documents", ctypes.c_void_p)]


def _scores(layout, cap, slopes, positions, limits, documents):
    import torch
    p = layout.problem
    for name, t, shape, dtype in (("slopes", slopes, (p.num_heads,), torch.float32), ("positions", positions, (p.batch, layout.n_tokens_real), torch.int32),
                                  ("limits", limits, (p.batch, layout.n_tokens_real), torch.int32),
                                  ("documents", documents, (p.batch, layout.n_tokens_real), torch.int32)):
        if t is None:
            continue
        _on_current_device(t, name)
        if t.shape != shape or t.dtype != dtype or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {shape}")
    return ca_scores(cap, *(None if t is None else t.data_ptr() for t in (slopes, positions, limits, documents)))


def _check_tiles(t, layout, name):
    _on_current_device(t, name)
    _check_tensor(t, layout, True, name)


def _check_lse(t, layout, name):
    import torch
    _on_current_device(t, name)
    if t.shape != layout.shape(True)[:3] or t.dtype != torch.float32 or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous float32 tensor of shape {layout.shape(True)[:3]}")


def _workspace(layout, scores, backward, q, stream):
    kind = backward, bool(scores.slopes), bool(scores.limits or scores.documents)   # all that its size depends on
    need = layout._scored_workspace.get(kind)
    if need is None:
        size = ctypes.c_int64()
        _check(load_library().compact_attn_scored_workspace(layout.handle, scores, backward, size))
        need = layout._scored_workspace[kind] = size.value
    if need == 0:
        return None, 0
    workspace = _lend(q, need, stream)
    if workspace is None or workspace is NotImplemented:
        raise CompactAttnError(CA_ERR_ALLOC, f"no memory for a workspace of {need} bytes, or a capture that torch does not run")
    return workspace, need


def compact_attn_forward_scored(q, k, v, layout, cap=0.0, slopes=None, positions=None, limits=None, documents=None, out=None, stream=None):
    """Sparse attention over tile-ordered, padded q/k/v [batch, heads, N_pad, D] with scores cap * tanh(s / cap) - slopes[head] * |position difference| (cap 0, slopes
    None: without), visible where documents are equal and not negative and a key's position is at most the query's limit.  slopes: float32
    [heads]; positions, limits, documents: int32 [batch, N_real] in natural order.  -> (out, lse), lse float32 [batch, heads, N_pad]; out: such a pair to write to."""
    for name, t in (("q", q), ("k", k), ("v", v)):
        _check_tiles(t, layout, name)
    scores = _scores(layout, cap, slopes, positions, limits, documents)
    if out is None:
        import torch
        with _on(stream, q.device):
            out = q.new_empty(q.shape), q.new_empty(q.shape[:3], dtype=torch.float32)
    else:
        _check_tiles(out[0], layout, "out")
        _check_lse(out[1], layout, "lse of out")
    workspace, need = _workspace(layout, scores, 0, q, stream)
    _check(load_library().compact_attn_forward_scored(q.data_ptr(), k.data_ptr(), v.data_ptr(), layout.handle, scores, out[0].data_ptr(), out[1].data_ptr(),
                                                      None if workspace is None else workspace.data_ptr(), need, _stream_ptr(stream)))
    return tuple(out)


def compact_attn_backward_scored(dout, q, k, v, out, lse, layout, cap=0.0, slopes=None, positions=None, limits=None, documents=None, grads=None, stream=None):
    """Gradients (dq, dk, dv) of compact_attn_forward_scored for the gradient dout of its first result, from its inputs and results and the same scores; all in tile
    order.  out and lse as that call left them, not merged from several (compact_attn.h); lse has no gradient.  grads: three tensors to write to."""
    for name, t in (("dout", dout), ("q", q), ("k", k), ("v", v), ("out", out)):
        _check_tiles(t, layout, name)
    _check_lse(lse, layout, "lse")
    scores = _scores(layout, cap, slopes, positions, limits, documents)
    if grads is None:
        with _on(stream, q.device):
            grads = tuple(q.new_empty(q.shape) for _ in range(3))
    else:
        for name, t in zip(("dq", "dk", "dv"), grads, strict=True):
            _check_tiles(t, layout, name)
    workspace, need = _workspace(layout, scores, 1, q, stream)
    _check(load_library().compact_attn_backward_scored(dout.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), lse.data_ptr(), layout.handle, scores,
                                                       *(t.data_ptr() for t in grads), None if workspace is None else workspace.data_ptr(), need, _stream_ptr(stream)))
    return tuple(grads)


def compact_attn_layout_upload_scored(layout, backward=True):
    """Makes the lists that scored calls walk over (backward: and those of the gradients) and copies them to the device (the first call does it otherwise, but not
    under capture)."""
    _check(load_library().compact_attn_layout_upload_scored(layout.handle, int(bool(backward))))


def _declare(lib):
    vp, i64 = ctypes.c_void_p, ctypes.c_int64
    sc = ctypes.POINTER(ca_scores)
    lib.compact_attn_scored_workspace.argtypes = [vp, sc, ctypes.c_int32, ctypes.POINTER(i64)]
    lib.compact_attn_forward_scored.argtypes = [vp, vp, vp, vp, sc, vp, vp, vp, i64, vp]
    lib.compact_attn_layout_upload_scored.argtypes = [vp, ctypes.c_int32]
    lib.compact_attn_backward_scored.argtypes = [vp, vp, vp, vp, vp, vp, vp, sc, vp, vp, vp, vp, i64, vp]


binding._declarations.append(_declare)
