"""Rotary positions, and norms of queries and keys with the rotation in the same pass: argument marshalling for the entry points of
that part of include/compact_attn.h, as binding.py does it for the others.  Tensors are device buffers; there is no autograd here, gradients have
calls of their own."""
import contextlib
import ctypes

from . import binding
from .binding import CA_ERR_ALLOC, CompactAttnError, _check, _lend, _stream_ptr, _torch_dtype, _torch_stream, load_library

CA_PAIRINGS = {"interleaved": 0, "half": 1}
CA_STRETCHES = {"linear": 0, "base": 1, "bands": 2}


class ca_rotary_axis(ctypes.Structure):
    _fields_ = [("channels", ctypes.c_int32), ("positions", ctypes.c_int32), ("base", ctypes.c_double), ("stretch", ctypes.c_double),
                ("trained", ctypes.c_double), ("turns_low", ctypes.c_double), ("turns_high", ctypes.c_double)]


class ca_strides(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int64), ("head", ctypes.c_int64), ("token", ctypes.c_int64)]


class ca_where(ctypes.Structure):
    _fields_ = [("origin", ctypes.c_int32 * 3), ("positions", ctypes.c_void_p)]


class ca_norm(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("q_strides", ctypes.POINTER(ca_strides)), ("k_strides", ctypes.POINTER(ca_strides)),
                ("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p), ("rotary", ctypes.c_void_p), ("where", ctypes.POINTER(ca_where)),
                ("eps", ctypes.c_float), ("tiled", ctypes.c_int32)]


class Rotary:
    """Owner of a ca_rotary*."""

    def __init__(self, handle, channels, lengths):
        self.handle = handle
        self.channels, self.lengths = channels, lengths

    def free(self):
        if self.handle is not None:
            load_library().compact_attn_free_rotary(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.free()
        except Exception:
            pass


def _three(value):
    return tuple(value) if isinstance(value, (tuple, list)) else (value,) * 3


def compact_attn_build_rotary(channels, lengths, pairing="interleaved", base=10000.0, stretch=1.0, method="linear", trained=0.0, turns=(1.0, 32.0),
                              magnitude=1.0):
    """Table of angles for three axes (frame, row, column).  channels: rotated channels of each axis; lengths: how many positions each has.
    base, stretch, trained: a number for all axes or one for each; method "linear", "base" or "bands" says what a stretch does (compact_attn.h);
    turns: (low, high) of "bands"."""
    if pairing not in CA_PAIRINGS:
        raise ValueError(f"pairing must be one of {tuple(CA_PAIRINGS)}")
    if method not in CA_STRETCHES:
        raise ValueError(f"method must be one of {tuple(CA_STRETCHES)}")
    per_axis = [_three(v) for v in (channels, lengths, base, stretch, trained)]
    if any(len(v) != 3 for v in per_axis):
        raise ValueError("channels, lengths, base, stretch and trained have a value for each of three axes, or one for all")
    axes = (ca_rotary_axis * 3)(*(ca_rotary_axis(*v, *turns) for v in zip(*per_axis)))
    handle = ctypes.c_void_p()
    _check(load_library().compact_attn_build_rotary(axes, CA_PAIRINGS[pairing], CA_STRETCHES[method], magnitude, ctypes.byref(handle)))
    return Rotary(handle, per_axis[0], per_axis[1])


def compact_attn_rotary_angles(rotary, axis):
    """float32 [positions, channels / 2, 2] copied out of the table: (cos, sin) of an axis; None for an axis without channels."""
    import numpy as np
    at = ctypes.POINTER(ctypes.c_float)()
    _check(load_library().compact_attn_rotary_angles(rotary.handle, axis, ctypes.byref(at)))
    return np.ctypeslib.as_array(at, shape=(rotary.lengths[axis], rotary.channels[axis] // 2, 2)).copy() if at else None


def compact_attn_rotary_upload(rotary):
    _check(load_library().compact_attn_rotary_upload(rotary.handle))


def compact_attn_free_rotary(rotary):
    rotary.free()


def _on_current_device(t, name):
    import torch
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.get_device() != torch._C._cuda_getDevice():
        raise ValueError(f"{name} is on {t.device}, the current device is cuda:{torch.cuda.current_device()}")


def _check_rows(t, layout, padded, name):
    """A tensor of rows; the strides to hand over, None where it is contiguous."""
    _on_current_device(t, name)
    if t.dtype != _torch_dtype(layout):
        raise ValueError(f"{name} has dtype {t.dtype}, layout expects {_torch_dtype(layout)}")
    if t.shape != layout.shape(padded):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {layout.shape(padded)}")
    if t.is_contiguous():
        return None
    if padded:
        raise ValueError(f"{name} is in tile order and must be contiguous")
    if t.stride(3) != 1 and t.shape[3] > 1:
        raise ValueError(f"channels of {name} must be contiguous")
    return ca_strides(*(t.stride(i) if t.shape[i] > 1 else 0 for i in range(3)))


def _table(rotary):
    if rotary is not None and rotary.handle is None:
        raise ValueError("rotary has been freed")
    return None if rotary is None else rotary.handle


def _where(layout, origin, positions):
    if len(origin) != 3:
        raise ValueError("origin has a value for each of three axes")
    if positions is None:
        return None if tuple(origin) == (0, 0, 0) else ca_where((ctypes.c_int32 * 3)(*origin), None)
    import torch
    _on_current_device(positions, "positions")
    expected = (layout.problem.batch, layout.n_tokens_real, 3)
    if positions.shape != expected or positions.dtype != torch.int32 or not positions.is_contiguous():
        raise ValueError(f"positions must be a contiguous int32 tensor of shape {expected}")
    return ca_where((ctypes.c_int32 * 3)(*origin), positions.data_ptr())


_here = contextlib.nullcontext()


def _on(stream, device):
    """Where results of a call on `stream` are allocated: from that stream's memory."""
    import torch
    return _here if stream is None else torch.cuda.stream(_torch_stream(stream, device))


def compact_attn_rotate(src, layout, rotary, origin=(0, 0, 0), positions=None, tiled=True, transpose=False, out=None, stream=None):
    """Rotary positions.  transpose=False: src [batch, heads, N_real, D] in natural order, any strides with contiguous channels, -> rotated, in
    tile order (tiled) or natural order.  transpose=True: src in tile (tiled) or natural order -> natural order, turned back: the gradient."""
    tiled, transpose = bool(tiled), bool(transpose)
    padded_in, padded_out = tiled and transpose, tiled and not transpose
    src_strides = _check_rows(src, layout, padded_in, "src")
    dst_strides = None
    if out is not None:
        dst_strides = _check_rows(out, layout, padded_out, "out")
    else:
        with _on(stream, src.device):
            out = src.new_empty(layout.shape(padded_out))
    where = _where(layout, origin, positions)
    _check(load_library().compact_attn_rotate(src.data_ptr(), src_strides, out.data_ptr(), dst_strides, layout.handle, _table(rotary), where, int(tiled),
                                              int(transpose), _stream_ptr(stream)))
    return out


def _norm(q, k, q_weight, k_weight, layout, rotary, eps, origin, positions, tiled):
    strides = [_check_rows(t, layout, False, name) for name, t in (("q", q), ("k", k))]
    for name, w in (("q_weight", q_weight), ("k_weight", k_weight)):
        if w is not None:
            _on_current_device(w, name)
            if w.dtype != _torch_dtype(layout) or tuple(w.shape) != (layout.problem.head_dim,) or not w.is_contiguous():
                raise ValueError(f"{name} must be a contiguous {_torch_dtype(layout)} tensor of {layout.problem.head_dim} elements")
    pointers = [None if s is None else ctypes.pointer(s) for s in strides]
    weights = [None if w is None else w.data_ptr() for w in (q_weight, k_weight)]
    where = _where(layout, origin, positions)
    return ca_norm(q.data_ptr(), k.data_ptr(), *pointers, *weights, _table(rotary), None if where is None else ctypes.pointer(where), eps,
                   int(bool(tiled)))


def compact_attn_norm_rotate(q, k, q_weight, k_weight, layout, rotary, eps=1e-6, origin=(0, 0, 0), positions=None, tiled=True, out=None, stream=None):
    """Norm of every query and key head, times the weight [D] (None: ones), and the rotation (rotary None: none) in one pass.  q, k: natural order, any strides
    with contiguous channels -> (q, k) contiguous in tile order (tiled) or natural order.  out: a pair of tensors to write to."""
    norm = _norm(q, k, q_weight, k_weight, layout, rotary, eps, origin, positions, tiled)
    if out is None:
        with _on(stream, q.device):
            out = q.new_empty(layout.shape(tiled)), q.new_empty(layout.shape(tiled))
    else:
        for name, t in zip(("q of out", "k of out"), out, strict=True):
            if _check_rows(t, layout, bool(tiled), name) is not None:
                raise ValueError(f"{name} must be contiguous")
    _check(load_library().compact_attn_norm_rotate(norm, out[0].data_ptr(), out[1].data_ptr(), layout.handle, _stream_ptr(stream)))
    return tuple(out)


def compact_attn_norm_rotate_backward(dq_out, dk_out, q, k, q_weight, k_weight, layout, rotary, eps=1e-6, origin=(0, 0, 0), positions=None, tiled=True,
                                      out=None, stream=None):
    """Gradients of compact_attn_norm_rotate: dq_out, dk_out as its results, the other arguments as given to it -> (dq, dk, dq_weight, dk_weight).  dq and dk are
    laid out as q and k where these are dense; out: a pair of tensors to write them to (natural order, any strides with contiguous
    channels).  The weight gradients are float32 [D], None where neither weight is given."""
    import torch
    norm = _norm(q, k, q_weight, k_weight, layout, rotary, eps, origin, positions, tiled)
    for name, t in (("dq_out", dq_out), ("dk_out", dk_out)):
        if _check_rows(t, layout, bool(tiled), name) is not None:
            raise ValueError(f"{name} must be contiguous")
    weighted = q_weight is not None or k_weight is not None
    with _on(stream, q.device):
        if out is None:
            out = torch.empty_like(q), torch.empty_like(k)
        dw = q.new_empty((2, layout.problem.head_dim), dtype=torch.float32) if weighted else None
    strides = [_check_rows(t, layout, False, name) for name, t in zip(("dq of out", "dk of out"), out, strict=True)]
    need, workspace = ctypes.c_int64(), None
    if weighted:
        _check(load_library().compact_attn_norm_workspace(layout.handle, need))
        workspace = _lend(q, need.value, stream)
        if workspace is None or workspace is NotImplemented:
            raise CompactAttnError(CA_ERR_ALLOC, f"no memory for a workspace of {need.value} bytes, or a capture that torch does not run")
    _check(load_library().compact_attn_norm_rotate_backward(norm, dq_out.data_ptr(), dk_out.data_ptr(), out[0].data_ptr(), strides[0], out[1].data_ptr(), strides[1],
                                                            dw[0].data_ptr() if weighted else None, dw[1].data_ptr() if weighted else None, layout.handle,
                                                            workspace.data_ptr() if weighted else None, need.value, _stream_ptr(stream)))
    return (*out, dw[0] if q_weight is not None else None, dw[1] if k_weight is not None else None)


def _declare(lib):
    vp, i32, i64p = ctypes.c_void_p, ctypes.c_int32, ctypes.POINTER(ctypes.c_int64)
    st, wh, nm = ctypes.POINTER(ca_strides), ctypes.POINTER(ca_where), ctypes.POINTER(ca_norm)
    lib.compact_attn_build_rotary.argtypes = [ctypes.POINTER(ca_rotary_axis), i32, i32, ctypes.c_double, ctypes.POINTER(vp)]
    lib.compact_attn_rotary_angles.argtypes = [vp, i32, ctypes.POINTER(ctypes.POINTER(ctypes.c_float))]
    lib.compact_attn_rotary_upload.argtypes = [vp]
    lib.compact_attn_free_rotary.argtypes = [vp]
    lib.compact_attn_free_rotary.restype = None
    lib.compact_attn_rotate.argtypes = [vp, st, vp, st, vp, vp, wh, i32, i32, vp]
    lib.compact_attn_norm_rotate.argtypes = [nm, vp, vp, vp, vp]
    lib.compact_attn_norm_workspace.argtypes = [vp, i64p]
    lib.compact_attn_norm_rotate_backward.argtypes = [nm, vp, vp, vp, st, vp, st, vp, vp, vp, vp, ctypes.c_int64, vp]


binding._declarations.append(_declare)
