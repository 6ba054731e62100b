"""A paged cache of keys and values: argument marshalling for the entry points of that part of include/compact_attn.h, as binding.py does it for the others."""
import ctypes

from . import binding
from .binding import CA_BF16, CA_ERR_ALLOC, CA_F32, CompactAttnError, _check, _lend, _stream_ptr, load_library
from .rotary import _on, _on_current_device, _table, ca_strides, ca_where


class ca_cache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("num_pages", ctypes.c_int64), ("page_tokens", ctypes.c_int32), ("kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32), ("sequences", ctypes.c_int32), ("table_width", ctypes.c_int32), ("table", ctypes.c_void_p),
                ("lengths", ctypes.c_void_p), ("starts", ctypes.c_void_p), ("origins", ctypes.c_void_p), ("tokens", ctypes.c_int32), ("frame_height", ctypes.c_int32),
                ("frame_width", ctypes.c_int32)]


class ca_append(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("q_strides", ctypes.POINTER(ca_strides)), ("k_strides", ctypes.POINTER(ca_strides)),
                ("v_strides", ctypes.POINTER(ca_strides)), ("q_out", ctypes.c_void_p), ("heads", ctypes.c_int32), ("normed", ctypes.c_int32), ("q_weight", ctypes.c_void_p),
                ("k_weight", ctypes.c_void_p), ("eps", ctypes.c_float), ("rotary", ctypes.c_void_p), ("where", ctypes.POINTER(ca_where))]


class ca_reach(ctypes.Structure):
    _fields_ = [("scale", ctypes.c_float), ("cap", ctypes.c_float), ("slopes", ctypes.c_void_p), ("causal", ctypes.c_int32), ("window", ctypes.c_int32),
                ("tree", ctypes.c_void_p)]


def _check_ints(t, shape, name, device=None):
    import torch
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if device is not None and t.device != device:
        raise ValueError(f"{name} is on {t.device}, the pages are on {device}")
    if tuple(t.shape) != shape or t.dtype != torch.int32 or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous int32 tensor of shape {shape}")


class Cache:
    """Pages of keys and values, and whose tokens lie where: k, v [num_pages, kv_heads, page_tokens, head_dim]; table int32 [sequences, pages of the longest], -1 where there is
    none; lengths int32 [sequences], tokens with those of the next call; starts int32 [sequences + 1], rows of the next call's packed tensors; origins int32
    [sequences] or None, tokens of the prompts; frame: (height, width) of a frame.  Device tensors, which a program changes in place from call to call, or it makes
    another Cache of the same pages."""

    def __init__(self, k, v, table, lengths, starts, origins=None, frame=(1, 1)):
        import torch
        if k.dim() != 4 or k.dtype not in (torch.float32, torch.bfloat16):
            raise ValueError("pages are bfloat16 or float32 [num_pages, kv_heads, page_tokens, head_dim]")
        for name, t in (("k", k), ("v", v)):
            if not t.is_cuda or t.device != k.device or t.shape != k.shape or t.dtype != k.dtype or not t.is_contiguous():
                raise ValueError(f"pages of {name} must be a contiguous device tensor, those of k and v alike")
        if table.dim() != 2:
            raise ValueError("table has a row for every sequence")
        sequences = table.shape[0]
        for name, t, shape in (("table", table, tuple(table.shape)), ("lengths", lengths, (sequences,)), ("starts", starts, (sequences + 1,)), ("origins", origins, (sequences,))):
            if t is not None:
                _check_ints(t, shape, name, k.device)
        if len(frame) != 2:
            raise ValueError("frame has a height and a width")
        self.k, self.v, self.table, self.lengths, self.starts, self.origins, self.frame = k, v, table, lengths, starts, origins, tuple(frame)
        pages, kv_heads, page_tokens, head_dim = k.shape
        self._args = (k.data_ptr(), v.data_ptr(), pages, page_tokens, kv_heads, head_dim, CA_BF16 if k.dtype == torch.bfloat16 else CA_F32, sequences, table.shape[1],
                      table.data_ptr(), lengths.data_ptr(), starts.data_ptr(), None if origins is None else origins.data_ptr())
        self._workspace = {}   # bytes by (tokens, heads)

    def _of(self, tokens):
        return ca_cache(*self._args, tokens, *self.frame)


def _packed(t, cache, heads, name):
    """A packed tensor of rows; the strides to hand over, None where it is contiguous."""
    _on_current_device(t, name)
    if t.dtype != cache.k.dtype:
        raise ValueError(f"{name} has dtype {t.dtype}, the cache {cache.k.dtype}")
    if t.dim() != 3 or t.shape[2] != cache.k.shape[3] or (heads is not None and t.shape[1] != heads):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected [tokens, {'heads' if heads is None else heads}, {cache.k.shape[3]}]")
    if t.is_contiguous():
        return None
    if t.stride(2) != 1 and t.shape[2] > 1:
        raise ValueError(f"channels of {name} must be contiguous")
    return ca_strides(0, *(t.stride(i) if t.shape[i] > 1 else 0 for i in (1, 0)))


def compact_attn_cache_append(k, v, cache, q=None, norm=True, q_weight=None, k_weight=None, rotary=None, eps=1e-6, origin=(0, 0, 0), positions=None, out=None, stream=None):
    """Stores keys and values [tokens, kv_heads, D] of new tokens in their pages, keys with norm (times k_weight [D]) and rotation, and returns the queries q [tokens, heads, D] with theirs
    (None without q).  Any strides with contiguous channels.  Tokens are turned by origin + (frame, row, column), or by positions int32 [tokens, 3].  out: where to write the queries."""
    _on_current_device(cache.k, "the cache")
    tokens = k.shape[0]
    kv_heads = cache.k.shape[1]
    strides = [None if t is None else _packed(t, cache, heads, name) for name, t, heads in (("q", q, None), ("k", k, kv_heads), ("v", v, kv_heads))]
    for name, t in (("q", q), ("v", v)):
        if t is not None and t.shape[0] != tokens:
            raise ValueError(f"{name} has {t.shape[0]} tokens, k has {tokens}")
    for name, w in (("q_weight", q_weight), ("k_weight", k_weight)):
        if w is not None:
            _on_current_device(w, name)
            if w.dtype != cache.k.dtype or tuple(w.shape) != (cache.k.shape[3],) or not w.is_contiguous():
                raise ValueError(f"{name} must be a contiguous {cache.k.dtype} tensor of {cache.k.shape[3]} elements")
    if len(origin) != 3:
        raise ValueError("origin has a value for each of three axes")
    if positions is not None:
        _on_current_device(positions, "positions")
        _check_ints(positions, (tokens, 3), "positions")
    if q is None:
        if out is not None:
            raise ValueError("out without q")
    elif out is None:
        with _on(stream, q.device):
            out = q.new_empty(q.shape)
    elif _packed(out, cache, q.shape[1], "out") is not None or out.shape[0] != tokens:
        raise ValueError("out must be contiguous, of the shape of q")
    where = None if positions is None and tuple(origin) == (0, 0, 0) else ctypes.pointer(ca_where((ctypes.c_int32 * 3)(*origin), None if positions is None else positions.data_ptr()))
    at = lambda t: None if t is None else t.data_ptr()
    append = ca_append(at(q), at(k), at(v), *(None if s is None else ctypes.pointer(s) for s in strides), at(out), 0 if q is None else q.shape[1], int(bool(norm)), at(q_weight),
                       at(k_weight), eps, _table(rotary), where)
    _check(load_library().compact_attn_cache_append(append, cache._of(tokens), _stream_ptr(stream)))
    return out


def compact_attn_cache_attend(q, cache, scale=0.0, cap=0.0, slopes=None, causal=True, window=0, tree=None, out=None, stream=None):
    """Attention of the new tokens' queries q [tokens, heads, D] over the cache: scores cap * tanh(scale q.k / cap) - slopes[head] * |frame difference| (cap 0, slopes None:
    without) over the prompt and the frames up to their own (causal), the last `window` of them (0: all), or the drafts that the bits of tree (int64 or uint64 [tokens]) say.
    -> (out [tokens, heads, D], lse float32 [tokens, heads]); out: such a pair to write to."""
    import torch
    _on_current_device(cache.k, "the cache")
    strides = _packed(q, cache, None, "q")
    tokens, heads = q.shape[:2]
    if slopes is not None:
        _on_current_device(slopes, "slopes")
        if tuple(slopes.shape) != (heads,) or slopes.dtype != torch.float32 or not slopes.is_contiguous():
            raise ValueError(f"slopes must be a contiguous float32 tensor of shape {(heads,)}")
    if tree is not None:
        _on_current_device(tree, "tree")
        if tuple(tree.shape) != (tokens,) or tree.dtype not in (torch.int64, torch.uint64) or not tree.is_contiguous():
            raise ValueError(f"tree must be a contiguous int64 or uint64 tensor of shape {(tokens,)}")
    if out is None:
        with _on(stream, q.device):
            out = q.new_empty(q.shape), q.new_empty((tokens, heads), dtype=torch.float32)
    else:
        if _packed(out[0], cache, heads, "out") is not None or out[0].shape[0] != tokens:
            raise ValueError("out must be contiguous, of the shape of q")
        _on_current_device(out[1], "lse of out")
        if tuple(out[1].shape) != (tokens, heads) or out[1].dtype != torch.float32 or not out[1].is_contiguous():
            raise ValueError(f"lse of out must be a contiguous float32 tensor of shape {(tokens, heads)}")
    args, lib = cache._of(tokens), load_library()
    need = cache._workspace.get((tokens, heads))
    if need is None:
        size = ctypes.c_int64()
        _check(lib.compact_attn_cache_workspace(args, heads, size))
        need = cache._workspace[tokens, heads] = size.value
    workspace = None
    if need:
        workspace = _lend(q, need, stream)
        if workspace is None or workspace is NotImplemented:
            raise CompactAttnError(CA_ERR_ALLOC, f"no memory for a workspace of {need} bytes, or a capture that torch does not run")
    reach = ca_reach(scale, cap, None if slopes is None else slopes.data_ptr(), int(bool(causal)), window, None if tree is None else tree.data_ptr())
    _check(lib.compact_attn_cache_attend(q.data_ptr(), strides, heads, args, reach, out[0].data_ptr(), out[1].data_ptr(), None if workspace is None else workspace.data_ptr(), need,
                                         _stream_ptr(stream)))
    return tuple(out)


def compact_attn_cache_keep(cache, kept, counts, stream=None):
    """Keeps some of the last call's new tokens (those of lengths and starts): new token kept[s, j] becomes new token j, for j < counts[s], in the pages.  kept: int32 [sequences, up to 64],
    counts: int32 [sequences]."""
    _on_current_device(cache.k, "the cache")
    if kept.dim() != 2:
        raise ValueError("kept has a row for every sequence")
    sequences = cache.table.shape[0]
    _check_ints(kept, (sequences, kept.shape[1]), "kept", cache.k.device)
    _check_ints(counts, (sequences,), "counts", cache.k.device)
    _check(load_library().compact_attn_cache_keep(cache._of(2 ** 31 - 1), kept.data_ptr(), kept.shape[1], counts.data_ptr(), _stream_ptr(stream)))


def _declare(lib):
    vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    cache = ctypes.POINTER(ca_cache)
    lib.compact_attn_cache_append.argtypes = [ctypes.POINTER(ca_append), cache, vp]
    lib.compact_attn_cache_workspace.argtypes = [cache, i32, ctypes.POINTER(i64)]
    lib.compact_attn_cache_attend.argtypes = [vp, ctypes.POINTER(ca_strides), i32, cache, ctypes.POINTER(ca_reach), vp, vp, vp, i64, vp]
    lib.compact_attn_cache_keep.argtypes = [cache, vp, i32, vp, vp]


binding._declarations.append(_declare)
