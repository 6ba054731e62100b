"""A paged cache of keys and values: argument marshalling for the entry points of that part of include/compact_attn.h, as binding.py does it for the others."""
import ctypes
import operator

from . import binding
from .binding import CA_BF16, CA_ERR_ALLOC, CA_F32, CompactAttnError, _lend, load_library
from .binding import _check as _check_status
from .rotary import _on, _table, ca_strides, ca_where


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


def _check(t, cache, shape, dtype, name):
    """A contiguous tensor beside the pages."""
    if t.get_device() != cache._device:   # (-1: not a device tensor)
        raise ValueError(f"{name} is on {t.device}, the cache on cuda:{cache._device}")
    if t.shape != shape or t.dtype is not dtype or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)}")


def _fixed(name):
    """An attribute that calls know by its address: it stays what the Cache was made with."""
    def refuse(self, value):
        raise AttributeError(f"{name} of a Cache cannot be replaced: change it in place, or make another Cache of the same pages")
    return property(operator.attrgetter("_" + name), refuse)


class Cache:
    """Pages of keys and values, and whose tokens lie where: k, v [num_pages, kv_heads, page_tokens, head_dim]; table int32 [sequences, pages of the longest], -1 where there is
    none; lengths int32 [sequences], tokens with those of the next call; starts int32 [sequences + 1], rows of the next call's packed tensors; origins int32
    [sequences] or None, tokens of the prompts; frame: (height, width) of a frame.  Device tensors, which a program changes in place from call to call (their
    memory stays where it is), or it makes another Cache of the same pages; as attributes they can be read, not replaced."""

    k, v, table, lengths, starts, origins, frame = map(_fixed, ("k", "v", "table", "lengths", "starts", "origins", "frame"))

    def __init__(self, k, v, table, lengths, starts, origins=None, frame=(1, 1)):
        import torch
        if k.dim() != 4 or k.dtype not in (torch.float32, torch.bfloat16):
            raise ValueError("pages are bfloat16 or float32 [num_pages, kv_heads, page_tokens, head_dim]")
        for name, t in (("k", k), ("v", v)):
            if not t.is_cuda or t.device != k.device or t.shape != k.shape or t.dtype != k.dtype or not t.is_contiguous():
                raise ValueError(f"pages of {name} must be a contiguous device tensor, those of k and v alike")
        if table.dim() != 2:
            raise ValueError("table has a row for every sequence")
        if len(frame) != 2:
            raise ValueError("frame has a height and a width")
        self._device = k.get_device()
        sequences = table.shape[0]
        for name, t, shape in (("table", table, table.shape), ("lengths", lengths, (sequences,)), ("starts", starts, (sequences + 1,)), ("origins", origins, (sequences,))):
            if t is not None:
                _check(t, self, shape, torch.int32, name)
        self._k, self._v, self._table, self._lengths, self._starts, self._origins, self._frame = k, v, table, lengths, starts, origins, tuple(frame)
        pages, self._kv_heads, page_tokens, self._head_dim = k.shape
        self._sequences = sequences
        self._dtype = k.dtype
        self._args = (k.data_ptr(), v.data_ptr(), pages, page_tokens, self._kv_heads, self._head_dim, CA_BF16 if k.dtype == torch.bfloat16 else CA_F32, sequences, table.shape[1],
                      table.data_ptr(), lengths.data_ptr(), starts.data_ptr(), None if origins is None else origins.data_ptr())
        self._current_device, self._current_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream
        self._of = {}          # ca_cache by tokens of a call
        self._workspace = {}   # bytes by (tokens, heads)


def _of(cache, tokens):
    """The ca_cache of a call of so many tokens, on the current device."""
    if cache._current_device() != cache._device:
        raise ValueError(f"the cache is on cuda:{cache._device}, the current device is cuda:{cache._current_device()}")
    args = cache._of.get(tokens)
    if args is None:
        if len(cache._of) >= 64:
            cache._of.clear()
            cache._workspace.clear()
        args = cache._of[tokens] = ca_cache(*cache._args, tokens, *cache._frame)
    return args


def _packed(t, cache, tokens, heads, name):
    """A packed tensor of rows; the strides to hand over, None where it is contiguous."""
    if t.get_device() != cache._device:
        raise ValueError(f"{name} is on {t.device}, the cache on cuda:{cache._device}")
    if t.dtype is not cache._dtype:
        raise ValueError(f"{name} has dtype {t.dtype}, the cache {cache._dtype}")
    if t.shape != (tokens, heads, cache._head_dim):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {(tokens, heads, cache._head_dim)}")
    if t.is_contiguous():
        return None
    token, head, channel = t.stride()
    if channel != 1 and cache._head_dim > 1:
        raise ValueError(f"channels of {name} must be contiguous")
    return ctypes.pointer(ca_strides(0, head if heads > 1 else 0, token if tokens > 1 else 0))


def _stream_of(cache, stream):
    """The handle of a call's stream, the current device's if it has none."""
    return cache._current_stream(cache._device) if stream is None else stream.cuda_stream


def _rows(t, name):
    """(tokens, heads) of a packed tensor."""
    if t.dim() != 3:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected tokens, heads and channels")
    return t.shape[:2]


def compact_attn_cache_append(k, v, cache, q=None, norm=True, q_weight=None, k_weight=None, rotary=None, eps=1e-6, origin=(0, 0, 0), positions=None, out=None, stream=None):
    """Stores keys and values [tokens, kv_heads, D] of new tokens in their pages, keys with norm (times k_weight [D]) and rotation, and returns the queries q [tokens, heads, D] with theirs
    (None without q).  Any strides with contiguous channels.  Tokens are turned by origin + (frame, row, column), or by positions int32 [tokens, 3].  out: where to write the queries."""
    tokens, heads = k.shape[0], 0
    args = _of(cache, tokens)
    append = ca_append(None, k.data_ptr(), v.data_ptr())
    append.k_strides, append.v_strides = _packed(k, cache, tokens, cache._kv_heads, "k"), _packed(v, cache, tokens, cache._kv_heads, "v")
    if q is not None:
        heads = _rows(q, "q")[1]
        append.q_strides = _packed(q, cache, tokens, heads, "q")
        if out is None:
            if stream is None:
                out = q.new_empty(tokens, heads, cache._head_dim)  # (0.9 us; 1.4 of q.shape)
            else:
                with _on(stream, q.device):
                    out = q.new_empty(tokens, heads, cache._head_dim)
        elif _packed(out, cache, tokens, heads, "out") is not None:
            raise ValueError("out must be contiguous")
        append.q, append.q_out, append.heads = q.data_ptr(), out.data_ptr(), heads
    elif out is not None:
        raise ValueError("out without q")
    append.normed, append.eps = bool(norm), eps
    if q_weight is not None:
        _check(q_weight, cache, (cache._head_dim,), cache._dtype, "q_weight")
        append.q_weight = q_weight.data_ptr()
    if k_weight is not None:
        _check(k_weight, cache, (cache._head_dim,), cache._dtype, "k_weight")
        append.k_weight = k_weight.data_ptr()
    append.rotary = _table(rotary)
    if len(origin) != 3:
        raise ValueError("origin has a value for each of three axes")
    if positions is not None or tuple(origin) != (0, 0, 0):
        where = ca_where((ctypes.c_int32 * 3)(*origin), None)
        if positions is not None:
            import torch
            _check(positions, cache, (tokens, 3), torch.int32, "positions")
            where.positions = positions.data_ptr()
        append.where = ctypes.pointer(where)
    _check_status(load_library().compact_attn_cache_append(append, args, _stream_of(cache, stream)))
    return out


def compact_attn_cache_attend(q, cache, scale=0.0, cap=0.0, slopes=None, causal=True, window=0, tree=None, out=None, stream=None):
    """Attention of the new tokens' queries q [tokens, heads, D] over the cache: scores cap * tanh(scale q.k / cap) - slopes[head] * |frame difference| (cap 0, slopes None:
    without) over the prompt and the frames up to their own (causal), the last `window` of them (0: all), or the drafts that the bits of tree (int64 or uint64 [tokens]) say.
    -> (out [tokens, heads, D], lse float32 [tokens, heads]); out: such a pair to write to."""
    import torch
    tokens, heads = _rows(q, "q")
    args, lib = _of(cache, tokens), load_library()
    strides = _packed(q, cache, tokens, heads, "q")
    reach = ca_reach(scale, cap, None, bool(causal), window)
    if slopes is not None:
        _check(slopes, cache, (heads,), torch.float32, "slopes")
        reach.slopes = slopes.data_ptr()
    if tree is not None:
        _check(tree, cache, (tokens,), torch.int64 if tree.dtype is torch.int64 else torch.uint64, "tree")
        reach.tree = tree.data_ptr()
    if out is None:
        if stream is None:
            out = q.new_empty(tokens, heads, cache._head_dim), q.new_empty(tokens, heads, dtype=torch.float32)
        else:
            with _on(stream, q.device):
                out = q.new_empty(tokens, heads, cache._head_dim), q.new_empty(tokens, heads, dtype=torch.float32)
    else:
        if _packed(out[0], cache, tokens, heads, "out") is not None:
            raise ValueError("out must be contiguous")
        _check(out[1], cache, (tokens, heads), torch.float32, "lse of out")
    need = cache._workspace.get((tokens, heads))
    if need is None:
        size = ctypes.c_int64()
        _check_status(lib.compact_attn_cache_workspace(args, heads, size))
        need = cache._workspace[tokens, heads] = size.value
    workspace = None
    if need:
        workspace = _lend(q, need, stream)
        if workspace is None or workspace is NotImplemented:
            raise CompactAttnError(CA_ERR_ALLOC, f"no memory for a workspace of {need} bytes, or a capture that torch does not run")
    _check_status(lib.compact_attn_cache_attend(q.data_ptr(), strides, heads, args, reach, out[0].data_ptr(), out[1].data_ptr(),
                                                None if workspace is None else workspace.data_ptr(), need, _stream_of(cache, stream)))
    return tuple(out)


def compact_attn_cache_keep(cache, kept, counts, stream=None):
    """Keeps some of the last call's new tokens (those of lengths and starts): new token kept[s, j] becomes new token j, for j < counts[s], in the pages.  kept: int32 [sequences, up to 64],
    counts: int32 [sequences]."""
    import torch
    args, sequences = _of(cache, 2 ** 31 - 1), cache._sequences
    if kept.dim() != 2:
        raise ValueError("kept has a row for every sequence")
    _check(kept, cache, (sequences, kept.shape[1]), torch.int32, "kept")
    _check(counts, cache, (sequences,), torch.int32, "counts")
    _check_status(load_library().compact_attn_cache_keep(args, kept.data_ptr(), kept.shape[1], counts.data_ptr(), _stream_of(cache, stream)))


def _declare(lib):
    vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    cache = ctypes.POINTER(ca_cache)
    lib.compact_attn_cache_append.argtypes = [ctypes.POINTER(ca_append), cache, vp]
    lib.compact_attn_cache_workspace.argtypes = [cache, i32, ctypes.POINTER(i64)]
    lib.compact_attn_cache_attend.argtypes = [vp, ctypes.POINTER(ca_strides), i32, cache, ctypes.POINTER(ca_reach), vp, vp, vp, i64, vp]
    lib.compact_attn_cache_keep.argtypes = [cache, vp, i32, vp, vp]


binding._declarations.append(_declare)
