"""Python binding of the C ABI in include/focused_attention.h: a key/value cache in 8 bits, attention over it, and attention over the
blocks that a score selects.

Argument marshalling only, as in `binding`: every step runs in the HIP kernels of libfocused_conv.so, and there is no fallback.

    cache = KVCache(blocks=4096, kv_heads=8, head_dim=128)
    kv_append(cache, k, v, table, lengths)                      # the new tokens' keys and values, the last ones of every sequence
    out = cache_attention(cache, q, table, lengths)             # every new token over its sequence
    out, selected = focused_attention(cache, q, table, lengths, first=1, last=2, top=13)

The calls' semantics (blocks of 64 tokens, scales, selection, bounds) are stated in the header.  A serving loop that makes the same call
on the same tensors again and again marshals it once: PreparedAppend, PreparedRead, PreparedAttention, PreparedFocusedAttention.

Kernels and their grids are chosen by the bounds.  Without starts they follow from the tensors' shapes; with starts, max_new is every row of the call
unless it is given, right for one sequence alone: sequences of single tokens want max_new=1, others their largest number of new tokens.
"""
from __future__ import annotations

import ctypes
import math

from . import binding as B

BLOCK = 64
MAX_HEAD_DIM = 256
MAX_SELECTED = 1024
CAUSAL = 1

FUNCTIONS = ("fc_kv_cache_bytes", "fc_kv_append", "fc_kv_read", "fc_cache_attention_workspace_bytes",
             "fc_focused_attention_workspace_bytes", "fc_cache_attention", "fc_focused_attention")


class AttentionDesc(ctypes.Structure):
    """Mirror of fc_attention_desc."""
    _fields_ = ([(k, ctypes.c_int32) for k in ("blocks", "kv_heads", "head_dim", "batch", "tokens", "max_new", "max_len", "table_width",
                                               "heads", "dtype")] + [("flags", ctypes.c_uint32)] +
                [(k, ctypes.c_int32) for k in ("first", "last", "top")] + [("scale", ctypes.c_float), ("reserved", ctypes.c_int32)] +
                [(k, ctypes.c_int64) for k in ("q_row", "q_head", "k_row", "k_head", "v_row", "v_head")])


_lib = None


def lib():
    """The loaded C library (binding.lib) with these functions' types set."""
    global _lib
    if _lib is None:
        L = B.lib()
        vp, desc, size = ctypes.c_void_p, ctypes.POINTER(AttentionDesc), ctypes.c_size_t
        for name, args in (("fc_kv_cache_bytes", [desc, ctypes.POINTER(size)]),
                           ("fc_kv_append", [desc] + [vp] * 7),
                           ("fc_kv_read", [desc] + [vp] * 7),
                           ("fc_cache_attention_workspace_bytes", [desc, ctypes.POINTER(size)]),
                           ("fc_focused_attention_workspace_bytes", [desc, ctypes.POINTER(size)]),
                           ("fc_cache_attention", [desc] + [vp] * 8 + [size, vp]),
                           ("fc_focused_attention", [desc] + [vp] * 9 + [size, vp])):
            f = getattr(L, name)
            f.restype, f.argtypes = ctypes.c_int32, args
        _lib = L
    return _lib


def _bytes(name: str, desc: AttentionDesc) -> int:
    b = ctypes.c_size_t()
    B._check(getattr(lib(), name)(ctypes.byref(desc), ctypes.byref(b)), name)
    return b.value


def cache_bytes(blocks: int, kv_heads: int, head_dim: int) -> int:
    """Bytes of a cache (fc_kv_cache_bytes)."""
    return _bytes("fc_kv_cache_bytes", AttentionDesc(blocks=blocks, kv_heads=kv_heads, head_dim=head_dim))


class KVCache:
    """A pool of `blocks` blocks of 64 tokens: keys and values of `kv_heads` heads of `head_dim` channels in 8 bits."""

    def __init__(self, blocks: int, kv_heads: int, head_dim: int, device="cuda"):
        self.blocks, self.kv_heads, self.head_dim = int(blocks), int(kv_heads), int(head_dim)
        self.data = B._torch().empty((cache_bytes(blocks, kv_heads, head_dim),), dtype=B._torch().uint8, device=device)

    @property
    def device(self):
        return self.data.device


def _desc(cache: KVCache, table, lengths, starts, tokens, max_new, max_len) -> AttentionDesc:
    """The cache and the sequences, checked."""
    torch = B._torch()
    B._require_cuda(cache.data, table, lengths, starts)
    for t in (table, lengths, starts):
        if t is not None and (t.dtype != torch.int32 or t.device != cache.device):
            raise ValueError("table, lengths and starts must be int32 on the cache's device")
    if table.dim() != 2 or lengths.shape != (table.shape[0],) or (starts is not None and starts.shape != (table.shape[0] + 1,)):
        raise ValueError("table is [batch, blocks], lengths [batch], starts [batch + 1]")
    batch, width = table.shape
    if max_new is None:
        max_new = tokens if starts is not None else tokens // batch if batch else 0
    if starts is None and tokens and max_new * batch != tokens:
        raise ValueError("without starts every sequence has the same number of new tokens")
    if max_len is None:
        max_len = min(width * BLOCK, 2 ** 31 - 1)
    if tokens == 0:     # (nothing to do: the library takes no sizes of zero)
        batch, width, max_new, max_len = max(batch, 1), max(width, 1), max(max_new, 1), max(max_len, 1)
    return AttentionDesc(blocks=cache.blocks, kv_heads=cache.kv_heads, head_dim=cache.head_dim, batch=batch, tokens=tokens,
                         max_new=int(max_new), max_len=int(max_len), table_width=width)


def _rows(x, cache: KVCache, heads, what: str):
    """(stride of rows, stride of heads) of x [tokens, heads, head_dim]."""
    if not x.is_cuda or x.device != cache.device:
        raise ValueError("%s must be on the cache's device" % what)
    if x.dim() != 3 or x.shape[2] != cache.head_dim or (heads is not None and x.shape[1] != heads):
        raise ValueError("%s is [tokens, heads, head_dim]" % what)
    if x.stride(2) != 1 and x.shape[2] > 1:
        raise ValueError("the channels of %s must lie next to each other" % what)
    return x.stride(0), x.stride(1)


def _dtype(x):
    torch = B._torch()
    if x.dtype == torch.bfloat16:
        return B.BF16
    if x.dtype == torch.float16:
        return B.F16
    raise ValueError("keys, values and queries are bfloat16 or float16")


def _made(shape, dtype, device, stream):
    t = B._torch().empty(shape, dtype=dtype, device=device)
    if stream is not None:
        t.record_stream(stream)
    return t


class _Prepared:
    """A call with its arguments marshalled once: the same tensors every time."""

    def __call__(self, stream=None):
        rc = self._fn(*self._args, B._current_raw_stream() if stream is None else stream.cuda_stream)
        if rc != 0:
            raise B.FcError(rc, self._fn.__name__)
        return self._result


class PreparedAppend(_Prepared):
    """kv_append with its arguments marshalled once."""

    def __init__(self, cache, k, v, table, lengths, starts=None, max_new=None, max_len=None):
        desc = _desc(cache, table, lengths, starts, k.shape[0], max_new, max_len)
        if v.shape != k.shape or v.dtype != k.dtype:
            raise ValueError("k and v must be alike")
        desc.dtype = _dtype(k)
        desc.k_row, desc.k_head = _rows(k, cache, cache.kv_heads, "k")
        desc.v_row, desc.v_head = _rows(v, cache, cache.kv_heads, "v")
        self._keep = (desc, cache.data, k, v, table, lengths, starts)
        self._fn = lib().fc_kv_append
        self._args = (ctypes.byref(desc), cache.data.data_ptr(), k.data_ptr(), v.data_ptr(), table.data_ptr(), lengths.data_ptr(),
                      B._ptr(starts))
        self._result = cache


class PreparedRead(_Prepared):
    """kv_read with its arguments marshalled once."""

    def __init__(self, cache, table, lengths, starts=None, tokens=None, max_new=None, max_len=None, k=None, v=None, stream=None):
        if tokens is None:
            if starts is not None:
                raise ValueError("tokens: the rows that starts counts")
            if max_new is None:
                raise ValueError("max_new: the tokens of every sequence to be read, or tokens: those of all of them")
            tokens = table.shape[0] * max_new
        desc = _desc(cache, table, lengths, starts, tokens, max_new, max_len)
        torch = B._torch()
        shape = (tokens, cache.kv_heads, cache.head_dim)
        for t in (k, v):
            B._require_cuda(t)
            if t is not None and (t.shape != shape or t.dtype != torch.float32 or t.device != cache.device):
                raise ValueError("k and v are float32 [tokens, kv_heads, head_dim]")
        k = _made(shape, torch.float32, cache.device, stream) if k is None else k
        v = _made(shape, torch.float32, cache.device, stream) if v is None else v
        self._keep = (desc, cache.data, table, lengths, starts)
        self._fn = lib().fc_kv_read
        self._args = (ctypes.byref(desc), cache.data.data_ptr(), table.data_ptr(), lengths.data_ptr(), B._ptr(starts), k.data_ptr(), v.data_ptr())
        self._result = (k, v)


class _PreparedAttend(_Prepared):
    def _prepare(self, name, desc, cache, q, table, lengths, starts, scale, out, lse, selected, workspace, stream):
        torch = B._torch()
        desc.dtype, desc.heads = _dtype(q), q.shape[1]
        desc.q_row, desc.q_head = _rows(q, cache, None, "q")
        desc.scale = 1.0 / math.sqrt(cache.head_dim) if scale is None else scale
        B._require_cuda(out, lse, selected, workspace)
        if out is None:
            out = _made(tuple(q.shape), q.dtype, q.device, stream)
        elif out.shape != q.shape or out.dtype != q.dtype or out.device != q.device:
            raise ValueError("out must be like q")
        if lse is not None and (lse.shape != q.shape[:2] or lse.dtype != torch.float32 or lse.device != q.device):
            raise ValueError("lse is float32 [tokens, heads]")
        need = _bytes(name + "_workspace_bytes", desc)
        if workspace is None and need:
            workspace = self._workspace(need, q.device, stream, desc)
        self._keep = (desc, cache.data, q, table, lengths, starts, out, lse, selected, workspace)
        self._fn = getattr(lib(), name)
        outputs = (out.data_ptr(), B._ptr(lse)) + (() if selected is None else (selected.data_ptr(),))
        self._args = (ctypes.byref(desc), cache.data.data_ptr(), q.data_ptr(), table.data_ptr(), lengths.data_ptr(), B._ptr(starts), *outputs,
                      B._ptr(workspace), 0 if workspace is None else workspace.numel() * workspace.element_size())
        self._result = out if selected is None else (out, selected)

    def _workspace(self, need, device, stream, desc):
        """A workspace of the call's own, cleared here once: the calls leave its counters zero."""
        torch = B._torch()
        desc.flags |= B.WORKSPACE_READY
        with torch.cuda.stream(stream if stream is not None else torch.cuda.current_stream(device)):
            workspace = torch.zeros((need,), dtype=torch.uint8, device=device)
            if not torch.cuda.is_current_stream_capturing():
                torch.cuda.current_stream(device).synchronize()     # (a call may come on any stream)
        return workspace


class PreparedAttention(_PreparedAttend):
    """cache_attention with its arguments marshalled once."""

    def __init__(self, cache, q, table, lengths, starts=None, max_new=None, max_len=None, causal=True, scale=None, out=None, lse=None,
                 workspace=None, stream=None):
        desc = _desc(cache, table, lengths, starts, q.shape[0], max_new, max_len)
        desc.flags = CAUSAL if causal else 0
        self._prepare("fc_cache_attention", desc, cache, q, table, lengths, starts, scale, out, lse, None, workspace, stream)


class PreparedFocusedAttention(_PreparedAttend):
    """focused_attention with its arguments marshalled once."""

    def __init__(self, cache, q, table, lengths, first, last, top, starts=None, max_new=None, max_len=None, scale=None, out=None, lse=None,
                 selected=None, workspace=None, stream=None):
        desc = _desc(cache, table, lengths, starts, q.shape[0], max_new, max_len)
        desc.flags, desc.first, desc.last, desc.top = CAUSAL, first, last, top
        torch = B._torch()
        shape = (q.shape[0], cache.kv_heads, first + last + top)
        if selected is None:
            if min(shape) < 0:
                raise ValueError("first, last and top count blocks")
            selected = _made(shape, torch.int32, q.device, stream)
        elif selected.shape != shape or selected.dtype != torch.int32 or selected.device != q.device:
            raise ValueError("selected is int32 [tokens, kv_heads, first + last + top]")
        self._prepare("fc_focused_attention", desc, cache, q, table, lengths, starts, scale, out, lse, selected, workspace, stream)


def _kept_workspace(self, need, device, stream, desc):
    return B._own_workspace(need, device, B._stream(stream), stream)


class _Attention(PreparedAttention):
    _workspace = _kept_workspace        # a call made once: the thread's kept workspace


class _FocusedAttention(PreparedFocusedAttention):
    _workspace = _kept_workspace


def kv_append(cache, k, v, table, lengths, starts=None, max_new=None, max_len=None, stream=None):
    """fc_kv_append.  k, v [tokens, kv_heads, head_dim], bfloat16 or float16, any strides of tokens and heads."""
    return PreparedAppend(cache, k, v, table, lengths, starts, max_new, max_len)(stream)


def kv_read(cache, table, lengths, starts=None, tokens=None, max_new=None, max_len=None, k=None, v=None, stream=None):
    """fc_kv_read: (keys, values) of the sequences' last tokens, float32 [tokens, kv_heads, head_dim]: max_new of every sequence, or with
    starts as many as it counts (tokens in all)."""
    return PreparedRead(cache, table, lengths, starts, tokens, max_new, max_len, k, v, stream)(stream)


def cache_attention(cache, q, table, lengths, starts=None, max_new=None, max_len=None, causal=True, scale=None, out=None, lse=None,
                    workspace=None, stream=None):
    """fc_cache_attention.  q [tokens, heads, head_dim]; scale None: 1 / sqrt(head_dim).  Returns out."""
    return _Attention(cache, q, table, lengths, starts, max_new, max_len, causal, scale, out, lse, workspace, stream)(stream)


def focused_attention(cache, q, table, lengths, first, last, top, starts=None, max_new=None, max_len=None, scale=None, out=None, lse=None,
                      selected=None, workspace=None, stream=None):
    """fc_focused_attention.  Returns (out, selected [tokens, kv_heads, first + last + top])."""
    return _FocusedAttention(cache, q, table, lengths, first, last, top, starts, max_new, max_len, scale, out, lse, selected, workspace,
                             stream)(stream)
