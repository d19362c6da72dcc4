"""Python binding of the C ABI in include/focused_pages.h: the pages of a key/value cache, kept on the device.

Argument marshalling only, as in `binding`: every step runs in the HIP kernels of libfocused_conv.so, and there is no fallback.

    cache, users = KVCache(blocks=4096, kv_heads=8, head_dim=128), kv_users(cache)
    kv_resize(cache, users, table, lengths)             # blocks for the lengths, before kv_append; a length of zero frees a sequence
    kv_fork(cache, users, table, lengths, parents)      # slot b becomes what slot parents[b] was; -1 frees it
    kv_compact(cache, users, table, other, other_users) # the blocks in use move to another cache
    kv_copy(cache, sources, other, targets)             # single blocks

The calls' semantics are stated in the header.  A serving loop that makes the same call on the same tensors again and again marshals it
once: PreparedResize, PreparedFork, PreparedCompact, PreparedCopy.
"""
from __future__ import annotations

import ctypes

from . import binding as B
from .attention import _Prepared, _check_workspace, _kept_workspace, _made, _ready_workspace

FUNCTIONS = ("fc_kv_resize_workspace_bytes", "fc_kv_fork_workspace_bytes", "fc_kv_compact_workspace_bytes", "fc_kv_resize", "fc_kv_fork",
             "fc_kv_compact", "fc_kv_copy")


class PagesDesc(ctypes.Structure):
    """Mirror of fc_pages_desc."""
    _fields_ = [(k, ctypes.c_int32) for k in ("blocks", "kv_heads", "head_dim", "blocks_to", "batch", "table_width", "pairs")] + [("flags", ctypes.c_uint32)]


_lib = None


def lib():
    """The loaded C library (binding.lib) with these functions' types set."""
    global _lib
    if _lib is None:
        L = B.lib()
        vp, desc, size = ctypes.c_void_p, ctypes.POINTER(PagesDesc), ctypes.c_size_t
        for name, args in (("fc_kv_resize_workspace_bytes", [desc, ctypes.POINTER(size)]),
                           ("fc_kv_fork_workspace_bytes", [desc, ctypes.POINTER(size)]),
                           ("fc_kv_compact_workspace_bytes", [desc, ctypes.POINTER(size)]),
                           ("fc_kv_resize", [desc] + [vp] * 6 + [size, vp]),
                           ("fc_kv_fork", [desc] + [vp] * 7 + [size, vp]),
                           ("fc_kv_compact", [desc] + [vp] * 8 + [size, vp]),
                           ("fc_kv_copy", [desc] + [vp] * 5)):
            f = getattr(L, name)
            f.restype, f.argtypes = ctypes.c_int32, args
        _lib = L
    return _lib


def kv_users(cache):
    """How many sequences hold each block of a new cache: none."""
    torch = B._torch()
    return torch.zeros((cache.blocks,), dtype=torch.int32, device=cache.device)


def _int32(t, shape, device, what):
    torch = B._torch()
    B._require_cuda(t)
    if t.dtype != torch.int32 or t.device != device or tuple(t.shape) != shape:
        raise ValueError("%s is int32 %s on the cache's device" % (what, list(shape)))


def _desc(cache, users, table, lengths=None, missing=None):
    B._require_cuda(cache.data, table)
    if table.dim() != 2 or 0 in table.shape:
        raise ValueError("table is [batch, blocks]")
    _int32(users, (cache.blocks,), cache.device, "users")
    _int32(table, tuple(table.shape), cache.device, "table")
    if lengths is not None:
        _int32(lengths, (table.shape[0],), cache.device, "lengths")
    if missing is not None:
        _int32(missing, (1,), cache.device, "missing")
    return PagesDesc(blocks=cache.blocks, kv_heads=cache.kv_heads, head_dim=cache.head_dim, batch=table.shape[0], table_width=table.shape[1])


def _other(cache, to):
    B._require_cuda(to.data)
    if (to.kv_heads, to.head_dim, to.device) != (cache.kv_heads, cache.head_dim, cache.device):
        raise ValueError("both caches must have the same heads, channels and device")


class _OnDevice(_Prepared):
    """A call whose tensors are on device `_device`, which the stream has to be of."""

    def __call__(self, stream=None):
        device = B._torch()._C._cuda_getDevice() if stream is None else stream.device_index
        if device != self._device:
            raise ValueError("the tensors are on cuda:%d, the stream on cuda:%d" % (self._device, device))
        return super().__call__(stream)


class _PreparedPages(_OnDevice):
    def _finish(self, name, desc, cache, pointers, keep, missing, workspace, stream):
        """pointers: what lies between the descriptor and missing"""
        torch = B._torch()
        if missing is None:
            missing = _made((1,), torch.int32, cache.device, stream)
        need = ctypes.c_size_t()
        B._check(getattr(lib(), name + "_workspace_bytes")(ctypes.byref(desc), ctypes.byref(need)), name + "_workspace_bytes")
        _check_workspace(workspace, cache.device)
        if workspace is None:
            workspace = self._workspace(need.value, cache.device, stream, desc)
        self._keep, self._device = (desc, cache.data, missing, workspace) + keep, cache.device.index
        self._fn = getattr(lib(), name)
        self._args = (ctypes.byref(desc),) + pointers + (missing.data_ptr(), workspace.data_ptr(), workspace.numel() * workspace.element_size())
        self._result = missing

    def _workspace(self, need, device, stream, desc):
        return _ready_workspace(need, device, stream, desc)


class PreparedResize(_PreparedPages):
    """kv_resize with its arguments marshalled once."""

    def __init__(self, cache, users, table, lengths, missing=None, workspace=None, stream=None):
        desc = _desc(cache, users, table, lengths, missing)
        self._finish("fc_kv_resize", desc, cache, (cache.data.data_ptr(), users.data_ptr(), table.data_ptr(), lengths.data_ptr()),
                     (users, table, lengths), missing, workspace, stream)


class PreparedFork(_PreparedPages):
    """kv_fork with its arguments marshalled once."""

    def __init__(self, cache, users, table, lengths, parents, missing=None, workspace=None, stream=None):
        desc = _desc(cache, users, table, lengths, missing)
        _int32(parents, (table.shape[0],), cache.device, "parents")
        self._finish("fc_kv_fork", desc, cache, (cache.data.data_ptr(), users.data_ptr(), table.data_ptr(), lengths.data_ptr(), parents.data_ptr()),
                     (users, table, lengths, parents), missing, workspace, stream)


class PreparedCompact(_PreparedPages):
    """kv_compact with its arguments marshalled once."""

    def __init__(self, cache, users, table, cache_to, users_to, table_to, missing=None, workspace=None, stream=None):
        desc = _desc(cache, users, table, None, missing)
        _other(cache, cache_to)
        _int32(users_to, (cache_to.blocks,), cache.device, "users_to")
        _int32(table_to, tuple(table.shape), cache.device, "table_to")
        desc.blocks_to = cache_to.blocks
        self._finish("fc_kv_compact", desc, cache, (cache.data.data_ptr(), users.data_ptr(), table.data_ptr(), cache_to.data.data_ptr(),
                                                    users_to.data_ptr(), table_to.data_ptr()),
                     (users, table, cache_to.data, users_to, table_to), missing, workspace, stream)


class PreparedCopy(_OnDevice):
    """kv_copy with its arguments marshalled once."""

    def __init__(self, cache, sources, cache_to, targets):
        B._require_cuda(cache.data)
        _other(cache, cache_to)
        if sources.dim() != 1:
            raise ValueError("sources and targets are lists of blocks")
        for t, what in ((sources, "sources"), (targets, "targets")):
            _int32(t, tuple(sources.shape), cache.device, what)
        desc = PagesDesc(blocks=cache.blocks, kv_heads=cache.kv_heads, head_dim=cache.head_dim, blocks_to=cache_to.blocks, pairs=sources.shape[0])
        self._keep, self._device = (desc, cache.data, sources, cache_to.data, targets), cache.device.index
        self._fn = lib().fc_kv_copy
        self._args = (ctypes.byref(desc), cache.data.data_ptr(), sources.data_ptr(), cache_to.data.data_ptr(), targets.data_ptr())
        self._result = cache_to


class _Resize(PreparedResize):
    _workspace = _kept_workspace        # a call made once: the thread's kept workspace


class _Fork(PreparedFork):
    _workspace = _kept_workspace


class _Compact(PreparedCompact):
    _workspace = _kept_workspace


def kv_resize(cache, users, table, lengths, missing=None, workspace=None, stream=None):
    """fc_kv_resize: every sequence holds the blocks that its length needs.  Returns missing (int32 [1]): places that got none."""
    return _Resize(cache, users, table, lengths, missing, workspace, stream)(stream)


def kv_fork(cache, users, table, lengths, parents, missing=None, workspace=None, stream=None):
    """fc_kv_fork: slot b becomes what slot parents[b] was, or is freed where that is no slot.  Returns missing."""
    return _Fork(cache, users, table, lengths, parents, missing, workspace, stream)(stream)


def kv_compact(cache, users, table, cache_to, users_to, table_to=None, missing=None, workspace=None, stream=None):
    """fc_kv_compact: the blocks in use move to cache_to.  Returns (table_to, missing)."""
    if table_to is None:
        table_to = _made(tuple(table.shape), table.dtype, table.device, stream)
    return table_to, _Compact(cache, users, table, cache_to, users_to, table_to, missing, workspace, stream)(stream)


def kv_copy(cache, sources, cache_to, targets, stream=None):
    """fc_kv_copy: blocks targets of cache_to become blocks sources of cache.  Returns cache_to."""
    return PreparedCopy(cache, sources, cache_to, targets)(stream)
