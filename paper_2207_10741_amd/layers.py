"""Python binding of the C ABI in include/focused_layers.h: the matrix product with bias, activation and residual, and group norm.

Argument marshalling only, as in `binding`: every step runs in the HIP kernels of libfocused_conv.so, and there is no fallback.

    qkv = linear(rows, w_qkv, bias)                                         # out = rows @ w_qkv.T + bias
    y = linear(attended, w_out, residual=rows)                              # ... + rows
    h = group_norm(x, 32, weight, bias, mask=mask, activation="silu")       # x [images, height, width, channels]

The calls' semantics are stated in the header.  A serving loop that makes the same call on the same tensors again and again marshals it
once: PreparedLinear, PreparedGroupNorm.
"""
from __future__ import annotations

import ctypes

from . import binding as B
from .attention import _check_workspace, _kept_workspace, _made, _ready_workspace
from .pages import _OnDevice

ACTIVATIONS = {None: 0, "none": 0, "relu": 1, "silu": 2, "gelu": 3}
RESIDUAL_FIRST, ANY_POINTERS, COUNTED = 128, 256, 512
MAX_STRIDE = 4194304
GROUP_MAX_CHANNELS = 16384
NORM_MAX_ROWS = 1073741824

LINEAR_KERNELS = ("rings", "rows", "stages", "stages_any", "tiles", "large")

FUNCTIONS = ("fc_linear_workspace_bytes", "fc_group_norm_workspace_bytes", "fc_linear_cut_of", "fc_linear", "fc_group_norm")


class LinearDesc(ctypes.Structure):
    """Mirror of fc_linear_desc."""
    _fields_ = ([(k, ctypes.c_int32) for k in ("rows", "n", "k", "dtype", "out_dtype", "activation")] + [("flags", ctypes.c_uint32)] +
                [("reserved", ctypes.c_int32)] + [(k, ctypes.c_int64) for k in ("x_row", "w_row", "residual_row", "out_row")])


class LinearCut(ctypes.Structure):
    """Mirror of fc_linear_cut."""
    _fields_ = [(k, ctypes.c_int32) for k in ("kernel", "tile_rows", "tile_columns", "pieces", "anew_x", "anew_w")]


class GroupNormDesc(ctypes.Structure):
    """Mirror of fc_group_norm_desc."""
    _fields_ = ([(k, ctypes.c_int32) for k in ("images", "rows", "max_rows", "channels", "groups", "dtype", "activation")] +
                [("flags", ctypes.c_uint32), ("eps", ctypes.c_float), ("reserved", ctypes.c_int32)] +
                [(k, ctypes.c_int64) for k in ("x_row", "out_row")])


_lib = None


def lib():
    """The loaded C library (binding.lib) with these functions' types set."""
    global _lib
    if _lib is None:
        L = B.lib()
        vp, size = ctypes.c_void_p, ctypes.c_size_t
        linear, norm = ctypes.POINTER(LinearDesc), ctypes.POINTER(GroupNormDesc)
        for name, args in (("fc_linear_workspace_bytes", [linear, ctypes.POINTER(size)]),
                           ("fc_group_norm_workspace_bytes", [norm, ctypes.POINTER(size)]),
                           ("fc_linear_cut_of", [linear, ctypes.POINTER(LinearCut)]),
                           ("fc_linear", [linear] + [vp] * 7 + [size, vp]),
                           ("fc_group_norm", [norm] + [vp] * 7 + [size, vp])):
            f = getattr(L, name)
            f.restype, f.argtypes = ctypes.c_int32, args
        _lib = L
    return _lib


def _dtype(x, names="float32, bfloat16 or float16"):
    torch = B._torch()
    code = {torch.float32: B.F32, torch.bfloat16: B.BF16, torch.float16: B.F16}.get(x.dtype)
    if code is None or (code == B.F32 and "float32" not in names):
        raise ValueError("expected %s, got %s" % (names, x.dtype))
    return code


def _activation(name):
    if name not in ACTIVATIONS:
        raise ValueError("activation is one of %s" % sorted(k for k in ACTIVATIONS if k))
    return ACTIVATIONS[name]


def _matrix(x, what, device=None):
    """The stride of the rows of x [rows, columns] on the device."""
    if not x.is_cuda or (device is not None and x.device != device):
        raise ValueError("%s must be a device tensor, all on one device" % what)
    if x.dim() != 2 or (x.stride(1) != 1 and x.shape[1] > 1 and x.shape[0] > 0):
        raise ValueError("%s is [rows, columns], the columns next to each other" % what)
    return x.stride(0) if x.shape[0] > 1 else max(x.stride(0), x.shape[1])


def _vector(t, n, dtype, device, what):
    if t is not None and (not t.is_cuda or t.device != device or t.dtype != dtype or tuple(t.shape) != (n,) or not t.is_contiguous()):
        raise ValueError("%s is %s [%d], contiguous, on the same device" % (what, str(dtype).replace("torch.", ""), n))


def _aligned(*tensors):
    return all(t.data_ptr() % 16 == 0 for t in tensors)


def _in_order(mask, rows):
    """Does a mask of this shape go over rows of that shape in their order?  Dimensions of one, and neighbouring dimensions as one, make no difference."""
    def lengths(shape):
        found, n = set(), 1
        for d in reversed(shape):
            n *= d
            found.add(n)
        return found - {1}
    a, b = lengths(mask), lengths(rows)
    return a <= b or b <= a


def linear_cut(desc):
    """fc_linear_cut_of: how a product (LinearDesc) is cut."""
    cut = LinearCut()
    B._check(lib().fc_linear_cut_of(ctypes.byref(desc), ctypes.byref(cut)), "fc_linear_cut_of")
    return cut


class _PreparedLayer(_OnDevice):
    def _bytes(self, desc):
        b = ctypes.c_size_t()
        name = self._name + "_workspace_bytes"
        B._check(getattr(lib(), name)(ctypes.byref(desc), ctypes.byref(b)), name)
        return b.value

    def _workspace(self, need, device, stream, desc):
        return _ready_workspace(need, device, stream, desc)

    def _finish(self, desc, pointers, keep, workspace, device, stream, result):
        need = self._bytes(desc)
        _check_workspace(workspace, device)
        if workspace is None and need:
            workspace = self._workspace(need, device, stream, desc)
        self._keep, self._device = (desc, workspace) + keep, device.index
        self._fn = getattr(lib(), self._name)
        self._args = (ctypes.byref(desc),) + pointers + (B._ptr(workspace), 0 if workspace is None else workspace.numel() * workspace.element_size())
        self._result = result


class PreparedLinear(_PreparedLayer):
    """linear with its arguments marshalled once."""
    _name = "fc_linear"

    @property
    def cut(self):
        """How the product is cut (LinearCut)."""
        return linear_cut(self._keep[0])

    def __init__(self, x, w, bias=None, residual=None, activation=None, residual_first=False, count=None, out=None, out_dtype=None,
                 workspace=None, stream=None):
        torch = B._torch()
        device = x.device
        desc = LinearDesc(rows=x.shape[0], x_row=_matrix(x, "x"), w_row=_matrix(w, "w", device), n=w.shape[0], k=w.shape[1],
                          dtype=_dtype(x, "bfloat16 or float16"), activation=_activation(activation), flags=RESIDUAL_FIRST if residual_first else 0)
        if w.dtype != x.dtype or x.shape[1] != w.shape[1]:
            raise ValueError("x is [rows, k], w [n, k], of one type")
        shape = (x.shape[0], w.shape[0])
        _vector(bias, shape[1], torch.float32, device, "bias")
        _vector(count, 1, torch.int32, device, "count")
        if out is None:
            if residual is not None and out_dtype is None:
                out_dtype = residual.dtype
            out = _made(shape, x.dtype if out_dtype is None else out_dtype, device, stream)
        elif out_dtype is not None and out.dtype != out_dtype:
            raise ValueError("out is not of out_dtype")
        desc.out_row, desc.out_dtype = _matrix(out, "out", device), _dtype(out)
        if tuple(out.shape) != shape or out.dtype not in (x.dtype, torch.float32):
            raise ValueError("out is [rows, n], of x's type or float32")
        if residual is not None:
            desc.residual_row = _matrix(residual, "residual", device)
            if tuple(residual.shape) != shape or residual.dtype != out.dtype:
                raise ValueError("residual must be like out")
        desc.flags |= (0 if _aligned(x, w) else ANY_POINTERS) | (0 if count is None else COUNTED)
        self._finish(desc, (x.data_ptr(), w.data_ptr(), B._ptr(bias), B._ptr(residual), B._ptr(count), out.data_ptr()),
                     (x, w, bias, residual, count, out), workspace, device, stream, out)


class PreparedGroupNorm(_PreparedLayer):
    """group_norm with its arguments marshalled once."""
    _name = "fc_group_norm"

    def __init__(self, x, groups, weight=None, bias=None, mask=None, starts=None, max_rows=None, eps=1e-5, activation=None, keep_out=False,
                 out=None, workspace=None, stream=None):
        torch = B._torch()
        if x.dim() < 2 or (starts is None and x.dim() < 3):
            raise ValueError("x is [images, ..., channels], or with starts [rows, channels]")
        device, channels = x.device, x.shape[-1]
        if out is None:
            out = _made(tuple(x.shape), x.dtype, device, stream)
        elif out.shape != x.shape or out.dtype != x.dtype:
            raise ValueError("out must be like x")
        rows = x.numel() // channels if channels else 0
        try:
            flat, flat_out = x.view(rows, channels), out.view(rows, channels)
        except RuntimeError:
            raise ValueError("the rows of x and of out must lie in order, with one stride") from None
        desc = GroupNormDesc(rows=rows, channels=channels, groups=int(groups), dtype=_dtype(x), activation=_activation(activation), eps=eps,
                             x_row=_matrix(flat, "x"), out_row=_matrix(flat_out, "out", device), flags=B.SKIP_ZERO_FILL if keep_out else 0)
        if starts is not None:
            if starts.dim() != 1 or starts.shape[0] < 2:
                raise ValueError("starts is int32 [images + 1]")
            _vector(starts, starts.shape[0], torch.int32, device, "starts")
            desc.images = starts.shape[0] - 1
            desc.max_rows = rows if max_rows is None else max_rows
        else:
            desc.images = x.shape[0]
            desc.max_rows = rows // x.shape[0] if x.shape[0] else 0
            if max_rows is not None and max_rows != desc.max_rows:
                raise ValueError("max_rows: without starts every image has the same number of rows")
            if rows == 0:
                desc.images, desc.max_rows = max(desc.images, 1), 0     # (nothing to do: the library takes no sizes of zero)
        _vector(weight, channels, torch.float32, device, "weight")
        _vector(bias, channels, torch.float32, device, "bias")
        if mask is not None:
            if mask.numel() != rows or not mask.is_cuda or mask.device != device or not mask.is_contiguous() or mask.element_size() != 1:
                raise ValueError("mask is a byte a row, contiguous, on the same device")
            if rows and not _in_order(mask.shape, x.shape[:-1]):
                raise ValueError("mask %s does not go over the rows %s in their order" % (list(mask.shape), list(x.shape[:-1])))
        if not _aligned(x, out):
            desc.flags |= ANY_POINTERS
        self._finish(desc, (x.data_ptr(), B._ptr(weight), B._ptr(bias), B._ptr(mask), B._ptr(starts), out.data_ptr()),
                     (x, weight, bias, mask, starts, out), workspace, device, stream, out)


class _Linear(PreparedLinear):
    _workspace = _kept_workspace        # a call made once: the thread's kept workspace


class _GroupNorm(PreparedGroupNorm):
    _workspace = _kept_workspace


def linear(x, w, bias=None, residual=None, activation=None, residual_first=False, count=None, out=None, out_dtype=None, workspace=None,
           stream=None):
    """fc_linear.  x [rows, k], w [n, k], bfloat16 or float16, any stride of rows; bias float32 [n]; residual [rows, n] of out's type;
    activation None, "relu", "silu" or "gelu"; count int32 [1]: the rows that there are, known on the device (the work is laid out for half of
    them, which changes the order of sums).  Returns out [rows, n] of residual's type, or x's."""
    return _Linear(x, w, bias, residual, activation, residual_first, count, out, out_dtype, workspace, stream)(stream)


def group_norm(x, groups, weight=None, bias=None, mask=None, starts=None, max_rows=None, eps=1e-5, activation=None, keep_out=False, out=None,
               workspace=None, stream=None):
    """fc_group_norm.  x [images, ..., channels], or with starts (int32 [images + 1]) [rows, channels]; mask a byte a row: relevant ones are
    normed by their own statistics, the others become zero, or with keep_out stay.  Returns out like x."""
    return _GroupNorm(x, groups, weight, bias, mask, starts, max_rows, eps, activation, keep_out, out, workspace, stream)(stream)
