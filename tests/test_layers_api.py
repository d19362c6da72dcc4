"""Host-side checks of the layers' and pages' C ABI that need no GPU: exported symbols, sizes, refusals before anything is launched."""
import ctypes
import os
import re

import pytest

from paper_2207_10741_amd import attention as A, binding as B, layers as L, pages as P

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NULL, SHAPE, DTYPE, ALIGN, WORKSPACE, RANGE = -1, -2, -3, -4, -5, -6


def _header(name):
    return open(os.path.join(ROOT, "include", name)).read()


def _fields(text, struct):
    body = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    body = re.search(r"typedef struct \{([^}]*)\} %s;" % struct, body).group(1)
    return [n.strip() for line in body.split(";") if line.strip() for n in line.strip().split(" ", 1)[1].split(",")]


@pytest.mark.parametrize("header,module", [("focused_layers.h", L), ("focused_pages.h", P)])
def test_every_declared_symbol_is_exported_and_bound(header, module):
    names = set(re.findall(r"\b(fc_[a-z0-9_]+)\s*\(", re.sub(r"/\*.*?\*/", "", _header(header), flags=re.S)))
    assert names == set(module.FUNCTIONS)
    for n in names:
        assert getattr(module.lib(), n) is not None


def test_descriptors_and_constants_mirror_the_headers():
    layers, pages = _header("focused_layers.h"), _header("focused_pages.h")
    assert _fields(layers, "fc_linear_desc") == [n for n, _ in L.LinearDesc._fields_]
    assert _fields(layers, "fc_group_norm_desc") == [n for n, _ in L.GroupNormDesc._fields_]
    assert _fields(pages, "fc_pages_desc") == [n for n, _ in P.PagesDesc._fields_]
    for name, value in (("FC_RESIDUAL_FIRST", L.RESIDUAL_FIRST), ("FC_ANY_POINTERS", L.ANY_POINTERS), ("FC_COUNTED", L.COUNTED), ("FC_NORM_MAX_ROWS", L.NORM_MAX_ROWS), ("FC_LAYERS_MAX_STRIDE", L.MAX_STRIDE),
                        ("FC_GROUP_MAX_CHANNELS", L.GROUP_MAX_CHANNELS), ("FC_ACT_RELU", L.ACTIVATIONS["relu"]), ("FC_ACT_SILU", L.ACTIVATIONS["silu"]),
                        ("FC_ACT_GELU", L.ACTIVATIONS["gelu"])):
        assert value == int(re.search(name + r"\s*=\s*(\d+)", layers).group(1))


def _p(n):
    return ctypes.c_void_p(16 * n)      # (never read: the call is refused first)


def _linear_desc(**kw):
    base = dict(rows=100, n=64, k=128, dtype=B.BF16, out_dtype=B.BF16, activation=0, x_row=128, w_row=128, residual_row=64, out_row=64)
    base.update(kw)
    return L.LinearDesc(**base)


def _linear(d, x=_p(1), w=_p(2), bias=None, residual=None, count=None, out=_p(3), ws=_p(4), ws_bytes=1 << 40):
    return L.lib().fc_linear(None if d is None else ctypes.byref(d), x, w, bias, residual, count, out, ws, ws_bytes, None)


def _norm_desc(**kw):
    base = dict(images=2, rows=200, max_rows=100, channels=64, groups=8, dtype=B.BF16, eps=1e-5, x_row=64, out_row=64)
    base.update(kw)
    return L.GroupNormDesc(**base)


def _norm(d, x=_p(1), weight=None, bias=None, mask=None, starts=None, out=_p(3), ws=_p(4), ws_bytes=1 << 40):
    return L.lib().fc_group_norm(None if d is None else ctypes.byref(d), x, weight, bias, mask, starts, out, ws, ws_bytes, None)


def _bytes(module, name, d):
    b = ctypes.c_size_t()
    rc = getattr(module.lib(), name + "_workspace_bytes")(ctypes.byref(d), ctypes.byref(b))
    return rc if rc else b.value


def test_linear_refuses():
    assert _linear(None) == NULL
    for bad in (dict(rows=-1), dict(n=0), dict(k=0), dict(n=-4), dict(x_row=-1), dict(w_row=-1), dict(residual_row=-1), dict(out_row=63)):
        assert _linear(_linear_desc(**bad)) == SHAPE and _bytes(L, "fc_linear", _linear_desc(**bad)) == SHAPE
    for bad in (dict(dtype=B.F32), dict(dtype=B.FP8), dict(dtype=7), dict(out_dtype=B.F16), dict(out_dtype=B.FP8), dict(activation=4), dict(activation=-1),
                dict(flags=1), dict(flags=1024), dict(reserved=1)):
        assert _linear(_linear_desc(**bad)) == DTYPE
    most = L.MAX_STRIDE
    for bad in (dict(k=most + 1), dict(n=most + 1, out_row=most + 1), dict(x_row=most + 1), dict(w_row=most + 1), dict(out_row=most + 1),
                dict(rows=2 ** 31 - 1, n=most, out_row=most)):
        assert _linear(_linear_desc(**bad)) == RANGE
    assert _linear(_linear_desc(residual_row=most + 1), residual=_p(5)) == RANGE
    assert _linear(_linear_desc(), x=None) == NULL and _linear(_linear_desc(), w=None) == NULL and _linear(_linear_desc(), out=None) == NULL
    odd = ctypes.c_void_p(33)
    for name in ("x", "w", "out", "residual", "bias", "count"):
        assert _linear(_linear_desc(), **{name: odd}) == ALIGN
    assert _linear(_linear_desc(), x=ctypes.c_void_p(34)) == ALIGN and _linear(_linear_desc(out_dtype=B.F32), out=ctypes.c_void_p(34)) == ALIGN
    assert _linear(_linear_desc(rows=0), x=None, w=None, out=None, ws=None) == 0


def test_linear_workspace():
    long = _linear_desc(rows=100, k=4096, x_row=4096, w_row=4096)       # few tiles, a long reduction: in pieces
    need = _bytes(L, "fc_linear", long)
    assert need > 100 * 64 * 4
    assert _linear(long, ws=None) == WORKSPACE and _linear(long, ws_bytes=need - 1) == WORKSPACE and _linear(long, ws=ctypes.c_void_p(24)) == ALIGN
    assert _bytes(L, "fc_linear", _linear_desc(rows=0)) == 0
    # many rows of any alignment are laid out anew
    sizes = dict(rows=4096, n=4096, out_row=4096, residual_row=4096, x_row=4096, w_row=4096)
    plain, odd = _linear_desc(k=4096, **sizes), _linear_desc(k=4095, **sizes)
    room = 2 * 4096 * 4096 * 2
    assert _bytes(L, "fc_linear", odd) >= _bytes(L, "fc_linear", plain) + room
    assert _bytes(L, "fc_linear", _linear_desc(k=4096, flags=L.ANY_POINTERS, **sizes)) >= _bytes(L, "fc_linear", plain) + room
    b = ctypes.c_size_t()
    assert L.lib().fc_linear_workspace_bytes(None, ctypes.byref(b)) == NULL and L.lib().fc_linear_workspace_bytes(ctypes.byref(plain), None) == NULL


def test_group_norm_refuses():
    assert _norm(None) == NULL
    for bad in (dict(images=0), dict(rows=-1), dict(max_rows=-1), dict(channels=0), dict(groups=0), dict(groups=7), dict(eps=-1.0), dict(eps=float("nan")),
                dict(eps=float("inf")), dict(x_row=-1), dict(out_row=63)):
        assert _norm(_norm_desc(**bad)) == SHAPE and _bytes(L, "fc_group_norm", _norm_desc(**bad)) == SHAPE
    assert _norm(_norm_desc(rows=199)) == SHAPE                 # (no starts: images * max_rows)
    for bad in (dict(dtype=B.FP8), dict(dtype=9), dict(activation=4), dict(activation=-1), dict(flags=1), dict(flags=128), dict(reserved=1)):
        assert _norm(_norm_desc(**bad)) == DTYPE
    most = L.MAX_STRIDE
    for bad in (dict(channels=L.GROUP_MAX_CHANNELS + 1, groups=1, out_row=most), dict(x_row=most + 1), dict(out_row=most + 1),
                dict(images=1, max_rows=2 ** 30 + 1, rows=2 ** 30 + 1), dict(images=2 ** 30, max_rows=1, rows=2 ** 30, channels=512, groups=512, out_row=512)):
        assert _norm(_norm_desc(**bad)) == RANGE
    assert _norm(_norm_desc(), x=None) == NULL and _norm(_norm_desc(), out=None) == NULL
    for name in ("x", "out", "weight", "bias", "mask", "starts"):
        assert _norm(_norm_desc(), **{name: ctypes.c_void_p(24)}) == ALIGN
    assert _norm(_norm_desc(flags=L.ANY_POINTERS), x=ctypes.c_void_p(17)) == ALIGN
    large = _norm_desc(max_rows=50000, rows=100000)
    need = _bytes(L, "fc_group_norm", large)
    assert need > 0
    assert _norm(large, ws=None) == WORKSPACE and _norm(large, ws_bytes=need - 1) == WORKSPACE and _norm(large, ws=ctypes.c_void_p(24)) == ALIGN
    assert _norm(_norm_desc(rows=0, max_rows=0), x=None, out=None, ws=None) == 0
    assert _norm(_norm_desc(rows=0), x=None, out=None, starts=_p(5), ws=None) == 0


def _pages_desc(**kw):
    base = dict(blocks=100, kv_heads=2, head_dim=64, blocks_to=50, batch=3, table_width=8, pairs=4)
    base.update(kw)
    return P.PagesDesc(**base)


def _resize(d, cache=_p(1), users=_p(2), table=_p(3), lengths=_p(4), missing=_p(5), ws=_p(6), ws_bytes=1 << 40):
    return P.lib().fc_kv_resize(None if d is None else ctypes.byref(d), cache, users, table, lengths, missing, ws, ws_bytes, None)


def _fork(d, cache=_p(1), users=_p(2), table=_p(3), lengths=_p(4), parents=_p(7), missing=_p(5), ws=_p(6), ws_bytes=1 << 40):
    return P.lib().fc_kv_fork(None if d is None else ctypes.byref(d), cache, users, table, lengths, parents, missing, ws, ws_bytes, None)


def _compact(d, cache=_p(1), users=_p(2), table=_p(3), cache_to=_p(8), users_to=_p(9), table_to=_p(10), missing=_p(5), ws=_p(6), ws_bytes=1 << 40):
    return P.lib().fc_kv_compact(None if d is None else ctypes.byref(d), cache, users, table, cache_to, users_to, table_to, missing, ws, ws_bytes, None)


def _copy(d, cache=_p(1), sources=_p(2), cache_to=_p(3), targets=_p(4)):
    return P.lib().fc_kv_copy(None if d is None else ctypes.byref(d), cache, sources, cache_to, targets, None)


@pytest.mark.parametrize("call,name", [(_resize, "fc_kv_resize"), (_fork, "fc_kv_fork"), (_compact, "fc_kv_compact")])
def test_pages_refuse(call, name):
    assert call(None) == NULL
    for field in ("blocks", "kv_heads", "head_dim", "batch", "table_width"):
        for value in (0, -1):
            assert call(_pages_desc(**{field: value})) == SHAPE and _bytes(P, name, _pages_desc(**{field: value})) == SHAPE
    assert call(_pages_desc(head_dim=257)) == SHAPE
    assert call(_pages_desc(flags=1)) == DTYPE
    for bad in (dict(batch=65536), dict(batch=60000, table_width=40000), dict(blocks=2 ** 29 + 1, kv_heads=1), dict(blocks=2 ** 28, kv_heads=8)):
        assert call(_pages_desc(**bad)) == RANGE
    for pointer in ("cache", "users", "table", "missing"):
        assert call(_pages_desc(), **{pointer: None}) == NULL and call(_pages_desc(), **{pointer: ctypes.c_void_p(24)}) == ALIGN
    need = _bytes(P, name, _pages_desc())
    assert call(_pages_desc(), ws=None) == WORKSPACE and call(_pages_desc(), ws_bytes=need - 1) == WORKSPACE and call(_pages_desc(), ws=ctypes.c_void_p(24)) == ALIGN


def test_pages_of_two_caches_refuse():
    for call in (_compact, _copy):
        assert call(_pages_desc(blocks_to=0)) == SHAPE and call(_pages_desc(blocks_to=2 ** 30)) == RANGE
        assert call(_pages_desc(), cache_to=None) == NULL and call(_pages_desc(), cache_to=ctypes.c_void_p(24)) == ALIGN
    for same in (dict(cache_to=_p(1)), dict(users_to=_p(2)), dict(table_to=_p(3))):
        assert _compact(_pages_desc(), **same) == SHAPE
    assert _copy(None) == NULL and _copy(_pages_desc(pairs=-1)) == SHAPE and _copy(_pages_desc(), cache_to=_p(1)) == SHAPE
    assert _copy(_pages_desc(), sources=None) == NULL and _copy(_pages_desc(), targets=ctypes.c_void_p(24)) == ALIGN
    assert _copy(_pages_desc(pairs=0), cache=None, sources=None, cache_to=None, targets=None) == 0


def test_the_binding_refuses_tensors_it_cannot_take():
    torch = pytest.importorskip("torch")
    x = torch.zeros((4, 8), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="device"):
        L.linear(x, x)
    with pytest.raises(ValueError, match="device"):
        L.group_norm(x[None], 2)
    with pytest.raises(ValueError, match="images"):
        L.group_norm(x, 2)
    cache = A.KVCache(4, 2, 64, device="cpu")
    table = torch.zeros((2, 3), dtype=torch.int32)
    with pytest.raises(ValueError, match="device"):
        P.kv_resize(cache, P.kv_users(cache), table, table[:, 0].contiguous())
    with pytest.raises(ValueError, match="device"):
        P.kv_copy(cache, table[0], cache, table[0])


def test_group_norm_takes_groups_that_do_not_divide():
    """A prime number of groups is no reason to refuse: slices of one group then."""
    for groups, per_group, dtype in ((65537, 1, B.BF16), (65537, 8, B.BF16), (65537, 16, B.F32), (4099, 5, B.F16), (7, 16384, B.F32)):
        channels = groups * per_group
        rows = 10000
        d = _norm_desc(images=1, rows=rows, max_rows=rows, channels=channels, groups=groups, dtype=dtype, x_row=channels, out_row=channels)
        assert _bytes(L, "fc_group_norm", d) >= 0


class _Stream:
    device_index, cuda_stream = 1, 0


def test_a_stream_of_another_device_is_refused():
    call = L.PreparedLinear.__new__(L.PreparedLinear)
    call._device = 0
    with pytest.raises(ValueError, match="cuda:0, the stream on cuda:1"):
        call(_Stream())
    call = P.PreparedFork.__new__(P.PreparedFork)
    call._device = 0
    with pytest.raises(ValueError, match="cuda:0, the stream on cuda:1"):
        call(_Stream())
