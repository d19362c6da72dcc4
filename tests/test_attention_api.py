"""Host-side checks of the attention operators' C ABI that need no GPU: exported symbols, sizes, refusals before anything is launched."""
import ctypes
import os
import re

import pytest

from paper_2207_10741_amd import attention as A, binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER_TEXT = open(os.path.join(ROOT, "include", "focused_attention.h")).read()
NULL, SHAPE, DTYPE, ALIGN, WORKSPACE, RANGE = -1, -2, -3, -4, -5, -6


def test_every_declared_symbol_is_exported_and_bound():
    text = re.sub(r"/\*.*?\*/", "", HEADER_TEXT, flags=re.S)
    names = set(re.findall(r"\b(fc_[a-z0-9_]+)\s*\(", text))
    assert names == set(A.FUNCTIONS)
    for n in names:
        assert getattr(A.lib(), n) is not None


def test_constants_and_the_descriptor_mirror_the_header():
    for name, value in (("FC_KV_BLOCK", A.BLOCK), ("FC_KV_MAX_HEAD_DIM", A.MAX_HEAD_DIM), ("FC_MAX_SELECTED", A.MAX_SELECTED)):
        assert value == int(re.search(name + r"\s*=\s*(\d+)", HEADER_TEXT).group(1))
    body = re.search(r"typedef struct \{(.*?)\} fc_attention_desc;", HEADER_TEXT, re.S).group(1)
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
    fields = [n.strip() for line in body.split(";") if line.strip() for n in line.strip().split(" ", 1)[1].split(",")]
    assert fields == [n for n, _ in A.AttentionDesc._fields_]


def _desc(**kw):
    base = dict(blocks=100, kv_heads=2, head_dim=64, batch=3, tokens=6, max_new=2, max_len=500, table_width=8, heads=8, dtype=B.BF16,
                flags=A.CAUSAL, first=1, last=1, top=4, scale=0.125, q_row=512, q_head=64, k_row=128, k_head=64, v_row=128, v_head=64)
    base.update(kw)
    return A.AttentionDesc(**base)


def _p(n):
    return ctypes.c_void_p(16 * n)      # (never read: the call is refused first)


def _append(d, cache=_p(1), k=_p(2), v=_p(3), table=_p(4), lengths=_p(5), starts=None):
    return A.lib().fc_kv_append(None if d is None else ctypes.byref(d), cache, k, v, table, lengths, starts, None)


def _read(d, cache=_p(1), table=_p(4), lengths=_p(5), starts=None, k=_p(2), v=_p(3)):
    return A.lib().fc_kv_read(None if d is None else ctypes.byref(d), cache, table, lengths, starts, k, v, None)


def _attend(d, cache=_p(1), q=_p(2), table=_p(4), lengths=_p(5), starts=None, out=_p(6), lse=None, ws=_p(7), ws_bytes=1 << 40):
    return A.lib().fc_cache_attention(None if d is None else ctypes.byref(d), cache, q, table, lengths, starts, out, lse, ws, ws_bytes, None)


def _focused(d, cache=_p(1), q=_p(2), table=_p(4), lengths=_p(5), starts=None, out=_p(6), lse=None, selected=_p(8), ws=_p(7), ws_bytes=1 << 40):
    return A.lib().fc_focused_attention(None if d is None else ctypes.byref(d), cache, q, table, lengths, starts, out, lse, selected, ws, ws_bytes,
                                        None)


CALLS = [_append, _read, _attend, _focused]


@pytest.mark.parametrize("call", CALLS)
def test_sequences_and_cache_are_checked(call):
    assert call(None) == NULL
    for name in ("blocks", "kv_heads", "head_dim", "batch", "max_new", "max_len", "table_width"):
        assert call(_desc(**{name: 0})) == SHAPE and call(_desc(**{name: -1})) == SHAPE
    assert call(_desc(tokens=-1)) == SHAPE and call(_desc(tokens=7)) == SHAPE       # (no starts: batch * max_new rows)
    assert call(_desc(head_dim=257)) == SHAPE
    assert call(_desc(blocks=2 ** 30, kv_heads=4, heads=8)) == RANGE
    assert call(_desc(batch=70000, tokens=140000)) == RANGE
    assert call(_desc(flags=2)) == DTYPE and call(_desc(reserved=1)) == DTYPE
    assert call(_desc(), cache=None) == NULL and call(_desc(), table=None) == NULL and call(_desc(), lengths=None) == NULL
    for name in ("cache", "table", "lengths", "starts"):
        assert call(_desc(), **{name: ctypes.c_void_p(24)}) == ALIGN


@pytest.mark.parametrize("call", CALLS)
def test_no_rows_is_nothing_to_do(call):
    assert call(_desc(tokens=0), cache=None, table=None, lengths=None, starts=_p(9)) == 0


def test_append_and_read_refuse():
    assert _append(_desc(dtype=B.F32)) == DTYPE and _append(_desc(dtype=B.FP8)) == DTYPE
    for name in ("k_row", "k_head", "v_row", "v_head"):
        assert _append(_desc(**{name: -1})) == SHAPE
    assert _append(_desc(), k=None) == NULL and _append(_desc(), v=None) == NULL
    assert _append(_desc(), k=ctypes.c_void_p(33)) == ALIGN
    assert _read(_desc(), k=None, v=None) == NULL and _read(_desc(), v=ctypes.c_void_p(20)) == ALIGN


@pytest.mark.parametrize("call", [_append, _read])
def test_more_blocks_than_a_grid_holds_are_refused(call):
    many = dict(batch=1, kv_heads=16, heads=16, max_new=2 ** 26, max_len=2 ** 30, table_width=2 ** 24)
    assert call(_desc(tokens=2 ** 26, **many), starts=_p(9)) == RANGE
    assert call(_desc(tokens=0, **many), starts=_p(9)) == 0         # (the rows bound the blocks that new tokens touch)


@pytest.mark.parametrize("call", [_attend, _focused])
def test_attention_refuses(call):
    assert call(_desc(heads=7)) == SHAPE and call(_desc(heads=0)) == SHAPE and call(_desc(heads=-2)) == SHAPE
    assert call(_desc(dtype=B.F32)) == DTYPE
    for scale in (float("nan"), float("inf")):
        assert call(_desc(scale=scale)) == SHAPE
    assert call(_desc(q_row=-1)) == SHAPE and call(_desc(q_head=-1)) == SHAPE
    assert call(_desc(tokens=2 ** 29, heads=8), starts=_p(9)) == RANGE
    assert call(_desc(), q=None) == NULL and call(_desc(), out=None) == NULL
    assert call(_desc(), q=ctypes.c_void_p(33)) == ALIGN and call(_desc(), out=ctypes.c_void_p(34)) == ALIGN
    assert call(_desc(), lse=ctypes.c_void_p(36)) == ALIGN
    many = dict(max_len=100000, table_width=2000)
    if call is _focused:
        many.update(top=60)
    assert call(_desc(**many), ws=None) == WORKSPACE and call(_desc(**many), ws_bytes=16) == WORKSPACE
    assert call(_desc(**many), ws=ctypes.c_void_p(24)) == ALIGN


def test_selection_refuses():
    for bad in (dict(first=-1), dict(last=0), dict(top=-1), dict(first=1000, last=20, top=10), dict(top=2 ** 31 - 1)):
        assert _focused(_desc(**bad)) == SHAPE
    assert _focused(_desc(), selected=None) == NULL and _focused(_desc(), selected=ctypes.c_void_p(20)) == ALIGN
    assert _focused(_desc(table_width=40000, max_len=64 * 32768 + 1)) == RANGE
    need = ctypes.c_size_t()
    d = _desc(table_width=40000, max_len=64 * 32768 + 1)
    assert A.lib().fc_focused_attention_workspace_bytes(ctypes.byref(d), ctypes.byref(need)) == RANGE
    assert A.lib().fc_cache_attention_workspace_bytes(ctypes.byref(d), ctypes.byref(need)) == 0


def test_sizes():
    assert A.cache_bytes(10, 2, 128) >= 10 * 2 * 128 * 128
    assert A.cache_bytes(10, 2, 65) == A.cache_bytes(10, 2, 96) < A.cache_bytes(10, 2, 97) == A.cache_bytes(10, 2, 128)
    assert A.cache_bytes(2 ** 20, 16, 128) > 2 ** 37
    with pytest.raises(B.FcError) as e:
        A.cache_bytes(0, 2, 128)
    assert e.value.status == SHAPE
    assert A.lib().fc_kv_cache_bytes(ctypes.byref(_desc()), None) == NULL
    # the table bounds the length: what it cannot hold needs no workspace
    short, long = _desc(table_width=8, max_len=2 ** 30), _desc(table_width=8, max_len=512)
    sizes = []
    for d in (short, long):
        b = ctypes.c_size_t()
        assert A.lib().fc_cache_attention_workspace_bytes(ctypes.byref(d), ctypes.byref(b)) == 0
        sizes.append(b.value)
    assert sizes[0] == sizes[1]


def test_the_binding_refuses_tensors_it_cannot_take():
    torch = pytest.importorskip("torch")
    cache = A.KVCache(4, 2, 64, device="cpu")
    k = torch.zeros((2, 2, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="device tensors"):
        A.kv_append(cache, k, k, torch.zeros((1, 2), dtype=torch.int32), torch.ones((1,), dtype=torch.int32))
