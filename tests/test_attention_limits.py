"""Refusals of sizes that the attention operators cannot take: found on the host before anything is launched (no GPU needed)."""
import ctypes

import pytest

from paper_2207_10741_amd import attention as A
from tests.test_attention_api import CALLS, RANGE, SHAPE, _append, _attend, _desc, _focused, _p


def _workspace(d, name="fc_focused_attention"):
    need = ctypes.c_size_t()
    return getattr(A.lib(), name + "_workspace_bytes")(ctypes.byref(d), ctypes.byref(need))


def test_more_heads_a_key_head_than_a_score_can_sum():
    """A group's rounded queries are held in three 8-bit digits: up to 255 each, 32767 heads and no more."""
    most = dict(kv_heads=1, batch=1, tokens=1, max_new=1)
    assert _workspace(_desc(heads=32767, **most)) == 0
    for heads in (32768, 2 ** 20):
        assert _workspace(_desc(heads=heads, **most)) == RANGE
        assert _focused(_desc(heads=heads, **most), starts=_p(9)) == RANGE
        assert _workspace(_desc(heads=heads, **most), "fc_cache_attention") == 0


def _refused(call, name, **kw):
    """Both the workspace's size (where there is one) and the call."""
    if name:
        assert _workspace(_desc(**kw), name) == RANGE
    assert call(_desc(**kw), starts=_p(9)) == RANGE


def test_more_threads_than_a_launch_of_the_selection_holds():
    """A dimension of a grid holds fewer than 2^32 threads."""
    # a token a workgroup of 1024 (sequences of more than 8192 blocks)
    long = dict(batch=1, kv_heads=8, heads=8, max_len=640000, table_width=10000)
    _refused(_focused, "fc_focused_attention", tokens=600000, max_new=600000, **long)
    assert _workspace(_desc(tokens=500000, max_new=500000, **long)) == 0
    # 16 tokens a workgroup of 256; the bound counts, not the tokens
    many = dict(batch=512, kv_heads=8, heads=8, max_new=131072, max_len=131072, table_width=2048)
    _refused(_focused, "fc_focused_attention", tokens=131583, **many)
    assert _workspace(_desc(tokens=131583, **{**many, "batch": 250})) == 0


def test_more_threads_than_a_launch_of_attention_holds():
    few = dict(batch=65535, max_new=1, tokens=65535, max_len=64, table_width=1)
    _refused(_attend, "fc_cache_attention", kv_heads=512, heads=512, **few)
    assert _workspace(_desc(kv_heads=128, heads=128, **few), "fc_cache_attention") == 0
    prompts = dict(batch=65535, max_new=4096, tokens=70000, max_len=4096, table_width=64, heads=16)
    _refused(_attend, "fc_cache_attention", kv_heads=16, **prompts)
    # lists: a wave a token and key head
    tokens = dict(batch=60000, max_new=1000, tokens=70000, max_len=1000, table_width=16)
    _refused(_focused, "fc_focused_attention", kv_heads=2, heads=64, **tokens)


def test_more_threads_than_a_launch_of_appending_holds():
    many = dict(batch=65535, max_new=1, tokens=65535, max_len=64, table_width=1, heads=1100)
    _refused(_append, None, kv_heads=1100, **many)


@pytest.mark.parametrize("call", CALLS)
def test_no_rows_without_starts(call):
    """Whatever the bound of new tokens is: nothing to do."""
    for max_new in (1, 7):
        assert call(_desc(tokens=0, max_new=max_new), cache=None, table=None, lengths=None) == 0
    assert call(_desc(tokens=1)) == SHAPE
