"""Refusals of sizes that the attention operators cannot take: found on the host before anything is launched (no GPU needed)."""
import ctypes

import pytest

from paper_2207_10741_amd import attention as A, binding as B
from tests.test_attention_api import RANGE, _desc, _focused, _p


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
