"""Sizes up to group norm's limits are not refused.  No GPU is needed."""
import ctypes

import pytest

from paper_2207_10741_amd import binding as B, layers as L


def _bytes(groups, per_group, dtype, rows, images=1, flags=0):
    channels, b = groups * per_group, ctypes.c_size_t()
    d = L.GroupNormDesc(images=images, rows=images * rows, max_rows=rows, channels=channels, groups=groups, dtype=dtype, eps=1e-5, x_row=channels, out_row=channels, flags=flags)
    rc = L.lib().fc_group_norm_workspace_bytes(ctypes.byref(d), ctypes.byref(b))
    return rc if rc else b.value


# pieces of 16 bytes put several groups into a slice
@pytest.mark.parametrize("rows", [1, 10, 10000])
@pytest.mark.parametrize("groups,per_group,dtype", [(8, 2561, B.BF16), (4, 5122, B.BF16), (16, 3001, B.BF16), (8, 16383, B.F16), (2, 16380, B.F16), (4, 16383, B.F32), (4, 16382, B.F32),
                                                    (8, 16383, B.F32)])
def test_long_groups_that_are_not_whole_pieces(groups, per_group, dtype, rows):
    assert _bytes(groups, per_group, dtype, rows) >= 0


def test_every_group_size_is_taken():
    for dtype, most in ((B.BF16, 8), (B.F16, 8), (B.F32, 4)):
        for groups in (1, 2, 3, 4, 5, 8, 12, 16, 64):
            for per_group in list(range(1, 40)) + list(range(40, L.GROUP_MAX_CHANNELS, 101)) + list(range(L.GROUP_MAX_CHANNELS - 20, L.GROUP_MAX_CHANNELS + 1)):
                for rows in (3, 5000):
                    assert _bytes(groups, per_group, dtype, rows) >= 0, (dtype, groups, per_group, rows)
