"""Values near the ends of what bf16 and the cache's scales hold: sums of weighted values pass 32 bits' range where the result, which is no
larger than the values, does not.  Rows are compared with the definition in 64 bits, with the bounds of the other attention tests."""
import numpy as np
import pytest

from paper_2207_10741_amd import attention as A, binding as B
from tests import attention_oracle as O, gpu_util as G
from tests.test_gpu_attention import LAST_PLACE, LEAST, Setup, _int32

pytestmark = pytest.mark.gpu


def _check(setup, out, qn, picks, lists=None, causal=True):
    """picks: (row of the call, position)"""
    for row, position in picks:
        want, _, error = O.attend(setup.oracle[0], qn[row], position, setup.dim ** -0.5, causal, None if lists is None else lists[row])
        allowed = error + LAST_PLACE[setup.dtype] * (np.abs(want) + error) + LEAST[setup.dtype]
        off = np.abs(G.to_f64(out[row]) - want)
        assert (off <= allowed).all(), "row %d: off by %g where %g is allowed, %g wanted" % (
            row, np.nanmax(off), allowed.flat[np.nanargmax(off)], want.flat[np.nanargmax(off)])


def _rows(new):
    return sorted({0, new - 1, new // 2, min(31, new - 1), min(128, new - 1)})


def _attend(setup, new, group, causal=True, magnitude=0.05):
    """Rows that weigh all tokens about alike."""
    q, qn = setup.queries(new, group, magnitude)
    out = A.cache_attention(setup.cache, q, setup.table, setup.lengths_dev, causal=causal)
    _check(setup, out, qn, [(r, setup.lengths[0] - new + r) for r in _rows(new)], causal=causal)


def _focus(setup, batch, new, group, first, last, top, magnitude=0.05):
    """`batch` sequences of the same blocks."""
    length = setup.lengths[0]
    table = setup.table.expand(batch, -1).contiguous()
    q, qn = setup.queries(batch * new, group, magnitude)
    out, selected = A.focused_attention(setup.cache, q, table, _int32([length] * batch), first, last, top)
    picks = [(b * new + i, length - new + i) for b, i in ((0, 0), (0, new - 1), (batch - 1, new // 2))]
    lists = {r: O.select(setup.oracle[0], qn[r], position, first, last, top) for r, position in picks}
    for r, _ in picks:
        assert np.array_equal(selected[r].cpu().numpy(), lists[r])
    _check(setup, out, qn, picks, lists)


# (length, new tokens, key heads, group, head size, causal)
DENSE = [
    (300, 1, 2, 4, 64, True),               # one piece
    (6000, 1, 1, 8, 128, True),             # pieces
    (20001, 1, 1, 16, 64, True),            # pieces of eight waves
    (3000, 3, 1, 8, 128, True),             # 24 rows
    (1000, 2, 1, 4, 256, True),
    (300, 300, 1, 2, 64, True),             # many rows
    (3000, 100, 1, 1, 80, False),           # many rows in pieces
    (700, 60, 1, 3, 192, True),
    (2100, 2100, 16, 4, 128, True),         # 256 rows a workgroup
]
# (length, sequences, new tokens, group, head size, first, last, top)
FOCUSED = [
    (6000, 1, 1, 4, 128, 1, 2, 60),         # pieces of lists
    (1000, 1100, 1, 3, 64, 1, 1, 5),        # a list a wave
    (2000, 1100, 19, 4, 96, 1, 1, 5),       # neighbouring tokens' lists
]


@pytest.mark.parametrize("length,new,heads,group,dim,causal", DENSE)
def test_means_of_large_values(length, new, heads, group, dim, causal):
    setup = Setup([length], heads, dim, B.BF16, scale_of=lambda n: np.full(n, 2.0 ** 124))
    _attend(setup, new, group, causal)


@pytest.mark.parametrize("length,batch,new,group,dim,first,last,top", FOCUSED)
def test_means_of_large_values_over_selected_blocks(length, batch, new, group, dim, first, last, top):
    setup = Setup([length], 1, dim, B.BF16, scale_of=lambda n: np.full(n, 2.0 ** 124))
    _focus(setup, batch, new, group, first, last, top)


@pytest.mark.parametrize("length,new,heads,group,dim,causal", DENSE)
def test_means_of_small_values(length, new, heads, group, dim, causal):
    """Below the least scale's 448: the codes get smaller, and so do the sums."""
    setup = Setup([length], heads, dim, B.BF16, scale_of=lambda n: np.full(n, 2.0 ** -64))
    _attend(setup, new, group, causal)
