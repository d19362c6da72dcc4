"""Selection with many query heads a key head: the sum of a group's rounded queries does not fit two 8-bit digits any more.

Selected blocks are compared for equality: the scores are sums of whole numbers."""
import numpy as np
import pytest

from paper_2207_10741_amd import attention as A, binding as B
from tests import attention_oracle as O, gpu_util as G
from tests.test_gpu_attention import Setup, _int32, _tensor

pytestmark = pytest.mark.gpu


def _selected(setup, rows, top, first=0, last=1):
    """rows [tokens, heads, dim] on the host, of values that the type holds."""
    q, qn = _tensor(rows.copy(), setup.dtype)
    assert np.array_equal(qn, rows)
    _, selected = A.focused_attention(setup.cache, q, setup.table, setup.lengths_dev, first, last, top)
    return selected.cpu().numpy()


@pytest.mark.parametrize("new", [1, 3])
@pytest.mark.parametrize("dim,dtype", [(64, B.BF16), (128, B.F16), (256, B.BF16)])
@pytest.mark.parametrize("group", [127, 128, 129, 130, 256, 515, 600])
def test_heads_that_agree(group, dim, dtype, new):
    """All heads of a group have the same queries, most channels at the largest magnitude: the largest sums there can be."""
    setup = Setup([64 * 40 + 5], 1, dim, dtype)
    signs = np.where(setup.rng.random((new, 1, dim)) < 0.5, -1.0, 1.0)
    sizes = np.where(setup.rng.random((new, 1, dim)) < 0.8, 127.0, 65.0)
    rows = np.broadcast_to(signs * sizes, (new, group, dim))
    got = _selected(setup, rows, 7)
    for i in range(new):
        assert np.array_equal(got[i], O.select(setup.oracle[0], rows[i], setup.lengths[0] - new + i, 0, 1, 7))


@pytest.mark.parametrize("new", [1, 3])
@pytest.mark.parametrize("group", [64, 65, 128, 140])
def test_queries_at_the_end_of_the_range(group, new):
    """Above 127 * 2^120 the unit of the queries does not grow any more: a rounded query is up to 255."""
    setup = Setup([64 * 30], 1, 64, B.BF16)
    most = 3.3895313892515355e38
    rows = np.broadcast_to(np.where(setup.rng.random((new, 1, 64)) < 0.5, -most, most), (new, group, 64))
    got = _selected(setup, rows, 5)
    for i in range(new):
        assert np.array_equal(got[i], O.select(setup.oracle[0], rows[i], setup.lengths[0] - new + i, 0, 1, 5))


@pytest.mark.parametrize("batch,new", [(1, 20), (70, 1)])
def test_several_key_heads_and_heads_that_differ(batch, new):
    """Ordinary queries of 160 heads a key head, and attention over what is selected."""
    length, dim, group = 64 * 20 + 9, 64, 160
    setup = Setup([length], 2, dim, B.BF16)
    table = setup.table.expand(batch, -1).contiguous()
    q, qn = setup.queries(batch * new, group)
    out, selected = A.focused_attention(setup.cache, q, table, _int32([length] * batch), 1, 1, 3)
    for b, i in {(0, 0), (0, new - 1), (batch - 1, new // 2)}:
        row, position = b * new + i, length - new + i
        blocks = O.select(setup.oracle[0], qn[row], position, 1, 1, 3)
        assert np.array_equal(selected[row].cpu().numpy(), blocks)
        want, _, error = O.attend(setup.oracle[0], qn[row], position, dim ** -0.5, True, blocks)
        off = np.abs(G.to_f64(out[row]) - want)
        assert (off <= error + 2.0 ** -8 * (np.abs(want) + error) + 2.0 ** -133).all()
