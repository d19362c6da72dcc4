"""Lengths that count tokens which were never appended: the blocks hold what the memory held.  Results mean nothing then, but lists are whole and name blocks
of the sequence."""
import numpy as np
import pytest

from paper_2207_10741_amd import attention as A, binding as B
from tests import gpu_util as G
from tests.test_gpu_attention import Setup, _int32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("new", [1, 20])
@pytest.mark.parametrize("blocks,top", [(40, 3), (200, 20), (300, 64), (300, 65), (1100, 40)])
def test_blocks_that_were_never_written(blocks, top, new):
    """As many of them among the candidates as are chosen, fewer, and more; their weights are NaN, infinite or zero."""
    torch = G.torch_mod()
    setup = Setup([64 * blocks], 1, 64, B.BF16, pool_more=top + 7)
    unused = np.setdiff1d(np.arange(setup.pool), setup.table_np)
    q, _ = setup.queries(new, 2)
    for bits in (0x7fffffff, -1, 0x7f800000, -0x800000, 0):
        cache = A.KVCache(setup.pool, 1, 64, device=G.dev())
        cache.data.view(torch.int32).fill_(bits)
        A.kv_append(cache, setup.k, setup.v, setup.table, setup.lengths_dev)
        for never in (top, top // 2, top + 7):
            table = setup.table_np.copy()
            table[0, np.random.default_rng(7).permutation(blocks - 4)[:never] + 2] = unused[:never]
            selected = torch.full((new, 1, 2 + top), 2 ** 29, dtype=torch.int32, device=G.dev())
            A.focused_attention(cache, q, _int32(table), setup.lengths_dev, 1, 1, top, selected=selected)
            lists = selected.cpu().numpy()[:, 0]
            assert (np.diff(lists, axis=1) > 0).all() and (lists[:, 0] == 0).all() and (lists[:, -1] == blocks - 1).all()
