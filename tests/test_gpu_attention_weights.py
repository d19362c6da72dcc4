"""Tokens that weigh little beside one that dominates, but are many: what their weights lose in 16 bits.

A row's weights are held so that its largest is 2^6 at least when they are rounded to f16, twice at most (as they are and, in the kernel of many rows, once more when
the row's reference rises), to half of 2^-24 each time: at most 2^-30 of the sum of weights is lost a token."""
import numpy as np
import pytest

from paper_2207_10741_amd import attention as A, binding as B
from tests import attention_oracle as O, gpu_util as G
from tests.test_gpu_attention import LAST_PLACE, LEAST, Setup, _int32, _tensor

pytestmark = pytest.mark.gpu

STEP = 2.0 ** -30


def _dominated(size, at):
    """All keys zero but one token's, which has no value itself: its rows get what the others add."""
    def tokens(b, k, v):
        k[:], v = 0.0, 1.0 + 0.1 * v
        k[at], v[at] = size, 0.0
        return k, v
    return tokens


@pytest.mark.parametrize("at", [0, 70, 4000])
@pytest.mark.parametrize("length,batch,new,group,dim,size,dtype", [
    (64 * 4 * 65 + 37, 530, 1, 2, 64, 2.25, B.BF16),        # a wave goes over 65 blocks
    (64 * 4 * 40, 530, 1, 3, 128, 1.625, B.F16),
    (64 * 131 + 9, 260, 40, 1, 64, 2.25, B.F16),            # a workgroup over 132
    (64 * 131 + 9, 260, 40, 1, 128, 1.625, B.BF16),
    (20000, 1, 1, 4, 64, 2.25, B.BF16),                     # pieces
    (9000, 1, 100, 4, 96, 1.875, B.BF16),                   # pieces of many rows
])
def test_many_tokens_of_small_weights(length, batch, new, group, dim, size, dtype, at):
    """Weights of about 2^-26 of the largest (scale * size * dim = 18.0 to 18.4)."""
    setup = Setup([length], 1, dim, dtype, tokens=_dominated(size, at))
    table = setup.table.expand(batch, -1).contiguous()
    q, qn = _tensor(np.ones((batch * new, group, dim)), dtype)
    out = A.cache_attention(setup.cache, q, table, _int32([length] * batch))
    v = setup.oracle[0].values("v")[:, 0]
    for b, i in {(0, 0), (batch // 2, new // 2), (batch - 1, new - 1)}:
        position = length - new + i
        want, _, error = O.attend(setup.oracle[0], qn[b * new + i], position, dim ** -0.5)
        total = np.abs(v[:position + 1]).sum(axis=0)
        error = error - 2.0 ** -25 * total + STEP * total
        off = np.abs(G.to_f64(out[b * new + i]) - want)
        allowed = error + LAST_PLACE[dtype] * (np.abs(want) + error) + LEAST[dtype]
        assert (off <= allowed).all(), "off by %g where %g is allowed, %g wanted" % (off.max(), allowed.min(), np.abs(want).max())
