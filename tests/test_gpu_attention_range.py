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


def _blocks_of(exponents, poison=()):
    """Values of about 2^e in the blocks, one exponent after another (None: zeros), every other channel of a block: those of the next one's are zero there, so
    that nothing hides what a block of small values adds.  poison: (token, channel) of values that are infinite."""
    def tokens(b, k, v):
        n = v.shape[0]
        nth = np.arange(n) // 64 % len(exponents)
        v = v * np.array([0.0 if e is None else 2.0 ** e for e in exponents])[nth][:, None, None]
        v *= ((np.arange(n)[:, None] // 64 + np.arange(v.shape[2])[None, :]) % 2)[:, None, :]
        for t, c in poison:
            v[t, :, c] = np.inf
        return k, v
    return tokens


PATTERNS = [
    (66, None),                     # what a block of zeros has for a scale is far below
    (None, 66),
    (None, None, 124),
    (-64, 124),
    (124, -64, 0, 60, -20),
    (-64, -20, 20, 60, 100, 124),
    (10, -50),                      # (the sums follow the blocks)
]


@pytest.mark.parametrize("exponents", PATTERNS)
@pytest.mark.parametrize("length,new,heads,group,dim,causal", DENSE)
def test_blocks_of_very_different_values(length, new, heads, group, dim, causal, exponents):
    setup = Setup([length], heads, dim, B.BF16, tokens=_blocks_of(exponents))
    _attend(setup, new, group, causal, magnitude=0.3)


@pytest.mark.parametrize("exponents", [(66, None), (124, -64, 0, 60, -20), (10, -50)])
@pytest.mark.parametrize("length,batch,new,group,dim,first,last,top", FOCUSED)
def test_selected_blocks_of_very_different_values(length, batch, new, group, dim, first, last, top, exponents):
    setup = Setup([length], 1, dim, B.BF16, tokens=_blocks_of(exponents))
    _focus(setup, batch, new, group, first, last, top, magnitude=0.3)


@pytest.mark.parametrize("new", [1, 5, 140])
@pytest.mark.parametrize("exponents", [(124, -64), (-64, 124)])
def test_nan_in_blocks_of_very_different_values(exponents, new):
    """A value that later rows see and earlier ones do not, in the last block or the one before it."""
    for at in (190, 255):
        length = 64 * 4
        setup = Setup([length], 1, 64, B.BF16, tokens=_blocks_of(exponents, [(at, 3)]))
        q, qn = setup.queries(new, 2, 0.3)
        out = A.cache_attention(setup.cache, q, setup.table, setup.lengths_dev)
        sees = np.arange(length - new, length) >= at
        got = G.to_f64(out)
        assert np.isnan(got[sees][:, :, 3]).all() and np.isfinite(got[~sees]).all()
        got = np.delete(got, 3, axis=2)
        assert np.isfinite(got).all()
        for row in _rows(new):
            want, _, error = O.attend(setup.oracle[0], qn[row], length - new + row, 0.125)
            off = np.abs(got[row] - np.delete(want, 3, axis=1))
            assert (off <= np.delete(error + LAST_PLACE[B.BF16] * (np.abs(want) + error) + LEAST[B.BF16], 3, axis=1)).all()


@pytest.mark.parametrize("new", [1, 90])
@pytest.mark.parametrize("key_size,scale", [(1.0, 3.4e38), (2.0 ** 122, 2.0 ** 20), (2.0 ** 122, -3.4e38)])
def test_factors_of_scores_beyond_32_bits(key_size, scale, new):
    """A factor of the scores, with the keys' scale in it, that 32 bits do not hold: scores of zero are still zero."""
    setup = Setup([700], 1, 64, B.BF16, tokens=lambda b, k, v: (k * key_size, v))
    q, qn = setup.queries(new, 2, 0.0)
    out = A.cache_attention(setup.cache, q, setup.table, setup.lengths_dev, scale=scale)
    listed, selected = A.focused_attention(setup.cache, q, setup.table, setup.lengths_dev, 1, 1, 3, scale=scale)
    for row in _rows(new):
        position = 700 - new + row
        for got, blocks in ((out, None), (listed, selected[row].cpu().numpy())):
            want, _, error = O.attend(setup.oracle[0], qn[row], position, scale, True, blocks)
            allowed = error + LAST_PLACE[B.BF16] * (np.abs(want) + error) + LEAST[B.BF16]
            assert (np.abs(G.to_f64(got[row]) - want) <= allowed).all()


@pytest.mark.parametrize("new", [1, 90])
def test_scores_that_are_all_minus_infinity(new):
    """A query of infinity against keys of the other sign: nothing is attended to; of the same sign: NaN."""
    torch = G.torch_mod()

    def positive(b, k, v):
        k[:, :, 3] = 0.5 + np.abs(k[:, :, 3])
        return k, v
    setup = Setup([700], 1, 64, B.BF16, tokens=positive)
    q, _ = setup.queries(new, 2)
    q[:, 0, 3], q[:, 1, 3] = float("-inf"), float("inf")
    lse = torch.empty(q.shape[:2], dtype=torch.float32, device=G.dev())
    out = A.cache_attention(setup.cache, q, setup.table, setup.lengths_dev, lse=lse)
    listed, _ = A.focused_attention(setup.cache, q, setup.table, setup.lengths_dev, 1, 1, 3)
    for got in (G.to_f64(out), G.to_f64(listed)):
        assert (got[:, 0] == 0).all() and np.isnan(got[:, 1]).all()
    assert torch.isneginf(lse[:, 0]).all()
