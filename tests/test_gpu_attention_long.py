"""Attention over long axes and many rows: the cuts into pieces, tiles and whole lists that only larger calls take.  Rows are sampled, since the definition
in 64 bits takes its time.  Sequences may share blocks that nobody appends to, so many of them need no more cache than one."""
import numpy as np
import pytest

from paper_2207_10741_amd import attention as A, binding as B
from tests import attention_oracle as O, gpu_util as G
from tests.test_gpu_attention import LAST_PLACE, LEAST, Setup, _int32

pytestmark = pytest.mark.gpu


def _check(setup, out, q, picks, news, lists=None, causal=True, lse=None):
    """picks: (sequence of the oracle, row of the call, position)"""
    scale = 1.0 / np.sqrt(setup.dim)
    for b, row, position in picks:
        want, want_lse, error = O.attend(setup.oracle[b], q[row], position, scale, causal, None if lists is None else lists[row])
        allowed = error + LAST_PLACE[setup.dtype] * (np.abs(want) + error) + LEAST[setup.dtype]
        off = np.abs(G.to_f64(out[row]) - want)
        assert (off <= allowed).all(), "row %d: off by %g where %g is allowed" % (row, (off - allowed).max(), allowed.flat[np.argmax(off - allowed)])
        if lse is not None:
            assert np.abs(G.to_f64(lse[row]) - want_lse).max() < 1e-4 * (1 + np.abs(want_lse).max())


LONG = [
    # (length, new tokens, key heads, group, head size, type, causal)
    (9000, 1, 1, 8, 128, B.BF16, True),             # pieces of four waves
    (40000, 1, 1, 4, 64, B.F16, True),              # pieces of eight
    (20001, 1, 2, 16, 128, B.BF16, True),
    (9000, 3, 1, 8, 128, B.F16, True),              # 24 rows
    (9000, 2, 1, 13, 64, B.BF16, False),
    (5000, 1, 1, 3, 256, B.BF16, True),
    (3000, 100, 1, 1, 64, B.BF16, True),            # many rows, in pieces
    (2000, 300, 2, 3, 128, B.F16, True),
    (1500, 70, 1, 4, 256, B.BF16, True),
    (900, 40, 1, 5, 192, B.F16, False),
    (2100, 2100, 16, 4, 128, B.BF16, True),         # 256 rows a workgroup
    (2100, 2050, 16, 4, 120, B.F16, False),
    (1300, 1300, 4, 2, 128, B.BF16, True),
]


@pytest.mark.parametrize("length,new,heads,group,dim,dtype,causal", LONG)
def test_rows_of_long_calls(length, new, heads, group, dim, dtype, causal):
    torch = G.torch_mod()
    setup = Setup([length], heads, dim, dtype)
    q, qn = setup.queries(new, group)
    lse = torch.empty(q.shape[:2], dtype=torch.float32, device=G.dev())
    out = A.cache_attention(setup.cache, q, setup.table, setup.lengths_dev, causal=causal, lse=lse)
    rows = sorted({0, new - 1, new // 2, new // 3, min(31, new - 1), min(32, new - 1), min(127, new - 1), min(128, new - 1)})
    _check(setup, out, qn, [(0, r, length - new + r) for r in rows], [new], causal=causal, lse=lse)


def _shared(length, batch, dim, dtype, heads=1):
    """`batch` sequences of the same blocks."""
    setup = Setup([length], heads, dim, dtype)
    table = setup.table.expand(batch, -1).contiguous()
    return setup, table, _int32([length] * batch)


@pytest.mark.parametrize("dim,dtype", [(64, B.BF16), (128, B.F16)])
def test_more_than_64_blocks_a_wave(dim, dtype):
    """As many sequences as leave each its axis in one piece: a wave looks more than 64 blocks up."""
    length, batch = 64 * 4 * 65 + 37, 530
    setup, table, lengths = _shared(length, batch, dim, dtype)
    q, qn = setup.queries(batch, 2)
    out = A.cache_attention(setup.cache, q, table, lengths)
    _check(setup, out, qn, [(0, r, length - 1) for r in (0, 263, batch - 1)], None)


@pytest.mark.parametrize("dim,dtype", [(64, B.F16), (128, B.BF16), (192, B.BF16)])
def test_more_than_64_blocks_a_tile(dim, dtype):
    length, batch, new = 64 * 131 + 9, 260, 40
    setup, table, lengths = _shared(length, batch, dim, dtype)
    q, qn = setup.queries(batch * new, 1)
    out = A.cache_attention(setup.cache, q, table, lengths)
    _check(setup, out, qn, [(0, b * new + i, length - new + i) for b, i in ((0, 0), (101, 17), (259, 39))], None)


@pytest.mark.parametrize("top", [3, 70])
def test_whole_lists_of_a_wave(top):
    """Enough tokens for a wave each; lists of more than 64 blocks."""
    length, batch = 64 * 90 + 5, 1100
    setup, table, lengths = _shared(length, batch, 64, B.BF16)
    q, qn = setup.queries(batch, 3)
    out, selected = A.focused_attention(setup.cache, q, table, lengths, first=1, last=2, top=top)
    picks = (0, 513, batch - 1)
    lists = {r: O.select(setup.oracle[0], qn[r], length - 1, 1, 2, top) for r in picks}
    for r in picks:
        assert np.array_equal(selected[r].cpu().numpy(), lists[r])
    _check(setup, out, qn, [(0, r, length - 1) for r in picks], None, lists=lists)


@pytest.mark.parametrize("heads,group,dim,dtype", [(2, 4, 128, B.BF16), (1, 18, 64, B.F16), (1, 2, 200, B.BF16)])
def test_lists_of_a_piece_of_a_prompt(heads, group, dim, dtype):
    length, new = 4000, 1100
    setup = Setup([length], heads, dim, dtype)
    q, qn = setup.queries(new, group)
    out, selected = A.focused_attention(setup.cache, q, setup.table, setup.lengths_dev, first=2, last=1, top=5)
    picks = (0, 15, 16, 555, new - 1)
    lists = {r: O.select(setup.oracle[0], qn[r], length - new + r, 2, 1, 5) for r in picks}
    for r in picks:
        assert np.array_equal(selected[r].cpu().numpy(), lists[r])
    _check(setup, out, qn, [(0, r, length - new + r) for r in picks], None, lists=lists)


@pytest.mark.parametrize("top", [1, 64, 65, 200])
def test_thresholds_with_many_equal_keys(top):
    """Scores of three values only: the threshold lies among equal ones, for one token and for sixteen at once."""
    def three(b, k, v):
        blocks = k.shape[0] // 64
        kinds = np.random.default_rng(5).integers(0, 3, size=blocks).repeat(64)
        base = k[:64]
        return np.tile(base, (blocks, 1, 1)) * (1.0 + kinds[:, None, None]), v
    setup = Setup([64 * 300], 1, 64, B.BF16, tokens=three)
    for new in (1, 5):
        q, qn = setup.queries(new, 2)
        _, selected = A.focused_attention(setup.cache, q, setup.table, setup.lengths_dev, first=0, last=1, top=top)
        for r in range(new):
            assert np.array_equal(selected[r].cpu().numpy(), O.select(setup.oracle[0], qn[r], 64 * 300 - new + r, 0, 1, top))


@pytest.mark.parametrize("new", [200, 1])
def test_nan_in_pieces(new):
    """NaN of later tokens in a call whose axis is cut, and of tokens that all rows see."""
    length = 3000

    def poisoned(b, k, v):
        v[2900, :, 3] = np.inf
        v[100, :, 5] = np.nan
        return k, v
    setup = Setup([length], 1, 128, B.BF16, tokens=poisoned)
    q, qn = setup.queries(new, 2)
    out = G.to_f64(A.cache_attention(setup.cache, q, setup.table, setup.lengths_dev))
    assert np.isnan(out[:, :, 5]).all()
    sees = np.arange(length - new, length) >= 2900
    assert np.isnan(out[sees][:, :, 3]).all() and np.isfinite(out[~sees][:, :, 3]).all()
    others = [c for c in range(128) if c not in (3, 5)]
    assert np.isfinite(out[:, :, others]).all()


@pytest.mark.parametrize("group,dim,dtype,top", [(1, 64, B.BF16, 2), (2, 128, B.F16, 9), (3, 64, B.BF16, 5), (5, 96, B.F16, 20), (8, 192, B.BF16, 3)])
def test_neighbouring_tokens_together(group, dim, dtype, top):
    """Tokens whose lists a wave takes together: rows that share some blocks and not others, sequences' last tokens that do not fill a wave."""
    length, batch, new = 64 * 40 + 13, 1100, 19
    setup, table, lengths = _shared(length, batch, dim, dtype)
    q, qn = setup.queries(batch * new, group)
    out, selected = A.focused_attention(setup.cache, q, table, lengths, first=1, last=1, top=top)
    picks = [(b * new + i, length - new + i) for b, i in ((0, 0), (0, 18), (311, 4), (311, 5), (1099, 15), (1099, 16), (1099, 18))]
    lists = {r: O.select(setup.oracle[0], qn[r], position, 1, 1, top) for r, position in picks}
    for r, _ in picks:
        assert np.array_equal(selected[r].cpu().numpy(), lists[r])
    _check(setup, out, qn, [(0, r, position) for r, position in picks], None, lists=lists)


def test_blocks_of_other_tokens_have_no_influence():
    """Keys and values that are NaN or infinite in a block that neighbours select and a token does not."""
    length, batch, new = 64 * 40, 2100, 8

    def poisoned(b, k, v):
        k[64 * 7 + 3, :, 2] = np.nan
        v[64 * 9 + 5, :, 4] = np.inf
        return k, v
    setup = Setup([length], 1, 64, B.BF16, tokens=poisoned)
    table, lengths = setup.table.expand(batch, -1).contiguous(), _int32([length] * batch)
    q, qn = setup.queries(batch * new, 2)
    out, selected = A.focused_attention(setup.cache, q, table, lengths, first=0, last=1, top=4)
    out, selected = G.to_f64(out), selected.cpu().numpy()[:, 0]
    key, value = (selected == 7).any(axis=1), (selected == 9).any(axis=1)
    assert 0 < key.sum() < len(key) and 0 < value.sum() < len(value)
    assert np.isnan(out[key]).all()
    assert np.isfinite(out[~key & ~value]).all()
    assert np.isnan(out[~key & value][:, :, 4]).all() and np.isfinite(np.delete(out[~key & value], 4, axis=2)).all()
    # the same rows one by one
    for r in np.flatnonzero(~key)[:3]:
        want, _, error = O.attend(setup.oracle[0], qn[r], length - new + r % new, 0.125, True, selected[r][None])
        assert (np.abs(out[r] - want)[~np.isnan(want)] <= (error + LAST_PLACE[B.BF16] * (np.abs(want) + error))[~np.isnan(want)]).all()
