"""Attention over the 8-bit key/value cache against its definition in 64 bits (tests/attention_oracle.py).

What a cache holds is compared bit for bit, and so are selected blocks.  An output may be off by its own rounding (half a unit of the last
place of bf16 or f16) and by the error that 32-bit sums and 11-bit weights allow, which the oracle gives for each output."""
import numpy as np
import pytest

from paper_2207_10741_amd import attention as A, binding as B
from tests import attention_oracle as O, gpu_util as G

pytestmark = pytest.mark.gpu

LAST_PLACE = {B.BF16: 2.0 ** -8, B.F16: 2.0 ** -11}
LEAST = {B.BF16: 2.0 ** -133, B.F16: 2.0 ** -24}


def _tensor(x, dtype):
    """float64 array -> device tensor of the type, and the values it holds."""
    torch = G.torch_mod()
    t = torch.from_numpy(np.asarray(x, dtype=np.float64)).to(B.torch_dtype(dtype))
    return t.to(G.dev()), t.to(torch.float64).numpy()


def _int32(x):
    return G.torch_mod().from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(G.dev())


class Setup:
    """Sequences of given lengths in a cache on the device and in the oracle's."""

    def __init__(self, lengths, heads, dim, dtype, seed=3, pool_more=2, scale_of=None, tokens=None):
        rng = np.random.default_rng(seed)
        self.lengths, self.heads, self.dim, self.dtype, self.rng = list(lengths), heads, dim, dtype, rng
        width = max(1, max(-(-n // 64) for n in lengths))
        self.pool = sum(-(-n // 64) for n in lengths) + pool_more
        order, at = rng.permutation(self.pool), 0
        self.table_np = np.full((len(lengths), width), -1, dtype=np.int32)
        for b, n in enumerate(lengths):
            self.table_np[b, :-(-n // 64)] = order[at:at + -(-n // 64)]
            at += -(-n // 64)
        self.table = _int32(self.table_np)
        self.cache = A.KVCache(self.pool, heads, dim, device=G.dev())
        self.cache.data.fill_(0xff)                 # (NaN codes: nothing may read what was not written)
        self.oracle = [O.Cache(heads, dim) for _ in lengths]
        parts = []
        for b, n in enumerate(lengths):
            mean = rng.normal(size=(-(-n // 64), 1, heads, dim)).repeat(64, 1).reshape(-1, heads, dim)[:n]
            k = 0.7 * rng.normal(size=(n, heads, dim)) + 0.7 * mean
            v = rng.normal(size=(n, heads, dim)) * (1.0 if scale_of is None else scale_of(n)[:, None, None])
            parts.append((k, v) if tokens is None else tokens(b, k, v))
        self.k, k = _tensor(np.concatenate([p[0] for p in parts]), dtype)
        self.v, v = _tensor(np.concatenate([p[1] for p in parts]), dtype)
        starts = np.concatenate([[0], np.cumsum(lengths)])
        for b in range(len(lengths)):
            self.oracle[b].append(k[starts[b]:starts[b + 1]], v[starts[b]:starts[b + 1]])
        self.lengths_dev = _int32(lengths)
        if self.k.shape[0]:
            A.kv_append(self.cache, self.k, self.v, self.table, self.lengths_dev, starts=_int32(starts), max_new=max(lengths))

    def queries(self, rows, group, magnitude=1.5):
        return _tensor(magnitude * self.rng.normal(size=(rows, self.heads * group, self.dim)), self.dtype)


def _compare(setup, got, lse, q, news, causal=True, lists=None, scale=None):
    scale = 1.0 / np.sqrt(setup.dim) if scale is None else scale
    got, lse = G.to_f64(got), None if lse is None else G.to_f64(lse)
    row = 0
    for b, n in enumerate(news):
        for i in range(n):
            position = setup.lengths[b] - n + i
            want, want_lse, error = O.attend(setup.oracle[b], q[row], position, scale, causal, None if lists is None else lists[row])
            allowed = error + LAST_PLACE[setup.dtype] * (np.abs(want) + error) + LEAST[setup.dtype]
            off = np.abs(got[row] - want)
            assert np.array_equal(np.isnan(got[row]), np.isnan(want)), "NaN at row %d" % row
            assert not (off > allowed).any(), "row %d of sequence %d: off by %g where %g is allowed" % (
                i, b, np.nanmax(off - allowed), allowed.flat[np.nanargmax(off - allowed)])
            if lse is not None:
                assert np.array_equal(np.isneginf(lse[row]), np.isneginf(want_lse))
                some = np.isfinite(want_lse)
                assert np.array_equal(np.isnan(lse[row]), np.isnan(want_lse))
                # |z| 2^-23 a rounding of the exponent, its factor, the logarithm and the product behind it, dz of the oracle's bound
                bound = 2.0 ** -20 * (1 + np.abs(want_lse[some])) + 2.0 ** -20 * scale * np.abs(q[row][some]).sum(axis=1) * 16
                assert (np.abs(lse[row][some] - want_lse[some]) <= bound).all()
            row += 1


# ---- the cache ------------------------------------------------------------------

@pytest.mark.parametrize("dim", [1, 40, 64, 80, 128, 192, 250, 256])
@pytest.mark.parametrize("dtype", [B.BF16, B.F16])
def test_appends_of_all_sizes_and_read_back(dim, dtype):
    """Blocks begun, continued, filled and left; a later token may raise a block's scale, and codes that are there are rounded again."""
    torch = G.torch_mod()
    rng = np.random.default_rng(dim)
    heads, batch, steps = 3, 2, [1, 62, 1, 1, 130, 0, 5, 64, 7]
    total = sum(steps)
    width = -(-total // 64)
    cache = A.KVCache(batch * width + 1, heads, dim, device=G.dev())
    cache.data.fill_(0x7f)
    table = _int32(rng.permutation(batch * width + 1)[:batch * width].reshape(batch, width))
    oracle = [O.Cache(heads, dim) for _ in range(batch)]
    length = 0
    for step in steps:
        if step == 0:
            continue
        length += step
        magnitude = 2.0 ** rng.uniform(-9, 9, size=(batch * step, 1, 1))
        k, kn = _tensor(rng.normal(size=(batch * step, heads, dim)) * magnitude, dtype)
        v, vn = _tensor(rng.normal(size=(batch * step, heads, dim)) * magnitude[::-1], dtype)
        lengths = _int32([length] * batch)
        A.kv_append(cache, k, v, table, lengths)
        for b in range(batch):
            oracle[b].append(kn[b * step:(b + 1) * step], vn[b * step:(b + 1) * step])
        got = A.kv_read(cache, table, lengths, max_new=length)
        for n, t in zip("kv", got):
            want = np.concatenate([o.values(n) for o in oracle])
            assert np.array_equal(G.to_f64(t), want), "%s after %d tokens" % (n, length)
    # the last 70 tokens by themselves; one of the two only
    some = torch.empty((batch * 70, heads, dim), dtype=torch.float32, device=G.dev())
    A.kv_read(cache, table, lengths, max_new=70, v=some)
    assert np.array_equal(G.to_f64(some), np.concatenate([o.values("v")[-70:] for o in oracle]))


@pytest.mark.parametrize("dim,offset", [(64, 0), (80, 3), (33, 1)])
def test_append_from_slices_of_one_tensor(dim, offset):
    """Keys and values as slices of one projection's output: strides, and addresses off every alignment."""
    torch = G.torch_mod()
    rng = np.random.default_rng(1)
    heads, n = 2, 75
    flat, values = _tensor(rng.normal(size=(n * (6 * heads * dim) + 8,)), B.BF16)
    rows = flat[offset:offset + n * 6 * heads * dim].view(n, 6 * heads, dim)
    host = values[offset:offset + n * 6 * heads * dim].reshape(n, 6 * heads, dim)
    k, v = rows[:, 2 * heads:3 * heads], rows[:, 1:1 + 2 * heads:2]
    cache = A.KVCache(3, heads, dim, device=G.dev())
    table, lengths = _int32([[2, 0]]), _int32([n])
    A.kv_append(cache, k, v, table, lengths)
    oracle = O.Cache(heads, dim)
    oracle.append(host[:, 2 * heads:3 * heads], host[:, 1:1 + 2 * heads:2])
    for t, name in zip(A.kv_read(cache, table, lengths, max_new=n), "kv"):
        assert np.array_equal(G.to_f64(t), oracle.values(name))
    # one token's row for all (a stride of zero)
    A.kv_append(cache, k[:1].expand(n, heads, dim), v[:1].expand(n, heads, dim), table, lengths)
    again = O.Cache(heads, dim)
    again.append(np.broadcast_to(host[:1, 2 * heads:3 * heads], (n, heads, dim)), np.broadcast_to(host[:1, 1:1 + 2 * heads:2], (n, heads, dim)))
    for t, name in zip(A.kv_read(cache, table, lengths, max_new=n), "kv"):
        assert np.array_equal(G.to_f64(t), again.values(name))


@pytest.mark.parametrize("dtype", [B.BF16, B.F16])
def test_values_at_the_ends_of_the_range(dtype):
    """Not-finite values become NaN and do not count for the scale; the largest, the smallest and zeros."""
    heads, dim, n = 1, 64, 64
    x = np.zeros((4 * n, heads, dim))
    x[:n, 0, 0], x[3, 0, 5], x[7, 0, 1], x[9, 0, 2] = 3.0, np.inf, -np.inf, np.nan
    most = 65504.0 if dtype == B.F16 else 3.3895313892515355e38
    x[n:2 * n, 0, 3], x[n + 1, 0, 4] = most, 1.0
    x[2 * n:3 * n, 0, 6] = 2.0 ** -24 if dtype == B.F16 else 2.0 ** -133
    t, host = _tensor(x, dtype)
    cache = A.KVCache(4, heads, dim, device=G.dev())
    table, lengths = _int32([[1, 3, 0, 2]]), _int32([4 * n])
    A.kv_append(cache, t, t, table, lengths)
    oracle = O.Cache(heads, dim)
    oracle.append(host, host)
    for got, name in zip(A.kv_read(cache, table, lengths, max_new=4 * n), "kv"):
        got, want = G.to_f64(got), oracle.values(name)
        assert np.array_equal(np.isnan(got), np.isnan(want)) and np.isnan(got).sum() == 3
        with np.errstate(over="ignore"):        # (the largest bf16 rounds up to 2^128: infinite as a 32-bit value)
            want = want.astype(np.float32).astype(np.float64)
        assert np.array_equal(np.nan_to_num(got), np.nan_to_num(want))


def test_blocks_that_are_not_there_and_rows_without_a_position():
    torch = G.torch_mod()
    heads, dim = 2, 64
    rng = np.random.default_rng(2)
    cache = A.KVCache(4, heads, dim, device=G.dev())
    cache.data.zero_()
    before = cache.data.clone()
    k, kn = _tensor(rng.normal(size=(200, heads, dim)), B.BF16)
    A.kv_append(cache, k, k, _int32([[4, -1, 2 ** 30, -2 ** 31]]), _int32([200]))
    assert torch.equal(cache.data, before)
    # 200 rows for a sequence of 130 tokens: the first 70 have no position; block 1 is not there
    table, lengths = _int32([[3, 9, 1]]), _int32([130])
    A.kv_append(cache, k, k, table, lengths)
    got = G.to_f64(A.kv_read(cache, table, lengths, max_new=200)[0])
    oracle = O.Cache(heads, dim)
    oracle.append(kn[70:], kn[70:])
    want = np.concatenate([np.zeros((70, heads, dim)), oracle.values("k")])
    want[70 + 64:70 + 128] = 0
    assert np.array_equal(got, want)


# ---- attention --------------------------------------------------------------------

CASES = [
    # (lengths, new tokens of each, key heads, group, head size, type, causal)
    ([1], [1], 1, 1, 64, B.BF16, True),
    ([1, 0, 63, 64, 65, 129], [1] * 6, 2, 4, 128, B.BF16, True),
    ([700, 1, 64], [1] * 3, 1, 16, 128, B.F16, True),
    ([700, 1, 64], [1] * 3, 2, 17, 64, B.BF16, True),
    ([3000], [1], 1, 5, 80, B.F16, True),
    ([1000, 300], [1, 1], 1, 8, 256, B.BF16, True),
    ([130], [1], 2, 3, 40, B.BF16, True),
    ([130], [1], 1, 2, 1, B.F16, True),
    ([200, 65], [3, 2], 2, 4, 192, B.BF16, True),
    ([150], [150], 2, 2, 128, B.BF16, True),
    ([150], [150], 2, 2, 128, B.BF16, False),
    ([97, 0, 64, 31], [97, 0, 20, 31], 1, 3, 96, B.F16, True),
    ([97, 0, 64, 31], [40, 2, 64, 50], 1, 3, 33, B.BF16, True),       # (more new tokens than the length)
    ([333], [77], 1, 1, 64, B.F16, False),
    ([70], [70], 1, 9, 256, B.F16, True),
]


@pytest.mark.parametrize("lengths,news,heads,group,dim,dtype,causal", CASES)
def test_attention_over_the_cache(lengths, news, heads, group, dim, dtype, causal):
    torch = G.torch_mod()
    setup = Setup(lengths, heads, dim, dtype)
    q, qn = setup.queries(sum(news), group)
    starts = None if len(set(news)) == 1 else _int32(np.concatenate([[0], np.cumsum(news)]))
    lse = torch.empty(q.shape[:2], dtype=torch.float32, device=G.dev())
    out = A.cache_attention(setup.cache, q, setup.table, setup.lengths_dev, starts=starts, max_new=max(news), causal=causal, lse=lse)
    _compare(setup, out, lse, qn, news, causal)


@pytest.mark.parametrize("news", [[1], [90]])
def test_scales_that_differ_between_blocks(news):
    """Values of one block 2^40 times the next one's: a weight's part does not depend on the other blocks' scales."""
    setup = Setup([400], 2, 64, B.BF16, scale_of=lambda n: 2.0 ** (20.0 * np.where(np.arange(n) // 64 % 2, 1, -1)))
    q, qn = setup.queries(news[0], 2)
    out = A.cache_attention(setup.cache, q, setup.table, setup.lengths_dev)
    _compare(setup, out, None, qn, news)


@pytest.mark.parametrize("scale", [0.0, -0.3, 4.0])
def test_scales_of_the_products(scale):
    setup = Setup([300], 1, 64, B.F16)
    q, qn = setup.queries(2, 4)
    out = A.cache_attention(setup.cache, q, setup.table, setup.lengths_dev, scale=scale)
    _compare(setup, out, None, qn, [2], scale=scale)


@pytest.mark.parametrize("news", [1, 80])
def test_queries_in_slices_and_rows_of_others_left_alone(news):
    torch = G.torch_mod()
    setup = Setup([150], 2, 72, B.BF16)
    wide, values = _tensor(np.random.default_rng(0).normal(size=(news, 9, 73)), B.BF16)
    q, qn = wide[:, 1:9:2, 1:], values[:, 1:9:2, 1:]
    out = torch.full((news + 3, 4, 72), 7.0, dtype=torch.bfloat16, device=G.dev())
    q = torch.cat([torch.zeros_like(q[:1]), q, torch.zeros_like(q[:1]), torch.zeros_like(q[:1])])
    A.cache_attention(setup.cache, q, setup.table, setup.lengths_dev, starts=_int32([1, news + 1]), max_new=news, out=out)
    assert (out[0] == 7).all() and (out[news + 1:] == 7).all()
    _compare(setup, out[1:news + 1], None, qn, [news])
    straight = A.cache_attention(setup.cache, wide[:, 1:9:2, 1:], setup.table, setup.lengths_dev)
    assert torch.equal(straight, out[1:news + 1])


def _poisoned(which, at):
    def tokens(b, k, v):
        for t, c in at:
            if "k" in which:
                k[t, :, c] = np.nan
            if "v" in which:
                v[t, :, c] = np.inf
        return k, v
    return tokens


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("which", ["k", "v", "kv"])
@pytest.mark.parametrize("news", [5, 140])
def test_what_is_not_attended_to_has_no_influence(which, news, dim):
    """NaN in keys and values of later tokens: rows before them are clean, the channel of rows that see them is NaN."""
    setup = Setup([140], 2, dim, B.BF16, tokens=_poisoned(which, [(137, 3), (70, 5)] if news > 5 else [(137, 3)]))
    q, qn = setup.queries(news, 2)
    out = A.cache_attention(setup.cache, q, setup.table, setup.lengths_dev)
    assert np.isfinite(G.to_f64(out)[0]).all()
    _compare(setup, out, None, qn, [news])


def test_what_lies_behind_a_shortened_sequence_has_no_influence():
    """Tokens taken back (a shorter length) leave their NaN in the block."""
    setup = Setup([100], 1, 64, B.BF16, tokens=_poisoned("kv", [(98, 3), (99, 0)]))
    full = setup.oracle[0]
    for n in (97, 65, 64, 1):
        setup.oracle[0] = O.Cache(1, 64)
        setup.oracle[0].codes = {k: c[:n] for k, c in full.codes.items()}
        setup.oracle[0].scales = {k: c[:-(-n // 64)] for k, c in full.scales.items()}
        setup.lengths = [n]
        q, qn = setup.queries(1, 2)
        out = A.cache_attention(setup.cache, q, setup.table, _int32([n]))
        assert np.isfinite(G.to_f64(out)).all()
        _compare(setup, out, None, qn, [1])


def test_contents_beyond_the_bounds_are_cut_off():
    """Lengths, starts and table entries out of range: cut to the call's bounds, nothing is read or written outside."""
    torch = G.torch_mod()
    setup = Setup([130], 1, 64, B.BF16)
    q, qn = setup.queries(4, 2)
    out = torch.full((4, 2, 64), 7.0, dtype=torch.bfloat16, device=G.dev())
    A.cache_attention(setup.cache, q, setup.table, _int32([-5]), out=out)
    assert (out == 0).all()
    A.cache_attention(setup.cache, q, setup.table, _int32([2 ** 31 - 1]), max_len=130, out=out)
    _compare(setup, out, None, qn, [4])
    out.fill_(7)
    A.cache_attention(setup.cache, q, setup.table, _int32([130]), starts=_int32([-9, 2 ** 31 - 1]), max_new=4, out=out)
    _compare(setup, out, None, qn, [4])
    out.fill_(7)
    A.cache_attention(setup.cache, q, setup.table, _int32([130]), starts=_int32([3, 1]), max_new=4, out=out)
    assert (out == 7).all()
    # a block that is not there: the softmax over the others
    table = setup.table.clone()
    table[0, 1] = setup.pool
    A.cache_attention(setup.cache, q, table, setup.lengths_dev, out=out)
    holes = np.broadcast_to(np.array([[0, 2]]), (4, 1, 2))
    _compare(setup, out, None, qn, [4], lists=holes)


def test_blocks_past_32_bits_of_bytes():
    """A pool of more than 4 GB, and of more than 2^31 bytes of codes before the sequence's blocks."""
    torch = G.torch_mod()
    heads, dim = 8, 128
    blocks = (5 << 30) // (heads * 128 * dim)
    cache = A.KVCache(blocks, heads, dim, device=G.dev())
    setup = Setup([200], heads, dim, B.BF16)
    table = _int32([[blocks - 1, 1, blocks // 2 + 7, blocks - 2]])
    A.kv_append(cache, setup.k, setup.v, table, setup.lengths_dev)
    q, qn = setup.queries(1, 2)
    _compare(setup, A.cache_attention(cache, q, table, setup.lengths_dev), None, qn, [1])
    out, selected = A.focused_attention(cache, q, table, setup.lengths_dev, first=0, last=1, top=1)
    _compare(setup, out, None, qn, [1], lists=selected.cpu().numpy())


# ---- selection -----------------------------------------------------------------------

FOCUSED = [
    # (lengths, new tokens, key heads, group, head size, type, first, last, top)
    ([1], [1], 1, 1, 64, B.BF16, 1, 1, 2),
    ([640, 0, 64, 65, 1500], [1] * 5, 2, 4, 128, B.BF16, 1, 2, 3),
    ([2000, 900], [1, 1], 1, 16, 64, B.F16, 0, 1, 5),
    ([2000], [1], 1, 20, 64, B.BF16, 2, 1, 4),
    ([700, 449], [30, 449], 2, 3, 80, B.BF16, 1, 1, 2),
    ([600], [600], 1, 1, 128, B.F16, 0, 1, 0),
    ([500], [37], 2, 5, 256, B.BF16, 0, 2, 3),
    ([500], [500], 1, 2, 33, B.F16, 3, 1, 1),
    ([120], [200], 1, 2, 64, B.BF16, 1, 1, 1),              # (more new tokens than the length)
    ([5000], [3], 1, 4, 64, B.BF16, 1, 2, 60),
]


def _lists(setup, qn, news, first, last, top):
    out, row = [], 0
    for b, n in enumerate(news):
        for i in range(n):
            out.append(O.select(setup.oracle[b], qn[row], setup.lengths[b] - n + i, first, last, top))
            row += 1
    return np.stack(out)


@pytest.mark.parametrize("lengths,news,heads,group,dim,dtype,first,last,top", FOCUSED)
def test_selected_blocks_and_attention_over_them(lengths, news, heads, group, dim, dtype, first, last, top):
    torch = G.torch_mod()
    setup = Setup(lengths, heads, dim, dtype)
    q, qn = setup.queries(sum(news), group)
    lse = torch.empty(q.shape[:2], dtype=torch.float32, device=G.dev())
    out, selected = A.focused_attention(setup.cache, q, setup.table, setup.lengths_dev, first, last, top, max_new=max(news),
                                        starts=None if len(set(news)) == 1 else _int32(np.concatenate([[0], np.cumsum(news)])), lse=lse)
    want = _lists(setup, qn, news, first, last, top)
    assert np.array_equal(selected.cpu().numpy(), want)
    _compare(setup, out, lse, qn, news, lists=want)


def test_ties_go_to_the_lowest_blocks():
    """All blocks alike, and queries of zero: every score is the same."""
    def same(b, k, v):
        return np.broadcast_to(k[:64], (k.shape[0] // 64, 64) + k.shape[1:]).reshape(k.shape), v
    setup = Setup([64 * 90], 2, 64, B.BF16, tokens=same)
    for magnitude in (1.0, 0.0):
        q, qn = setup.queries(1, 2, magnitude)
        _, selected = A.focused_attention(setup.cache, q, setup.table, setup.lengths_dev, first=2, last=2, top=70)
        assert np.array_equal(selected.cpu().numpy()[0, 0], list(range(72)) + [88, 89])
        assert np.array_equal(selected.cpu().numpy(), _lists(setup, qn, [1], 2, 2, 70))


@pytest.mark.parametrize("width", [100, 2100, 9000])
def test_selection_among_many_blocks(width):
    """Long tables: as many scores as there is room for decide how many tokens a workgroup takes.  All blocks of the table are eight of the pool."""
    heads, dim, news = 1, 64, 20
    setup = Setup([512], heads, dim, B.BF16)
    table = _int32(setup.table_np[:, np.random.default_rng(1).integers(0, 8, size=width)])
    whole = O.Cache(heads, dim)
    at = table.cpu().numpy()[0]
    place = {int(p): i for i, p in enumerate(setup.table_np[0])}
    rows = np.concatenate([np.arange(64) + 64 * place[int(p)] for p in at])
    whole.codes = {n: c[rows] for n, c in setup.oracle[0].codes.items()}
    whole.scales = {n: c[[place[int(p)] for p in at]] for n, c in setup.oracle[0].scales.items()}
    setup.oracle, setup.lengths = [whole], [64 * width]
    q, qn = setup.queries(news, 2)
    _, selected = A.focused_attention(setup.cache, q, table, _int32([64 * width]), first=1, last=1, top=9)
    for i in (0, 7, 19):
        want = O.select(whole, qn[i], 64 * width - news + i, 1, 1, 9)
        assert np.array_equal(selected.cpu().numpy()[i], want)


def test_queries_that_are_not_finite_select_by_the_others():
    setup = Setup([1000], 1, 64, B.BF16)
    q, qn = setup.queries(2, 2)
    q[0, 0, 3], q[0, 1, 7] = float("nan"), float("inf")
    qn[0, 0, 3], qn[0, 1, 7] = np.nan, np.inf
    out, selected = A.focused_attention(setup.cache, q, setup.table, setup.lengths_dev, first=0, last=1, top=3)
    assert np.array_equal(selected.cpu().numpy(), _lists(setup, qn, [2], 0, 1, 3))
    got = G.to_f64(out)
    assert np.isnan(got[0]).all()
    _compare(setup, out[1:], None, qn[1:], [1], lists=selected.cpu().numpy()[1:])


def test_all_blocks_selected_is_attention_over_all():
    setup = Setup([500, 260], 2, 128, B.BF16)
    q, _ = setup.queries(2, 4)
    torch = G.torch_mod()
    dense = A.cache_attention(setup.cache, q, setup.table, setup.lengths_dev)
    out, selected = A.focused_attention(setup.cache, q, setup.table, setup.lengths_dev, first=1, last=1, top=6)
    assert torch.equal(out, dense)


# ---- streams, graphs, repeated calls ----------------------------------------------------

def test_calls_on_another_stream_and_in_a_graph():
    """A step (append, attention, selection) recorded once and replayed with eager work between: the eager result every time."""
    torch = G.torch_mod()
    setup = Setup([900, 70], 2, 128, B.BF16)
    q, _ = setup.queries(2, 4)
    k, v = setup.k[-2:].clone(), setup.v[-2:].clone()
    calls = [A.PreparedAppend(setup.cache, k, v, setup.table, setup.lengths_dev),
             A.PreparedAttention(setup.cache, q, setup.table, setup.lengths_dev),
             A.PreparedFocusedAttention(setup.cache, q, setup.table, setup.lengths_dev, first=1, last=1, top=3)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    eager = [c(side) for c in calls][1:]
    side.synchronize()
    eager = [eager[0].clone(), eager[1][0].clone(), eager[1][1].clone()]
    one = A.cache_attention(setup.cache, q, setup.table, setup.lengths_dev, stream=side)
    side.synchronize()
    assert torch.equal(one, eager[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        for c in calls:
            c()
    outs = [calls[1]._result, *calls[2]._result]
    for _ in range(4):
        for t in outs:
            t.fill_(5)
        A.cache_attention(setup.cache, q, setup.table, setup.lengths_dev)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for got, want in zip(outs, eager):
            assert torch.equal(got, want)


def test_results_do_not_change_from_call_to_call():
    torch = G.torch_mod()
    setup = Setup([4000, 1300], 4, 128, B.F16)
    for news in (1, 33):
        q, _ = setup.queries(2 * news, 4)
        first = A.cache_attention(setup.cache, q, setup.table, setup.lengths_dev)
        focused = A.focused_attention(setup.cache, q, setup.table, setup.lengths_dev, first=1, last=1, top=5)
        for _ in range(3):
            assert torch.equal(A.cache_attention(setup.cache, q, setup.table, setup.lengths_dev), first)
            again = A.focused_attention(setup.cache, q, setup.table, setup.lengths_dev, first=1, last=1, top=5)
            assert torch.equal(again[0], focused[0]) and torch.equal(again[1], focused[1])


def test_no_tokens():
    torch = G.torch_mod()
    setup = Setup([10], 1, 64, B.BF16)
    q = torch.empty((0, 2, 64), dtype=torch.bfloat16, device=G.dev())
    assert A.cache_attention(setup.cache, q, setup.table, setup.lengths_dev, starts=_int32([0, 0])).shape == (0, 2, 64)
    out, selected = A.focused_attention(setup.cache, q, setup.table, setup.lengths_dev, 1, 1, 1, starts=_int32([0, 0]))
    assert out.shape == (0, 2, 64) and selected.shape == (0, 1, 3)
