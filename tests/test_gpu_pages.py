"""The pages of the cache against the oracle, step by step: tables, users and lengths for equality, contents by what is read back."""
import random

import pytest
import torch

from paper_2207_10741_amd import attention as A, pages as P
from tests.pages_oracle import Pages

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _dev(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _labels(cache, blocks, width=64):
    """Writes a label into every block: its number in all tokens of keys, its negative in the values (whole numbers to 240 are exact in the cache)."""
    token = torch.arange(blocks, device=DEV).repeat_interleave(64)
    k = (token % 15 + 1).to(torch.bfloat16)[:, None, None].expand(-1, cache.kv_heads, cache.head_dim).contiguous()
    v = (-(token // 15 % 15) - 1).to(torch.bfloat16)[:, None, None].expand(-1, cache.kv_heads, cache.head_dim).contiguous()
    A.kv_append(cache, k, v, torch.arange(blocks, dtype=torch.int32, device=DEV)[None], _dev([blocks * 64]))


def _read_labels(cache, blocks):
    """Of the given blocks; every token and channel of a block says the same."""
    if not blocks:
        return []
    k, v = A.kv_read(cache, _dev([blocks]), _dev([len(blocks) * 64]), max_new=len(blocks) * 64)
    both = torch.stack([k, v]).view(2, len(blocks), -1)
    assert bool((both == both[:, :, :1]).all())
    return [int(a - 1) + 15 * int(-b - 1) for a, b in zip(both[0, :, 0].tolist(), both[1, :, 0].tolist())]


class _Both:
    """The same pages on the device and in the oracle."""

    def __init__(self, blocks, batch, width, kv_heads=2, dim=64):
        self.cache = A.KVCache(blocks, kv_heads, dim, device=DEV)
        self.cache.data.zero_()
        assert blocks <= 225
        _labels(self.cache, blocks)
        self.users, self.table = P.kv_users(self.cache), torch.full((batch, width), -1, dtype=torch.int32, device=DEV)
        self.lengths = torch.zeros((batch,), dtype=torch.int32, device=DEV)
        self.oracle = Pages([0] * blocks, [[-1] * width] * batch, [0] * batch, range(blocks))
        self.blocks = blocks

    def check(self, missing, want):
        assert missing.tolist() == [want]
        assert self.table.tolist() == self.oracle.table
        assert self.users.tolist() == self.oracle.users
        assert self.lengths.tolist() == self.oracle.lengths
        assert sum(self.oracle.users) == sum(e >= 0 for r in self.oracle.table for e in r)
        used = [b for b in range(self.blocks) if self.oracle.users[b]]
        assert _read_labels(self.cache, used) == [self.oracle.contents[b] for b in used]

    def resize(self, lengths):
        self.lengths.copy_(_dev(lengths))
        self.oracle.lengths = list(lengths)
        self.check(P.kv_resize(self.cache, self.users, self.table, self.lengths), self.oracle.resize(lengths))

    def fork(self, parents):
        self.check(P.kv_fork(self.cache, self.users, self.table, self.lengths, _dev(parents)), self.oracle.fork(parents))


def test_blocks_are_given_lowest_first_and_go_back():
    s = _Both(20, 3, 6)
    s.resize([1, 64, 65])
    s.resize([128, 0, 200])
    s.resize([0, 300, 64])
    s.resize([6 * 64, 6 * 64, 6 * 64])
    s.resize([10 ** 6, -5, 2 ** 31 - 1])        # (the table's 384 tokens, nothing, the table's)
    s.resize([0, 0, 0])
    assert not bool(s.users.any())


def test_too_few_blocks():
    s = _Both(7, 4, 5)
    s.resize([100, 300, 130, 64])
    s.resize([100, 300, 130, 64])               # still too few
    s.resize([100, 64, 130, 64])                # now the others have theirs
    s.fork([0, 0, 2, 2])
    s.fork([0, 1, 2, 0])


def test_forks_share_full_blocks_and_copy_unfinished_ones():
    s = _Both(40, 6, 5)
    s.resize([200, 0, 128, 0, 0, 1])
    s.fork([0, 0, 2, 2, 0, 5])
    s.fork([1, 0, 3, 3, 5, -1])                 # slots change places, copies of copies, one is freed
    s.fork([0, 1, 2, 3, 4, 5])                  # everything stays
    s.fork([4, 4, 4, 4, 4, 4])                  # all of one that stays
    s.fork([1, 2, 3, 4, 5, 0])                  # in a ring
    s.fork([3, 3, 3, 9, -7, 2 ** 31 - 1])       # the parent itself goes
    s.fork([-1] * 6)
    assert not bool(s.users.any())


def test_cut_within_a_shared_block():
    s = _Both(40, 4, 5)
    s.resize([256, 0, 0, 0])
    s.fork([0, 0, 0, -1])
    s.resize([256, 100, 256, 0])                # one of three: a copy
    s.resize([100, 100, 200, 0])                # two that hold the same blocks: a copy each where it is shared
    s.resize([256, 101, 201, 1])
    s.resize([64, 64, 64, 64])


def test_cut_within_a_shared_block_without_a_free_one():
    s = _Both(4, 2, 4)
    s.resize([256, 0])
    s.fork([0, 0])
    s.resize([256, 100])
    s.resize([256, 64])


def test_entries_out_of_range_are_no_blocks():
    s = _Both(10, 2, 4)
    s.table.copy_(_dev([[-7, 10, 2 ** 31 - 1, -2 ** 31], [99, 3, 3000, -1]]))
    s.oracle.table = s.table.tolist()
    s.users[3] = 1
    s.oracle.users[3] = 1
    s.resize([130, 128])
    s.table[1, 0] = 10
    s.oracle.table[1][0] = 10
    s.users[s.oracle.table[0][0]] = 1
    s.oracle.users = s.users.tolist()
    missing = P.kv_fork(s.cache, s.users, s.table, s.lengths, _dev([1, 1]))
    want = s.oracle.fork([1, 1])
    assert missing.tolist() == [want] and s.table.tolist() == s.oracle.table and s.users.tolist() == s.oracle.users


@pytest.mark.parametrize("seed", range(12))
def test_random_steps(seed):
    rng = random.Random(seed)
    batch, width = rng.choice([(1, 1), (5, 3), (40, 7), (130, 2), (3, 70)]), None
    batch, width = batch
    s = _Both(rng.choice([1, 30, 100, 225]), batch, width, rng.choice([1, 2, 3]), rng.choice([16, 64, 80, 256]))
    for _ in range(6):
        s.resize([rng.choice([0, 0, 1, 64, rng.randint(0, width * 64), rng.randint(0, width * 64)]) for _ in range(batch)])
        s.fork([rng.choice([b, b, rng.randrange(batch), rng.randrange(batch), -1]) for b in range(batch)])


def _table_check(users, table, lengths, batch, width, blocks):
    cache = A.KVCache(blocks, 1, 16, device=DEV)
    oracle = Pages(users.tolist(), table.tolist(), lengths.tolist(), range(blocks))
    return cache, oracle


@pytest.mark.parametrize("batch,width,blocks", [(256, 129, 60000), (3000, 9, 20000), (2, 5000, 9000), (600, 3, 1200)])
def test_many_sequences_and_large_pools(batch, width, blocks):
    """Pools of several rounds of looking for free blocks, more sequences than workgroups."""
    rng = random.Random(batch)
    users, table = torch.zeros((blocks,), dtype=torch.int32, device=DEV), torch.full((batch, width), -1, dtype=torch.int32, device=DEV)
    busy = torch.rand((blocks,), generator=torch.Generator().manual_seed(1)) < 0.5
    users.copy_(busy.to(torch.int32))           # (of somebody else's table)
    lengths = torch.zeros((batch,), dtype=torch.int32, device=DEV)
    cache, oracle = _table_check(users, table, lengths, batch, width, blocks)
    for step in range(3):
        want = [rng.choice([0, rng.randint(0, width * 64)]) for _ in range(batch)]
        lengths.copy_(_dev(want))
        oracle.lengths = want
        missing = P.kv_resize(cache, users, table, lengths)
        assert missing.tolist() == [oracle.resize(want)]
        assert table.tolist() == oracle.table and users.tolist() == oracle.users
        parents = [rng.choice([b, rng.randrange(batch), -1]) for b in range(batch)]
        missing = P.kv_fork(cache, users, table, lengths, _dev(parents))
        assert missing.tolist() == [oracle.fork(parents)]
        assert table.tolist() == oracle.table and users.tolist() == oracle.users and lengths.tolist() == oracle.lengths


@pytest.mark.parametrize("blocks_to", [1, 30, 60, 200])
def test_compact(blocks_to):
    s = _Both(150, 6, 20)
    s.resize([1000, 500, 1200, 64, 0, 130])
    s.fork([0, 0, 2, 3, 2, 5])
    s.resize([0, 500, 700, 64, 1200, 0])
    to = A.KVCache(blocks_to, 2, 64, device=DEV)
    users_to = torch.full((blocks_to,), 77, dtype=torch.int32, device=DEV)
    before = [t.clone() for t in (s.cache.data, s.users, s.table)]
    table_to, missing = P.kv_compact(s.cache, s.users, s.table, to, users_to)
    table, users, contents, lost = s.oracle.compact(blocks_to)
    assert table_to.tolist() == table and users_to.tolist() == users and missing.tolist() == [lost]
    assert _read_labels(to, list(range(len(contents)))) == contents
    assert all(torch.equal(a, b) for a, b in zip(before, (s.cache.data, s.users, s.table)))


@pytest.mark.parametrize("blocks", [4095, 4097, 20000])
def test_compact_large_pools(blocks):
    gen = torch.Generator().manual_seed(blocks)
    users = (torch.rand((blocks,), generator=gen) < 0.3).to(torch.int32) * torch.randint(1, 4, (blocks,), generator=gen, dtype=torch.int32)
    table = torch.randint(-1, blocks, (7, 300), generator=gen, dtype=torch.int32)
    cache, to = A.KVCache(blocks, 1, 16, device=DEV), A.KVCache(blocks // 3, 1, 16, device=DEV)
    users_to = torch.full((blocks // 3,), 77, dtype=torch.int32, device=DEV)
    table_to, missing = P.kv_compact(cache, users.to(DEV), table.to(DEV), to, users_to)
    want = Pages(users.tolist(), table.tolist(), [0] * 7, range(blocks)).compact(blocks // 3)
    assert table_to.tolist() == want[0] and users_to.tolist() == want[1] and missing.tolist() == [want[3]]


def test_copy_within_a_cache_and_to_another():
    cache, to = A.KVCache(60, 3, 96, device=DEV), A.KVCache(9, 3, 96, device=DEV)
    _labels(cache, 60)
    _labels(to, 9)
    P.kv_copy(cache, _dev([50, 3, 60, 7, -1, 2 ** 31 - 1]), to, _dev([0, 8, 1, 9, 2, 3]))      # (pairs out of range: nothing)
    assert _read_labels(to, list(range(9))) == [50, 1, 2, 3, 4, 5, 6, 7, 3]
    P.kv_copy(cache, _dev([1, 2]), cache, _dev([59, 58]))
    assert _read_labels(cache, [1, 2, 57, 58, 59]) == [1, 2, 57, 2, 1]
    P.kv_copy(cache, _dev([]), to, _dev([]))


@pytest.mark.parametrize("dim", [16, 64, 96, 128, 200])
def test_a_copied_block_is_the_block(dim):
    """Codes, scales and what the selection reads: attention over the copy gives the same bits."""
    heads, tokens = 2, 64 * 9 + 17
    gen = torch.Generator().manual_seed(dim)
    k, v, q = (torch.randn((n, heads, dim), generator=gen).to(torch.bfloat16).to(DEV) for n in (tokens, tokens, 3))
    cache, users = A.KVCache(40, heads, dim, device=DEV), None
    users, table, lengths = P.kv_users(cache), torch.full((2, 12), -1, dtype=torch.int32, device=DEV), _dev([tokens, 0])
    P.kv_resize(cache, users, table, lengths)
    A.kv_append(cache, k, v, table, lengths, starts=_dev([0, tokens, tokens]), max_new=tokens)
    want = A.focused_attention(cache, q, table[:1].contiguous(), lengths[:1].clone(), 1, 1, 3)
    to, users_to = A.KVCache(11, heads, dim, device=DEV), None
    users_to = P.kv_users(to)
    table_to, _ = P.kv_compact(cache, users, table, to, users_to)
    got = A.focused_attention(to, q, table_to[:1].contiguous(), lengths[:1].clone(), 1, 1, 3)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    P.kv_fork(cache, users, table, lengths, _dev([0, 0]))
    got = A.focused_attention(cache, q, table[1:].contiguous(), lengths[1:].clone(), 1, 1, 3)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_captured_and_on_another_stream():
    cache, lengths = A.KVCache(500, 2, 64, device=DEV), _dev([700, 0, 0, 64])
    users, table = P.kv_users(cache), torch.full((4, 20), -1, dtype=torch.int32, device=DEV)
    parents = _dev([0, 0, 0, 3])
    resize, fork = P.PreparedResize(cache, users, table, lengths), P.PreparedFork(cache, users, table, lengths, parents)
    other = P.PreparedResize(cache, users, table, lengths)
    resize(), fork()
    state = [t.clone() for t in (users, table, lengths)]
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        resize()
        fork()
    for _ in range(4):
        lengths.zero_()
        assert other().tolist() == [0] and not bool(users.any())
        lengths.copy_(_dev([700, 0, 0, 64]))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(state, (users, table, lengths)))
    side.wait_stream(torch.cuda.current_stream())
    missing = P.kv_fork(cache, users, table, lengths, _dev([-1] * 4), stream=side)
    side.synchronize()
    assert missing.tolist() == [0] and not bool(users.any())
