"""Cuts within blocks that only cut sequences hold, in pools with too few blocks for a copy each: what is cached there stays with the lowest of them."""
import random

import pytest
import torch

from paper_2207_10741_amd import attention as A, pages as P
from tests.pages_oracle import Pages
from tests.test_gpu_pages import DEV, _Both, _dev, _read_labels

pytestmark = pytest.mark.gpu


def _state(s):
    return s.table.tolist(), s.users.tolist()


def test_all_holders_are_cut_without_a_free_block():
    s = _Both(4, 2, 4)
    s.resize([256, 0])
    s.fork([0, 0])
    s.resize([200, 200])
    assert _state(s) == ([[0, 1, 2, 3], [0, 1, 2, -1]], [2, 2, 2, 1])
    assert _read_labels(s.cache, [0, 1, 2, 3]) == [0, 1, 2, 3]


def test_the_lowest_of_those_that_are_cut_keeps_it():
    s = _Both(4, 5, 4)
    s.resize([0, 0, 0, 256, 0])
    s.fork([-1, 3, 3, 3, 3])
    s.resize([0, 256, 150, 150, 150])           # the first holds the block whole: nothing is kept by those that are cut
    assert _state(s) == ([[-1] * 4, [0, 1, 2, 3], [0, 1, -1, -1], [0, 1, -1, -1], [0, 1, -1, -1]], [4, 4, 1, 1])
    s.resize([0, 128, 100, 100, 100])           # (now blocks 2 and 3 are free)
    assert _state(s) == ([[-1] * 4, [0, 1, -1, -1], [0, 2, -1, -1], [0, 3, -1, -1], [0, -1, -1, -1]], [4, 1, 1, 1])
    s = _Both(2, 4, 2)
    s.resize([0, 128, 0, 0])
    s.fork([-1, 1, 1, 1])
    s.resize([0, 100, 90, 65])
    assert _state(s) == ([[-1, -1], [0, 1], [0, -1], [0, -1]], [3, 1])


def test_a_pool_that_has_exactly_enough():
    s = _Both(5, 2, 4)
    s.resize([256, 0])
    s.fork([0, 0])
    s.resize([200, 200])
    assert _state(s) == ([[0, 1, 2, 3], [0, 1, 2, 4]], [2, 2, 2, 1, 1])
    assert _read_labels(s.cache, [3, 4]) == [3, 3]
    s = _Both(6, 3, 4)                          # one free block for a sequence that begins
    s.resize([256, 0, 0])
    s.fork([0, 0, -1])
    s.resize([200, 200, 1])
    assert _state(s) == ([[0, 1, 2, 3], [0, 1, 2, 4], [5, -1, -1, -1]], [2, 2, 2, 1, 1, 1])


def test_blocks_that_are_no_longer_wanted_stay_free():
    """Two blocks, of two sequences each: four copies are wanted, three blocks are free, two are given."""
    s = _Both(5, 4, 1)
    s.resize([64, 64, 0, 0])
    s.fork([0, 1, 0, 1])
    s.resize([10, 20, 30, 40])
    assert _state(s) == ([[0], [1], [2], [3]], [1, 1, 1, 1, 0])
    assert _read_labels(s.cache, [0, 1, 2, 3]) == [0, 1, 0, 1]
    s.resize([64, 64, 64, 64])
    assert _state(s) == ([[0], [1], [2], [3]], [1, 1, 1, 1, 0])


def test_with_enough_blocks_everyone_gets_a_copy():
    s = _Both(6, 2, 4)
    s.resize([256, 0])
    s.fork([0, 0])
    s.resize([200, 200])
    assert _state(s) == ([[0, 1, 2, 4], [0, 1, 2, 5]], [2, 2, 2, 0, 1, 1])


def test_another_tables_sequences_hold_it_too():
    s = _Both(4, 2, 4)
    s.resize([256, 0])
    s.fork([0, 0])
    s.users[3] += 1                             # (of another table)
    assert P.kv_resize(s.cache, s.users, s.table, _dev([200, 200])).tolist() == [2]
    assert _state(s) == ([[0, 1, 2, -1], [0, 1, 2, -1]], [2, 2, 2, 1])


@pytest.mark.parametrize("seed", range(24))
def test_random_cuts_in_small_pools(seed):
    rng = random.Random(seed)
    batch, width = rng.choice([(4, 2), (9, 3), (60, 4), (130, 2)])
    s = _Both(rng.choice([batch * width // 4 + 1, batch * width // 2, batch * width]) % 225 + 1, batch, width, 1, 16)
    for _ in range(4):
        s.resize([rng.choice([0, 64 * width, rng.randint(0, width * 64)]) for _ in range(batch)])
        s.fork([rng.choice([b, rng.randrange(batch), rng.randrange(max(batch // 8, 1))]) for b in range(batch)])
        s.resize([min(int(n), rng.randint(1, width * 64)) for n in s.lengths.tolist()])


@pytest.mark.parametrize("batch,width,blocks", [(3000, 3, 1100), (5000, 2, 600), (1025, 5, 900), (20000, 2, 1500), (65535, 1, 300)])
def test_many_sequences(batch, width, blocks):
    """More sequences than threads, blocks that hundreds hold."""
    rng = random.Random(batch)
    cache = A.KVCache(blocks, 1, 16, device=DEV)
    users, table, lengths = P.kv_users(cache), torch.full((batch, width), -1, dtype=torch.int32, device=DEV), torch.zeros((batch,), dtype=torch.int32, device=DEV)
    oracle = Pages([0] * blocks, [[-1] * width] * batch, [0] * batch, range(blocks))

    def check(missing, want):
        assert missing.tolist() == [want] and table.tolist() == oracle.table and users.tolist() == oracle.users and lengths.tolist() == oracle.lengths

    for _ in range(3):
        want = [64 * width if b < 64 else 0 for b in range(batch)]
        lengths.copy_(_dev(want))
        oracle.lengths = list(want)
        check(P.kv_resize(cache, users, table, lengths), oracle.resize(want))
        parents = [b if b < 64 else rng.randrange(64) for b in range(batch)]
        check(P.kv_fork(cache, users, table, lengths, _dev(parents)), oracle.fork(parents))
        want = [rng.randint(1, 64 * width) if b % 64 < 60 else rng.randint(64 * width - 63, 64 * width - 1) for b in range(batch)]
        lengths.copy_(_dev(want))
        oracle.lengths = list(want)
        check(P.kv_resize(cache, users, table, lengths), oracle.resize(want))
