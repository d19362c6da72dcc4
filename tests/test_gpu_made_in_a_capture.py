"""Prepared calls that are made while a graph is captured: their eager calls, before the graph's first replay too, find their workspace as they need it."""
import pytest
import torch

from paper_2207_10741_amd import attention as A, layers as L, pages as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _normal(shape, seed, scale=1.0):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).mul_(scale).to(torch.bfloat16).to(DEV)


def _dirty():
    """Memory that the graph's allocations are made of holds no zeros."""
    torch.full((1 << 26,), 0x5a, dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()


@pytest.mark.parametrize("rows,k,n", [(3, 1001, 37), (130, 4104, 60), (50, 4104, 70)])
def test_linear(rows, k, n):
    x, w = _normal((rows, k), 1), _normal((n, k), 2, k ** -0.5)
    want = L.linear(x, w).clone()
    _dirty()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call = L.PreparedLinear(x, w)
        got = call()
    assert call.cut.pieces > 1
    for _ in range(3):
        got.zero_()
        assert torch.equal(call(), want)
        got.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want)


def test_pages():
    cache, lengths, parents = A.KVCache(300, 2, 64, device=DEV), _int32([700, 0, 0, 64]), _int32([0, 0, 0, 3])
    users, table = P.kv_users(cache), torch.full((4, 20), -1, dtype=torch.int32, device=DEV)
    start = [t.clone() for t in (users, table, lengths)]

    def again():
        for t, s in zip((users, table, lengths), start):
            t.copy_(s)

    P.kv_resize(cache, users, table, lengths)
    P.kv_fork(cache, users, table, lengths, parents)
    want = [t.clone() for t in (users, table, lengths)]
    _dirty()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        resize, fork = P.PreparedResize(cache, users, table, lengths), P.PreparedFork(cache, users, table, lengths, parents)
        resize()
        fork()
    for _ in range(3):
        again()
        assert resize().tolist() == [0] and fork().tolist() == [0]
        assert all(torch.equal(a, b) for a, b in zip(want, (users, table, lengths)))
        again()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (users, table, lengths)))


def test_attention():
    tokens, heads, dim = 3000, 2, 64
    cache, table, lengths = A.KVCache(50, heads, dim, device=DEV), torch.arange(48, dtype=torch.int32, device=DEV)[None], _int32([tokens])
    A.kv_append(cache, _normal((tokens, heads, dim), 1), _normal((tokens, heads, dim), 2), table, lengths)
    q = _normal((1, heads, dim), 3)
    want, (want_of, blocks) = A.cache_attention(cache, q, table, lengths).clone(), [t.clone() for t in A.focused_attention(cache, q, table, lengths, 1, 1, 6)]
    _dirty()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call, of = A.PreparedAttention(cache, q, table, lengths), A.PreparedFocusedAttention(cache, q, table, lengths, 1, 1, 6)
        got = call()
        got_of = of()
    for _ in range(3):
        assert torch.equal(call(), want)
        out, selected = of()
        assert torch.equal(out, want_of) and torch.equal(selected, blocks)
        got.zero_()
        got_of[0].zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(got_of[0], want_of) and torch.equal(got_of[1], blocks)
