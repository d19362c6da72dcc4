"""Workspaces that a caller gives: as they come, with anything in them; refused where their bytes do not lie next to each other."""
import pytest
import torch

from paper_2207_10741_amd import attention as A, layers as L, pages as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _normal(shape, seed, scale=1.0):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).mul_(scale).to(torch.bfloat16).to(DEV)


def _workspaces():
    whole = torch.full((1 << 24,), 0x5a, dtype=torch.uint8, device=DEV)
    return whole, whole[::2]


def test_linear_and_group_norm():
    x, w = _normal((50, 4104), 1), _normal((70, 4104), 2, 4104 ** -0.5)
    whole, apart = _workspaces()
    want = L.linear(x, w)
    for _ in range(3):
        assert torch.equal(L.linear(x, w, workspace=whole), want)
    with pytest.raises(ValueError, match="contiguous"):
        L.linear(x, w, workspace=apart)
    y = _normal((1, 9000, 64), 3)
    want = L.group_norm(y, 8)
    assert torch.equal(L.group_norm(y, 8, workspace=whole), want)
    with pytest.raises(ValueError, match="contiguous"):
        L.group_norm(y, 8, workspace=apart)


def test_pages_and_attention():
    cache, lengths = A.KVCache(60, 2, 64, device=DEV), torch.tensor([700, 3], dtype=torch.int32, device=DEV)
    users, table = P.kv_users(cache), torch.full((2, 20), -1, dtype=torch.int32, device=DEV)
    whole, apart = _workspaces()
    with pytest.raises(ValueError, match="contiguous"):
        P.kv_resize(cache, users, table, lengths, workspace=apart)
    for _ in range(2):
        assert P.kv_resize(cache, users, table, lengths, workspace=whole).tolist() == [0]
        assert int(users.sum()) == 12
        whole.fill_(0x5a)
    k, v, q = _normal((703, 2, 64), 4), _normal((703, 2, 64), 5), _normal((2, 2, 64), 6)
    A.kv_append(cache, k, v, table, lengths, starts=torch.tensor([0, 700, 703], dtype=torch.int32, device=DEV), max_new=700)
    want = A.cache_attention(cache, q, table, lengths)
    assert torch.equal(A.cache_attention(cache, q, table, lengths, workspace=whole), want)
    with pytest.raises(ValueError, match="contiguous"):
        A.cache_attention(cache, q, table, lengths, workspace=apart)
