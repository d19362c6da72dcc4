"""Calls without new tokens, and without sequences: nothing to do, whichever way the rows are counted."""
import pytest

from paper_2207_10741_amd import attention as A, binding as B
from tests import gpu_util as G
from tests.test_gpu_attention import Setup, _int32

pytestmark = pytest.mark.gpu


def _calls(cache, table, lengths, **kw):
    torch = G.torch_mod()
    k = torch.empty((0, 2, 64), dtype=torch.bfloat16, device=G.dev())
    q = torch.empty((0, 6, 64), dtype=torch.bfloat16, device=G.dev())
    before = cache.data.clone()
    assert A.kv_append(cache, k, k, table, lengths, **kw) is cache
    for got in A.kv_read(cache, table, lengths, tokens=0, **kw):
        assert got.shape == (0, 2, 64)
    assert A.cache_attention(cache, q, table, lengths, **kw).shape == (0, 6, 64)
    out, selected = A.focused_attention(cache, q, table, lengths, 1, 1, 2, **kw)
    assert out.shape == (0, 6, 64) and selected.shape == (0, 2, 4)
    torch.cuda.synchronize()
    assert torch.equal(cache.data, before)


@pytest.mark.parametrize("kw", [{}, {"max_new": 0}, {"max_new": 1}, {"max_new": 7, "max_len": 100}])
def test_no_new_tokens(kw):
    setup = Setup([100, 70], 2, 64, B.BF16)
    _calls(setup.cache, setup.table, setup.lengths_dev, **kw)
    _calls(setup.cache, setup.table, setup.lengths_dev, starts=_int32([0, 0, 0]), **kw)


@pytest.mark.parametrize("width", [0, 3])
def test_no_sequences(width):
    torch = G.torch_mod()
    setup = Setup([100], 2, 64, B.BF16)
    table = torch.empty((0, width), dtype=torch.int32, device=G.dev())
    _calls(setup.cache, table, table.new_empty((0,)))


def test_reading_needs_the_number_of_rows():
    setup = Setup([100], 2, 64, B.BF16)
    with pytest.raises(ValueError, match="max_new"):
        A.kv_read(setup.cache, setup.table, setup.lengths_dev)
    with pytest.raises(ValueError, match="tokens"):
        A.kv_read(setup.cache, setup.table, setup.lengths_dev, starts=_int32([0, 5]))
    assert A.kv_read(setup.cache, setup.table, setup.lengths_dev, max_new=5)[0].shape == (5, 2, 64)
