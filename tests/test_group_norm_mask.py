"""Masks of group norm whose bytes are not the rows' in order are refused."""
import pytest

from paper_2207_10741_amd import layers as L


@pytest.mark.parametrize("mask", [(2, 9, 13), (234,), (2, 117), (18, 13), (2, 1, 9, 13), (2, 9, 13, 1), (1, 234), (2, 3, 3, 13)])
def test_shapes_that_go_over_the_rows(mask):
    assert L._in_order(mask, (2, 9, 13)) and L._in_order((2, 9, 13), mask)


@pytest.mark.parametrize("mask", [(2, 13, 9), (9, 13, 2), (13, 18), (9, 26), (117, 2), (9, 2, 13)])
def test_shapes_that_do_not(mask):
    assert not L._in_order(mask, (2, 9, 13))


@pytest.mark.gpu
def test_group_norm_refuses_them():
    import torch
    x = torch.zeros((2, 9, 13, 32), dtype=torch.bfloat16, device="cuda:0")
    mask = torch.ones((2, 13, 9), dtype=torch.uint8, device="cuda:0")
    with pytest.raises(ValueError, match="in their order"):
        L.group_norm(x, 4, mask=mask)
    assert torch.equal(L.group_norm(x, 4, mask=mask.view(2, 117)), L.group_norm(x, 4))
    assert L.group_norm(x[:0], 4, mask=mask[:0]).shape == (0, 9, 13, 32)
