"""Workspaces on another device than the call's tensors are refused.  No GPU is needed."""
import pytest

from paper_2207_10741_amd import attention as A


class _Tensor:
    is_cuda = True

    def __init__(self, device):
        self.device = device

    def is_contiguous(self):
        return True


def test_another_device_is_refused():
    torch = pytest.importorskip("torch")
    A._check_workspace(None, torch.device("cuda:0"))
    A._check_workspace(_Tensor(torch.device("cuda:1")), torch.device("cuda:1"))
    with pytest.raises(ValueError, match="same device"):
        A._check_workspace(_Tensor(torch.device("cuda:1")), torch.device("cuda:0"))
