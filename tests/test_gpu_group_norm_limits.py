"""Group norm at its limits against its definition in 64 bits: long groups that are not whole pieces of 16 bytes, more images than 2^31 threads."""
import pytest
import torch

from paper_2207_10741_amd import layers as L
from tests import layers_oracle as O

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.mark.parametrize("images,rows,groups,per_group,dtype", [(1, 10, 8, 2561, BF16), (2, 300, 8, 2561, F16), (1, 5, 4, 5122, BF16), (1, 2, 8, 16383, BF16), (1, 70, 2, 16380, F16),
                                                                (2, 3, 4, 16383, F32), (1, 40, 4, 16382, F32)])
def test_long_groups_that_are_not_whole_pieces(images, rows, groups, per_group, dtype):
    channels = groups * per_group
    gen = torch.Generator().manual_seed(channels)
    x = torch.randn((images, rows, channels), generator=gen).mul_(1.5).add_(0.7).to(dtype).to(DEV)
    weight, bias = (torch.randn((channels,), generator=gen).to(DEV) for _ in range(2))
    mask = torch.rand((images, rows), generator=gen) < 0.7
    mask[:, 0] = True
    for m in (None, mask):
        got = L.group_norm(x, groups, weight, bias, mask=None if m is None else m.to(torch.uint8).to(DEV), activation="silu")
        for b in range(images):
            want, error = O.group_norm(x[b], groups, weight, bias, None if m is None else m[b], activation="silu")
            O.check(got[b], want, error, "image %d" % b)


def test_more_images_than_2_to_the_31_threads():
    images, channels = 2 ** 21 + 5, 8
    counts = torch.ones((images,), dtype=torch.int64)
    counts[7], counts[-1] = 0, 3
    starts = torch.cat([torch.zeros(1, dtype=torch.int64), counts.cumsum(0)])
    x = torch.randn((int(starts[-1]), channels), generator=torch.Generator().manual_seed(1)).to(BF16).to(DEV)
    got = L.group_norm(x, 2, starts=starts.to(torch.int32).to(DEV), max_rows=4096)
    want, error = O.group_norm(x[-3:], 2)
    O.check(got[-3:], want, error, "the last image")
    part = x[:-3].double().view(-1, 2, 4)
    mean = part.mean(2, keepdim=True)
    variance = (part - mean).square().mean(2, keepdim=True)
    factor = 1.0 / torch.sqrt(variance + 1e-5)
    want = (part - mean) * factor
    # (layers_oracle.group_norm's bound, an image a row)
    off = want.abs() * (2.0 ** -18 + 2.0 ** -22) + torch.sqrt(variance) * factor * 2.0 ** -20 + mean.abs() * factor * 2.0 ** -23
    off = off + 2.0 ** -8 * (want.abs() + off) + 2.0 ** -134
    assert bool(((got[:-3].double().view(-1, 2, 4) - want).abs() <= off).all())
