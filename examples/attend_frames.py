"""A camera's frames, one after another: the relevant positions of each frame attend to those of all frames so far.

A frame's features go through a focused 3x3 layer that hands on the kept positions only, as rows in list order; a 1x1 layer makes queries, keys and values of
the rows; the keys and values enter the 8-bit cache; every row attends to the blocks of earlier rows that its score selects; and a last 1x1 layer puts the result
back into a feature map.  How many positions a mask keeps is known on the device only, and nothing here asks for it: the rows are bounded by the frame's
size, and the device's count tells the calls how many there are.

    python examples/attend_frames.py
"""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

from paper_2207_10741_amd import attention as A, binding as B, synth


class FrameAttention:
    """One layer of attention over the kept positions of up to `frames` frames of height x width positions with `channels` channels."""

    def __init__(self, height, width, channels=64, heads=4, kv_heads=2, head_dim=64, frames=8, first=1, last=4, top=11, seed=0, device="cuda:0"):
        self.height, self.width, self.channels = height, width, channels
        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, head_dim
        self.first, self.last, self.top = first, last, top
        self.rows = height * width                              # of a frame, at most
        gen = torch.Generator(device=device).manual_seed(seed)

        def weights(c_out, k, c_in):
            w = torch.randn((c_out, k, k, c_in), generator=gen, device=device)
            return w.mul_((2.0 / (k * k * c_in)) ** 0.5).to(torch.bfloat16)

        self.w_in = weights(channels, 3, channels)
        self.w_qkv = weights((heads + 2 * kv_heads) * head_dim, 1, channels)
        self.w_out = weights(channels, 1, heads * head_dim)
        blocks = -(-frames * self.rows // A.BLOCK)
        self.cache = A.KVCache(blocks, kv_heads, head_dim, device=device)
        self.table = torch.arange(blocks, dtype=torch.int32, device=device)[None]       # one sequence: the pool in order
        self.length = torch.zeros((1,), dtype=torch.int32, device=device)

    def _layer(self, c_in, c_out, k, flags, x, w, idx, count, mask=None):
        desc = B.conv_desc(1, self.height, self.width, c_in, c_out, (k, k), pad=(k // 2, k // 2), in_dtype=B.BF16, flags=flags)
        return B.focused_conv2d(desc, x, w, mask_in=mask, mask_out=mask, idx=idx, count=count)

    def __call__(self, x, mask):
        """x [1, height, width, channels] bf16, mask [1, height, width] uint8 -> (features like x, zero at irrelevant positions; the rows of
        queries, keys and values; the attention's rows and selected blocks; the number of rows)"""
        idx, count = B.active_index_compact(mask)
        kept = self._layer(self.channels, self.channels, 3, B.RELU | B.COMPACT_OUT, x, self.w_in, idx, count, mask)
        width = (self.heads + 2 * self.kv_heads) * self.head_dim
        qkv = self._layer(self.channels, width, 1, B.COMPACT_IN | B.COMPACT_OUT, kept, self.w_qkv, idx, count, mask)
        qkv = qkv.view(self.rows, self.heads + 2 * self.kv_heads, self.head_dim)
        q, k, v = qkv.split([self.heads, self.kv_heads, self.kv_heads], dim=1)          # slices: nothing is copied
        starts = torch.zeros((2,), dtype=torch.int32, device=x.device)
        starts[1:] = count
        self.length += count
        A.kv_append(self.cache, k, v, self.table, self.length, starts=starts, max_new=self.rows)
        attended, selected = A.focused_attention(self.cache, q, self.table, self.length, self.first, self.last, self.top, starts=starts,
                                                 max_new=self.rows)
        y = self._layer(self.heads * self.head_dim, self.channels, 1, B.COMPACT_IN, attended, self.w_out, idx, count, mask)
        return y, qkv, attended, selected, count


def main():
    height, width, frames = 60, 80, 6
    layer = FrameAttention(height, width, frames=frames)
    gen = torch.Generator(device="cuda:0").manual_seed(1)
    for frame in range(frames):
        x = torch.randn((1, height, width, layer.channels), generator=gen, device="cuda:0").relu_().to(torch.bfloat16)
        mask = torch.from_numpy(synth.mask_objects(1, height, width, 0.48, frame)).to("cuda:0")
        y, _, _, selected, count = layer(x, mask)
        kept = int(count)                                       # (for the printed line only)
        print("frame %d: %d of %d positions kept, %d in the cache, rms of the output at them %.3f, blocks of the last row %s" % (
            frame, kept, layer.rows, int(layer.length), float((y.float().square().sum() / (kept * layer.channels)).sqrt()),
            [b for b in selected[kept - 1, 0].tolist() if b >= 0]))


if __name__ == "__main__":
    main()
