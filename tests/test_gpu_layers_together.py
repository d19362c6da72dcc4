"""The layers, the pages and the attention together, as a model over a camera's frames uses them: group norm over the kept positions of a feature map, projections of
the kept rows, blocks for them, the cache, attention, the projection back with the residual, and samples that go on from a shared prefix."""
import math

import pytest
import torch

from paper_2207_10741_amd import attention as A, binding as B, layers as L, pages as P
from tests import layers_oracle as O

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16 = torch.bfloat16


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _normal(shape, seed, scale=1.0, dtype=BF16):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).mul_(scale).to(dtype).to(DEV)


class _Block:
    """One layer: norm, projection, cache, attention, projection and residual; two sequences in a pool."""

    def __init__(self, channels, heads, kv_heads, dim, blocks, width, batch):
        self.channels, self.heads, self.kv_heads, self.dim, self.batch = channels, heads, kv_heads, dim, batch
        self.weight, self.bias = _normal((channels,), 1, 0.2, torch.float32), _normal((channels,), 2, 0.2, torch.float32)
        self.w_qkv = _normal(((heads + 2 * kv_heads) * dim, channels), 3, channels ** -0.5)
        self.b_qkv = _normal(((heads + 2 * kv_heads) * dim,), 4, 0.1, torch.float32)
        self.w_out = _normal((channels, heads * dim), 5, (heads * dim) ** -0.5)
        self.cache = A.KVCache(blocks, kv_heads, dim, device=DEV)
        self.users, self.table = P.kv_users(self.cache), torch.full((batch, width), -1, dtype=torch.int32, device=DEV)
        self.lengths = torch.zeros((batch,), dtype=torch.int32, device=DEV)

    def rows(self, x, counts):
        """x [rows, channels], the sequences' new rows behind each other (counts: how many each has) -> out and what lies between."""
        starts = _int32([0] + torch.tensor(counts).cumsum(0).tolist())
        qkv = L.linear(x, self.w_qkv, self.b_qkv).view(-1, self.heads + 2 * self.kv_heads, self.dim)
        q, k, v = qkv.split([self.heads, self.kv_heads, self.kv_heads], dim=1)
        self.lengths += _int32(counts)
        missing = P.kv_resize(self.cache, self.users, self.table, self.lengths)
        A.kv_append(self.cache, k, v, self.table, self.lengths, starts=starts, max_new=max(counts))
        attended = A.cache_attention(self.cache, q, self.table, self.lengths, starts=starts, max_new=max(counts))
        out = L.linear(attended.view(-1, self.heads * self.dim), self.w_out, residual=x)
        return out, qkv, attended, missing

    def cached(self, slot):
        n = int(self.lengths[slot])
        k, v = A.kv_read(self.cache, self.table[slot:slot + 1].clone(), self.lengths[slot:slot + 1].clone(), max_new=max(n, 1))
        return k[:n].double().cpu(), v[:n].double().cpu()

    def check(self, x, counts, got):
        out, qkv, attended, missing = got
        assert missing.tolist() == [0]
        want, error = O.linear(x, self.w_qkv, self.b_qkv, out_dtype=BF16)
        O.check(qkv.reshape(x.shape[0], -1), want, error, "queries, keys, values")
        want, error = O.linear(attended.reshape(x.shape[0], -1), self.w_out, residual=x, out_dtype=BF16)
        O.check(out, want, error, "projection back")
        at = 0
        for slot, n in enumerate(counts):
            if n == 0:
                continue
            k, v = self.cached(slot)
            # (the cache's own rounding is 2^-4 of a value; its contents are what is attended to)
            new = qkv[at:at + n, self.heads:].double().cpu()
            most = torch.cat([k, v], 1)[-n:].abs().amax()
            assert float((torch.cat([k, v], 1)[-n:] - new).abs().max()) <= 2.0 ** -4 * float(most)
            group = self.heads // self.kv_heads
            for i in {0, n // 2, n - 1}:
                position = k.shape[0] - n + i
                q = qkv[at + i, :self.heads].double().cpu().view(self.kv_heads, group, self.dim)
                z = torch.matmul(q, k[:position + 1].permute(1, 2, 0)) / math.sqrt(self.dim)
                p = torch.softmax(z, 2)
                want = torch.matmul(p, v[:position + 1].transpose(0, 1)).reshape(self.heads, self.dim)
                # half a step of bf16, 2^-11 of the weights, 2^-20 of the scores
                size = torch.matmul(p, v[:position + 1].transpose(0, 1).abs()).reshape(self.heads, self.dim)
                off = (attended[at + i].double().cpu() - want).abs()
                assert bool((off <= 2.0 ** -8 * want.abs() + 2.0 ** -9 * size + 1e-6).all())
            at += n


def test_a_prefix_two_samples_and_a_move():
    block = _Block(96, 4, 2, 64, 40, 10, 3)
    # a feature map of two images: norm over the kept positions, whose rows go on
    x = _normal((2, 9, 13, 96), 7, 2.0)
    mask = (torch.rand((2, 9, 13), generator=torch.Generator().manual_seed(8)) < 0.6)
    normed = L.group_norm(x, 8, block.weight, block.bias, mask=mask.to(torch.uint8).to(DEV), activation="silu")
    for b in range(2):
        want, error = O.group_norm(x[b].view(-1, 96), 8, block.weight, block.bias, mask[b].view(-1), activation="silu")
        O.check(normed[b].view(-1, 96), want, error, "norm")
    counts = [int(m.sum()) for m in mask] + [0]
    rows = normed[mask.to(DEV)]
    block.check(rows, counts, block.rows(rows, counts))
    # slot 2 goes on from slot 0, by itself; then all three have one more token
    before = block.cached(0)
    assert P.kv_fork(block.cache, block.users, block.table, block.lengths, _int32([0, 1, 0])).tolist() == [0]
    assert all(torch.equal(a, b) for a, b in zip(before, block.cached(2)))
    for step in range(70):          # over the end of the unfinished block
        token = _normal((3, 96), 100 + step)
        got = block.rows(token, [1, 1, 1])
        if step % 23 == 0:
            block.check(token, [1, 1, 1], got)
    full = counts[0] // 64
    assert torch.equal(block.table[0, :full], block.table[2, :full]) and not torch.equal(block.table[0], block.table[2])
    kept = [block.cached(b) for b in range(3)]
    n = counts[0] // 64 * 64
    assert all(torch.equal(kept[0][i][:n], kept[2][i][:n]) for i in range(2)) and not torch.equal(kept[0][0], kept[2][0])
    # slot 1 ends, what is left moves to a smaller cache and goes on there
    block.lengths[1] = 0
    assert P.kv_resize(block.cache, block.users, block.table, block.lengths).tolist() == [0]
    to = A.KVCache(12, 2, 64, device=DEV)
    users = P.kv_users(to)
    table, missing = P.kv_compact(block.cache, block.users, block.table, to, users)
    assert missing.tolist() == [0]
    block.cache, block.users, block.table = to, users, table
    assert all(torch.equal(a, b) for s in (0, 2) for a, b in zip(kept[s], block.cached(s)))
    token = _normal((2, 96), 300)
    block.check(token, [1, 0, 1], block.rows(token, [1, 0, 1]))


def test_a_captured_step_of_all_of_them():
    """One graph: norm, projection, blocks, cache, attention, projection back and a fork; replayed, with eager work of the same kinds between."""
    block, eager = (_Block(64, 4, 2, 64, 60, 8, 4) for _ in range(2))
    x = _normal((4, 64), 1)
    parents = _int32([0, 1, 0, 3])

    def step(b):
        h = L.group_norm(x[:, None], 4, b.weight, b.bias)[:, 0]
        qkv = L.linear(h, b.w_qkv, b.b_qkv, activation="gelu").view(4, -1, 64)
        q, k, v = qkv.split([4, 2, 2], dim=1)
        b.lengths += 1
        P.kv_resize(b.cache, b.users, b.table, b.lengths)
        A.kv_append(b.cache, k, v, b.table, b.lengths)
        attended = A.cache_attention(b.cache, q, b.table, b.lengths)
        out = L.linear(attended.view(4, -1), b.w_out, residual=x)
        P.kv_fork(b.cache, b.users, b.table, b.lengths, parents)
        return out

    step(block), step(eager)                # (kernels' limits are raised before a capture)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(block)
    for i in range(70):
        x.copy_(_normal((4, 64), 50 + i))
        graph.replay()
        want = step(eager)
        assert torch.equal(got, want)
        assert torch.equal(block.table, eager.table) and torch.equal(block.users, eager.users) and torch.equal(block.lengths, eager.lengths)


def test_compacted_rows_of_a_convolution():
    """Rows that a focused convolution hands on in list order go through a projection with the device's count and back into the map."""
    from paper_2207_10741_amd import synth
    n, h, w, c = 2, 20, 31, 64
    x = _normal((n, h, w, c), 1)
    mask = torch.from_numpy(synth.mask_objects(n, h, w, 0.5, 3)).to(DEV)
    idx, count = B.active_index_compact(mask)
    w_conv = _normal((c, 3, 3, c), 2, 0.05)
    rows = B.focused_conv2d(B.conv_desc(n, h, w, c, c, in_dtype=B.BF16, flags=B.COMPACT_OUT | B.RELU), x, w_conv, mask_in=mask, mask_out=mask, idx=idx, count=count)
    rows = rows.view(-1, c)
    weight, bias = _normal((100, c), 3, 0.1), _normal((100,), 4, 1.0, torch.float32)
    out = torch.full((n * h * w, 100), 3.0, dtype=BF16, device=DEV)
    L.linear(rows, weight, bias, activation="silu", count=count, out=out)
    kept = int(count)
    assert 0 < kept < n * h * w
    want, error = O.linear(rows[:kept], weight, bias, activation="silu", out_dtype=BF16)
    O.check(out[:kept], want, error)
    assert bool((out[kept:] == 3).all())
