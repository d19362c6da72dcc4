"""The attention operators from their definition, in 64 bits on the host: what a cache holds after each append, attention over it with
the error that its rounding allows, and the selection of blocks."""
import math

import numpy as np

BLOCK = 64


def least_power(a, limit, lo, hi):
    """The least 2^e, lo <= e <= hi, with a <= limit * 2^e."""
    e = lo
    while e < hi and a > limit * 2.0 ** e:
        e += 1
    return 2.0 ** e


def e4m3(x):
    """The nearest 8-bit value, ties to even, of magnitudes up to 448; NaN stays."""
    x = np.asarray(x, dtype=np.float64)
    m, e = np.frexp(np.where(np.isfinite(x), x, 0.0))
    step = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)
    return np.where(np.isnan(x), np.nan, np.rint(x / step) * step)


def _codes(x, scale):
    """x / scale as codes; what is not finite is NaN."""
    return e4m3(np.where(np.isfinite(x), x / scale, np.nan))


class Cache:
    """One sequence's keys and values: codes [tokens, heads, dim] and the scales [blocks, heads] of either."""

    def __init__(self, heads, dim):
        self.codes = {n: np.zeros((0, heads, dim)) for n in "kv"}
        self.scales = {n: np.zeros((0, heads)) for n in "kv"}
        self.heads, self.dim = heads, dim

    def __len__(self):
        return self.codes["k"].shape[0]

    def append(self, k, v):
        for n, x in (("k", k), ("v", v)):
            x = np.asarray(x, dtype=np.float64)
            had, codes, scales = len(self.codes[n]), self.codes[n], self.scales[n].copy()
            total = had + len(x)
            out = np.concatenate([codes, np.zeros_like(x)])
            grown = np.zeros((-(-total // BLOCK), self.heads))
            grown[:len(scales)] = scales
            for block in range(had // BLOCK, -(-total // BLOCK)):
                lo, hi = max(had, block * BLOCK), min(total, (block + 1) * BLOCK)
                for h in range(self.heads):
                    part = x[lo - had:hi - had, h]
                    finite = np.abs(part[np.isfinite(part)])
                    s = least_power(finite.max() if finite.size else 0.0, 448.0, -64, 120)
                    old = grown[block, h] if lo > block * BLOCK else 0.0
                    if old > s:
                        s = old
                    if old and old != s:
                        out[block * BLOCK:lo, h] = e4m3(out[block * BLOCK:lo, h] * (old / s))
                    out[lo:hi, h] = _codes(part, s)
                    grown[block, h] = s
            self.codes[n], self.scales[n] = out, grown

    def values(self, n):
        return self.codes[n] * np.repeat(self.scales[n], BLOCK, axis=0)[:len(self), :, None]

    def sketches(self):
        """(whole numbers [full blocks, heads, dim], weights [full blocks, heads])"""
        full = len(self) // BLOCK
        sums = np.nan_to_num(self.codes["k"][:full * BLOCK]).reshape(full, BLOCK, self.heads, self.dim).sum(axis=1)
        unit = np.array([[least_power(np.abs(sums[b, h]).max(), 127.0, -126, 120) for h in range(self.heads)] for b in range(full)])
        unit = unit.reshape(full, self.heads)
        return np.rint(sums / unit[:, :, None]), unit / BLOCK * self.scales["k"][:full]


def select(cache, q, position, first, last, top):
    """q [heads, dim] -> ascending blocks of every key head, -1 behind the last."""
    width = first + last + top
    out = np.full((cache.heads, width), -1, dtype=np.int32)
    if position < 0:
        return out
    own = position // BLOCK
    sketch, weight = cache.sketches()
    q = np.asarray(q, dtype=np.float64).reshape(cache.heads, -1, cache.dim)
    for h in range(cache.heads):
        finite = np.where(np.isfinite(q[h]), q[h], 0.0)
        q8 = np.rint(finite / least_power(np.abs(finite).max(), 127.0, -126, 120)).sum(axis=0)
        always = [b for b in range(own + 1) if b < first or b > own - last]
        others = [b for b in range(own + 1) if b not in always]
        others.sort(key=lambda b: (-np.float32(np.float32(q8 @ sketch[b, h]) * np.float32(weight[b, h])), b))
        chosen = sorted(always + others[:top])
        out[h, :len(chosen)] = chosen
    return out


def attend(cache, q, position, scale, causal=True, blocks=None, length=None):
    """One row: q [heads, dim] -> (out, lse, error allowed in 32-bit sums and 11-bit weights), [heads, dim], [heads], [heads, dim].
    blocks: the blocks of every key head; None: all.  position < 0: nothing is attended to."""
    q = np.asarray(q, dtype=np.float64)
    heads, group = q.shape[0], q.shape[0] // cache.heads
    length = len(cache) if length is None else length
    out, lse, error = np.zeros_like(q), np.full(heads, -np.inf), np.zeros_like(q)
    k, v = cache.values("k"), cache.values("v")
    seen = np.arange(length) <= (position if causal else length)
    if position < 0 and causal:
        return out, lse, error
    for h in range(heads):
        rows = seen.copy()
        if blocks is not None:
            rows &= np.isin(np.arange(length) // BLOCK, blocks[h // group][blocks[h // group] >= 0])
        at = np.flatnonzero(rows)
        if at.size == 0:
            continue
        kk, vv = k[at, h // group], v[at, h // group]
        with np.errstate(invalid="ignore", over="ignore"):
            z = scale * (kk @ q[h])
            most = np.max(z) if not np.isnan(z).any() else np.nan
            p = np.exp(z - most)
            total = p.sum()
            lse[h] = most + math.log(total) if np.isfinite(total) else np.nan
            p = p / total
            out[h] = p @ vv
            # a product of stored values: exact; their sum in 32 bits: |q|.|k| 2^-24 an addition and channel, and as much again from
            # the factor of the exponent; the weight's own 2^-11, its least step 2^-25, and the division and sums behind it
            dz = 2.0 ** -23 * scale * np.max(np.abs(kk) @ np.abs(q[h])) * math.sqrt(cache.dim) + 2.0 ** -21
            error[h] = (2.0 ** -11 + 2 * dz + 2.0 ** -18) * (p @ np.abs(vv)) + 2.0 ** -25 * np.abs(vv).sum(axis=0)
    return out, lse, error
