"""The matrix product with its epilogue and group norm, from their definitions in 64 bits on the CPU, with how far a kernel's output may be off."""
import math

import torch

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
LEAST = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150}     # half the least step


def activate(y, activation):
    if activation == "relu":
        return torch.where(y < 0, torch.zeros_like(y), y)
    if activation == "silu":
        return y / (1.0 + torch.exp(-y))
    if activation == "gelu":
        return 0.5 * y * (1.0 + torch.erf(y / math.sqrt(2.0)))
    return y


def _after(y, error, activation):
    """The activation and its error: slopes are below 1.13, its own arithmetic is good to 2^-20 of its argument."""
    out = activate(y, activation)
    return out, error if activation in (None, "none") else 1.13 * error + (0.0 if activation == "relu" else 2.0 ** -20) * y.abs()


def linear(x, w, bias=None, residual=None, activation=None, residual_first=False, out_dtype=None):
    """(out, the most it may be off).  A sum is rounded once for each product at most, in 32 bits: k 2^-24 of the sum of magnitudes; a quarter of that
    is allowed, as four products at least are added between two roundings."""
    x, w = x.double().cpu(), w.double().cpu()
    y, size = x @ w.t(), x.abs() @ w.abs().t()
    error = (x.shape[1] / 4 + 64) * 2.0 ** -24 * size
    dtype = out_dtype
    more = 0.0 if residual is None else residual.double().cpu()
    if bias is not None:
        y = y + bias.double().cpu()
        error = error + 2.0 ** -24 * y.abs()
    if residual_first:
        y = y + more
        error = error + 2.0 ** -24 * y.abs()
    y, error = _after(y, error, activation)
    if not residual_first:
        y = y + more
        error = error + 2.0 ** -24 * y.abs()
    return y, error + HALF_STEP[dtype] * (y.abs() + error) + LEAST[dtype]


def group_norm(x, groups, weight=None, bias=None, mask=None, eps=1e-5, activation=None):
    """One image's rows [rows, channels] -> (out, the most it may be off); mask [rows] truth values.  The mean is off by 2^-20 of the spread and by a rounding of
    itself (2^-23 with the subtraction), the factor by 2^-18."""
    dtype, (rows, channels) = x.dtype, x.shape
    x = x.double().cpu()
    keep = torch.ones(rows, dtype=torch.bool) if mask is None else mask.cpu()
    out, error = torch.zeros(rows, channels, dtype=torch.float64), torch.zeros(rows, channels, dtype=torch.float64)
    if not bool(keep.any()):
        return out, error
    part = x[keep].view(-1, groups, channels // groups)
    mean = part.mean(dim=(0, 2), keepdim=True)
    variance = (part - mean).square().mean(dim=(0, 2), keepdim=True)
    factor = 1.0 / torch.sqrt(variance + eps)
    z = (part - mean) * factor
    off = z.abs() * 2.0 ** -18 + torch.sqrt(variance) * factor * 2.0 ** -20 + mean.abs() * factor * 2.0 ** -23
    z, off = z.reshape(-1, channels), off.reshape(-1, channels)
    if weight is not None:
        z, off = z * weight.double().cpu(), off * weight.double().cpu().abs()
    if bias is not None:
        z = z + bias.double().cpu()
    off = off + 2.0 ** -22 * z.abs()
    y, off = _after(z, off, activation)
    out[keep] = y
    error[keep] = off + HALF_STEP[dtype] * (y.abs() + off) + LEAST[dtype]
    return out, error


def check(got, want, error, what=""):
    """NaN and infinities in the same places, everything else within its error."""
    got = got.double().cpu()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)]), what
    over = (got - want).abs()[fine] > error[fine]
    assert not bool(over.any()), "%s: %d of %d off, worst %g of what is allowed" % (
        what, int(over.sum()), over.numel(), float(((got - want).abs()[fine] / error[fine].clamp_min(1e-300)).max()))
