"""Products of every way in which they are cut, with what each is cut into, and their definition in 64 bits with the most a kernel's output may be off."""
import torch

from paper_2207_10741_amd import binding as B, layers as L
from tests import layers_oracle as O

# rows, columns of x, columns of out, the operands whose rows are not whole 16-byte pieces -> kernel, rows and columns of a tile, in several pieces, operands laid out anew.
# Remainders of rows, columns and reduction on either side of the tiles; the reductions of the large tiles end in each of the six stages of their loop.
FORMS = [
    ((1, 4096, 500, ""), ("rings", 16, 16, False, "")), ((16, 72, 5000, ""), ("rings", 16, 32, False, "")), ((17, 520, 203, ""), ("rings", 32, 16, False, "")),
    ((31, 72, 5001, ""), ("rings", 32, 32, False, "")), ((20, 72, 16377, ""), ("rings", 32, 64, False, "")), ((50, 1000, 130, ""), ("rings", 64, 16, False, "")),
    ((33, 200, 5003, ""), ("rings", 64, 32, False, "")), ((129, 72, 3001, ""), ("rings", 64, 64, False, "")),
    ((5, 77, 130, "xw"), ("rows", 16, 16, False, "")), ((3, 1001, 37, "xw"), ("rows", 16, 16, True, "")), ((20, 200, 99, "x"), ("rows", 32, 16, False, "")),
    ((29, 1000, 50, "w"), ("rows", 32, 16, True, "")),
    ((7, 72, 16385, ""), ("stages", 64, 128, False, "")), ((50, 4104, 70, ""), ("stages", 64, 128, True, "")), ((67, 40, 3903, ""), ("stages", 128, 128, False, "")),
    ((130, 4104, 60, ""), ("stages", 128, 128, True, "")),
    ((40, 203, 150, "xw"), ("stages_any", 64, 128, False, "")), ((61, 1003, 131, "xw"), ("stages_any", 64, 128, True, "")),
    ((300, 72, 130, "x"), ("stages_any", 128, 128, False, "")), ((131, 1000, 260, "w"), ("stages_any", 128, 128, True, "")),
    ((4099, 72, 1100, ""), ("tiles", 128, 128, False, "")), ((127, 4104, 3899, ""), ("tiles", 128, 128, True, "")), ((4099, 72, 1101, "x"), ("tiles", 128, 128, False, "x")),
    ((4100, 136, 1004, "w"), ("tiles", 128, 128, False, "w")), ((4100, 67, 1003, "xw"), ("tiles", 128, 128, False, "xw")),
    ((700, 4104, 1501, "x"), ("tiles", 128, 128, True, "x")), ((700, 4104, 1499, "w"), ("tiles", 128, 128, True, "w")), ((700, 4097, 1501, "xw"), ("tiles", 128, 128, True, "xw")),
    ((4100, 400, 2048, ""), ("large", 256, 256, False, "")), ((4099, 456, 2044, ""), ("large", 256, 256, False, "")), ((2000, 520, 5001, ""), ("large", 256, 256, False, "")),
    ((3841, 640, 2056, ""), ("large", 256, 256, False, "")), ((4097, 704, 2049, ""), ("large", 256, 256, False, "")), ((4095, 768, 2305, ""), ("large", 256, 256, False, "")),
    ((4100, 400, 2051, "x"), ("large", 256, 256, False, "x")), ((4001, 448, 2100, "w"), ("large", 256, 256, False, "w")), ((4100, 403, 2051, "xw"), ("large", 256, 256, False, "xw")),
]


def desc_of(rows, k, n, odd, **kw):
    """A descriptor of the size, as the binding makes it where the operands named in odd have one more element between their rows."""
    base = dict(rows=rows, n=n, k=k, dtype=B.BF16, out_dtype=B.BF16, x_row=k + ("x" in odd), w_row=k + ("w" in odd), residual_row=n, out_row=n)
    base.update(kw)
    return L.LinearDesc(**base)


def described(cut):
    return (L.LINEAR_KERNELS[cut.kernel], cut.tile_rows, cut.tile_columns, cut.pieces > 1, "x" * cut.anew_x + "w" * cut.anew_w)


def sums(x, w):
    """(x w^T in 64 bits, the sums of magnitudes), on the operands' device."""
    x, w = x.double().contiguous(), w.double().t().contiguous()
    return x @ w, x.abs() @ w.abs()


def finished(both, k, bias, residual, activation, first, dtype):
    """(out, the most it may be off) from the sums: the bounds of layers_oracle.linear, which says where they come from."""
    y, size = both
    error = (k / 4 + 64) * 2.0 ** -24 * size
    if bias is not None:
        y = y + bias.double()
        error = error + 2.0 ** -24 * y.abs()
    if first and residual is not None:
        y = y + residual.double()
        error = error + 2.0 ** -24 * y.abs()
    y, error = O._after(y, error, activation)
    if not first and residual is not None:
        y = y + residual.double()
        error = error + 2.0 ** -24 * y.abs()
    return y, error + O.HALF_STEP[dtype] * (y.abs() + error) + O.LEAST[dtype]


def check(got, want, error, what=""):
    """layers_oracle.check on the device."""
    got = got.double()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    assert torch.equal(got.nan_to_num(0.0)[~fine], want.nan_to_num(0.0)[~fine]), what
    over = (torch.where(fine, got - want, 0.0).abs() > error.nan_to_num(0.0)) & fine
    at = torch.nonzero(over)
    assert at.shape[0] == 0, "%s: %d of %d off, the first at %s" % (what, at.shape[0], over.numel(), at[0].tolist())
