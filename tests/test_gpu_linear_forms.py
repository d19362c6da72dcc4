"""The matrix product in every way that it is cut, each size asserted to be cut so, against its definition in 64 bits."""
import pytest
import torch

from paper_2207_10741_amd import layers as L
from tests.linear_forms import FORMS, check, described, finished, sums

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
ACTS = [None, "relu", "silu", "gelu"]
NAMES = lambda v: "x".join(str(p) for p in v)


def _normal(shape, dtype, seed, scale=1.0):
    return torch.randn(shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV).mul_(scale).to(dtype)


def _operands(size, dtype, seed=1):
    rows, k, n, odd = size
    x, w = _normal((rows, k + ("x" in odd)), dtype, seed)[:, :k], _normal((n, k + ("w" in odd)), dtype, seed + 1, k ** -0.5)[:, :k]
    return x, w


def _made_as(call, form):
    assert described(call.cut) == form
    return call()


@pytest.mark.parametrize("dtype,out", [(BF16, BF16), (BF16, F32), (F16, F16), (F16, F32)], ids=["bf16", "bf16-f32", "f16", "f16-f32"])
@pytest.mark.parametrize("size,form", FORMS, ids=NAMES)
def test_every_form(size, form, dtype, out):
    rows, k, n, _ = size
    x, w = _operands(size, dtype)
    both = sums(x, w)
    bias, residual = _normal((n,), F32, 3), _normal((rows, n), out, 4)
    i = (rows + n + (out == F32)) % 4
    for act, b, r, first in ((None, None, None, False), (ACTS[i], bias, residual, i % 2 == 0), (ACTS[(i + 2) % 4], None, residual, i % 2 == 1)):
        got = _made_as(L.PreparedLinear(x, w, b, residual=r, activation=act, residual_first=first, out_dtype=out), form)
        assert got.dtype == out and got.shape == (rows, n)
        check(got, *finished(both, k, b, r, act, first, out), "%s, %s" % (size, act))


# one of each kernel; the epilogue differs where out's rows are whole pieces of eight columns and where not
EPILOGUES = [((4100, 400, 2048, ""), "large"), ((4099, 456, 2044, ""), "large"), ((4099, 72, 1104, ""), "tiles"), ((127, 4104, 3899, ""), "tiles"), ((127, 4104, 3904, ""), "tiles"),
             ((130, 4104, 64, ""), "stages"), ((50, 4104, 70, ""), "stages"), ((131, 1000, 264, "w"), "stages_any"), ((61, 1003, 131, "xw"), "stages_any"), ((50, 1000, 130, ""), "rings")]


@pytest.mark.parametrize("dtype,out", [(BF16, BF16), (BF16, F32), (F16, F16), (F16, F32)], ids=["bf16", "bf16-f32", "f16", "f16-f32"])
@pytest.mark.parametrize("size,kernel", EPILOGUES, ids=lambda v: v if isinstance(v, str) else NAMES(v))
def test_epilogues(size, kernel, dtype, out):
    rows, k, n, _ = size
    x, w = _operands(size, dtype, 11)
    both = sums(x, w)
    bias, residual = _normal((n,), F32, 13), _normal((rows, n), out, 14)
    for act in ACTS:
        for b, r, first in ((None, None, False), (bias, None, False), (None, residual, False), (bias, residual, False), (None, residual, True), (bias, residual, True)):
            call = L.PreparedLinear(x, w, b, residual=r, activation=act, residual_first=first, out_dtype=out)
            assert described(call.cut)[0] == kernel
            check(call(), *finished(both, k, b, r, act, first, out), "%s, %s, first %s" % (size, act, first))


# rows of the call, what a plan for half of them is
COUNTED = [((8200, 400, 2048, ""), "large"), ((8001, 403, 2051, "xw"), "large"), ((8200, 72, 1100, ""), "tiles"), ((8200, 67, 1003, "xw"), "tiles"), ((1400, 4097, 1501, "xw"), "tiles"),
           ((260, 4104, 60, ""), "stages"), ((262, 1000, 260, "w"), "stages_any"), ((100, 1000, 130, ""), "rings"), ((10, 1001, 37, "xw"), "rows")]


@pytest.mark.parametrize("size,kernel", COUNTED, ids=lambda v: v if isinstance(v, str) else NAMES(v))
def test_rows_that_are_there(size, kernel):
    rows, k, n, _ = size
    x, w = _operands(size, BF16, 21)
    bias = _normal((n,), F32, 23)
    want, error = finished(sums(x, w), k, bias, None, "silu", False, BF16)
    for there in (0, 1, rows // 3, rows // 2 + 1, rows - 1, rows, rows + 5, -3):
        held = min(max(there, 0), rows)
        out = torch.full((rows, n), 5.0, dtype=BF16, device=DEV)
        y = torch.as_strided(torch.empty((rows * x.stride(0),), dtype=BF16, device=DEV), x.shape, x.stride()).copy_(x)
        y[held:] = float("nan")
        call = L.PreparedLinear(y, w, bias, count=torch.tensor([there], dtype=torch.int32, device=DEV), out=out, activation="silu")
        assert described(call.cut)[0] == kernel
        call()
        check(out[:held], want[:held], error[:held], "%d of %s" % (there, size))
        assert bool((out[held:] == 5).all())


@pytest.mark.parametrize("size", [(4100, 400, 2048, ""), (4099, 72, 1104, ""), (130, 4104, 64, "")], ids=NAMES)
def test_strides_in_place_and_one_row_for_all(size):
    rows, k, n, _ = size
    x, w = _normal((rows, k + 24), F16, 31)[:, 8:8 + k], _normal((n, k + 16), F16, 32, k ** -0.5)[:, 16:]
    big = _normal((rows, n + 16), F16, 33)
    for at in (0, 5, 8):            # (rows of out of any alignment and not)
        out, before = big[:, at:at + n], big.clone()
        want, error = finished(sums(x, w), k, None, before[:, at:at + n], None, False, F16)
        assert L.linear(x, w, residual=out, out=out) is out
        check(out, want, error, "from column %d" % at)
        assert torch.equal(big[:, :at], before[:, :at]) and torch.equal(big[:, at + n:], before[:, at + n:])
    one = x[:1].expand(rows, k)
    check(L.linear(one, w), *finished(sums(one, w), k, None, None, None, False, F16), "one row for all")


@pytest.mark.parametrize("size", [(4100, 400, 2048, ""), (4100, 403, 2051, "xw"), (4099, 72, 1100, ""), (127, 4104, 3899, "")], ids=NAMES)
def test_not_finite_values_stay_in_their_rows_and_columns(size):
    rows, k, n, _ = size
    x, w = _operands(size, BF16, 41)
    x[1, k - 1] = float("nan")
    x[rows - 1, 0] = float("inf")
    w[3, 5] = float("inf")
    w[n - 1, k - 1] = float("nan")
    got = L.linear(x, w, out_dtype=F32)
    want, error = finished(sums(x, w), k, None, None, None, False, F32)
    check(got, want, error)


# every kernel whose workgroups share a reduction: pieces asserted
SHARED = [((3, 4097, 37, "xw"), "rows"), ((29, 4097, 50, "w"), "rows"), ((50, 4104, 70, ""), "stages"), ((130, 4104, 60, ""), "stages"), ((61, 4097, 131, "xw"), "stages_any"),
          ((131, 4097, 260, "w"), "stages_any"), ((127, 4104, 3899, ""), "tiles"), ((700, 4097, 1501, "xw"), "tiles")]


@pytest.mark.parametrize("size,kernel", SHARED, ids=lambda v: v if isinstance(v, str) else NAMES(v))
def test_shared_reductions_do_not_depend_on_arrival(size, kernel):
    rows, k, n, _ = size
    x, w = _operands(size, BF16, 51)
    call = L.PreparedLinear(x, w, out_dtype=F32)
    assert described(call.cut)[0] == kernel and call.cut.pieces > 1
    first = call().clone()
    check(first, *finished(sums(x, w), k, None, None, None, False, F32), str(size))
    for _ in range(20):
        assert torch.equal(call(), first)


@pytest.mark.parametrize("size,kernel", [((4100, 400, 2048, ""), "large"), ((4100, 403, 2051, "xw"), "large"), ((127, 4104, 3904, ""), "tiles"), ((700, 4097, 1501, "xw"), "tiles")],
                         ids=lambda v: v if isinstance(v, str) else NAMES(v))
def test_captured(size, kernel):
    """A captured call, replayed, with eager work of the same kind between."""
    rows, k, n, _ = size
    x, w = _operands(size, BF16, 61)
    residual = _normal((rows, n), BF16, 63)
    call, other = L.PreparedLinear(x, w, residual=residual, activation="gelu"), L.PreparedLinear(x, w)
    assert described(call.cut)[0] == kernel
    eager, eager_other = call().clone(), other().clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call()
    for _ in range(4):
        got.zero_()
        graph.replay()
        assert torch.equal(other(), eager_other)
        torch.cuda.synchronize()
        assert torch.equal(got, eager)
        x.copy_(x.flip(0))
        eager, eager_other = L.linear(x, w, residual=residual, activation="gelu").clone(), L.linear(x, w).clone()
