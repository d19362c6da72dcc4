"""The matrix product with bias, activation and residual against its definition in 64 bits."""
import pytest
import torch

from paper_2207_10741_amd import binding as B, layers as L
from tests import layers_oracle as O

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


def _normal(shape, dtype, seed, scale=1.0):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).mul_(scale).to(dtype).to(DEV)


def _case(rows, k, n, dtype, out, bias, residual, activation, first=False, **kw):
    x, w = _normal((rows, k), dtype, rows * 7 + k), _normal((n, k), dtype, n * 5 + k, k ** -0.5)
    b = _normal((n,), F32, 3) if bias else None
    r = _normal((rows, n), out, 4) if residual else None
    got = L.linear(x, w, b, residual=r, activation=activation, residual_first=first, out_dtype=out, **kw)
    assert got.dtype == out and got.shape == (rows, n)
    want, error = O.linear(x, w, b, r, activation, first, out)
    O.check(got, want, error, "%d x %d x %d" % (rows, k, n))


# rows on either side of the kernels' tiles, reductions from one element on, odd sizes
SIZES = [(1, 1, 1), (1, 64, 16), (1, 1000, 37), (1, 4096, 512), (2, 65, 5), (3, 8, 1000), (15, 200, 130), (16, 128, 64), (17, 63, 33), (31, 1001, 100),
         (32, 512, 256), (33, 72, 48), (63, 520, 515), (64, 640, 200), (64, 64, 16400), (5, 96, 16390), (20, 40, 17000),
         (65, 1, 1), (65, 64, 64), (100, 1001, 515), (127, 200, 8), (128, 128, 128), (129, 136, 136), (300, 520, 264), (513, 72, 1000), (70, 4100, 33),
         (2100, 200, 5600), (2049, 64, 5633), (256, 65, 49200)]


@pytest.mark.parametrize("size", SIZES, ids=lambda s: "%dx%dx%d" % s)
@pytest.mark.parametrize("dtype,out", [(BF16, BF16), (F16, F32)], ids=["bf16", "f16-f32"])
def test_sizes(size, dtype, out):
    rows, k, n = size
    _case(rows, k, n, dtype, out, rows % 2 == 0 or k % 2 == 0, n % 3 == 0, [None, "relu", "silu", "gelu"][(rows + n) % 4])


@pytest.mark.parametrize("rows", [7, 200])
@pytest.mark.parametrize("dtype,out", [(BF16, F32), (F16, F16)], ids=["bf16-f32", "f16"])
@pytest.mark.parametrize("activation", [None, "relu", "silu", "gelu"])
@pytest.mark.parametrize("first", [False, True])
def test_epilogues(rows, dtype, out, activation, first):
    for bias, residual in ((False, False), (True, False), (False, True), (True, True)):
        _case(rows, 72, 104, dtype, out, bias, residual, activation, first)


@pytest.mark.parametrize("rows", [9, 150])
@pytest.mark.parametrize("offset,k,extra", [(0, 64, 16), (8, 72, 8), (1, 64, 8), (3, 77, 5), (0, 64, 1)])
def test_strides(rows, offset, k, extra):
    n = 56
    x = _normal((rows, offset + k + extra), BF16, 1)[:, offset:offset + k]
    w = _normal((n, offset + k + extra), BF16, 2, 0.1)[:, offset:offset + k]
    res = _normal((rows, n + 3), BF16, 3)[:, 1:1 + n]
    big = torch.full((rows, n + 9), 7.0, dtype=BF16, device=DEV)
    out = big[:, 5:5 + n]
    L.linear(x, w, residual=res, out=out)
    want, error = O.linear(x, w, None, res, out_dtype=BF16)
    O.check(out, want, error)
    assert bool((big[:, :5] == 7).all()) and bool((big[:, 5 + n:] == 7).all())


@pytest.mark.parametrize("rows", [12, 140])
def test_one_row_for_all_and_residual_in_place(rows):
    x = _normal((1, 96), F16, 1).expand(rows, 96)
    w = _normal((40, 96), F16, 2, 0.1)
    out = _normal((rows, 40), F16, 3)
    before = out.clone()
    assert L.linear(x, w, residual=out, out=out, activation="gelu") is out
    want, error = O.linear(x, w, None, before, "gelu", out_dtype=F16)
    O.check(out, want, error)


@pytest.mark.parametrize("rows,k,n", [(10, 100, 50), (64, 64, 64), (400, 200, 136), (400, 201, 77), (3000, 64, 4400)])
def test_rows_that_are_there(rows, k, n):
    x, w, bias = _normal((rows, k), BF16, 1), _normal((n, k), BF16, 2, 0.1), _normal((n,), F32, 3)
    for there in (0, 1, rows // 3, rows - 1, rows, rows + 5, -3):
        held = min(max(there, 0), rows)
        y = x.clone()
        y[held:] = float("nan")
        out = torch.full((rows, n), 5.0, dtype=BF16, device=DEV)
        L.linear(y, w, bias, count=torch.tensor([there], dtype=torch.int32, device=DEV), out=out, activation="silu")
        want, error = O.linear(x[:held], w, bias, activation="silu", out_dtype=BF16)
        O.check(out[:held], want, error)
        assert bool((out[held:] == 5).all())


@pytest.mark.parametrize("rows", [5, 90])
@pytest.mark.parametrize("k", [64, 50])
def test_not_finite_values_stay_in_their_rows_and_columns(rows, k):
    x, w = _normal((rows, k), BF16, 1), _normal((24, k), BF16, 2)
    x[1, k - 1] = float("nan")
    x[2, 0] = float("inf")
    w[3, 5] = float("inf")
    w[23, k - 1] = float("nan")
    got = L.linear(x, w, out_dtype=F32)
    want, error = O.linear(x, w, out_dtype=F32)
    O.check(got, want, error)


@pytest.mark.parametrize("rows,k,n", [(1, 8192, 64), (50, 4096, 100), (200, 4096, 260)])
def test_results_do_not_depend_on_arrival(rows, k, n):
    """Reductions that several workgroups share are added in order."""
    x, w = _normal((rows, k), BF16, 1), _normal((n, k), BF16, 2)
    call = L.PreparedLinear(x, w, out_dtype=F32)
    first = call().clone()
    want, error = O.linear(x, w, out_dtype=F32)
    O.check(first, want, error)
    for _ in range(20):
        assert torch.equal(call(), first)


def test_no_rows():
    w = _normal((40, 64), BF16, 2)
    assert L.linear(torch.empty((0, 64), dtype=BF16, device=DEV), w).shape == (0, 40)


@pytest.mark.parametrize("rows,k,n", [(3, 4096, 96), (300, 1001, 200), (300, 2048, 128)])
def test_captured_and_on_another_stream(rows, k, n):
    x, w, r = _normal((rows, k), BF16, 1), _normal((n, k), BF16, 2, 0.05), _normal((rows, n), BF16, 3)
    call = L.PreparedLinear(x, w, residual=r, activation="gelu")
    other = L.PreparedLinear(x, w, residual=r)
    eager, eager_other = call().clone(), other().clone()
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        got = call()
    for i in range(4):
        got.zero_()
        graph.replay()
        assert torch.equal(other(), eager_other)
        torch.cuda.synchronize()
        assert torch.equal(got, eager)
        x.copy_(x.flip(0))
        eager, eager_other = L.linear(x, w, residual=r, activation="gelu").clone(), L.linear(x, w, residual=r).clone()
    side.wait_stream(torch.cuda.current_stream())
    out = L.linear(x, w, residual=r, activation="gelu", stream=side)
    side.synchronize()
    assert torch.equal(out, eager)


def test_a_captured_call_brings_its_own_workspace():
    x, w = _normal((200, 2048), BF16, 1), _normal((128, 2048), BF16, 2, 0.05)
    want = L.linear(x, w).clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = L.linear(x, w)
    for _ in range(4):
        got.zero_()
        graph.replay()
        assert torch.equal(L.linear(x, w), want)
        torch.cuda.synchronize()
        assert torch.equal(got, want)
