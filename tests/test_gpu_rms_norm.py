"""zi_rms_norm and zi_rms_norm_backward against their formulas in 64 bits.

Sums over a row of n take at most 64 steps in a thread and 16 over threads in fp32: 80 * 2^-24 < 5e-6 of the sum of
magnitudes.  What is made of them has up to six more roundings; results are rounded once to their type."""
import pytest
import torch

import paper_2104_07857_amd as zi
from fp8_util import DT, HALF_ULP, LEAST, Matrix, block_most, normal, numbers, powers, rounded, same, scale_bytes, spread, view_of

pytestmark = pytest.mark.gpu
SUM, EPS = 5e-6, 1e-5
HALF = [torch.bfloat16, torch.float16]
SIZES = [(1, 1), (1, 4096), (3, 7), (2, 8), (5, 127), (4, 128), (9, 129), (70, 512), (6, 513), (33, 1000), (3, 2048), (2, 2049), (5, 4097), (17, 8192), (3, 8200),
         (2, 16385), (2, 32768), (3, 40001), (2, 65536), (3000, 256)]


def _near(got, want, dtype, extra):
    return bool(((got.double() - want).abs() <= want.abs() * HALF_ULP[dtype] * 1.01 + LEAST[dtype] + extra).all())


def _norm(x, gamma, residual=None, wide=True, eps=EPS, stream=None, pad=0, inplace=None):
    rows, cols = x.shape
    new = lambda: view_of(torch.full((rows, cols), float("nan"), dtype=x.dtype, device="cuda:0"), pad)          # noqa: E731
    total = None if residual is None else (x if inplace == "x" else residual if inplace == "residual" else new())
    y = (x if inplace == "y" else new()) if wide else None
    rstd, y8 = torch.full((rows,), float("nan"), device="cuda:0"), Matrix(rows, cols)
    args = zi.make_rms_norm(x, gamma, DT[x.dtype], eps, residual=residual, sum=total, y=y, rstd=rstd)
    torch.cuda.synchronize()
    zi.zi_rms_norm(args, y8.struct, stream)
    torch.cuda.synchronize()
    return total, y, rstd, y8


def _check(x, gamma, residual, result, eps=EPS):
    total, y, rstd, y8 = result
    dtype, cols = x.dtype, x.shape[1]
    h = x
    if residual is not None:
        h = (x.float() + residual.float()).to(dtype)
        assert same(total, h)
    h = h.double()
    r = (h.square().mean(1) + eps).rsqrt()
    assert bool(((rstd.double() - r).abs() <= r * (SUM + 4 * 2.0 ** -24)).all())
    want = h * r[:, None] * gamma.double()
    slack = SUM + 6 * 2.0 ** -24
    if y is not None:
        assert _near(y, want, dtype, want.abs() * slack)
    # a block's scale is one of those that the largest may have within the slack, its numbers within half a step of the scaled value
    most = block_most(want, 1)
    s = y8.scales()
    assert bool(((s >= scale_bytes(most * (1 - slack))) & (s <= scale_bytes(most * (1 + slack)))).all())
    scaled = want / spread(powers(s), *x.shape, 1)
    q = numbers(y8.codes())
    step = torch.maximum(torch.exp2(torch.floor(torch.log2(torch.maximum(scaled.abs(), q.abs()).clamp_min(2.0 ** -6)))) / 8, torch.full_like(scaled, 2.0 ** -9))
    assert bool(((q - scaled).abs() <= step / 2 + scaled.abs() * slack).all())
    if cols >= 1000:                                                         # nearly all of them are the very numbers
        assert float((q != rounded(scaled)).double().mean()) < 1e-3


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("dtype", HALF)
def test_norm(rows, cols, dtype):
    x, residual = normal((rows, cols), 1, 2.0, dtype), normal((rows, cols), 2, 1.0, dtype)
    gamma = (1 + normal((cols,), 3, 0.2)).to(dtype)
    _check(x, gamma, None, _norm(x, gamma))
    _check(x, gamma, residual, _norm(x, gamma, residual, wide=False))


@pytest.mark.parametrize("pad", [1, 5, 8])
@pytest.mark.parametrize("dtype", HALF)
def test_norm_of_views(pad, dtype):
    x, residual = view_of(normal((30, 777), 4, dtype=dtype), pad, 3), view_of(normal((30, 777), 5, dtype=dtype), pad)
    gamma = view_of(normal((1, 777), 6, dtype=dtype), 1, 1)[0]
    _check(x, gamma, residual, _norm(x, gamma, residual, pad=pad))


@pytest.mark.parametrize("inplace", ["x", "residual", "y"])
@pytest.mark.parametrize("cols", [100, 4096, 40001])
def test_norm_in_place(inplace, cols):
    x, residual, gamma = normal((20, cols), 7, dtype=torch.bfloat16), normal((20, cols), 8, dtype=torch.bfloat16), normal((cols,), 9, dtype=torch.bfloat16)
    x0, r0 = x.clone(), residual.clone()
    if inplace == "y":
        _check(x0, gamma, None, _norm(x, gamma, inplace="y"))
    else:
        _check(x0, gamma, r0, _norm(x, gamma, residual, inplace=inplace))


@pytest.mark.parametrize("cols", [5, 300, 9000])
def test_rows_of_zeros_infinities_and_nan(cols):
    x, gamma = normal((12, cols), 10, dtype=torch.bfloat16), normal((cols,), 11, dtype=torch.bfloat16)
    gamma[0] = 0.0
    x[1] = 0.0
    x[2, cols // 2], x[3, 0], x[4, cols - 1] = float("nan"), float("inf"), float("-inf")
    x[5] = 1e-30
    total, y, rstd, y8 = _norm(x, gamma)
    fine = [0, 1, 5, 6, 7, 8, 9, 10, 11]
    keep = Matrix(len(fine), cols).put(y8.codes()[fine], y8.scales()[fine])
    _check(x[fine], gamma, None, (None, y[fine], rstd[fine], keep))
    # an infinity leaves rstd 0 and is NaN itself, a NaN takes its row along
    assert float(rstd[1]) == pytest.approx(EPS ** -0.5, rel=1e-6) and bool(rstd[2].isnan()) and rstd[3:5].tolist() == [0.0, 0.0]
    assert bool(y[2].isnan().all()) and bool(numbers(y8.codes())[2].isnan().all())
    assert bool(y[3, 0].isnan()) and not bool(y[3, 1:].any()) and bool(y[4, cols - 1].isnan()) and not bool(y[4, :cols - 1].any())
    assert int(numbers(y8.codes())[3:5].isnan().sum()) == 2
    z = torch.zeros((2, cols), dtype=torch.float16, device="cuda:0")           # eps 0: 0 * infinity
    y = _norm(z, gamma.half(), eps=0.0)[1]
    assert bool(y.isnan().all())


def test_norm_outputs_one_at_a_time_streams_and_graphs():
    x, gamma = normal((50, 600), 12, dtype=torch.bfloat16), normal((600,), 13, dtype=torch.bfloat16)
    _, y, rstd, y8 = _norm(x, gamma, stream=torch.cuda.Stream())
    _check(x, gamma, None, (None, y, rstd, y8))
    only_y, only_rstd, only_8 = torch.empty_like(x), torch.empty(50, device="cuda:0"), Matrix(50, 600)
    zi.zi_rms_norm(zi.make_rms_norm(x, gamma, zi.ZI_BF16, EPS, y=only_y))
    zi.zi_rms_norm(zi.make_rms_norm(x, gamma, zi.ZI_BF16, EPS, rstd=only_rstd))
    zi.zi_rms_norm(zi.make_rms_norm(x, gamma, zi.ZI_BF16, EPS), only_8.struct)
    torch.cuda.synchronize()
    assert torch.equal(only_y, y) and torch.equal(only_rstd, rstd) and torch.equal(only_8.codes(), y8.codes()) and torch.equal(only_8.scales(), y8.scales())
    g = torch.cuda.CUDAGraph()
    args = zi.make_rms_norm(x, gamma, zi.ZI_BF16, EPS, y=only_y)
    with torch.cuda.graph(g):
        zi.zi_rms_norm(args, only_8.struct, torch.cuda.current_stream())
    for k in range(3):
        x.copy_(normal((50, 600), 20 + k))
        g.replay()
        torch.cuda.synchronize()
        _check(x, gamma, None, (None, only_y, _norm(x, gamma)[2], only_8))


# ---- backward -------------------------------------------------------------------------------------------------

def _forms(dy, h, gamma, rstd, dsum):
    """dx, dgamma and what bounds the errors of their sums, in 64 bits."""
    dy, h, gamma, r = dy.double(), h.double(), gamma.double(), rstd.double()[:, None]
    u, n = dy * gamma, h * r
    dot, size = (u * n).mean(1, keepdim=True), (u * n).abs().mean(1, keepdim=True)
    dx = r * (u - n * dot)
    extra = r * (SUM * n.abs() * size + 6 * 2.0 ** -24 * (u.abs() + n.abs() * dot.abs()))
    if dsum is not None:
        dx = dx + dsum.double()
        extra = extra + 2.0 ** -23 * (dx.abs() + dsum.double().abs())
    return dx, extra, (dy * n).sum(0), (dy * n).abs().sum(0)


def _backward(dy, h, gamma, rstd, dsum=None, dgamma32=True, accumulate=None, pad=0, inplace=None, stream=None, want=(True, True)):
    rows, cols = dy.shape
    dx = None
    if want[0]:
        dx = {"dy": dy, "dsum": dsum, None: view_of(torch.full((rows, cols), float("nan"), dtype=dy.dtype, device="cuda:0"), pad)}[inplace]
    dgamma = None
    if want[1]:
        dgamma = torch.full((cols,), float("nan"), dtype=torch.float32 if dgamma32 else dy.dtype, device="cuda:0") if accumulate is None else accumulate.clone()
    ws = torch.full((max(1, zi.zi_rms_norm_workspace_bytes(rows, cols)),), 0xFF, dtype=torch.uint8, device="cuda:0")
    args = zi.make_rms_norm_backward(dy, h, gamma, rstd, dx, dgamma, DT[dy.dtype], dsum=dsum, dgamma_dtype=zi.ZI_FP32 if dgamma32 else None,
                                     accumulate=accumulate is not None)
    torch.cuda.synchronize()
    zi.zi_rms_norm_backward(args, ws, stream=stream)
    torch.cuda.synchronize()
    return dx, dgamma


def _inputs(rows, cols, dtype, seed=30):
    dy, h, dsum = normal((rows, cols), seed, 0.1, dtype), normal((rows, cols), seed + 1, 1.5, dtype), normal((rows, cols), seed + 2, 0.1, dtype)
    gamma = (1 + normal((cols,), seed + 3, 0.2)).to(dtype)
    return dy, h, dsum, gamma, (h.float().square().mean(1) + EPS).rsqrt()


def _row_sum(rows):
    """Steps of the sum over rows in fp32 (one share a row, then shares), as a bound on its relative error."""
    return (rows + 80) * 2.0 ** -24


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("dtype", HALF)
def test_backward(rows, cols, dtype):
    dy, h, dsum, gamma, rstd = _inputs(rows, cols, dtype)
    for add in (None, dsum):
        want, extra, sums, size = _forms(dy, h, gamma, rstd, add)
        dx, dgamma = _backward(dy, h, gamma, rstd, add)
        assert _near(dx, want, dtype, extra)
        assert _near(dgamma, sums, torch.float32, size * _row_sum(rows))
    dx, dgamma = _backward(dy, h, gamma, rstd, dgamma32=False)
    assert _near(dgamma, sums, dtype, size * _row_sum(rows))


@pytest.mark.parametrize("dgamma32", [True, False])
def test_backward_accumulates_and_gives_one_output_at_a_time(dgamma32):
    dy, h, dsum, gamma, rstd = _inputs(40, 600, torch.bfloat16)
    want, extra, sums, size = _forms(dy, h, gamma, rstd, None)
    old = normal((600,), 40, dtype=torch.float32 if dgamma32 else torch.bfloat16)
    dx, dgamma = _backward(dy, h, gamma, rstd, dgamma32=dgamma32, accumulate=old)
    assert _near(dgamma, sums + old.double(), old.dtype, size * _row_sum(40) + 2.0 ** -23 * old.double().abs())
    assert torch.equal(_backward(dy, h, gamma, rstd, want=(True, False))[0], dx)
    assert torch.equal(_backward(dy, h, gamma, rstd, dgamma32=dgamma32, want=(False, True))[1], _backward(dy, h, gamma, rstd, dgamma32=dgamma32)[1])
    zero = _backward(dy[:0], h[:0], gamma, rstd[:0], want=(False, True))[1]
    assert not bool(zero.any())                                              # a sum over no rows


@pytest.mark.parametrize("cols", [100, 4096, 40001])
@pytest.mark.parametrize("inplace", ["dy", "dsum"])
def test_backward_in_place_and_of_views(cols, inplace):
    dy, h, dsum, gamma, rstd = _inputs(30, cols, torch.float16)
    want, extra, sums, size = _forms(dy, h, gamma, rstd, dsum)
    dx, dgamma = _backward(dy.clone(), h, gamma, rstd, dsum.clone(), inplace=inplace)
    assert _near(dx, want, torch.float16, extra) and _near(dgamma, sums, torch.float32, size * _row_sum(30))
    dx, dgamma = _backward(view_of(dy, 5, 1), view_of(h, 3), gamma, rstd, view_of(dsum, 8), pad=1)
    assert _near(dx, want, torch.float16, extra) and _near(dgamma, sums, torch.float32, size * _row_sum(30))


def test_backward_same_bits_every_time_and_in_a_graph():
    dy, h, dsum, gamma, rstd = _inputs(3000, 1000, torch.bfloat16)
    dx, dgamma = _backward(dy, h, gamma, rstd, dsum)
    for _ in range(3):
        again = _backward(dy, h, gamma, rstd, dsum, stream=torch.cuda.Stream())
        assert torch.equal(again[0], dx) and torch.equal(again[1], dgamma)
    out, total = torch.zeros_like(dx), torch.zeros_like(dgamma)
    ws = torch.empty(zi.zi_rms_norm_workspace_bytes(3000, 1000), dtype=torch.uint8, device="cuda:0")
    args = zi.make_rms_norm_backward(dy, h, gamma, rstd, out, total, zi.ZI_BF16, dsum=dsum, dgamma_dtype=zi.ZI_FP32)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        zi.zi_rms_norm_backward(args, ws, stream=torch.cuda.current_stream())
    for _ in range(3):
        out.zero_()
        ws.fill_(0xFF)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, dx) and torch.equal(total, dgamma)


def test_nan_in_a_row_reaches_its_gradient_and_every_share_of_gamma():
    dy, h, dsum, gamma, rstd = _inputs(40, 300, torch.bfloat16)
    dy[7, 3] = float("nan")
    dx, dgamma = _backward(dy, h, gamma, rstd)
    assert bool(dx[7].isnan().all()) and int(dx.isnan().sum()) == 300
    assert bool(dgamma[3].isnan()) and int(dgamma.isnan().sum()) == 1


@pytest.mark.parametrize("rows,cols", [(3, 17), (5, 600)])
def test_gradients_against_differences(rows, cols):
    """The loss sum(y * dy) of the norm in 64 bits: central differences in random directions.  Their own error is of the
    order of step^2, 1e-8 of the loss' size; the gradients are in fp16."""
    dy, h, _, gamma, _ = _inputs(rows, cols, torch.float16, 50)
    rstd = (h.double().square().mean(1) + EPS).rsqrt().float()
    dx, dgamma = _backward(dy, h, gamma, rstd)

    def loss(x, g):
        return float((x * (x.square().mean(1, keepdim=True) + EPS).rsqrt() * g * dy.double()).sum())

    step = 1e-4
    for seed in range(4):
        v, w = normal((rows, cols), 60 + seed).double(), normal((cols,), 70 + seed).double()
        x, g = h.double(), gamma.double()
        along = (loss(x + step * v, g) - loss(x - step * v, g)) / (2 * step)
        assert abs(float((dx.double() * v).sum()) - along) <= (HALF_ULP[torch.float16] + 1e-5) * float(dx.double().norm() * v.norm())
        along = (loss(x, g + step * w) - loss(x, g - step * w)) / (2 * step)
        assert abs(float((dgamma.double() * w).sum()) - along) <= 1e-5 * float(dgamma.double().norm() * w.norm())
