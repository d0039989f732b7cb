"""The norm and its backward pass where a workgroup goes over several rows, and the norm's kernels for many rows of 8193 to 16384 columns:
against the formulas in 64 bits, with the bounds of test_gpu_rms_norm.py."""
import pytest
import torch

import paper_2104_07857_amd as zi
from fp8_util import DT, Matrix, normal, numbers, view_of
from test_gpu_rms_norm import EPS, HALF, _backward, _check, _forms, _inputs, _near, _norm, _row_sum

pytestmark = pytest.mark.gpu

# more than 256 rows: 512 threads with three (to 12288) and four octets, whole and not
WIDE = [(300, 8200), (257, 8193), (300, 11001), (300, 12288), (300, 12296), (270, 12289), (300, 16383), (300, 16384)]


@pytest.mark.parametrize("rows,cols", WIDE)
@pytest.mark.parametrize("dtype", HALF)
def test_norm_of_many_wide_rows(rows, cols, dtype):
    x, residual = normal((rows, cols), 100, 2.0, dtype), normal((rows, cols), 101, 1.0, dtype)
    gamma = (1 + normal((cols,), 102, 0.2)).to(dtype)
    _check(x, gamma, None, _norm(x, gamma))
    _check(x, gamma, residual, _norm(x, gamma, residual))
    _check(x, gamma, residual, _norm(view_of(x, 3, 5), gamma, view_of(residual, 1), pad=7))


@pytest.mark.parametrize("inplace", ["x", "residual", "y"])
@pytest.mark.parametrize("cols", [8200, 11001, 12296, 16383])
def test_norm_of_many_wide_rows_in_place(inplace, cols):
    x, residual, gamma = normal((300, cols), 103, dtype=torch.bfloat16), normal((300, cols), 104, dtype=torch.bfloat16), normal((cols,), 105, dtype=torch.bfloat16)
    x0, r0 = x.clone(), residual.clone()
    if inplace == "y":
        _check(x0, gamma, None, _norm(x, gamma, inplace="y"))
    else:
        _check(x0, gamma, r0, _norm(x, gamma, residual, inplace=inplace))


@pytest.mark.parametrize("cols", [8200, 11001, 12296, 16383])
def test_rows_of_zeros_infinities_and_nan_among_many(cols):
    x, gamma = normal((300, cols), 106, dtype=torch.bfloat16), normal((cols,), 107, dtype=torch.bfloat16)
    x[1] = 0.0
    x[2, cols // 2], x[299, 0], x[4, cols - 1] = float("nan"), float("inf"), float("-inf")
    _, y, rstd, y8 = _norm(x, gamma)
    fine = [i for i in range(300) if i not in (2, 4, 299)]
    _check(x[fine], gamma, None, (None, y[fine], rstd[fine], Matrix(len(fine), cols).put(y8.codes()[fine], y8.scales()[fine])))
    assert bool(y[2].isnan().all()) and bool(numbers(y8.codes())[2].isnan().all()) and rstd[[4, 299]].tolist() == [0.0, 0.0]
    assert bool(y[299, 0].isnan()) and not bool(y[299, 1:].any()) and bool(y[4, cols - 1].isnan()) and not bool(y[4, :cols - 1].any())
    assert int(numbers(y8.codes())[[4, 299]].isnan().sum()) == 2


@pytest.mark.parametrize("cols", [5, 8, 13, 600, 1032, 1027])
def test_norm_of_more_rows_than_a_launch_has_workgroups(cols):
    """2^20 workgroups: the first of them have a second row."""
    rows = (1 << 20) + 77
    x = normal((rows, cols), 108, dtype=torch.float16)
    gamma = (1 + normal((cols,), 109, 0.2)).half()
    _, y, rstd, y8 = _norm(x, gamma)
    for part in (slice(0, 200), slice(rows - 277, rows)):
        n = len(range(*part.indices(rows)))
        _check(x[part], gamma, None, (None, y[part], rstd[part], Matrix(n, cols).put(y8.codes()[part], y8.scales()[part])))


# ---- backward: three rows and more of some workgroups -----------------------------------------------------------

# up to 512 columns 1536 workgroups, to 1024 1024, to 2048 512, to 16384 256; cut rows 768 over their cuts, and means from 4096 workgroups
ROWS = [(4000, 7), (4000, 8), (4000, 300), (4000, 301), (2500, 1000), (2500, 1001), (1300, 2048), (1300, 2047), (700, 4096), (700, 4001), (700, 8192),
        (700, 8191), (700, 12288), (700, 16384),
        (900, 8201), (500, 16392), (300, 40001), (160, 65536), (5000, 8201)]


@pytest.mark.parametrize("rows,cols", ROWS)
@pytest.mark.parametrize("dtype", HALF)
def test_backward_over_rows(rows, cols, dtype):
    dy, h, dsum, gamma, rstd = _inputs(rows, cols, dtype, 110)
    for add in (None, dsum):
        want, extra, sums, size = _forms(dy, h, gamma, rstd, add)
        dx, dgamma = _backward(dy, h, gamma, rstd, add)
        assert _near(dx, want, dtype, extra)
        assert _near(dgamma, sums, torch.float32, size * _row_sum(rows))
    assert torch.equal(_backward(dy, h, gamma, rstd, dsum, want=(True, False))[0], dx)
    assert torch.equal(_backward(dy, h, gamma, rstd, dsum, want=(False, True))[1], dgamma)


@pytest.mark.parametrize("rows,cols", [(4000, 301), (2500, 1000), (1300, 2047), (700, 4001), (700, 8192), (700, 16384), (900, 8201), (500, 16392)])
@pytest.mark.parametrize("inplace", ["dy", "dsum"])
def test_backward_over_rows_in_place_and_of_views(rows, cols, inplace):
    dy, h, dsum, gamma, rstd = _inputs(rows, cols, torch.bfloat16, 120)
    dx, dgamma = _backward(dy, h, gamma, rstd, dsum)
    want, extra, sums, size = _forms(dy, h, gamma, rstd, dsum)
    assert _near(dx, want, torch.bfloat16, extra) and _near(dgamma, sums, torch.float32, size * _row_sum(rows))
    again = _backward(dy.clone(), h, gamma, rstd, dsum.clone(), inplace=inplace)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dgamma)
    again = _backward(view_of(dy, 5, 1), view_of(h, 3), gamma, rstd, view_of(dsum, 8), pad=1)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dgamma)


@pytest.mark.parametrize("rows,cols", [(2500, 1000), (1300, 2047), (700, 8192), (700, 12288), (900, 8201), (500, 16392)])
def test_nan_keeps_to_its_row(rows, cols):
    """In a workgroup's second row: neither the one before it nor the one behind it sees it."""
    dy, h, dsum, gamma, rstd = _inputs(rows, cols, torch.float16, 130)
    clean = _backward(dy, h, gamma, rstd, dsum)
    spoilt = dy.clone()
    row = rows // 2
    spoilt[row, cols - 1] = float("nan")
    dx, dgamma = _backward(spoilt, h, gamma, rstd, dsum)
    assert bool(dx[row].isnan().all()) and int(dx.isnan().sum()) == cols
    assert bool(dgamma[cols - 1].isnan()) and torch.equal(dgamma[:-1], clean[1][:-1])
    keep = [i for i in range(rows) if i != row]
    assert torch.equal(dx[keep], clean[0][keep])


@pytest.mark.parametrize("rows,cols", [(700, 12288), (900, 8201), (500, 16392)])
def test_replays_over_rows(rows, cols):
    dy, h, dsum, gamma, rstd = _inputs(rows, cols, torch.bfloat16, 140)
    want = _backward(dy, h, gamma, rstd, dsum)
    out, total = torch.zeros_like(want[0]), torch.zeros_like(want[1])
    ws = torch.empty(zi.zi_rms_norm_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda:0")
    args = zi.make_rms_norm_backward(dy, h, gamma, rstd, out, total, DT[torch.bfloat16], dsum=dsum, dgamma_dtype=zi.ZI_FP32)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        zi.zi_rms_norm_backward(args, ws, stream=torch.cuda.current_stream())
    for _ in range(4):
        out.fill_(float("nan"))
        total.fill_(float("nan"))
        ws.fill_(0xFF)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(total, want[1])
        again = _backward(dy, h, gamma, rstd, dsum)
        assert torch.equal(again[0], want[0]) and torch.equal(again[1], want[1])


def test_differences_over_rows():
    """The loss sum(y * dy) in 64 bits, central differences in a random direction, as in test_gpu_rms_norm.py but over many rows a workgroup."""
    rows, cols = 1300, 2047
    dy, h, _, gamma, _ = _inputs(rows, cols, torch.float16, 150)
    rstd = (h.double().square().mean(1) + EPS).rsqrt().float()
    dx, dgamma = _backward(dy, h, gamma, rstd)
    loss = lambda x, g: float((x * (x.square().mean(1, keepdim=True) + EPS).rsqrt() * g * dy.double()).sum())      # noqa: E731
    v, w, step = normal((rows, cols), 160).double(), normal((cols,), 161).double(), 1e-4
    x, g = h.double(), gamma.double()
    along = (loss(x + step * v, g) - loss(x - step * v, g)) / (2 * step)
    assert abs(float((dx.double() * v).sum()) - along) <= (2.0 ** -11 + 1e-5) * float(dx.double().norm() * v.norm())
    along = (loss(x, g + step * w) - loss(x, g - step * w)) / (2 * step)
    assert abs(float((dgamma.double() * w).sum()) - along) <= 1e-5 * float(dgamma.double().norm() * w.norm())
