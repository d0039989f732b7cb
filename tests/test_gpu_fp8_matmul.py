"""zi_fp8_matmul against the product in 64 bits.

Small whole numbers times powers of two give products and sums that fp32 holds exactly, and none is small beside its
neighbours: there the result is the exact sum rounded once, bit for bit, so a wrong index or scale cannot hide.  Normal
numbers meet the matrix cores' own bound: of 16 neighbouring products what lies 2^-13 below the largest may be dropped,
15 * 2^-13 < 2^-9 of the sum of magnitudes in all, beside the rounding of the result and 2^-20 for sums of up to 2^4 * 2^12 terms
in fp32 whose order is free."""
import pytest
import torch

import paper_2104_07857_amd as zi
from fp8_util import DT, HALF_ULP, LEAST, Matrix, normal, view_of

pytestmark = pytest.mark.gpu
NUMBERS = [0x00, 0x38, 0xB8, 0x40, 0xC0, 0x44, 0x30, 0x80]                   # 0, 1, -1, 2, -2, 3, 0.5, -0


def _whole(rows, cols, block_rows, seed, **more):
    """Small numbers, scales from 2^-3 to 2^3."""
    g = torch.Generator(device="cuda:0").manual_seed(seed)
    pick = torch.randint(0, len(NUMBERS), (rows, cols), generator=g, device="cuda:0")
    codes = torch.tensor(NUMBERS, dtype=torch.uint8, device="cuda:0")[pick]
    m = Matrix(rows, cols, block_rows, **more)
    scales = torch.randint(124, 131, m.scales().shape, generator=g, device="cuda:0").to(torch.uint8)
    return m.put(codes, scales)


def _normal(rows, cols, block_rows, seed, outliers=False):
    x = normal((rows, cols), seed, dtype=torch.float32)
    if outliers:
        x[:, 7::64] *= 20.0
    m = Matrix(rows, cols, block_rows)
    zi.zi_fp8_quantize(x, zi.ZI_FP32, rows, cols, cols, m.struct)
    return m


def _call(a, b, dtype, c=None, pad=0, inplace=False, stream=None, workspace=None):
    m, n = a.rows, b.rows
    d = torch.full((m, n + pad), float("nan"), dtype=dtype, device="cuda:0")
    if c is not None:
        c = view_of(c, pad)
        if inplace:
            d.copy_(c if pad == 0 else torch.nn.functional.pad(c, (0, pad), value=float("nan")))
    ws = torch.full((max(1, zi.zi_fp8_matmul_workspace_bytes(m, n, a.cols)),), 0xFF, dtype=torch.uint8, device="cuda:0")
    torch.cuda.synchronize()
    zi.zi_fp8_matmul(a.struct, b.struct, d, DT[dtype], n + pad, d if inplace else c, ws, stream=stream)
    torch.cuda.synchronize()
    assert bool(d[:, n:].isnan().all())                                      # nothing between the rows
    return d[:, :n]


def _exact(a, b, c=None):
    d = a.values() @ b.values().t().contiguous()
    return d if c is None else d + c.double()


SIZES = [(1, 1, 1), (1, 16, 128), (2, 3, 5), (1, 300, 1000), (7, 129, 127), (13, 257, 384), (16, 1024, 2048), (17, 64, 129), (31, 500, 640), (33, 128, 256),
         (64, 512, 1111), (65, 70, 512), (100, 1000, 100), (128, 128, 128), (129, 255, 513), (200, 300, 4096), (256, 256, 256), (257, 511, 1030),
         (300, 40, 3000), (512, 768, 640), (1000, 1001, 130), (600, 1300, 96),
         # each kernel: k shared out (with an end inside a block and inside a group of four), each size of tile with ends on every side
         (40, 200, 16384), (33, 129, 12345), (100, 64, 7000), (16, 8192, 8000), (260, 4100, 700), (700, 6000, 900), (2050, 2047, 520), (1001, 8190, 250), (3900, 4099, 1100)]


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_whole_numbers_are_exact(m, n, k, dtype):
    for i, (ba, bb) in enumerate([(1, 128), (1, 1), (128, 128)]):
        a, b = _whole(m, k, ba, 10 + i), _whole(n, k, bb, 20 + i)
        assert torch.equal(_call(a, b, dtype), _exact(a, b).to(dtype))


@pytest.mark.parametrize("m,n,k", [(1, 300, 1000), (13, 257, 384), (40, 100, 260), (129, 255, 513), (300, 520, 640)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("inplace", [False, True])
def test_c_is_added_before_the_rounding(m, n, k, dtype, inplace):
    a, b = _whole(m, k, 1, 30), _whole(n, k, 1, 31)
    c = torch.randint(-64, 65, (m, n), generator=torch.Generator(device="cuda:0").manual_seed(1), device="cuda:0").to(dtype)
    for pad in (0, 3, 8):
        assert torch.equal(_call(a, b, dtype, c, pad, inplace), _exact(a, b, c).to(dtype))


@pytest.mark.parametrize("m,n,k", [(1, 512, 4096), (5, 100, 777), (24, 640, 2048), (100, 200, 300), (300, 260, 4000), (520, 1030, 8191)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("outliers", [False, True])
def test_normal_numbers_within_the_bound(m, n, k, dtype, outliers):
    a, b = _normal(m, k, 1, 40, outliers), _normal(n, k, 128, 41)
    d, e = _call(a, b, dtype).double(), _exact(a, b)
    size = a.values().abs() @ b.values().abs().t().contiguous()
    assert bool(((d - e).abs() <= size * (2.0 ** -9 + 2.0 ** -20) + e.abs() * HALF_ULP[dtype] * 1.01 + LEAST[dtype]).all())
    assert float((d - e).norm() / e.norm()) <= HALF_ULP[dtype] + 2e-4


@pytest.mark.parametrize("m", [1, 40, 300])
def test_garbage_around_the_operands(m):
    """Longer pitches, with NaN in every byte that belongs to no block."""
    a, b = _whole(m, 200, 1, 50, more_ld=48, more_scale=8), _whole(300, 200, 128, 51, more_ld=16, more_scale=4)
    assert torch.equal(_call(a, b, torch.bfloat16, pad=5), _exact(a, b).to(torch.bfloat16))


@pytest.mark.parametrize("m", [1, 20, 140, 300])
def test_nan_keeps_to_its_rows_and_columns(m):
    a, b = _whole(m, 300, 1, 60), _whole(270, 300, 1, 61)
    a.data[m - 1, 299], b.data[5, 0], b.scale[269, 1] = 0x7F, 0xFF, 0xFF
    d, e = _call(a, b, torch.bfloat16), _exact(a, b)
    assert torch.equal(d.isnan(), e.isnan()) and int(e.isnan().sum()) == 270 + 2 * (m - 1)
    assert torch.equal(d[~d.isnan()], e.to(torch.bfloat16)[~d.isnan()])


def test_results_beyond_the_type_and_the_smallest():
    a, b = Matrix(40, 128), Matrix(50, 128)
    for s, want in ((127, 448.0 * 448 * 128), (247, float("inf")), (0, 0.0)):
        a.put(torch.full((40, 128), 0x7E, dtype=torch.uint8, device="cuda:0"), torch.full((40, 1), s, dtype=torch.uint8, device="cuda:0"))
        b.put(torch.full((50, 128), 0x7E, dtype=torch.uint8, device="cuda:0"), torch.full((50, 1), s, dtype=torch.uint8, device="cuda:0"))
        want = torch.full((40, 50), want, dtype=torch.float64, device="cuda:0")
        assert torch.equal(_call(a, b, torch.bfloat16), want.to(torch.bfloat16))
        assert torch.equal(_call(a, b, torch.float16), want.to(torch.float16))


@pytest.mark.parametrize("m,n", [(1, 5), (40, 300), (300, 7)])
def test_k_of_zero(m, n):
    a, b = zi.zi_fp8_matrix(None, None, m, 0, 0, 0, 1, 0), zi.zi_fp8_matrix(None, None, n, 0, 0, 0, 128, 0)
    d = torch.full((m, n), float("nan"), dtype=torch.bfloat16, device="cuda:0")
    c = normal((m, n), 1, dtype=torch.bfloat16)
    zi.zi_fp8_matmul(a, b, d, zi.ZI_BF16, n)
    torch.cuda.synchronize()
    assert not bool(d.any())
    zi.zi_fp8_matmul(a, b, d, zi.ZI_BF16, n, c)
    torch.cuda.synchronize()
    assert torch.equal(d, c)


@pytest.mark.parametrize("m,n,k", [(1, 512, 4096), (20, 300, 2000), (150, 200, 3000), (700, 600, 900)])
def test_same_bits_every_time_on_any_stream_and_in_a_graph(m, n, k):
    a, b = _normal(m, k, 1, 70), _normal(n, k, 128, 71)
    d = _call(a, b, torch.bfloat16)
    for _ in range(3):
        assert torch.equal(_call(a, b, torch.bfloat16, stream=torch.cuda.Stream()), d)
    out = torch.zeros_like(d)
    ws = torch.empty(max(1, zi.zi_fp8_matmul_workspace_bytes(m, n, k)), dtype=torch.uint8, device="cuda:0")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        zi.zi_fp8_matmul(a.struct, b.struct, out, zi.ZI_BF16, out.stride(0), None, ws, stream=torch.cuda.current_stream())
    for k in range(3):
        out.zero_()
        ws.fill_(0xFF)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, d)


def test_operands_of_more_than_four_gib():
    """Offsets past 2^32 bytes in an operand and in D."""
    n, k = 2100, 2 << 20
    b = Matrix(n, k, 128)
    b.data.zero_()
    b.scale.fill_(127)
    rows = torch.tensor([0, 1, 1023, 2047, 2048, 2099], device="cuda:0")
    b.data[rows, k - 1] = torch.tensor([0x38, 0x40, 0x44, 0xB8, 0xC0, 0x30], dtype=torch.uint8, device="cuda:0")
    a = Matrix(1, k)
    a.data.fill_(0x38)
    a.scale.fill_(127)
    want = torch.zeros((1, n), dtype=torch.bfloat16, device="cuda:0")
    want[0, rows] = torch.tensor([1.0, 2.0, 3.0, -1.0, -2.0, 0.5], dtype=torch.bfloat16, device="cuda:0")
    assert torch.equal(_call(a, b, torch.bfloat16), want)
    assert torch.equal(_call(b, a, torch.bfloat16), want.t())


def test_the_gradients_of_a_layer():
    """y = x W^T: against the products in 64 bits of what the 8-bit operands stand for, and its directional derivative
    against differences."""
    m, n, k = 200, 300, 400
    x, w, dy = normal((m, k), 80), normal((n, k), 81, 0.05), normal((m, n), 82, 1e-3)
    x8, xt8, w8, wt8, dy8, dyt8 = Matrix(m, k), Matrix(k, m), Matrix(n, k, 128), Matrix(k, n, 128), Matrix(m, n), Matrix(n, m)
    zi.zi_fp8_quantize(x, zi.ZI_FP32, m, k, k, x8.struct, xt8.struct)
    zi.zi_fp8_quantize(w, zi.ZI_FP32, n, k, k, w8.struct, wt8.struct)
    zi.zi_fp8_quantize(dy, zi.ZI_FP32, m, n, n, dy8.struct, dyt8.struct)
    torch.cuda.synchronize()
    assert torch.equal(wt8.values(), w8.values().t())
    y, dx, dw = _call(x8, w8, torch.bfloat16), _call(dy8, wt8, torch.bfloat16), _call(dyt8, xt8, torch.bfloat16)
    near = lambda u, v, tol: float((u.double() - v).norm() / v.norm()) <= tol                         # noqa: E731
    # three products of rounded operands: 2^-4 / sqrt(3) of each number at most, independent, twice; and bf16
    for got, exact in ((y, x.double() @ w.double().t()), (dx, dy.double() @ w.double()), (dw, dy.double().t() @ x.double())):
        assert near(got, exact, 2.0 ** -4 / 3 ** 0.5 * 2 ** 0.5)
    for got, (p, q) in ((y, (x8, w8)), (dx, (dy8, wt8)), (dw, (dyt8, xt8))):
        assert near(got, _exact(p, q), HALF_ULP[torch.bfloat16] + 2e-4)
    # loss sum(y * dy) is linear in x and in W: a difference is exact up to the operands' rounding
    v, u = normal((m, k), 83).double(), normal((n, k), 84).double()
    loss = lambda a, b: float(((a @ b.t()) * dy.double()).sum())                                     # noqa: E731
    for got, diff, size in ((float((dx.double() * v).sum()), (loss(x.double() + v, w.double()) - loss(x.double() - v, w.double())) / 2, v),
                            (float((dw.double() * u).sum()), (loss(x.double(), w.double() + u) - loss(x.double(), w.double() - u)) / 2, u)):
        scale = float(size.norm()) * float((dx if size is v else dw).double().norm())
        assert abs(got - diff) <= 2.0 ** -4 / 3 ** 0.5 * 2 ** 0.5 * scale


# Products of each size of tile larger than the smallest (64 x 128, 128 x 128 with four and two steps in LDS, 256 x 128, 256 x 256): ends on every side,
# k that ends inside a block, with a block inside a group of four, and with a group.
TILES = [(1290, 3000, 384), (1290, 3001, 1667), (1290, 1544, 4001), (2049, 1000, 4001), (2500, 1544, 200), (2049, 2047, 1000), (1001, 4099, 4001),
         (2049, 2047, 4001), (1290, 3500, 4224), (2049, 6001, 1667), (3001, 4099, 2560), (3001, 4100, 3000)]


@pytest.mark.parametrize("m,n,k", TILES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_every_tile_is_exact(m, n, k, dtype):
    a, b = _whole(m, k, 1, 30), _whole(n, k, 128, 40)
    exact = _exact(a, b)
    assert torch.equal(_call(a, b, dtype), exact.to(dtype))
    c = torch.randint(-8, 9, (m, n), generator=torch.Generator(device="cuda:0").manual_seed(50), device="cuda:0").to(dtype)
    want = (exact + c.double()).to(dtype)
    assert torch.equal(_call(a, b, dtype, c=c, pad=3), want)
    assert torch.equal(_call(a, b, dtype, c=c, inplace=True), want)


@pytest.mark.parametrize("m,n,k", [(1290, 3001, 1667), (1290, 1544, 4001), (1001, 4099, 4001), (3001, 4100, 3000)])
def test_every_tile_keeps_nan_to_its_row_and_gives_the_same_bits(m, n, k):
    a, b = _normal(m, k, 1, 31), _normal(n, k, 128, 41)
    first = _call(a, b, torch.bfloat16)
    for _ in range(3):
        assert torch.equal(_call(a, b, torch.bfloat16), first)
    a.data[m - 2, k - 1] = 0x7F
    spoilt = _call(a, b, torch.bfloat16)
    assert bool(spoilt[m - 2].isnan().all())
    spoilt[m - 2] = first[m - 2]
    assert torch.equal(spoilt, first)
