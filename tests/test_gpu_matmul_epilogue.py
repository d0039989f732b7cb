"""zi_fp8_matmul_epilogue against the product in 64 bits and what follows it.  Whole numbers are exact, as test_gpu_fp8_matmul.py explains, through every kernel (test_epilogue_plans.py says that these sizes reach them);
normal numbers meet the matrix cores' own bound that it derives, on top of that of epilogue_util.py."""
import pytest
import torch

import paper_2104_07857_amd as zi
from epilogue_util import ACTIVATIONS, OFFSET, SEED, act, dropped, factor, kept, near, near8, same8
from epilogue_plans import ALONE, SUMS
from fp8_plans import FEW_16, FEW_32, PARTS, TILES
from fp8_util import DT, Matrix, normal, numbers, quantized, same, view_of
from test_gpu_epilogue import _empty, _is_quantised, _whole
from test_gpu_fp8_matmul import _exact, _normal
from test_gpu_fp8_matmul import _whole as _whole8

pytestmark = pytest.mark.gpu
HALF = [torch.bfloat16, torch.float16]


class Product:
    def __init__(self, a, b, dtype, activation="none", outputs="y", bias=None, residual=None, drop=0.0, pad=0, offset=0, at=OFFSET, d_offset=None, stream=None, y=None):
        m, n, k = a.rows, b.rows, a.cols
        wanted = outputs.split(",")
        self.z, self.y, self.y8, self.turned, checks = None, y, None, None, []
        for name in ("z", "y"):
            if name in wanted and getattr(self, name) is None:
                out, check = _empty(m, n, dtype, pad, offset)
                setattr(self, name, out)
                checks.append(check)
        more = dict(more_ld=16, more_scale=4) if pad else {}
        self.y8 = Matrix(m, n, **more) if "y8" in wanted else None
        self.turned = Matrix(n, m, **more) if "turned" in wanted else None
        self.args = zi.make_epilogue(m, n, DT[dtype], bias=bias, residual=residual, z=self.z, y=self.y, activation=ACTIVATIONS[activation], drop=drop, seed=SEED, offset=at,
                                     d_offset=d_offset)
        self.outputs8 = (zi.ZI_EPILOGUE_Y8 if self.y8 else 0) + (zi.ZI_EPILOGUE_TURNED if self.turned else 0)
        self.ws = torch.full((max(16, zi.zi_fp8_matmul_epilogue_workspace_bytes(m, n, k, self.outputs8)),), 0xFF, dtype=torch.uint8, device="cuda:0")
        self.a, self.b, self.checks = a, b, checks
        torch.cuda.synchronize()
        self.call(stream)
        torch.cuda.synchronize()
        self.check()

    def call(self, stream=None):
        zi.zi_fp8_matmul_epilogue(self.a.struct, self.b.struct, self.args, self.y8.struct if self.y8 else None, self.turned.struct if self.turned else None, self.ws, stream=stream)

    def check(self):
        assert all(c() for c in self.checks)
        for m, to in ((self.y8, 8), (self.turned, 16)):
            if m is not None:
                end = -(-m.cols // to) * to
                assert bool((m.data[:, end:] == 0xFF).all()) and not bool(m.data[:, m.cols:end].any())
                assert bool((m.scale[:, -(-m.cols // 128):] == 0xFF).all())

    def equals(self, other):
        return all((getattr(self, n) is None) or torch.equal(getattr(self, n), getattr(other, n)) for n in ("z", "y")) and \
            all((getattr(self, n) is None) or same8(getattr(self, n), getattr(other, n)) for n in ("y8", "turned"))


def _want(product, activation, drop, bias, residual):
    z = product if bias is None else product + bias.double()
    y = dropped(act(z, activation), drop)
    return z, y if residual is None else y + residual.double()


ALL = FEW_16 + FEW_32 + PARTS + TILES + SUMS + ALONE


@pytest.mark.parametrize("m,n,k", ALL)
@pytest.mark.parametrize("dtype", HALF)
def test_whole_numbers_are_exact(m, n, k, dtype):
    a, b = _whole8(m, k, 1, 1), _whole8(n, k, 128, 2)
    product = _exact(a, b)
    bias, residual = _whole(1, n, 3, dtype)[0], _whole(m, n, 4, dtype)
    z, y = _want(product, "relu", 0.5, bias, residual)
    for outputs in ("y", "z,y", "y8", "z,y8", "y8,turned", "z,y,y8,turned", "z,y8,turned", "turned"):
        for pad, offset in ((0, 0), (5, 1)):
            p = Product(a, b, dtype, "relu", outputs, bias, view_of(residual, pad), 0.5, pad, offset)
            assert p.z is None or torch.equal(p.z, z.to(dtype)), outputs
            assert p.y is None or torch.equal(p.y, y.to(dtype)), outputs
            assert p.y8 is None or _is_quantised(p.y8, y), outputs
            assert p.turned is None or _is_quantised(p.turned, y.t()), outputs
    p = Product(a, b, dtype, outputs="y,y8,turned")
    assert torch.equal(p.y, product.to(dtype)) and _is_quantised(p.y8, product) and _is_quantised(p.turned, product.t())
    p = Product(a, b, dtype, outputs="y", residual=residual, y=residual.clone())
    assert torch.equal(p.y, (product + residual.double()).to(dtype))
    inplace = residual.clone()
    p = Product(a, b, dtype, outputs="y", bias=bias, residual=inplace, drop=0.5, y=inplace)
    assert torch.equal(inplace, _want(product, "none", 0.5, bias, residual)[1].to(dtype))


@pytest.mark.parametrize("m,n,k", [FEW_16[1], FEW_16[3], FEW_32[0], PARTS[1], PARTS[5], TILES[0], TILES[5], TILES[7], TILES[9], TILES[12], TILES[16]] + ALONE)
@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("activation", list(ACTIVATIONS))
def test_normal_numbers_within_the_bounds(m, n, k, dtype, activation):
    """The product is within 2^-9 + 2^-20 of its magnitudes' sum (test_gpu_fp8_matmul.py); the activation passes 1.13 of that on, dropout its factor."""
    a, b = _normal(m, k, 1, 5), _normal(n, k, 128, 6)
    a.scale -= 1                                                        # results of a size where activations bend
    b.scale -= int(round(0.5 * torch.tensor(float(k)).log2().item())) - 1
    bias, residual = normal((n,), 7, 0.5, dtype), normal((m, n), 8, 2.0, dtype)
    product = _exact(a, b)
    size = a.values().abs() @ b.values().abs().t().contiguous()
    for drop in (0.0, 0.1):
        z, y = _want(product, activation, drop, bias, residual)
        off_z = size * (2.0 ** -9 + 2.0 ** -20) + z.abs() * 2.0 ** -23
        off = (1.13 * off_z + act(z, activation).abs() * 2.0 ** -16) * factor(drop) + y.abs() * 2.0 ** -23
        off = torch.where(kept(m, n, drop, device="cuda:0"), off, y.abs() * 2.0 ** -23)
        p = Product(a, b, dtype, activation, "z,y,y8,turned", bias, residual, drop)
        assert near(p.z, z, off_z) and near(p.y, y, off) and near8(p.y8, y, off) and near8(p.turned, y.t().contiguous(), off.t().contiguous())
        # and as near on the whole as the roundings let it be
        assert float((p.y.double() - y).norm() / y.norm()) <= 2.0 ** -8 + 2e-4
        codes, scales = quantized(y, 1)
        exact8 = (codes * torch.exp2(scales.double() - 127).repeat_interleave(128, 1)[:, :n])
        assert float((p.y8.values() - exact8).norm() / y.norm()) <= 0.01


@pytest.mark.parametrize("m,n,k", [FEW_16[3], FEW_32[2], PARTS[1], TILES[0], TILES[9], TILES[16]] + ALONE)
def test_nan_keeps_to_its_place(m, n, k):
    """A NaN in an operand makes NaN of a row, and no more in any output; what is dropped of it is 0."""
    a, b = _whole8(m, k, 1, 9), _whole8(n, k, 1, 10)
    a.data[m - 1, k - 1] = 0x7F
    product = _exact(a, b)
    _, y = _want(product, "none", 0.5, None, None)
    p = Product(a, b, torch.bfloat16, outputs="z,y,y8,turned", drop=0.5)
    assert bool(p.z[m - 1].isnan().all()) and int(p.z.isnan().sum()) == n
    assert torch.equal(p.y.isnan(), y.isnan()) and same(p.y.double(), y.to(torch.bfloat16).double())
    assert same(p.y8.values().isnan().double(), y.isnan().double()) and same(p.turned.values().t().isnan().double(), y.isnan().double())
    codes, scales = quantized(y, 1)
    assert torch.equal(p.y8.scales(), scales) and same(numbers(p.y8.codes()), codes)


@pytest.mark.parametrize("m,n,k", [FEW_16[3], PARTS[1], TILES[3], TILES[7], TILES[8], TILES[9], TILES[11], TILES[12], TILES[16]] + ALONE)
def test_infinities_have_no_part_in_a_scale(m, n, k):
    """A row of A whose products pass what fp32 holds: infinities in its row of y, NaN in 8 bits, and the scales of its columns' blocks those of the other rows."""
    a, b = _whole8(m, k, 1, 20), _whole8(n, k, 1, 21)
    b.data[:, 0], a.data[m // 2] = 0x38, 0
    a.data[m // 2, 0], a.scale[m // 2, 0] = 0x7E, 254                     # 448 * 2^127
    product = _exact(a, b)
    y = torch.where(product.abs() > 2.0 ** 128, torch.full_like(product, float("inf")), product)
    assert bool(y[m // 2].isinf().all()) and int(y.isinf().sum()) == n
    p = Product(a, b, torch.bfloat16, "relu", "y,y8,turned")
    want = y.clamp_min(0)
    assert torch.equal(p.y.double(), want.to(torch.bfloat16).double())
    for matrix, value in ((p.y8, want), (p.turned, want.t())):
        codes, scales = quantized(value, 1)
        assert torch.equal(matrix.scales(), scales) and same(numbers(matrix.codes()), codes)


@pytest.mark.parametrize("m,n", [(1, 5), (40, 300), (300, 700), (2100, 2200)])
def test_k_of_zero(m, n):
    a, b = zi.zi_fp8_matrix(None, None, m, 0, 0, 0, 1, 0), zi.zi_fp8_matrix(None, None, n, 0, 0, 0, 128, 0)
    bias = _whole(1, n, 11, torch.bfloat16)[0]
    y = torch.full((m, n), float("nan"), dtype=torch.bfloat16, device="cuda:0")
    y8, turned = Matrix(m, n), Matrix(n, m)
    ws = torch.empty(max(16, zi.zi_fp8_matmul_epilogue_workspace_bytes(m, n, 0, 3)), dtype=torch.uint8, device="cuda:0")
    zi.zi_fp8_matmul_epilogue(a, b, zi.make_epilogue(m, n, zi.ZI_BF16, bias=bias, y=y, activation=zi.ZI_ACT_RELU), y8.struct, turned.struct, ws)
    torch.cuda.synchronize()
    want = bias.double().clamp_min(0).expand(m, n)
    assert torch.equal(y.double(), want) and _is_quantised(y8, want) and _is_quantised(turned, want.t())


@pytest.mark.parametrize("m,n,k", [FEW_16[1], FEW_32[0], PARTS[1], TILES[0], TILES[8], TILES[9], TILES[16]] + ALONE)
def test_same_bits_every_time_on_any_stream_and_in_a_graph(m, n, k):
    a, b = _normal(m, k, 1, 12), _normal(n, k, 128, 13)
    bias, residual = normal((n,), 14, 0.5, torch.bfloat16), normal((m, n), 15, 2.0, torch.bfloat16)
    for outputs in ("y", "z,y8,turned"):
        first = Product(a, b, torch.bfloat16, "gelu", outputs, bias, residual, 0.1)
        for _ in range(2):
            assert Product(a, b, torch.bfloat16, "gelu", outputs, bias, residual, 0.1, stream=torch.cuda.Stream()).equals(first)
        at = torch.tensor([3], dtype=torch.int64, device="cuda:0")
        p = Product(a, b, torch.bfloat16, "gelu", outputs, bias, residual, 0.1, d_offset=at)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            p.call(torch.cuda.current_stream())
            at += 1
        for i in range(3):
            p.ws.fill_(0xFF)
            g.replay()
            torch.cuda.synchronize()
            p.check()
            assert p.equals(Product(a, b, torch.bfloat16, "gelu", outputs, bias, residual, 0.1, at=OFFSET + 3 + i))


def test_like_the_product_and_the_epilogue_by_itself():
    """Without what follows it is zi_fp8_matmul; z of one call and the epilogue of z are y within z's rounding; the backward pass' mask is the same."""
    m, n, k = 300, 520, 640
    a, b = _normal(m, k, 1, 16), _normal(n, k, 128, 17)
    residual = normal((m, n), 18, 1.0, torch.bfloat16)
    d = torch.empty((m, n), dtype=torch.bfloat16, device="cuda:0")
    zi.zi_fp8_matmul(a.struct, b.struct, d, zi.ZI_BF16, n, residual)
    assert torch.equal(Product(a, b, torch.bfloat16, residual=residual).y, d)
    p = Product(a, b, torch.bfloat16, "silu", "z,y", drop=0.2)
    dz = torch.empty_like(d)
    zi.zi_epilogue_backward(zi.make_epilogue_backward(torch.ones_like(d), None, dz, None, zi.ZI_BF16, drop=0.2, seed=SEED, offset=OFFSET))
    torch.cuda.synchronize()
    mask = kept(m, n, 0.2, device="cuda:0")
    assert torch.equal(dz != 0, mask) and not bool(p.y[~mask].any())
    again = torch.empty_like(d)
    zi.zi_epilogue(p.z, m, n, n, zi.make_epilogue(m, n, zi.ZI_BF16, y=again, activation=zi.ZI_ACT_SILU, drop=0.2, seed=SEED, offset=OFFSET))
    torch.cuda.synchronize()
    # z is off by 2^-8 of itself, silu's slope is 1.1 at most, and both are rounded to 2^-8
    assert bool(((again.double() - p.y.double()).abs() <= (1.1 * p.z.double().abs() * factor(0.2) + 2 * p.y.double().abs()) * 2.0 ** -8 + 2.0 ** -120).all())
