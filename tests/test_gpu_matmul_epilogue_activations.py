"""Every 16-bit number, infinities and NaN among them, through the activations of zi_fp8_matmul_epilogue, in every way that a product is made: of an operand of zeros z is the bias, exactly, so that nothing of the
product's own roundings hides what an activation does.  The bounds are those that zi_epilogue is held to (epilogue_util.py)."""
import pytest
import torch

from epilogue_plans import BOTH, TURNED, Y8, plan
from epilogue_util import forward, near
from fp8_plans import FEW, SHAPES
from fp8_util import block_most, numbers, powers, scale_bytes, spread
from test_gpu_fp8_matmul import _whole as _whole8
from test_gpu_matmul_epilogue import Product

HALF = [torch.bfloat16, torch.float16]
# the kernel for few rows (up to 16, up to 32), parts of k, and sums or tiles of each shape
SIZES = [(4, 2048, 16384), (32, 1024, 4000), (24, 1031, 12001), (17, 8192, 1111), (1290, 3000, 384), (1290, 1545, 4001), (2500, 1544, 200), (320, 6050, 8001), (1550, 7587, 4143), (3087, 1283, 9049)]


def test_every_way_is_gone():
    for outputs8 in (0, Y8, TURNED, BOTH):
        ways = {(p.whole, p.shape) for p in (plan(*s, outputs8) for s in SIZES)}
        least = 2 if outputs8 & TURNED else 1 if outputs8 else 0
        assert ways >= {(1, i) for i in range(least, len(SHAPES))} | {(0, 0), (0 if outputs8 else 1, FEW)} | ({(0, 1)} if outputs8 & TURNED else set()), outputs8


def _near8(codes, scales, want, off):
    """A row in 8 bits is want (64 bits) quantised, from at most `off` away; NaN where want is an infinity or NaN, which have no part in a scale."""
    fine = want.isfinite()
    off = torch.where(fine, off, torch.zeros_like(off))
    most, most_off = block_most(want, 1), block_most(off, 1)
    zero = most <= most_off                              # (then any smaller scale is right, and that of a block of zeros)
    least, largest = scale_bytes((most - most_off).clamp_min(0)), scale_bytes(most + most_off)
    assert bool(((scales >= least) | zero).all()) and bool(((scales <= largest) | (zero & (scales == 127))).all())
    v, s = numbers(codes), spread(powers(scales), *want.shape, 1)
    assert torch.equal(v.isnan(), ~fine)
    w = torch.where(fine, want, torch.zeros_like(want))
    _, e = torch.frexp((w.abs() + off).div(s).clamp_min(2.0 ** -6))
    assert bool(((v - w / s).abs() <= torch.exp2((e - 5).double()) + off / s)[fine].all())


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("activation", ["gelu", "gelu_tanh", "silu"])
def test_every_number_through_every_way(m, n, k, dtype, activation):
    a, b = _whole8(m, k, 1, 1), _whole8(n, k, 128, 2)
    a.data.view(torch.uint8)[:, :k] = 0
    every = torch.arange(65536, dtype=torch.int32, device="cuda:0").to(torch.int16).view(dtype)
    for first in range(0, 65536, n):
        bias = every[first:first + n]
        bias = torch.cat([bias, torch.zeros(n - bias.numel(), dtype=dtype, device="cuda:0")])
        row = bias.reshape(1, -1)
        _, y, off = forward(row, activation)
        off = torch.where(row.isinf(), torch.zeros_like(off), off)             # (it is 0 times infinity there, of a sum with a bias that is not added; y is 0, infinite or NaN)
        fine = y.isfinite()
        for outputs in ("z,y", "y,y8", "z,y8,turned"):
            p = Product(a, b, dtype, activation, outputs, bias)
            if p.z is not None:
                assert torch.equal(p.z.isnan(), bias.isnan().expand(m, n)) and bool(((p.z == bias) | bias.isnan()).all())
            if p.y is not None:
                assert torch.equal(p.y.isnan(), y.isnan().expand(m, n)) and torch.equal(p.y.isinf(), (y.isinf() & (p.y[:1] == y)).expand(m, n))
                assert bool(((p.y == p.y[:1]) | p.y.isnan()).all()) and near(p.y[:1][fine], y[fine], off[fine])
            if p.y8:
                assert bool((p.y8.codes() == p.y8.codes()[:1]).all()) and bool((p.y8.scales() == p.y8.scales()[:1]).all())
                _near8(p.y8.codes()[:1], p.y8.scales()[:1], y, off)
            if p.turned:
                codes, scales = p.turned.codes(), p.turned.scales()
                assert bool((codes == codes[:, :1]).all()) and bool((scales == scales[:, :1]).all())
                _near8(codes[:, :1], scales[:, :1], y.t().contiguous(), off.t().contiguous())
