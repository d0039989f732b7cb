"""zi_epilogue_backward where z or dy hold infinities and NaN: what dropout took out of y passes nothing back, whatever it was; at an infinite z, which is what a z beyond 65504 is stored as in fp16
though y is finite, the derivative is its limit; and in all forms of dz and in dbias nothing else is touched."""
import pytest
import torch

from epilogue_util import ACTIVATIONS, backward, derivative, dropped, kept, near
from fp8_util import block_most, normal, scale_bytes
from test_gpu_epilogue import Backward

pytestmark = pytest.mark.gpu
HALF = [torch.bfloat16, torch.float16]
INF, NAN = float("inf"), float("nan")
# one row of tiles; several, whose sums a second kernel adds; rows that end inside eight; rows of less than eight
SIZES = [(6, 304), (130, 1003), (40, 5), (261, 512)]


def _limit(z, name):
    """The derivative at any z, 64 bits: 0 and 1 at the infinities."""
    if name == "none":
        return torch.ones_like(z)
    slope = derivative(z, name)
    slope = torch.where(z == INF, torch.ones_like(z), torch.where(z == -INF, torch.zeros_like(z), slope))
    return slope if name == "relu" else torch.where(z.isnan(), z, slope)


def _sprinkle(x, values, first):
    flat = x.view(-1)
    for i, v in enumerate(values):
        flat[first + i::29] = v
    return x


def _check(a, dbias, want, off):
    """All forms of dz, and dbias, against dz in 64 bits."""
    fine = want.isfinite()
    off = torch.where(fine, off, torch.zeros_like(off))
    assert torch.equal(a.dz.isnan(), want.isnan()) and torch.equal(a.dz.isinf(), want.isinf())
    assert near(a.dz[fine], want[fine], off[fine])
    for matrix, w in ((a.dz8, want), (a.turned, want.t().contiguous())):
        assert torch.equal(matrix.values().isnan(), ~w.isfinite())
        most, slack, scales = block_most(w, 1), block_most(off if matrix is a.dz8 else off.t().contiguous(), 1), matrix.scales()
        zero = most <= slack                              # (then any smaller scale is right, and that of a block of zeros)
        assert bool(((scales >= scale_bytes((most - slack).clamp_min(0))) | zero).all()) and bool(((scales <= scale_bytes(most + slack)) | (zero & (scales == 127))).all())
    total = want.sum(0)
    assert torch.equal(dbias.isnan(), total.isnan()) and torch.equal(dbias.isinf(), total.isinf())
    # additions as test_backward_of_normal_numbers counts them
    good, depth = total.isfinite(), 30 + -(-want.shape[0] // 128)
    bound = off.sum(0) + want.nan_to_num(0, 0, 0).abs().sum(0) * depth * 2.0 ** -24
    assert bool(((dbias.double() - total).abs() <= bound)[good].all())


def _off(dy, z, name, p):
    """How far fp32 may be from dz where it is finite, as backward() has it."""
    return backward(dy.nan_to_num(0, 0, 0), z.nan_to_num(0, 0, 0), name, p)[1]


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("activation", list(ACTIVATIONS))
def test_what_is_dropped_has_no_gradient(rows, cols, dtype, activation):
    """Infinities and NaN in z and dy wherever dropout drops, and nowhere else: dz is 0 there, and finite throughout."""
    p = 0.5
    keep = kept(rows, cols, p, device="cuda:0")
    dy, z = normal((rows, cols), 51, 1e-3, dtype), normal((rows, cols), 52, 1.0, dtype)
    dy = torch.where(keep, dy, _sprinkle(dy.clone(), (INF, NAN, -INF), 1))
    z = torch.where(keep, z, _sprinkle(z.clone(), (NAN, -INF, INF, NAN, INF), 2))
    assert not bool(z.isfinite().all() or dy.isfinite().all())
    want = torch.where(keep, dropped(dy.double(), p) * _limit(z.double(), activation), torch.zeros_like(dy, dtype=torch.float64))
    assert bool(want.isfinite().all())
    dbias = torch.empty(cols, device="cuda:0")
    a = Backward(dy, z, activation, "dz,dz8,turned", p, dbias)
    assert not bool(a.dz[~keep].any())
    _check(a, dbias, want, _off(dy, z, activation, p))


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("activation", list(ACTIVATIONS))
@pytest.mark.parametrize("p", [0.0, 0.5])
def test_the_derivative_at_an_infinite_z_is_its_limit(rows, cols, dtype, activation, p):
    """1 at plus infinity, 0 at minus infinity; a NaN in z is one in dz (but for what does not look at it), and so is an infinite dy times 0."""
    dy, z = normal((rows, cols), 53, 1e-3, dtype), _sprinkle(normal((rows, cols), 54, 1.0, dtype), (INF, -INF, INF), 3)
    for more_z, more_dy in (((), ()), ((NAN,), (INF, -INF, NAN))):
        _sprinkle(z, more_z, 11)
        _sprinkle(dy, more_dy, 4)                                      # (at an infinite z too)
        d = dropped(dy.double(), p)
        want = d * _limit(z.double(), activation)
        if activation == "relu":                                       # 0 where the derivative is, whatever dy is
            want = torch.where(z.double() <= 0, torch.zeros_like(d), d)
        want = torch.where(kept(rows, cols, p, device="cuda:0"), want, torch.zeros_like(want))
        dbias = torch.empty(cols, device="cuda:0")
        _check(Backward(dy, z, activation, "dz,dz8,turned", p, dbias), dbias, want, _off(dy, z, activation, p))


@pytest.mark.parametrize("activation", ["gelu", "gelu_tanh", "silu"])
def test_the_derivative_of_far_numbers(activation):
    """Up to the largest of bf16 (fp16's numbers are in test_activations_of_every_number), as near as anywhere."""
    z = torch.cat([s * torch.logspace(0, 38.5, 4096, dtype=torch.float64, device="cuda:0") for s in (1.0, -1.0)]).to(torch.bfloat16).reshape(1, -1)
    one, dbias = torch.ones_like(z), torch.empty(z.shape[1], device="cuda:0")
    Backward(one, z, activation, "dbias", dbias=dbias)
    slope = derivative(z.double(), activation)
    assert bool(slope.isfinite().all())
    assert bool(((dbias.double() - slope).abs() <= slope.abs() * 2.0 ** -16 + 2.0 ** -20).all())
