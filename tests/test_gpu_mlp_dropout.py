"""The operators in one training step and one decoded token, as examples/mlp_dropout.py uses them: every stage is the layer of the operands that it had, its gradients those of the whole."""
import os
import sys

import pytest
import torch

import paper_2104_07857_amd as zi
from epilogue_util import act, backward, dropped, kept, near, near8
from fp8_util import HALF_ULP, Matrix, numbers, powers, spread

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu
DTYPE = torch.bfloat16


def _values(m):
    return numbers(m.data[:, :m.cols]) * spread(powers(m.scale[:, :-(-m.cols // 128)]), m.rows, m.cols, m.struct.block_rows)


class _As(Matrix):
    """A Matrix8 of the examples as the tests look at one."""

    def __init__(self, m):
        self.rows, self.cols, self.block_rows, self.data, self.scale = m.rows, m.cols, m.struct.block_rows, m.data, m.scale


def _near(got, exact):
    """A product: bf16's rounding, and 2e-4 for the matrix cores' (test_gpu_fp8_matmul.py)."""
    return float((got.double() - exact).norm() / exact.norm()) <= HALF_ULP[DTYPE] + 2e-4


@pytest.mark.parametrize("h,t", [(256, 384), (128, 100), (512, 1000)])
def test_every_stage_is_the_layer_of_its_operands(h, t):
    import mlp_dropout
    model = mlp_dropout.Mlp(h, t, drop=0.25, seed=3)
    model.step = 11
    x, _ = mlp_dropout.data(h, t, 5)
    dout = torch.randn((t, h), generator=torch.Generator(device="cuda:0").manual_seed(6), device="cuda:0").to(DTYPE)
    out, dx = model.forward(x), model.backward(x, dout)
    torch.cuda.synchronize()
    (w1, w1t), (w2, w2t) = [(_values(a), _values(b)) for a, b in model.w]
    where = dict(seed=mlp_dropout.SEED, offset=11)
    y8, u8, ut8, do8, dot8, dz8, dzt8, yt8 = (_values(m) for m in (model.y8, model.u8, model.ut8, model.do8, model.dot8, model.dz8, model.dzt8, model.yt8))
    # forward
    product = y8 @ w1.t().contiguous()
    off_z = (y8.abs() @ w1.abs().t().contiguous()) * (2.0 ** -9 + 2.0 ** -20)
    z = product + model.lp[2].double()
    assert near(model.z, z, off_z + z.abs() * 2.0 ** -23)
    u, off = act(z, "gelu"), 1.13 * off_z + act(z, "gelu").abs() * 2.0 ** -15
    assert near8(_As(model.u8), u, off) and near8(_As(model.ut8), u.t().contiguous(), off.t().contiguous())
    v = u8 @ w2.t().contiguous() + model.lp[4].double()
    want = dropped(v, 0.25, **where) + x.double()
    off = ((u8.abs() @ w2.abs().t().contiguous()) * (2.0 ** -9 + 2.0 ** -20) + v.abs() * 2.0 ** -23) * 4 / 3 + want.abs() * 2.0 ** -23
    assert near(out, want, off)
    assert torch.equal(out[~kept(t, h, 0.25, device="cuda:0", **where)], x[~kept(t, h, 0.25, device="cuda:0", **where)])
    # backward
    do, off = backward(dout, None, "none", 0.25, **where)
    assert near8(_As(model.do8), do, off) and near8(_As(model.dot8), do.t().contiguous(), off.t().contiguous())
    assert near(model.g[4], do.sum(0), off.sum(0) + do.abs().sum(0) * 64 * 2.0 ** -24)
    assert _near(model.du, do8 @ w2) and _near(model.g[3], dot8 @ ut8.t().contiguous())
    dz, off = backward(model.du, model.z, "gelu")
    assert near8(_As(model.dz8), dz, off) and near8(_As(model.dzt8), dz.t().contiguous(), off.t().contiguous())
    assert near(model.g[2], dz.sum(0), off.sum(0) + dz.abs().sum(0) * 64 * 2.0 ** -24)
    assert _near(model.dy, dz8 @ w1) and _near(model.g[1], dzt8 @ yt8.t().contiguous())
    xd, gamma = x.double().requires_grad_(), model.lp[0].double().requires_grad_()
    (xd * (xd.square().mean(1, keepdim=True) + 1e-5).rsqrt() * gamma).backward(model.dy.double())
    assert _near(dx, xd.grad + dout.double()) and _near(model.g[0], gamma.grad)


def test_gradients_of_the_whole():
    """Against autograd of the unrounded layer with the same mask: each operand of each product in 8 bits is off by 2^-4 / sqrt(3) of itself at most on the whole, independently, and so
    at most is what goes through gelu's slope with it: of W2 two roundings, of the biases one, of W1 and gamma (through du, dz and the operands of two products) five."""
    import mlp_dropout
    h, t = 512, 1024
    model = mlp_dropout.Mlp(h, t, drop=0.25, seed=4)
    x, _ = mlp_dropout.data(h, t, 8)
    dout = torch.randn((t, h), generator=torch.Generator(device="cuda:0").manual_seed(9), device="cuda:0").to(DTYPE)
    model.forward(x)
    dx = model.backward(x, dout)
    torch.cuda.synchronize()
    p = [model.lp[0].double(), model.p[1].double(), model.lp[2].double(), model.p[3].double(), model.lp[4].double()]
    p = [q.clone().requires_grad_() for q in p]
    xd = x.double().requires_grad_()
    norm = xd * (xd.square().mean(1, keepdim=True) + 1e-5).rsqrt() * p[0]
    u = act(norm @ p[1].t() + p[2], "gelu")
    mask = kept(t, h, 0.25, seed=mlp_dropout.SEED, offset=0, device="cuda:0").double() * 4 / 3
    (xd + mask * (u @ p[3].t() + p[4])).backward(dout.double())
    each = 2.0 ** -4 / 3 ** 0.5
    for got, want, count in ((model.g[4], p[4].grad, 1), (model.g[3], p[3].grad, 2 + 2), (model.g[2], p[2].grad, 5), (model.g[1], p[1].grad, 7), (model.g[0], p[0].grad, 7), (dx, xd.grad, 7)):
        assert float((got.double() - want).norm() / want.norm()) <= each * count ** 0.5 + 2 * HALF_ULP[DTYPE]


def test_it_runs_and_decodes():
    import mlp_dropout
    losses, model = mlp_dropout.train(256, 640, 4)
    assert len(losses) == 4 and all(loss == loss for loss in losses) and model.step == 4
    x, _ = mlp_dropout.data(256, 640, 7)
    model.drop = 0.0
    whole = model.forward(x)[:1].float()
    one = model.decode(x[:1].contiguous()).float()
    # the same operands and kernels of another order of sums: what it flips among u's numbers
    assert float((one - whole).norm() / whole.norm()) <= 0.02


def test_a_step_in_a_graph():
    """Forward and backward of a whole step captured, with the offset counted on in device memory: replays give what calls give one by one."""
    import mlp_dropout
    h, t = 256, 300
    model = mlp_dropout.Mlp(h, t, drop=0.5, seed=5)
    x, _ = mlp_dropout.data(h, t, 10)
    at = torch.zeros(1, dtype=torch.int64, device="cuda:0")
    u8, w2, bias = model.u8, model.w[1][0], model.lp[4]
    out, dz, dbias = torch.empty_like(x), torch.empty_like(x), torch.empty(h, device="cuda:0")
    model.forward(x)
    second = zi.make_epilogue(t, h, zi.ZI_BF16, bias=bias, residual=x, y=out, drop=0.5, seed=1, d_offset=at)
    back = zi.make_epilogue_backward(x, None, dz, dbias, zi.ZI_BF16, drop=0.5, seed=1, d_offset=at, dbias_dtype=zi.ZI_FP32)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s = torch.cuda.current_stream()
        zi.zi_fp8_matmul_epilogue(u8.struct, w2.struct, second, None, None, model.ws, stream=s)
        zi.zi_epilogue_backward(back, None, None, model.ws, stream=s)
        at += 1
    for i in range(3):
        g.replay()
        torch.cuda.synchronize()
        replayed = out.clone(), dz.clone(), dbias.clone()
        eager = zi.make_epilogue(t, h, zi.ZI_BF16, bias=bias, residual=x, y=out, drop=0.5, seed=1, offset=i)
        zi.zi_fp8_matmul_epilogue(u8.struct, w2.struct, eager, None, None, model.ws)
        zi.zi_epilogue_backward(zi.make_epilogue_backward(x, None, dz, dbias, zi.ZI_BF16, drop=0.5, seed=1, offset=i, dbias_dtype=zi.ZI_FP32), None, None, model.ws)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(replayed, (out, dz, dbias)))
