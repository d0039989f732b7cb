"""The operators together, as examples/fp8_mlp.py uses them: every stage of a training step, a run that learns, a token
by itself like the same token in a batch."""
import os
import sys

import pytest
import torch

from fp8_util import HALF_ULP, numbers, powers, spread

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def _values(m):
    return numbers(m.data[:, :m.cols]) * spread(powers(m.scale[:, :-(-m.cols // 128)]), m.rows, m.cols, m.struct.block_rows)


def test_every_stage_is_the_layer_of_its_operands():
    """Each product against the exact one of the numbers that it had: bf16's rounding of the result, and 2e-4 for the matrix cores'
    (see test_gpu_fp8_matmul.py).  (Autograd of the unrounded layer would not do: where rounding turns z's sign, relu's gradient
    is another.)"""
    import fp8_mlp
    h, t = 256, 384
    model = fp8_mlp.Mlp(h, t, seed=3)
    x, _ = fp8_mlp.data(h, t, 5)
    dout = torch.randn((t, h), generator=torch.Generator(device="cuda:0").manual_seed(6), device="cuda:0").bfloat16()
    out = model.forward(x)
    dx = model.backward(x, dout)
    torch.cuda.synchronize()
    (w1, w1t), (w2, w2t) = [(_values(a), _values(b)) for a, b in model.w]
    assert torch.equal(w1t, w1.t()) and torch.equal(w2t, w2.t())
    for w, p in ((w1, model.p[1]), (w2, model.p[2])):                        # rounding to three bits of fraction, uniform
        assert float((w - p.double()).norm() / p.double().norm()) <= 2.0 ** -4 / 3 ** 0.5
    near = lambda got, exact: float((got.double() - exact).norm() / exact.norm()) <= HALF_ULP[torch.bfloat16] + 2e-4      # noqa: E731
    y8, u8, ut8, do8, dot8, dz8, dzt8, yt8 = (_values(m) for m in (model.y8, model.u8, model.ut8, model.do8, model.dot8, model.dz8, model.dzt8, model.yt8))
    assert near(model.z, y8 @ w1.t().contiguous()) and near(model.out, u8 @ w2.t().contiguous())
    assert torch.equal(out, model.out + x)
    assert near(model.du, do8 @ w2) and near(model.dy, dz8 @ w1)
    assert near(model.g[2], dot8 @ ut8.t().contiguous()) and near(model.g[1], dzt8 @ yt8.t().contiguous())
    xd = x.double().requires_grad_()
    gamma = model.lp[0].double().requires_grad_()
    (xd * (xd.square().mean(1, keepdim=True) + 1e-5).rsqrt() * gamma).backward(model.dy.double())
    assert near(dx, xd.grad + dout.double()) and near(model.g[0], gamma.grad)


def test_it_learns_and_decodes():
    import fp8_mlp
    losses, model = fp8_mlp.train(256, 1024, 40)
    assert losses[-1] < 0.5 * losses[0] and all(later < 2 * losses[0] for later in losses)
    x, _ = fp8_mlp.data(256, 1024, 7)
    out, total = model.decode(x[:1] / 2, x[:1] / 2)
    whole = model.forward(x)[:1].float()
    # the same operands and kernels of another order of sums: bf16's rounding of z and of the sum, and what it flips in u's numbers
    assert float((out + total - whole).norm() / whole.norm()) <= 0.02
