"""A Transformer's MLP with biases, GELU and dropout, trained and decoded with what follows its products in their epilogues (include/zi_epilogue.h).

    out = x + drop(W2 gelu(W1 norm(x) + b1) + b2)

Beside fp8_mlp.py, whose relu, gradient and residual go over the widest matrices in passes of their own: here the first product leaves z in 16 bits for the backward pass and
its activation in 8 bits, as it is for the second product and transposed for the gradient of W2; the second adds its bias, drops and adds the residual stream; and the
gradients of both come in one pass each, with those of the biases.  Dropout's mask is made again in the backward pass from the seed and the step's number.

    python examples/mlp_dropout.py [hidden size [tokens [steps]]]
"""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

import torch

import paper_2104_07857_amd as zi
from fp8_mlp import BF16, DEV, Matrix8, data

SEED = 0x5EED


class Mlp:
    """Parameters in five tensors of one flat partition each (p, m, v in fp32, gradients and copy in bf16): gamma, W1, b1, W2, b2."""

    def __init__(self, hidden, tokens, drop=0.1, seed=0):
        self.h, self.t, self.drop = hidden, tokens, drop
        h, t = hidden, tokens
        shapes = [(h,), (4 * h, h), (4 * h,), (h, 4 * h), (h,)]
        gen = torch.Generator(device=DEV).manual_seed(seed)
        normal = lambda s: torch.randn(s, generator=gen, device=DEV) * (s[1] ** -0.5 if len(s) == 2 else 0.02)     # noqa: E731
        self.p = [torch.ones(h, device=DEV)] + [normal(s) for s in shapes[1:]]
        self.m, self.v = ([torch.zeros_like(x) for x in self.p] for _ in range(2))
        self.g, self.lp = ([torch.zeros(s, dtype=torch.bfloat16, device=DEV) for s in shapes] for _ in range(2))
        for lp, p in zip(self.lp, self.p):
            lp.copy_(p)
        self.tensors = zi.make_tensors(zip(self.p, self.m, self.v, self.g, self.lp))
        self.norm = torch.zeros(4, dtype=torch.float64, device=DEV)
        self.norm_ws = torch.empty(zi.zi_norm_workspace_bytes(), dtype=torch.uint8, device=DEV)
        self.w = [(Matrix8(r, c, 128), Matrix8(c, r, 128)) for r, c in (shapes[1], shapes[3])]       # as they are, transposed
        self.step = 0
        self.new_weights()
        # what a step leaves for its backward pass
        new = lambda *s: torch.empty(s, dtype=torch.bfloat16, device=DEV)                            # noqa: E731
        self.y, self.z, self.out, self.du, self.dy, self.dx = new(t, h), new(t, 4 * h), new(t, h), new(t, 4 * h), new(t, h), new(t, h)
        self.rstd = torch.empty(t, device=DEV)
        self.y8, self.yt8, self.u8, self.ut8 = Matrix8(t, h), Matrix8(h, t), Matrix8(t, 4 * h), Matrix8(4 * h, t)
        self.do8, self.dot8, self.dz8, self.dzt8 = Matrix8(t, h), Matrix8(h, t), Matrix8(t, 4 * h), Matrix8(4 * h, t)
        sizes = [zi.zi_fp8_matmul_workspace_bytes(*s) for s in ((t, 4 * h, h), (t, h, 4 * h), (4 * h, h, t), (h, 4 * h, t))]
        sizes += [zi.zi_fp8_matmul_epilogue_workspace_bytes(rows, *s) for rows in (t, 1)
                  for s in ((4 * h, h, zi.ZI_EPILOGUE_Y8 | zi.ZI_EPILOGUE_TURNED), (4 * h, h, zi.ZI_EPILOGUE_Y8), (h, 4 * h, 0))]
        sizes += [zi.zi_rms_norm_workspace_bytes(t, h), zi.zi_epilogue_workspace_bytes(t, 4 * h), 16]
        self.ws = torch.empty(max(sizes), dtype=torch.uint8, device=DEV)

    def new_weights(self):
        for (w, turned), p in zip(self.w, (self.p[1], self.p[3])):
            zi.zi_fp8_quantize(p, zi.ZI_FP32, *p.shape, p.shape[1], w.struct, turned.struct)

    def matmul(self, a, b, d):
        zi.zi_fp8_matmul(a.struct, b.struct, d, BF16, b.rows, None, self.ws)

    def forward(self, x):
        zi.zi_rms_norm(zi.make_rms_norm(x, self.lp[0], BF16, 1e-5, y=self.y, rstd=self.rstd), self.y8.struct)
        first = zi.make_epilogue(self.t, 4 * self.h, BF16, bias=self.lp[2], z=self.z, activation=zi.ZI_ACT_GELU)
        zi.zi_fp8_matmul_epilogue(self.y8.struct, self.w[0][0].struct, first, self.u8.struct, self.ut8.struct, self.ws)
        second = zi.make_epilogue(self.t, self.h, BF16, bias=self.lp[4], residual=x, y=self.out, drop=self.drop, seed=SEED, offset=self.step)
        zi.zi_fp8_matmul_epilogue(self.u8.struct, self.w[1][0].struct, second, None, None, self.ws)
        return self.out

    def backward(self, x, dout):
        """Gradients of the parameters into self.g; returns that of x."""
        dropped = zi.make_epilogue_backward(dout, None, None, self.g[4], BF16, drop=self.drop, seed=SEED, offset=self.step)
        zi.zi_epilogue_backward(dropped, self.do8.struct, self.dot8.struct, self.ws)
        self.matmul(self.do8, self.w[1][1], self.du)
        self.matmul(self.dot8, self.ut8, self.g[3])
        activated = zi.make_epilogue_backward(self.du, self.z, None, self.g[2], BF16, activation=zi.ZI_ACT_GELU)
        zi.zi_epilogue_backward(activated, self.dz8.struct, self.dzt8.struct, self.ws)
        self.matmul(self.dz8, self.w[0][1], self.dy)
        zi.zi_fp8_quantize(self.y, BF16, self.t, self.h, self.h, None, self.yt8.struct)
        self.matmul(self.dzt8, self.yt8, self.g[1])
        zi.zi_rms_norm_backward(zi.make_rms_norm_backward(self.dy, x, self.lp[0], self.rstd, self.dx, self.g[0], BF16, dsum=dout), self.ws)
        return self.dx

    def update(self, lr):
        self.step += 1
        zi.zi_grad_norm(self.tensors, BF16, 1.0, self.norm, self.norm_ws)
        zi.zi_adamw_step(self.tensors, BF16, zi.make_config(lr=lr, step=self.step, weight_decay=0.0, max_grad_norm=1.0), self.norm)
        self.new_weights()

    def decode(self, x):
        """One token, without dropout: the norm and two products."""
        y8, u8, out = Matrix8(1, self.h), Matrix8(1, 4 * self.h), torch.empty_like(x)
        zi.zi_rms_norm(zi.make_rms_norm(x, self.lp[0], BF16, 1e-5), y8.struct)
        first = zi.make_epilogue(1, 4 * self.h, BF16, bias=self.lp[2], activation=zi.ZI_ACT_GELU)
        zi.zi_fp8_matmul_epilogue(y8.struct, self.w[0][0].struct, first, u8.struct, None, self.ws)
        second = zi.make_epilogue(1, self.h, BF16, bias=self.lp[4], residual=x, y=out)
        zi.zi_fp8_matmul_epilogue(u8.struct, self.w[1][0].struct, second, None, None, self.ws)
        return out


def train(hidden=512, tokens=2048, steps=60, lr=2e-3, log=None):
    """Losses of all steps, and the trained model."""
    model, losses = Mlp(hidden, tokens), []
    for step in range(steps):
        x, want = data(hidden, tokens, 100 + step)
        diff = model.forward(x) - want
        losses.append(float(diff.float().square().mean()))
        model.backward(x, (diff * (2.0 / diff.shape[0])).contiguous())
        model.update(lr)
        if log and step % 10 == 0:
            log(f"step {step:3d}  loss {losses[-1]:.4f}  gradient norm {float(model.norm[1]):.3f}")
    return losses, model


if __name__ == "__main__":
    losses, model = train(*[int(a) for a in sys.argv[1:4]], log=lambda s: print(s, flush=True))
    x, _ = data(model.h, model.t, 7)
    model.drop = 0.0
    one, whole = model.decode(x[:1].contiguous()).float(), model.forward(x)[:1].float()
    print(f"last loss {losses[-1]:.4f}; one token by itself is {float((one - whole).norm() / whole.norm()):.1e} from the same token in the batch")
