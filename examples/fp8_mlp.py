"""A Transformer's MLP with its norm, trained and decoded with 8-bit products around the optimizer step.

    out = x + W2 relu(W1 norm(x))

Weights are fp32 masters that zi_adamw_step updates; after each step zi_fp8_quantize makes their 8-bit forms, as they are for the products and
transposed for the gradients of the inputs.  Activations and gradients are quantised where a product reads them: along their rows for
the product and its input's gradient, along their columns (transposed) for the weights' gradient.  Gradients come out of the
products in bf16, which is what zi_grad_norm and zi_adamw_step take.

    python examples/fp8_mlp.py [hidden size [tokens [steps]]]
"""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

import paper_2104_07857_amd as zi

BF16, DEV = zi.ZI_BF16, "cuda:0"


class Matrix8:
    """A matrix in 8 bits and the bytes that hold it."""

    def __init__(self, rows, cols, block_rows=1):
        data, scale = zi.fp8_layout(rows, cols, block_rows)
        self.data = torch.empty(data, dtype=torch.uint8, device=DEV)
        self.scale = torch.empty(scale, dtype=torch.uint8, device=DEV)
        self.rows, self.cols = rows, cols
        self.struct = zi.make_fp8_matrix(self.data, self.scale, rows, cols, block_rows)


class Mlp:
    """Parameters in three tensors of one flat partition each (p, m, v in fp32, gradients and copy in bf16)."""

    def __init__(self, hidden, tokens, seed=0):
        self.h, self.t = hidden, tokens
        shapes = [(hidden,), (4 * hidden, hidden), (hidden, 4 * hidden)]       # gamma, W1, W2
        gen = torch.Generator(device=DEV).manual_seed(seed)
        self.p = [torch.ones(hidden, device=DEV)] + [torch.randn(s, generator=gen, device=DEV) * s[1] ** -0.5 for s in shapes[1:]]
        self.m, self.v = ([torch.zeros_like(x) for x in self.p] for _ in range(2))
        self.g, self.lp = ([torch.zeros(s, dtype=torch.bfloat16, device=DEV) for s in shapes] for _ in range(2))
        self.lp[0].copy_(self.p[0])
        self.tensors = zi.make_tensors(zip(self.p, self.m, self.v, self.g, self.lp))
        self.norm = torch.zeros(4, dtype=torch.float64, device=DEV)
        self.norm_ws = torch.empty(zi.zi_norm_workspace_bytes(), dtype=torch.uint8, device=DEV)
        self.w = [(Matrix8(r, c, 128), Matrix8(c, r, 128)) for r, c in shapes[1:]]     # as they are, transposed
        self.step = 0
        self.new_weights()
        # what a step leaves for its backward pass
        h, t = hidden, tokens
        new = lambda *s: torch.empty(s, dtype=torch.bfloat16, device=DEV)              # noqa: E731
        self.y, self.z, self.out, self.du, self.dy, self.dx = new(t, h), new(t, 4 * h), new(t, h), new(t, 4 * h), new(t, h), new(t, h)
        self.rstd = torch.empty(t, device=DEV)
        self.y8, self.yt8, self.u8, self.ut8 = Matrix8(t, h), Matrix8(h, t), Matrix8(t, 4 * h), Matrix8(4 * h, t)
        self.do8, self.dot8, self.dz8, self.dzt8 = Matrix8(t, h), Matrix8(h, t), Matrix8(t, 4 * h), Matrix8(4 * h, t)
        most = max(zi.zi_fp8_matmul_workspace_bytes(*s) for s in (
            (t, 4 * h, h), (t, h, 4 * h), (4 * h, h, t), (h, 4 * h, t), (1, 4 * h, h), (1, h, 4 * h)))
        self.ws = torch.empty(max(most, zi.zi_rms_norm_workspace_bytes(t, h), 16), dtype=torch.uint8, device=DEV)

    def new_weights(self):
        for (w, turned), p in zip(self.w, self.p[1:]):
            zi.zi_fp8_quantize(p, zi.ZI_FP32, *p.shape, p.shape[1], w.struct, turned.struct)

    def matmul(self, a, b, d):
        zi.zi_fp8_matmul(a.struct, b.struct, d, BF16, b.rows, None, self.ws)

    def quantize(self, x, out, turned=None):
        zi.zi_fp8_quantize(x, BF16, *x.shape, x.shape[1], out.struct if out else None, turned.struct if turned else None)

    def forward(self, x):
        zi.zi_rms_norm(zi.make_rms_norm(x, self.lp[0], BF16, 1e-5, y=self.y, rstd=self.rstd), self.y8.struct)
        self.matmul(self.y8, self.w[0][0], self.z)
        self.quantize(self.z.relu(), self.u8, self.ut8)
        self.matmul(self.u8, self.w[1][0], self.out)
        return self.out + x

    def backward(self, x, dout):
        """Gradients of the parameters into self.g; returns that of x."""
        self.quantize(dout, self.do8, self.dot8)
        self.matmul(self.do8, self.w[1][1], self.du)                  # dout W2
        self.matmul(self.dot8, self.ut8, self.g[2])                   # dout^T u
        self.quantize(self.du * (self.z > 0), self.dz8, self.dzt8)
        self.matmul(self.dz8, self.w[0][1], self.dy)                  # dz W1
        self.quantize(self.y, None, self.yt8)
        self.matmul(self.dzt8, self.yt8, self.g[1])                   # dz^T y
        zi.zi_rms_norm_backward(zi.make_rms_norm_backward(self.dy, x, self.lp[0], self.rstd, self.dx, self.g[0], BF16, dsum=dout), self.ws)
        return self.dx

    def update(self, lr):
        self.step += 1
        zi.zi_grad_norm(self.tensors, BF16, 1.0, self.norm, self.norm_ws)
        zi.zi_adamw_step(self.tensors, BF16, zi.make_config(lr=lr, step=self.step, weight_decay=0.0, max_grad_norm=1.0), self.norm)
        self.new_weights()

    def decode(self, x, residual):
        """One token: the residual's addition, norm, both products; (out, what the residual stream holds now)."""
        total, z, out = torch.empty_like(x), torch.empty((1, 4 * self.h), dtype=x.dtype, device=DEV), torch.empty_like(x)
        y8, u8 = Matrix8(1, self.h), Matrix8(1, 4 * self.h)
        zi.zi_rms_norm(zi.make_rms_norm(x, self.lp[0], BF16, 1e-5, residual=residual, sum=total), y8.struct)
        self.matmul(y8, self.w[0][0], z)
        self.quantize(z.relu(), u8)
        self.matmul(u8, self.w[1][0], out)
        return out, total


def data(hidden, tokens, seed):
    """Inputs, and what a fixed random MLP makes of them."""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn((tokens, hidden), generator=gen, device=DEV)
    a, b = (torch.randn((hidden, hidden), generator=torch.Generator(device=DEV).manual_seed(s), device=DEV) * hidden ** -0.5 for s in (1, 2))
    return x.bfloat16(), (x + (x @ a).tanh() @ b).bfloat16()


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
    out, total = model.decode(x[:1] / 2, x[:1] / 2)
    whole = model.forward(x)[:1].float()
    print(f"last loss {losses[-1]:.4f}; one token by itself is {float((out + total - whole).norm() / whole.norm()):.1e} from the same token in the batch")
