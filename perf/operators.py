"""What the speed of the 8-bit layer operators is judged on: the calls of include/zi_fp8.h as a training or a serving
program makes them.

A matrix in 8 bits holds e4m3 numbers and, for each block of 128 columns in a row (or in 128 rows), one scale that is a
power of two (e8m0).  A case is one call:

  quantize   zi_fp8_quantize: weights after a step (blocks of 128 x 128) or activations and gradients (blocks of 1 x 128),
             as they are, transposed, or both in one pass
  matmul     zi_fp8_matmul: a layer's product (weights in 128 x 128), its input's gradient (the same with the transposed
             weights) or its weights' gradient (both in 1 x 128, added to what earlier micro-batches left)
  norm       zi_rms_norm: the residual's addition, root-mean-square norm, output in 8 bits
  backward   zi_rms_norm_backward: gradients of its input and of gamma

Sizes: the matrices of a Transformer block at a hidden size h of 1024 to 8192 (h x h, 4h x h, h x 4h), one token to 16384,
and odd ones between.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
EPS = 1e-5
BLOCK = 128


def _quantize(name, rows, cols, dtype, blocks, form, pad=0):
    return dict(name=name, op="quantize", rows=rows, cols=cols, dtype=dtype, blocks=blocks, form=form, pad=pad)


def _matmul(name, m, n, k, dtype, b_blocks, add=False):
    return dict(name=name, op="matmul", m=m, n=n, k=k, dtype=dtype, b_blocks=b_blocks, add=add)


def _norm(name, rows, cols, dtype, residual, wide=False, pad=0):
    return dict(name=name, op="norm", rows=rows, cols=cols, dtype=dtype, residual=residual, wide=wide, pad=pad)


def _backward(name, rows, cols, dtype, residual, gamma32, pad=0):
    return dict(name=name, op="backward", rows=rows, cols=cols, dtype=dtype, residual=residual, gamma32=gamma32, pad=pad)


def listed():
    return [
        # one token's activations before a product, a view of a wider buffer: latency
        _quantize("quantize_token_fp16", 1, 1000, "fp16", 1, "rows", pad=24),
        # the larger MLP weight at hidden size 4096 after a step, from the fp32 masters, for the product and its backward pass
        _quantize("quantize_weight_fp32", 16384, 4096, "fp32", 128, "both"),
        # the gradient of a layer's output at 8191 tokens: as it is for the input's gradient, transposed for the weights'
        _quantize("quantize_gradient_bf16", 8191, 8192, "bf16", 1, "both"),
        # one new token through the MLP at hidden size 4096
        _matmul("matmul_token_bf16", 1, 16384, 4096, "bf16", 128),
        # 13 sequences' new tokens through its second matrix
        _matmul("matmul_decode_fp16", 13, 4096, 16384, "fp16", 128),
        # a prompt of odd length at hidden size 2048
        _matmul("matmul_prompt_bf16", 1001, 8192, 2048, "bf16", 128),
        # weights' gradient of the attention's output projection at hidden size 4096 and 8191 tokens, accumulated
        _matmul("matmul_weight_grad_bf16", 4096, 4096, 8191, "bf16", 1, add=True),
        # the largest: 8192 tokens through the MLP's first matrix at hidden size 8192
        _matmul("matmul_mlp_bf16", 8192, 32768, 8192, "bf16", 128),
        # one new token's norm
        _norm("norm_token_bf16", 1, 4096, "bf16", residual=True),
        # a training batch's norm at hidden size 8192, with the 16-bit output that the backward pass keeps
        _norm("norm_batch_bf16", 16384, 8192, "bf16", residual=True, wide=True),
        # the backward pass of a small ragged batch
        _backward("backward_ragged_fp16", 333, 1000, "fp16", residual=False, gamma32=True, pad=5),
        # ... and of a training batch
        _backward("backward_batch_bf16", 16384, 4096, "bf16", residual=True, gamma32=False),
    ]


def _log_size(rng, lo, hi):
    """Spread over the logarithm; every other one a power of two, as a model's own sizes mostly are."""
    if rng.random() < 0.5:
        return 1 << rng.randint(math.ceil(math.log2(lo)), int(math.log2(hi)))
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    op = rng.choice(["quantize", "quantize", "matmul", "matmul", "matmul", "norm", "norm", "backward"])
    if op == "matmul":
        k, n = _log_size(rng, 128, 16384), _log_size(rng, 128, 32768)
        m = _log_size(rng, 1, 16384)
        m = min(m, (1 << 41) // (n * k), (1 << 28) // n)
        c = _matmul("", m, n, k, rng.choice(["bf16", "fp16"]), rng.choice([1, 128, 128]), rng.random() < 0.3)
    elif op == "quantize":
        rows = _log_size(rng, 1, 16384)
        cols = min(_log_size(rng, 64, 32768), (1 << 26) // rows)
        c = _quantize("", rows, cols, rng.choice(["bf16", "fp16", "fp32"]), rng.choice([1, 128]),
                      rng.choice(["rows", "turned", "both"]), rng.choice([0, 0, 8, 5]))
    else:
        rows = _log_size(rng, 1, 16384)
        cols = min(_log_size(rng, 64, 65536), (1 << 27) // rows)
        dtype, residual, pad = rng.choice(["bf16", "fp16"]), rng.random() < 0.6, rng.choice([0, 0, 8, 5])
        if op == "norm":
            c = _norm("", rows, cols, dtype, residual, rng.random() < 0.4, pad)
        else:
            c = _backward("", rows, cols, dtype, residual, rng.random() < 0.5, pad)
    del c["name"]
    return c


# ---- inputs ---------------------------------------------------------------------------------------------------

def _up(n, to):
    return -(-n // to) * to


class _State:
    pass


def _normal(gen, rows, cols, std):
    return torch.empty((rows, cols), dtype=torch.float32, device="cuda").normal_(0.0, std, generator=gen)


def _wide(x, pad, dtype):
    """x in its type, as a view of a buffer whose rows are `pad` elements longer."""
    if not pad:
        return x.to(dtype)
    buffer = torch.zeros((x.shape[0], x.shape[1] + pad), dtype=dtype, device=x.device)
    buffer[:, :x.shape[1]] = x
    return buffer[:, :x.shape[1]]


def _activations(gen, rows, cols, std=1.0):
    """Normal, with one channel in 64 twenty times larger, as activations have them."""
    x = _normal(gen, rows, cols, std)
    x[:, 7::64] *= 20.0
    return x


def _space(rows, cols, blocks):
    """Room for a matrix in 8 bits: rows of whole blocks, scales by rows of whole words."""
    data = torch.zeros((rows, _up(cols, BLOCK)), dtype=torch.uint8, device="cuda")
    scale = torch.zeros((-(-rows // blocks), _up(-(-cols // BLOCK), 4)), dtype=torch.uint8, device="cuda")
    return data.view(torch.float8_e4m3fn), scale.view(torch.float8_e8m0fnu)


def _filled(x, blocks):
    data, scale = _space(x.shape[0], x.shape[1], blocks)
    q, s = _plain_quantize(x, blocks)
    data.view(torch.uint8)[:, :x.shape[1]] = q.view(torch.uint8)
    scale.view(torch.uint8)[:, :s.shape[1]] = s.view(torch.uint8)
    return data, scale


def _shown(space, cols):
    """What a caller looks at of a matrix in 8 bits: its columns and their scales."""
    return space[0][:, :cols], space[1][:, :-(-cols // BLOCK)]


def prepare(case, seed):
    s = _State()
    s.case, s.op, s.dtype = case, case["op"], DTYPES[case["dtype"]]
    gen = torch.Generator(device="cuda").manual_seed(seed)
    if s.op == "matmul":
        m, n, k = case["m"], case["n"], case["k"]
        s.a = _filled(_activations(gen, m, k), 1)
        s.b = _filled(_normal(gen, n, k, 0.02), case["b_blocks"])
        s.c = _normal(gen, m, n, math.sqrt(k) * 0.02).to(s.dtype) if case["add"] else None
        s.d = torch.empty((m, n), dtype=s.dtype, device="cuda")
    else:
        rows, cols, pad = case["rows"], case["cols"], case["pad"]
        if s.op == "quantize":
            s.x = _wide(_normal(gen, rows, cols, 0.02) if case["blocks"] == 128 else _activations(gen, rows, cols), pad, s.dtype)
            s.rows = _space(rows, cols, case["blocks"]) if case["form"] != "turned" else None
            s.turned = _space(cols, rows, case["blocks"]) if case["form"] != "rows" else None
        else:
            s.x = _wide(_activations(gen, rows, cols), pad, s.dtype)
            s.gamma = (1.0 + _normal(gen, 1, cols, 0.1)[0]).to(s.dtype)
            if s.op == "norm":
                s.residual = _wide(_activations(gen, rows, cols), pad, s.dtype) if case["residual"] else None
                s.sum = torch.empty((rows, cols), dtype=s.dtype, device="cuda") if case["residual"] else None
                s.y = torch.empty((rows, cols), dtype=s.dtype, device="cuda") if case["wide"] else None
                s.rstd = torch.empty(rows, dtype=torch.float32, device="cuda")
                s.y8 = _space(rows, cols, 1)
            else:
                s.rstd = 1.0 / (s.x.float().square().mean(1) + EPS).sqrt()
                s.dy = _wide(_normal(gen, rows, cols, 1e-3), pad, s.dtype)
                s.dsum = _wide(_normal(gen, rows, cols, 1e-3), pad, s.dtype) if case["residual"] else None
                s.dx = torch.empty((rows, cols), dtype=s.dtype, device="cuda")
                s.dgamma = torch.empty(cols, dtype=torch.float32 if case["gamma32"] else s.dtype, device="cuda")
    if own:
        _plan(s)
    return s


def _plan(s):
    """The descriptors and workspaces that a program keeps between calls."""
    import paper_2104_07857_amd as zi
    c = s.case
    s.zi, s.dt = zi, {"bf16": zi.ZI_BF16, "fp16": zi.ZI_FP16, "fp32": zi.ZI_FP32}[c["dtype"]]
    if s.op == "matmul":
        s.a8 = zi.make_fp8_matrix(*s.a, c["m"], c["k"], block_rows=1)
        s.b8 = zi.make_fp8_matrix(*s.b, c["n"], c["k"], block_rows=c["b_blocks"])
        nbytes = zi.zi_fp8_matmul_workspace_bytes(c["m"], c["n"], c["k"])
    elif s.op == "quantize":
        s.rows8 = zi.make_fp8_matrix(*s.rows, c["rows"], c["cols"], block_rows=c["blocks"]) if s.rows else None
        s.turned8 = zi.make_fp8_matrix(*s.turned, c["cols"], c["rows"], block_rows=c["blocks"]) if s.turned else None
        nbytes = 0
    elif s.op == "norm":
        s.call = zi.make_rms_norm(s.x, s.gamma, s.dt, EPS, residual=s.residual, sum=s.sum, y=s.y, rstd=s.rstd)
        s.out8 = zi.make_fp8_matrix(*s.y8, c["rows"], c["cols"], block_rows=1)
        nbytes = 0
    else:
        s.call = zi.make_rms_norm_backward(s.dy, s.x, s.gamma, s.rstd, s.dx, s.dgamma, s.dt, dsum=s.dsum,
                                           dgamma_dtype=zi.ZI_FP32 if c["gamma32"] else s.dt)
        nbytes = zi.zi_rms_norm_workspace_bytes(c["rows"], c["cols"])
    s.ws = torch.empty(max(nbytes, 16), dtype=torch.uint8, device="cuda")
    s.stream = torch.cuda.current_stream()


# ---- the plain form -------------------------------------------------------------------------------------------

def _plain_quantize(x, blocks):
    """e4m3 numbers and e8m0 scales of x: the smallest power of two that brings a block's largest finite magnitude to 448
    or less (1 for a block of zeros).  Infinities and NaN become NaN and do not count."""
    rows, cols = x.shape
    x = x.float()
    padded = torch.zeros((_up(rows, blocks), _up(cols, BLOCK)), dtype=torch.float32, device=x.device)
    padded[:rows, :cols] = x
    tiles = padded.view(padded.shape[0] // blocks, blocks, -1, BLOCK)
    most = torch.where(torch.isfinite(tiles), tiles.abs(), torch.zeros_like(tiles)).amax((1, 3))
    fraction, exponent = torch.frexp(most)                   # 448 is 0.875 * 2^9
    exponent = (exponent - 9 + (fraction > 0.875)).clamp(-127, 127) * (most > 0)
    q = (tiles * torch.exp2(-exponent.float())[:, None, :, None]).reshape(padded.shape)[:rows, :cols]
    return q.to(torch.float8_e4m3fn), (exponent + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _spread(scale, blocks, rows, cols):
    return scale.repeat_interleave(blocks, 0)[:rows].repeat_interleave(BLOCK, 1)[:, :cols]


def _values(space, rows, cols, blocks, dtype):
    q, scale = _shown(space, cols)
    return q.to(dtype) * _spread(scale.to(dtype), blocks, rows, cols)


def _plain(s):
    c = s.case
    if s.op == "quantize":
        out = {}
        if s.rows:
            out["rows"] = _plain_quantize(s.x, c["blocks"])
        if s.turned:
            out["turned"] = _plain_quantize(s.x.t(), c["blocks"])
        return out
    if s.op == "matmul":
        d = _values(s.a, c["m"], c["k"], 1, torch.float32) @ _values(s.b, c["n"], c["k"], c["b_blocks"], torch.float32).t()
        return {"d": (d if s.c is None else d + s.c.float()).to(s.dtype)}
    if s.op == "norm":
        h, out = s.x, {}
        if s.residual is not None:
            h = out["sum"] = (s.x.float() + s.residual.float()).to(s.dtype)
        h = h.float()
        out["rstd"] = 1.0 / (h.square().mean(1) + EPS).sqrt()
        y = h * out["rstd"][:, None] * s.gamma.float()
        if s.y is not None:
            out["y"] = y.to(s.dtype)
        return {**out, "y8": _plain_quantize(y, 1)}
    dy, h = s.dy.float(), s.x.float() * s.rstd[:, None]
    u = dy * s.gamma.float()
    dx = s.rstd[:, None] * (u - h * (u * h).mean(1, keepdim=True))
    dx = dx if s.dsum is None else dx + s.dsum.float()
    return {"dx": dx.to(s.dtype), "dgamma": (dy * h).sum(0).to(s.dgamma.dtype)}


def run(s):
    if not own:
        return _plain(s)
    c, zi = s.case, s.zi
    if s.op == "quantize":
        zi.zi_fp8_quantize(s.x, s.dt, c["rows"], c["cols"], c["cols"] + c["pad"], s.rows8, s.turned8, s.stream)
        out = {}
        if s.rows:
            out["rows"] = _shown(s.rows, c["cols"])
        if s.turned:
            out["turned"] = _shown(s.turned, c["rows"])
        return out
    if s.op == "matmul":
        zi.zi_fp8_matmul(s.a8, s.b8, s.d, s.dt, c["n"], s.c, s.ws, stream=s.stream)
        return {"d": s.d}
    if s.op == "norm":
        zi.zi_rms_norm(s.call, s.out8, s.stream)
        out = {"rstd": s.rstd, "y8": _shown(s.y8, c["cols"])}
        if s.sum is not None:
            out["sum"] = s.sum
        if s.y is not None:
            out["y"] = s.y
        return out
    zi.zi_rms_norm_backward(s.call, s.ws, stream=s.stream)
    return {"dx": s.dx, "dgamma": s.dgamma}


# ---- what a call cannot do without ----------------------------------------------------------------------------

def _bytes8(rows, cols, blocks):
    return rows * cols + -(-rows // blocks) * -(-cols // BLOCK)


def work(case):
    c = case
    size = {"bf16": 2, "fp16": 2, "fp32": 4}[c["dtype"]]
    if c["op"] == "matmul":
        m, n, k = c["m"], c["n"], c["k"]
        return {"bytes": _bytes8(m, k, 1) + _bytes8(n, k, c["b_blocks"]) + m * n * size * (2 if c["add"] else 1),
                "flops": 2 * m * n * k}
    rows, cols = c["rows"], c["cols"]
    cells = rows * cols
    if c["op"] == "quantize":
        nbytes = cells * size
        nbytes += _bytes8(rows, cols, c["blocks"]) if c["form"] != "turned" else 0
        nbytes += _bytes8(cols, rows, c["blocks"]) if c["form"] != "rows" else 0
        return {"bytes": nbytes, "flops": 3 * cells}
    if c["op"] == "norm":
        passes = 1 + 2 * c["residual"] + c["wide"]
        return {"bytes": cells * size * passes + cols * size + 4 * rows + _bytes8(rows, cols, 1), "flops": 8 * cells}
    return {"bytes": cells * size * (3 + c["residual"]) + cols * (size + (4 if c["gamma32"] else size)) + 4 * rows, "flops": 11 * cells}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------

def _exact_quantize(x, blocks):
    """Codes and scales of x (64 bits), as the values they stand for, from the definition: log2 and rounding to a grid."""
    rows, cols = x.shape
    most = torch.nn.functional.pad(x.abs(), (0, -cols % BLOCK, 0, -rows % blocks))
    most = most.view(most.shape[0] // blocks, blocks, most.shape[1] // BLOCK, BLOCK).amax((1, 3))
    power = torch.ceil(torch.log2(most / 448.0).clamp(-127, 127))
    power = torch.where(most > 448.0 * torch.exp2(power), power + 1, power)          # where log2 rounded over a whole number
    power = torch.where((most <= 448.0 * torch.exp2(power - 1)) & (power > -127), power - 1, power)
    scale = torch.where(most > 0, torch.exp2(power), torch.ones_like(power))
    v = x / _spread(scale, blocks, rows, cols)
    grid = torch.exp2(torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6))) - 3)     # 3 bits of fraction; 2^-9 below 2^-6
    return torch.round(v / grid) * grid, scale


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if s.op == "quantize":
        x, out = s.x.double(), {}
        if s.rows:
            out["rows"] = _exact_quantize(x, c["blocks"])
        if s.turned:
            out["turned"] = _exact_quantize(x.t(), c["blocks"])
        return out
    if s.op == "matmul":
        a = s.a[0].double() * s.a[1].double().repeat_interleave(BLOCK, 1)[:, :s.a[0].shape[1]]
        b = s.b[0].double() * s.b[1].double().repeat_interleave(BLOCK, 1)[:, :s.b[0].shape[1]].repeat_interleave(c["b_blocks"], 0)[:c["n"]]
        d = torch.matmul(a, b.t().contiguous())
        return {"d": d if s.c is None else d + s.c.double()}
    if s.op == "norm":
        total, out = s.x.double(), {}
        if s.residual is not None:
            total = out["sum"] = total + s.residual.double()
        h = total.float().to(s.dtype).double()               # the norm is of what the residual stream holds
        out["rstd"] = (h.pow(2).sum(1) / c["cols"] + EPS).pow(-0.5)
        y = h * s.gamma.double() * out["rstd"].unsqueeze(1)
        if s.y is not None:
            out["y"] = y
        return {**out, "y8": _exact_quantize(y, 1)}
    r, dy, h, g = s.rstd.double().unsqueeze(1), s.dy.double(), s.x.double(), s.gamma.double()
    dot = (dy * g * h).sum(1, keepdim=True)
    dx = r * g * dy - h * r.pow(3) * dot / c["cols"]
    return {"dx": dx if s.dsum is None else dx + s.dsum.double(), "dgamma": (dy * h * r).sum(0)}
