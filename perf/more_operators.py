"""What the speed of the operators around the 8-bit products is judged on: the calls of include/zi_epilogue.h as a training or a
serving program makes them.

What follows a layer's product, element by element of its result (rows are tokens), is

  z = product + bias      y = residual + dropout(activation(z))

and a case is one call:

  matmul    zi_fp8_matmul_epilogue: the product of two matrices in 8 bits with all of that in its epilogue
  forward   zi_epilogue: the same of a 16-bit matrix that is there already (dropout by itself, an activation made again from z)
  backward  zi_epilogue_backward: the gradient of z from that of y, and the bias' gradient

Outputs are in 16 bits, or in 8 for the next product: e4m3 numbers with a power-of-two scale for each 128 columns of a row, as they are
and transposed (each 128 rows of a column).  Dropout's numbers come from the counter-based generator Philox4x32-10 (Salmon et al.,
"Parallel random numbers: as easy as 1, 2, 3", 2011): key = seed, counter = (column / 8, row, offset), eight numbers of 16 bits for eight
columns; an element is dropped where its number is below 65536 p, and the others are divided by 1 - p.

Sizes: the matrices of a Transformer's MLP and of its attention's output at a hidden size h of 1024 to 8192, one token to 16384, and odd ones
between.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
BLOCK = 128
ACTIVATIONS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


def _matmul(name, m, n, k, dtype, act, outputs, residual=False, drop=0.0):
    return dict(name=name, op="matmul", m=m, n=n, k=k, dtype=dtype, act=act, outputs=outputs, bias=True, residual=residual, drop=drop)


def _forward(name, rows, cols, dtype, act, outputs, bias=False, residual=False, drop=0.0, pad=0):
    return dict(name=name, op="forward", rows=rows, cols=cols, dtype=dtype, act=act, outputs=outputs, bias=bias, residual=residual,
                drop=drop, pad=pad)


def _backward(name, rows, cols, dtype, act, outputs, drop=0.0, dbias32=True, pad=0):
    return dict(name=name, op="backward", rows=rows, cols=cols, dtype=dtype, act=act, outputs=outputs, drop=drop, dbias32=dbias32, pad=pad)


def listed():
    return [
        # one new token through the MLP's first matrix at hidden size 4096, its activation in 8 bits for the second
        _matmul("matmul_token_fp16", 1, 16384, 4096, "fp16", "gelu", "y8"),
        # 13 sequences' new tokens through the second matrix, onto the residual stream
        _matmul("matmul_decode_bf16", 13, 4096, 16384, "bf16", "none", "y", residual=True),
        # a prompt of odd length through the first matrix at hidden size 2048
        _matmul("matmul_prompt_bf16", 1001, 8192, 2048, "bf16", "silu", "y8"),
        # a training batch through the second matrix at hidden size 4096: dropout and residual
        _matmul("matmul_down_fp16", 8191, 4096, 16384, "fp16", "none", "y", residual=True, drop=0.1),
        # the largest: a training batch through the first matrix at hidden size 8192, with all that the backward pass reads
        _matmul("matmul_up_bf16", 8192, 32768, 8192, "bf16", "gelu_tanh", "z,y8,turned"),
        # one token's activation by itself
        _forward("forward_token_bf16", 1, 16384, "bf16", "gelu", "y8", bias=True),
        # dropout of a small ragged batch, views of a wider buffer
        _forward("forward_ragged_fp16", 333, 1000, "fp16", "none", "y", residual=True, drop=0.25, pad=5),
        # dropout of the attention's output at hidden size 4096 and its addition to the residual stream
        _forward("forward_dropout_bf16", 16384, 4096, "bf16", "none", "y", residual=True, drop=0.1),
        # the activation made again from z in the backward pass, for the weights' gradient (and the product, when checkpointed)
        _forward("forward_batch_bf16", 8192, 16384, "bf16", "silu", "y8,turned"),
        # the backward pass of a small ragged batch
        _backward("backward_ragged_fp16", 333, 1000, "fp16", "relu", "dz", dbias32=False, pad=5),
        # the activation's in a training batch of odd length, for both products behind it
        _backward("backward_batch_bf16", 8191, 16384, "bf16", "gelu_tanh", "dz8,turned"),
        # dropout's in front of a product at hidden size 4096
        _backward("backward_dropout_bf16", 16384, 4096, "bf16", "none", "dz8,turned", drop=0.1),
    ]


def _log_size(rng, lo, hi):
    """Spread over the logarithm; every other one a power of two, as a model's own sizes mostly are."""
    if rng.random() < 0.5:
        return 1 << rng.randint(math.ceil(math.log2(lo)), int(math.log2(hi)))
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    op, act = rng.choice(["matmul", "matmul", "forward", "backward"]), rng.choice(ACTIVATIONS)
    dtype, drop = rng.choice(["bf16", "fp16"]), rng.choice([0.0, 0.0, 0.1, round(rng.uniform(0.01, 0.6), 3)])
    if op == "matmul":
        k, n = _log_size(rng, 128, 16384), _log_size(rng, 128, 32768)
        m = _log_size(rng, 1, 16384)
        m = min(m, (1 << 41) // (n * k), (1 << 28) // n)
        residual = rng.random() < 0.4
        c = _matmul("", m, n, k, dtype, act, rng.choice(["y", "y", "y8", "z,y8,turned"] if m > 16 else ["y", "y8"]), residual, drop)
    else:
        rows = _log_size(rng, 1, 16384)
        cols = min(_log_size(rng, 64, 32768), (1 << 27) // rows)
        pad = rng.choice([0, 0, 8, 5])
        if op == "forward":
            residual = rng.random() < 0.5
            c = _forward("", rows, cols, dtype, act, rng.choice(["y", "y8", "y,y8", "y8,turned"]), rng.random() < 0.5, residual, drop, pad)
        else:
            c = _backward("", rows, cols, dtype, act, rng.choice(["dz", "dz8,turned", "dz,dz8,turned"]), drop, rng.random() < 0.5, pad)
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


def _outliers(x):
    """One channel in 64 twenty times larger, as activations have them."""
    x[:, 7::64] *= 20.0
    return x


def _space(rows, cols, blocks=1):
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


def _shape(case):
    return (case["m"], case["n"]) if case["op"] == "matmul" else (case["rows"], case["cols"])


def prepare(case, seed):
    s = _State()
    s.case, s.op, s.dtype = case, case["op"], DTYPES[case["dtype"]]
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rows, cols = _shape(case)
    wanted = case["outputs"].split(",")
    empty = lambda name: torch.empty((rows, cols), dtype=s.dtype, device="cuda") if name in wanted else None          # noqa: E731
    s.seed, s.offset = (seed * 0x9E3779B97F4A7C15 + 0x1234567) % (1 << 64), (seed % 1000) << 30
    s.turned = _space(cols, rows) if "turned" in wanted else None
    if s.op == "backward":
        pad = case["pad"]
        s.dy = _wide(_normal(gen, rows, cols, 1e-3), pad, s.dtype)
        s.z = _wide(_normal(gen, rows, cols, 1.5), pad, s.dtype) if case["act"] != "none" else None
        s.dz, s.dz8 = empty("dz"), _space(rows, cols) if "dz8" in wanted else None
        s.dbias = torch.empty(cols, dtype=torch.float32 if case["dbias32"] else s.dtype, device="cuda")
    else:
        pad = case.get("pad", 0)
        if s.op == "matmul":
            # numbers of an activation and of weights whose product is of the size that activations have
            s.a = _filled(_outliers(_normal(gen, rows, case["k"], 1.0)), 1)
            s.b = _filled(_normal(gen, cols, case["k"], 0.4 / math.sqrt(case["k"])), BLOCK)
        else:
            s.x = _wide(_normal(gen, rows, cols, 1.5), pad, s.dtype)
        s.bias = _normal(gen, 1, cols, 0.2)[0].to(s.dtype) if case["bias"] else None
        s.residual = _wide(_outliers(_normal(gen, rows, cols, 1.0)), pad, s.dtype) if case["residual"] else None
        s.z, s.y, s.y8 = empty("z"), empty("y"), _space(rows, cols) if "y8" in wanted else None
    if own:
        _plan(s)
    return s


def _plan(s):
    """The descriptors and workspaces that a program keeps between calls."""
    import paper_2104_07857_amd as zi
    c = s.case
    rows, cols = _shape(c)
    s.zi, dt = zi, {"bf16": zi.ZI_BF16, "fp16": zi.ZI_FP16}[c["dtype"]]
    act = {"none": zi.ZI_ACT_NONE, "relu": zi.ZI_ACT_RELU, "gelu": zi.ZI_ACT_GELU, "gelu_tanh": zi.ZI_ACT_GELU_TANH, "silu": zi.ZI_ACT_SILU}[c["act"]]
    more = dict(activation=act, drop=c["drop"], seed=s.seed, offset=s.offset)
    matrix = lambda space, r, k, blocks=1: zi.make_fp8_matrix(*space, r, k, block_rows=blocks) if space else None       # noqa: E731
    s.turned8 = matrix(s.turned, cols, rows)
    nbytes = 0
    if s.op == "backward":
        s.args = zi.make_epilogue_backward(s.dy, s.z, s.dz, s.dbias, dt, dbias_dtype=zi.ZI_FP32 if c["dbias32"] else dt, **more)
        s.out8 = matrix(s.dz8, rows, cols)
        nbytes = zi.zi_epilogue_workspace_bytes(rows, cols)
    else:
        s.args = zi.make_epilogue(rows, cols, dt, bias=s.bias, residual=s.residual, z=s.z, y=s.y, **more)
        s.out8 = matrix(s.y8, rows, cols)
        if s.op == "matmul":
            s.a8, s.b8 = matrix(s.a, rows, c["k"]), matrix(s.b, cols, c["k"], BLOCK)
            outputs = (zi.ZI_EPILOGUE_Y8 if s.y8 else 0) | (zi.ZI_EPILOGUE_TURNED if s.turned else 0)
            nbytes = zi.zi_fp8_matmul_epilogue_workspace_bytes(rows, cols, c["k"], outputs)
    s.ws = torch.empty(max(nbytes, 16), dtype=torch.uint8, device="cuda")
    s.stream = torch.cuda.current_stream()


# ---- the plain form -------------------------------------------------------------------------------------------

def _plain_quantize(x, blocks=1):
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


def _threshold(p):
    return int(math.floor(p * 65536 + 0.5))


def _kept(rows, cols, p, seed, offset):
    """Where dropout keeps an element: the generator's 10 rounds on words of 32 bits, which 64-bit integers hold with their products (of
    those, which wrap around, only 64 bits are looked at)."""
    low = 0xFFFFFFFF
    octets = -(-cols // 8)
    x0 = torch.arange(octets, device="cuda").expand(rows, octets)
    x1 = torch.arange(rows, device="cuda")[:, None].expand(rows, octets)
    x2, x3 = torch.full_like(x0, offset & low), torch.full_like(x0, offset >> 32)
    k0, k1 = seed & low, seed >> 32
    for _ in range(10):
        a, b = x0 * 0xD2511F53, x2 * 0xCD9E8D57
        x0, x1, x2, x3 = (b >> 32 & low) ^ x1 ^ k0, b & low, (a >> 32 & low) ^ x3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    words = torch.stack([x0, x1, x2, x3], 2)
    halves = torch.stack([words & 0xFFFF, words >> 16], 3)
    return halves.reshape(rows, octets * 8)[:, :cols] >= _threshold(p)


def _activation(z, act):
    if act == "none":
        return z
    if act == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    return z / (1.0 + torch.exp(-z))


def _derivative(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if act == "gelu_tanh":
        t = torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * math.sqrt(2.0 / math.pi) * (1.0 + 3 * 0.044715 * z * z)
    sigmoid = 1.0 / (1.0 + torch.exp(-z))
    return sigmoid * (1.0 + z * (1.0 - sigmoid))


def _dropped(x, s):
    p = s.case["drop"]
    if _threshold(p) == 0:
        return x
    x = x * (65536.0 / (65536 - _threshold(p)))
    return torch.where(_kept(x.shape[0], x.shape[1], p, s.seed, s.offset), x, torch.zeros_like(x))


def _plain(s):
    c, out = s.case, {}
    rows, cols = _shape(c)
    if s.op == "backward":
        dz = _dropped(s.dy.float(), s)
        if c["act"] != "none":
            dz = dz * _derivative(s.z.float(), c["act"])
        if s.dz is not None:
            out["dz"] = dz.to(s.dtype)
        if s.dz8:
            out["dz8"] = _plain_quantize(dz)
        if s.turned:
            out["turned"] = _plain_quantize(dz.t())
        return {**out, "dbias": dz.sum(0).to(s.dbias.dtype)}
    if s.op == "matmul":
        z = _values(s.a, rows, c["k"], 1, torch.float32) @ _values(s.b, cols, c["k"], BLOCK, torch.float32).t()
    else:
        z = s.x.float()
    if s.bias is not None:
        z = z + s.bias.float()
    if s.z is not None:
        out["z"] = z.to(s.dtype)
    y = _dropped(_activation(z, c["act"]), s)
    if s.residual is not None:
        y = y + s.residual.float()
    if s.y is not None:
        out["y"] = y.to(s.dtype)
    if s.y8:
        out["y8"] = _plain_quantize(y)
    if s.turned:
        out["turned"] = _plain_quantize(y.t())
    return out


def run(s):
    if not own:
        return _plain(s)
    c, zi = s.case, s.zi
    rows, cols = _shape(c)
    out = {}
    if s.op == "backward":
        zi.zi_epilogue_backward(s.args, s.out8, s.turned8, s.ws, stream=s.stream)
        if s.dz is not None:
            out["dz"] = s.dz
        if s.dz8:
            out["dz8"] = _shown(s.dz8, cols)
        if s.turned:
            out["turned"] = _shown(s.turned, rows)
        return {**out, "dbias": s.dbias}
    if s.op == "matmul":
        zi.zi_fp8_matmul_epilogue(s.a8, s.b8, s.args, s.out8, s.turned8, s.ws, stream=s.stream)
    else:
        zi.zi_epilogue(s.x, rows, cols, cols + c["pad"], s.args, s.out8, s.turned8, s.stream)
    if s.z is not None:
        out["z"] = s.z
    if s.y is not None:
        out["y"] = s.y
    if s.y8:
        out["y8"] = _shown(s.y8, cols)
    if s.turned:
        out["turned"] = _shown(s.turned, rows)
    return out


# ---- what a call cannot do without ----------------------------------------------------------------------------

def _bytes8(rows, cols, blocks=1):
    return rows * cols + -(-rows // blocks) * -(-cols // BLOCK)


def work(case):
    c = case
    rows, cols = _shape(c)
    cells, wanted = rows * cols, c["outputs"].split(",")
    each = {"z": 2 * cells, "y": 2 * cells, "dz": 2 * cells, "y8": _bytes8(rows, cols), "dz8": _bytes8(rows, cols), "turned": _bytes8(cols, rows)}
    nbytes, flops = sum(each[w] for w in wanted), 0
    if c["op"] == "backward":
        nbytes += 2 * cells * (1 if c["act"] == "none" else 2) + cols * (4 if c["dbias32"] else 2)
        return {"bytes": nbytes, "flops": 4 * cells}
    nbytes += (2 * cols if c["bias"] else 0) + (2 * cells if c["residual"] else 0)
    if c["op"] == "matmul":
        nbytes += _bytes8(rows, c["k"]) + _bytes8(cols, c["k"], BLOCK)
        flops = 2 * cells * c["k"]
    else:
        nbytes += 2 * cells
    return {"bytes": nbytes, "flops": flops + 4 * cells}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------

def _exact_quantize(x, blocks=1):
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


def _exact_times(x, constant):
    """High and low 32 bits of the products of x (below 2^32) and a constant, by halves of 16 bits that nothing wraps around in."""
    x_high, x_low = torch.div(x, 65536, rounding_mode="floor"), x % 65536
    c_high, c_low = divmod(constant, 65536)
    middle = x_low * c_high + torch.div(x_low * c_low, 65536, rounding_mode="floor")
    other = x_high * c_low + middle % 65536
    high = x_high * c_high + torch.div(middle, 65536, rounding_mode="floor") + torch.div(other, 65536, rounding_mode="floor")
    return high, (other % 65536) * 65536 + (x_low * c_low) % 65536


def _exact_kept(rows, cols, p, seed, offset):
    """Of each octet of columns a counter of four words, through ten rounds: two multiplications, words change places, keys go on by the
    generator's two constants."""
    at = torch.arange(rows * _up(cols, 8) // 8, dtype=torch.int64, device="cuda")
    across = _up(cols, 8) // 8
    counter = [at % across, torch.div(at, across, rounding_mode="floor"), torch.zeros_like(at) + offset % (1 << 32), torch.zeros_like(at) + (offset >> 32)]
    for turn in range(10):
        first, second = _exact_times(counter[0], 0xD2511F53), _exact_times(counter[2], 0xCD9E8D57)
        keys = [(seed + turn * 0x9E3779B9) % (1 << 32), ((seed >> 32) + turn * 0xBB67AE85) % (1 << 32)]
        counter = [second[0].bitwise_xor(counter[1]).bitwise_xor(keys[0]), second[1], first[0].bitwise_xor(counter[3]).bitwise_xor(keys[1]), first[1]]
    kept = torch.empty((rows, across, 8), dtype=torch.bool, device="cuda")
    for j in range(8):
        number = counter[j // 2] if j % 2 == 0 else torch.div(counter[j // 2], 65536, rounding_mode="floor")
        kept[:, :, j] = (number % 65536 >= _threshold(p)).view(rows, across)
    return kept.view(rows, across * 8)[:, :cols]


def _exact_factor(s, shape):
    p = s.case["drop"]
    if _threshold(p) == 0:
        return 1.0
    return _exact_kept(*shape, p, s.seed, s.offset).double() / (1.0 - _threshold(p) / 65536)


def _exact_activation(z, act):
    if act == "none":
        return z
    if act == "relu":
        return z.clamp_min(0.0)
    if act == "gelu":
        return z * torch.special.erfc(-z / math.sqrt(2.0)) / 2.0
    if act == "gelu_tanh":
        return z * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (z + 0.044715 * z.pow(3)))
    return z * torch.sigmoid(z)


def _exact_derivative(z, act):
    if act == "none":
        return 1.0
    if act == "relu":
        return z.gt(0).double()
    if act == "gelu":
        return torch.special.erfc(-z / math.sqrt(2.0)) / 2.0 + z * torch.exp(-z.pow(2) / 2.0) / math.sqrt(2.0 * math.pi)
    if act == "gelu_tanh":
        inner = 2.0 * math.sqrt(2.0 / math.pi) * (z + 0.044715 * z.pow(3))
        slope = 2.0 * math.sqrt(2.0 / math.pi) * (1.0 + 0.134145 * z.pow(2))
        g = torch.sigmoid(inner)
        return g + z * slope * g * torch.sigmoid(-inner)
    return torch.sigmoid(z) + z * torch.sigmoid(z) * torch.sigmoid(-z)


def exact(case, seed):
    c, s = case, prepare(case, seed)
    shape, out = _shape(c), {}
    if s.op == "backward":
        dz = s.dy.double() * _exact_factor(s, shape)
        if s.z is not None:
            dz = dz * _exact_derivative(s.z.double(), c["act"])
        result, names = dz, ("dz", "dz8")
        out["dbias"] = dz.sum(0)
    else:
        if s.op == "matmul":
            a = s.a[0].double() * s.a[1].double().repeat_interleave(BLOCK, 1)[:, :s.a[0].shape[1]]
            b = s.b[0].double() * s.b[1].double().repeat_interleave(BLOCK, 1)[:, :s.b[0].shape[1]].repeat_interleave(BLOCK, 0)[:c["n"]]
            z = torch.matmul(a, b.t().contiguous())
            del a, b
        else:
            z = s.x.double()
        if s.bias is not None:
            z = z + s.bias.double()
        if s.z is not None:
            out["z"] = z
        result, names = _exact_activation(z, c["act"]) * _exact_factor(s, shape), ("y", "y8")
        if s.residual is not None:
            result = result + s.residual.double()
    wanted = c["outputs"].split(",")
    if names[0] in wanted:
        out[names[0]] = result
    if names[1] in wanted:
        out[names[1]] = _exact_quantize(result)
    if "turned" in wanted:
        out["turned"] = _exact_quantize(result.t().contiguous())
    return out
