"""The 8-bit operators' definitions in 64 bits, and matrices in 8 bits for the tests.  Works on any torch device."""
import math

import torch

import paper_2104_07857_amd as zi

DT = {torch.bfloat16: zi.ZI_BF16, torch.float16: zi.ZI_FP16, torch.float32: zi.ZI_FP32}
HALF_ULP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}   # of a result, whose significand has 8, 11 or 24 bits
LEAST = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25, torch.float32: 0.0}                      # half a step of fp16's subnormals


class Matrix:
    """A matrix in 8 bits whose bytes outside of it are 0xFF (NaN in both formats) before anything is written."""

    def __init__(self, rows, cols, block_rows=1, device="cuda:0", more_ld=0, more_scale=0):
        (r, ld), (sr, sld) = zi.fp8_layout(rows, cols, block_rows)
        self.rows, self.cols, self.block_rows = rows, cols, block_rows
        self.data = torch.full((r, ld + more_ld), 0xFF, dtype=torch.uint8, device=device)
        self.scale = torch.full((sr, sld + more_scale), 0xFF, dtype=torch.uint8, device=device)
        self.struct = zi.make_fp8_matrix(self.data, self.scale, rows, cols, block_rows)

    def put(self, codes, scales):
        self.data[:, :self.cols] = codes
        self.scale[:, :scales.shape[1]] = scales
        return self

    def codes(self):
        return self.data[:, :self.cols]

    def scales(self):
        return self.scale[:, :-(-self.cols // 128)]

    def values(self):
        return numbers(self.codes()) * spread(powers(self.scales()), self.rows, self.cols, self.block_rows)


def _e4m3(c):
    """Sign, 4 bits of exponent (bias 7), 3 of fraction; 0x7F is NaN."""
    e, f = (c >> 3) & 15, c & 7
    v = float("nan") if c & 0x7F == 0x7F else math.ldexp(8 + f, e - 10) if e else math.ldexp(f, -9)
    return -v if c & 0x80 else v


# (tables made on the host: a GPU's pow need not give the very power of two)
NUMBERS = torch.tensor([_e4m3(c) for c in range(256)], dtype=torch.float64)
POWERS = torch.tensor([math.ldexp(1.0, b - 127) for b in range(255)] + [float("nan")], dtype=torch.float64)


def numbers(codes):
    return NUMBERS.to(codes.device)[codes.to(torch.int64)]


def powers(scales):
    return POWERS.to(scales.device)[scales.to(torch.int64)]


def spread(blocks, rows, cols, block_rows):
    return blocks.repeat_interleave(block_rows, 0)[:rows].repeat_interleave(128, 1)[:, :cols]


def block_most(x, block_rows):
    """Largest finite magnitude of each block of x (64 bits)."""
    rows, cols = x.shape
    m = torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x))
    m = torch.nn.functional.pad(m, (0, -cols % 128, 0, -rows % block_rows))
    return m.view(m.shape[0] // block_rows, block_rows, -1, 128).amax((1, 3))


def scale_bytes(most):
    """Bytes of the smallest powers of two, 2^-127 at least, with most <= 448 * scale."""
    e = torch.full(most.shape, -127, dtype=torch.int64, device=most.device)
    for k in range(-126, 128):
        e = torch.where(most > 448.0 * 2.0 ** (k - 1), torch.full_like(e, k), e)
    return torch.where(most > 0, e + 127, torch.full_like(e, 127)).to(torch.uint8)


def rounded(v):
    """v (64 bits, 448 at most) to the nearest e4m3 value, ties to the even one."""
    _, e = torch.frexp(torch.where(torch.isfinite(v), v.abs(), torch.ones_like(v)).clamp_min(2.0 ** -6))
    step = powers(e - 4 + 127)
    return torch.where(torch.isfinite(v), torch.round(v / step) * step, torch.full_like(v, float("nan")))


def quantized(x, block_rows):
    """(values of the numbers, scale bytes) of x by the definition."""
    x = x.double()
    scales = scale_bytes(block_most(x, block_rows))
    return rounded(x / spread(powers(scales), *x.shape, block_rows)), scales


def same(a, b):
    """Equal, NaN at the same places, zeros of either sign."""
    return bool(((a == b) | (a.isnan() & b.isnan())).all())


def view_of(x, pad, offset=0):
    """x at `offset` elements into rows that are `pad` elements longer, NaN around it."""
    if not pad and not offset:
        return x.contiguous()
    wide = torch.full((x.shape[0], x.shape[1] + pad + offset), float("nan"), dtype=x.dtype, device=x.device)
    wide[:, offset:offset + x.shape[1]] = x
    return wide[:, offset:offset + x.shape[1]]


def normal(shape, seed, std=1.0, dtype=torch.float32):
    g = torch.Generator(device="cuda:0").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda:0") * std).to(dtype)
