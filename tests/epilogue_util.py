"""What follows a product, by its definition in 64 bits (include/zi_epilogue.h), on any torch device; the generator with Python's and numpy's whole numbers."""
import math

import numpy as np
import torch

import paper_2104_07857_amd as zi
from fp8_util import HALF_ULP, LEAST, numbers, powers, scale_bytes, block_most, spread

ACTIVATIONS = {"none": zi.ZI_ACT_NONE, "relu": zi.ZI_ACT_RELU, "gelu": zi.ZI_ACT_GELU, "gelu_tanh": zi.ZI_ACT_GELU_TANH, "silu": zi.ZI_ACT_SILU}
SEED, OFFSET = 0x0123456789ABCDEF, (5 << 32) + 77


def philox(counter, key):
    """Philox4x32-10 of a counter of four words (numbers or arrays of them) and a key of two."""
    x, k, low = [np.asarray(c, np.uint64) for c in counter], list(key), np.uint64(0xFFFFFFFF)
    for _ in range(10):
        a, b = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        x = [(b >> np.uint64(32)) ^ x[1] ^ np.uint64(k[0]), b & low, (a >> np.uint64(32)) ^ x[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return x


def threshold(p):
    return min(65535, round(float(np.float32(p)) * 65536))


def kept(rows, cols, p, seed=SEED, offset=OFFSET, row0=0, device="cpu"):
    """Where dropout keeps an element, of rows from row0 on."""
    octets = -(-cols // 8)
    octet, row = np.meshgrid(np.arange(octets, dtype=np.uint64), np.arange(row0, row0 + rows, dtype=np.uint64))
    words = philox((octet, row, offset & 0xFFFFFFFF, offset >> 32), (seed & 0xFFFFFFFF, seed >> 32))
    words = np.stack([np.broadcast_to(w, octet.shape) for w in words], -1)
    number = np.stack([words & np.uint64(0xFFFF), words >> np.uint64(16)], -1).reshape(rows, octets * 8)[:, :cols]
    return torch.from_numpy((number >= threshold(p)).copy()).to(device)


def factor(p):
    return 65536.0 / (65536 - threshold(p))


def dropped(x, p, **where):
    """drop(x), 64 bits."""
    if threshold(p) == 0:
        return x
    return torch.where(kept(x.shape[0], x.shape[1], p, device=x.device, **where), x * factor(p), torch.zeros_like(x))


def phi(z):
    return 0.5 * torch.special.erfc(-z / math.sqrt(2.0))


def act(z, name):
    if name == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if name == "gelu":
        return z * phi(z)
    if name == "gelu_tanh":
        return z * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))
    return z * torch.sigmoid(z) if name == "silu" else z


def derivative(z, name):
    if name == "relu":
        return torch.where(z <= 0, torch.zeros_like(z), torch.ones_like(z))
    if name == "gelu":
        return phi(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        u = 2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)
        return torch.sigmoid(u) * (1 + torch.sigmoid(-u) * z * 2 * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z * z))
    return torch.sigmoid(z) * (1 + z * torch.sigmoid(-z)) if name == "silu" else torch.ones_like(z)


def forward(x, name, p=0.0, bias=None, residual=None, **where):
    """(z, y, how far fp32 may be from y), 64 bits.  x and the bias in 16 bits are exact; their sum is rounded to 2^-24 of it, which the derivative (1.13 at most) and
    the factor pass on; act is within 2^-16 of itself and 2^-118; a product and a sum of two more steps."""
    z = x.double() if bias is None else x.double() + bias.double()
    v = dropped(act(z, name), p, **where)
    y = v if residual is None else v + residual.double()
    inexact = 0.0 if name in ("none", "relu") else 2.0 ** -16
    off = v.abs() * (inexact + 2.0 ** -23) + (0 if bias is None else 1.13 * 2.0 ** -24) * z.abs() * factor(p) + y.abs() * 2.0 ** -24 + (2.0 ** -118 * factor(p) if inexact else 0.0)
    return z, y, off


def backward(dy, z, name, p=0.0, **where):
    """(dz, how far fp32 may be from it): the derivative within 2^-16 of itself and 2^-20, two more roundings."""
    d = dropped(dy.double(), p, **where)
    slope = torch.ones_like(d) if name == "none" else derivative(z.double(), name)
    dz = torch.where(slope == 0, torch.zeros_like(d), d * slope) if name == "relu" else d * slope
    inexact = 0.0 if name in ("none", "relu") else 1.0
    return dz, dz.abs() * (2.0 ** -16 * inexact + 2.0 ** -23) + d.abs() * 2.0 ** -20 * inexact


def near(got, want, off, least=True):
    """got (16 bits) is want rounded once, from at most `off` away."""
    got, dtype = got.double(), got.dtype
    tol = off + (want.abs() + off) * HALF_ULP[dtype] + (LEAST[dtype] if least else 0)
    return bool((((got - want).abs() <= tol) | (got.isnan() & want.isnan()) | (got == want)).all())


def near8(matrix, want, off):
    """A matrix in 8 bits (blocks of a row) is want quantised, from at most `off` away: scales that are right for a largest magnitude that near, numbers that are within half a
    step of e4m3's there."""
    most, most_off = block_most(want, 1), block_most(off, 1)
    scales = matrix.scales().to(torch.int64)
    least, largest = scale_bytes((most - most_off).clamp_min(0)).to(torch.int64), scale_bytes(most + most_off).to(torch.int64)
    maybe_zero = most <= most_off                     # then any smaller scale is right, and that of a block of zeros
    ok = ((scales >= least) | maybe_zero) & ((scales <= largest) | (maybe_zero & (scales == 127)))
    s = spread(powers(matrix.scales()), matrix.rows, matrix.cols, 1)
    v = numbers(matrix.codes())
    _, e = torch.frexp((want.abs() + off).div(s).clamp_min(2.0 ** -6))
    half = torch.exp2((e - 5).double())
    return bool(ok.all()) and bool(((v - want / s).abs() <= half + off / s).all())


def same8(a, b):
    return torch.equal(a.codes(), b.codes()) and torch.equal(a.scales(), b.scales())
