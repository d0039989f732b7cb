"""zi_epilogue and zi_epilogue_backward against their definitions in 64 bits (epilogue_util.py, which derives the tolerances).  Where numbers are small whole ones and the factor of dropout
a power of two, results are exact and compared bit for bit, so that a wrong index, mask or scale cannot hide."""
import ctypes
import shutil

import pytest
import torch

import paper_2104_07857_amd as zi
from epilogue_util import ACTIVATIONS, OFFSET, SEED, backward, dropped, factor, forward, kept, near, near8, same8, threshold
from fp8_util import DT, Matrix, block_most, normal, quantized, same, view_of

pytestmark = pytest.mark.gpu
HALF = [torch.bfloat16, torch.float16]
ZI_ERR_HIP = -4
SIZES = [(1, 1), (1, 7), (3, 8), (2, 9), (5, 127), (1, 128), (7, 129), (16, 130), (17, 1000), (130, 257), (333, 1000), (128, 128), (129, 4100), (1, 16384), (2, 33001), (300, 640), (1025, 63)]


def _whole(rows, cols, seed, dtype, most=8):
    g = torch.Generator(device="cuda:0").manual_seed(seed)
    return torch.randint(-most, most + 1, (rows, cols), generator=g, device="cuda:0").to(dtype)


def _empty(rows, cols, dtype, pad=0, offset=0):
    """An output, NaN in it and around it; (the view, whether all around it is as it was)."""
    wide = torch.full((rows, cols + pad + offset), float("nan"), dtype=dtype, device="cuda:0")

    def untouched():
        return bool(wide[:, :offset].isnan().all()) and bool(wide[:, offset + cols:].isnan().all())
    return wide[:, offset:offset + cols], untouched


class Forward:
    """A call and its outputs: `outputs` of z, y, y8, turned."""

    def __init__(self, x, activation="none", outputs="y", bias=None, residual=None, drop=0.0, pad=0, offset=0, seed=SEED, at=OFFSET, d_offset=None, stream=None, y=None, z=None):
        rows, cols = x.shape
        wanted = outputs.split(",")
        self.z, self.y, self.y8, self.turned, checks = z, y, None, None, []
        for name in ("z", "y"):
            if name in wanted and getattr(self, name) is None:
                out, check = _empty(rows, cols, x.dtype, pad, offset)
                setattr(self, name, out)
                checks.append(check)
        if "y8" in wanted:
            self.y8 = Matrix(rows, cols, more_ld=16 if pad else 0, more_scale=4 if pad else 0)
        if "turned" in wanted:
            self.turned = Matrix(cols, rows, more_ld=16 if pad else 0, more_scale=4 if pad else 0)
        self.args = zi.make_epilogue(rows, cols, DT[x.dtype], bias=bias, residual=residual, z=self.z, y=self.y, activation=ACTIVATIONS[activation], drop=drop, seed=seed,
                                     offset=at, d_offset=d_offset)
        torch.cuda.synchronize()
        zi.zi_epilogue(x, rows, cols, x.stride(0) if rows > 1 else max(cols, x.stride(0)), self.args, self.y8.struct if self.y8 else None,
                       self.turned.struct if self.turned else None, stream)
        torch.cuda.synchronize()
        assert all(c() for c in checks)
        for m in (self.y8, self.turned):
            if m is not None:                      # up to the next multiple of 8 (16 in turned) zeros, nothing behind
                end = -(-m.cols // (8 if m is self.y8 else 16)) * (8 if m is self.y8 else 16)
                assert bool((m.data[:, end:] == 0xFF).all()) and not bool(m.data[:, m.cols:end].any())
                assert bool((m.scale[:, -(-m.cols // 128):] == 0xFF).all())


class Backward:
    def __init__(self, dy, z=None, activation="none", outputs="dz", drop=0.0, dbias=None, accumulate=False, pad=0, offset=0, seed=SEED, at=OFFSET, d_offset=None, stream=None, dz=None):
        rows, cols = dy.shape
        wanted = outputs.split(",")
        self.dz, self.dz8, self.turned, self.dbias, check = dz, None, None, dbias, None
        if "dz" in wanted and dz is None:
            self.dz, check = _empty(rows, cols, dy.dtype, pad, offset)
        if "dz8" in wanted:
            self.dz8 = Matrix(rows, cols)
        if "turned" in wanted:
            self.turned = Matrix(cols, rows)
        self.args = zi.make_epilogue_backward(dy, z, self.dz, dbias, DT[dy.dtype], activation=ACTIVATIONS[activation], drop=drop, seed=seed, offset=at, d_offset=d_offset,
                                              dbias_dtype=None if dbias is None else DT[dbias.dtype], accumulate=accumulate)
        self.ws = torch.full((max(16, zi.zi_epilogue_workspace_bytes(rows, cols)),), 0xFF, dtype=torch.uint8, device="cuda:0")
        torch.cuda.synchronize()
        zi.zi_epilogue_backward(self.args, self.dz8.struct if self.dz8 else None, self.turned.struct if self.turned else None, self.ws, stream=stream)
        torch.cuda.synchronize()
        assert check is None or check()


def _is_quantised(matrix, want):
    """Bit for bit, but for the sign of zeros."""
    codes, scales = quantized(want, 1)
    from fp8_util import numbers
    return torch.equal(matrix.scales(), scales) and same(numbers(matrix.codes()), codes)


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("dtype", HALF)
def test_whole_numbers_are_exact(rows, cols, dtype):
    """relu, a bias, half of the elements dropped (the others doubled), a residual; all outputs, and each by itself; views of wider buffers."""
    x, bias, residual = _whole(rows, cols, 1, dtype), _whole(1, cols, 2, dtype)[0], _whole(rows, cols, 3, dtype)
    for pad, offset in ((0, 0), (3, 1), (8, 0)):
        for drop in (0.0, 0.5):
            for activation in ("none", "relu"):
                z, y, _ = forward(x, activation, drop, bias, residual)
                a = Forward(view_of(x, pad, offset), activation, "z,y,y8,turned", bias, view_of(residual, pad), drop, pad, offset)
                assert torch.equal(a.z.double(), z) and torch.equal(a.y.double(), y)
                assert _is_quantised(a.y8, y) and _is_quantised(a.turned, y.t())
                b = Forward(view_of(x, pad, offset), activation, "z,y,y8", bias, view_of(residual, pad), drop, pad, offset)     # rows, not tiles
                assert torch.equal(b.z, a.z) and torch.equal(b.y, a.y) and same8(b.y8, a.y8)
        for outputs in ("z", "y", "y8", "turned"):
            c = Forward(view_of(x, pad, offset), "relu", outputs, bias, view_of(residual, pad), 0.5, pad, offset)
            z, y, _ = forward(x, "relu", 0.5, bias, residual)
            assert c.z is None or torch.equal(c.z.double(), z)
            assert c.y is None or torch.equal(c.y.double(), y)
            assert (c.y8 is None or _is_quantised(c.y8, y)) and (c.turned is None or _is_quantised(c.turned, y.t()))
        d = Forward(view_of(x, pad, offset), "none", "y", None, None, 0.5, pad, offset)
        assert torch.equal(d.y.double(), dropped(x.double(), 0.5))


@pytest.mark.parametrize("rows,cols", [(1, 1000), (7, 129), (130, 1003), (257, 640)])
@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("activation", list(ACTIVATIONS))
@pytest.mark.parametrize("drop", [0.0, 0.1])
def test_normal_numbers_within_the_bounds(rows, cols, dtype, activation, drop):
    x, bias, residual = normal((rows, cols), 4, 2.0, dtype), normal((cols,), 5, 0.5, dtype), normal((rows, cols), 6, 3.0, dtype)
    for b, r in ((bias, residual), (bias, None), (None, None)):
        z, y, off = forward(x, activation, drop, b, r)
        a = Forward(x, activation, "z,y,y8,turned", b, r, drop)
        assert near(a.z, z, z.abs() * 2.0 ** -24) and near(a.y, y, off) and near8(a.y8, y, off) and near8(a.turned, y.t().contiguous(), off.t().contiguous())
        c = Forward(x, activation, "y,y8", b, r, drop)
        assert torch.equal(c.y, a.y) and same8(c.y8, a.y8)


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("activation", ["gelu", "gelu_tanh", "silu"])
def test_activations_of_every_number(dtype, activation):
    """All finite numbers of 16 bits, forward and (in fp32, as the sums over one row) backward."""
    bits = torch.arange(65536, dtype=torch.int32, device="cuda:0").to(torch.int16).view(dtype)
    x = bits[bits.isfinite()].reshape(1, -1)
    _, y, off = forward(x, activation)
    assert near(Forward(x, activation).y, y, off)
    one, dbias = torch.ones_like(x), torch.empty(x.shape[1], device="cuda:0")
    Backward(one, x, activation, "dbias", dbias=dbias)
    dz, off = backward(one, x, activation)
    assert bool(((dbias.double() - dz).abs() <= off).all())


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("activation", list(ACTIVATIONS))
def test_infinities_and_nan(dtype, activation):
    """A NaN stays one; an infinity as the header says; dropped elements are 0 whatever they were; scales are those of the others."""
    inf, nan = float("inf"), float("nan")
    x = normal((6, 300), 7, 1.0, dtype)
    for i, v in enumerate((inf, -inf, nan)):
        x[i, 3 + i:300:17] = v
    for drop in (0.0, 0.5):
        z, y, off = forward(x, activation, drop)
        a = Forward(x, activation, "z,y,y8,turned", drop=drop)
        assert torch.equal(a.z.nan_to_num(7.0), x.nan_to_num(7.0))
        assert torch.equal(a.y.isnan(), y.isnan()) and torch.equal(a.y.isinf(), y.isinf())
        fine = y.isfinite()
        off = torch.where(off.isfinite(), off, torch.zeros_like(off))
        assert near(a.y[fine], y[fine], off[fine])
        v = a.y8.values()
        assert torch.equal(v.isnan(), ~fine) and torch.equal(a.turned.values().t().isnan(), ~fine)
        from fp8_util import scale_bytes
        most, slack = block_most(y, 1), 2.0 ** -14
        assert bool((a.y8.scales() >= scale_bytes(most * (1 - slack))).all()) and bool((a.y8.scales() <= scale_bytes(most * (1 + slack))).all())


@pytest.mark.parametrize("p", [2.0 ** -16, 0.1, 0.37, 0.999, 0.9999999])
def test_the_mask_and_its_factor(p):
    """Of ones: 0 or the factor, at every threshold; the backward pass has the same mask; seeds and offsets of 64 bits."""
    x = torch.ones((70, 523), dtype=torch.float16, device="cuda:0")
    for seed, offset in ((0, 0), (SEED, OFFSET), ((1 << 64) - 1, (1 << 64) - 1), (1 << 32, 1 << 32), (77, 1 << 63)):
        k = kept(70, 523, p, seed, offset, device="cuda:0")
        want = (k.double() * factor(p)).to(torch.float16)
        assert torch.equal(Forward(x, drop=p, seed=seed, at=offset).y, want)
        dbias = torch.empty(523, device="cuda:0")
        b = Backward(x, drop=p, seed=seed, at=offset, outputs="dz,dz8,turned", dbias=dbias)
        assert torch.equal(b.dz, want)
        assert bool(((dbias.double() - k.double().sum(0) * factor(p)).abs() <= 70 * 2.0 ** -23 * factor(p) * 70).all())
    assert threshold(p) > 0


def test_drop_that_rounds_to_nothing_has_no_part():
    x = normal((9, 100), 8, 1.0, torch.bfloat16)
    assert torch.equal(Forward(x, drop=2.0 ** -18).y, x)


@pytest.mark.parametrize("dtype", HALF)
def test_in_place(dtype):
    x, residual = normal((150, 1003), 9, 1.0, dtype), normal((150, 1003), 10, 1.0, dtype)
    for outputs in ("y", "y,turned"):
        want = Forward(x, "gelu", outputs, None, residual, 0.3)
        y = x.clone()
        assert torch.equal(Forward(y, "gelu", outputs, None, residual, 0.3, y=y).y, want.y)
        y = residual.clone()
        assert torch.equal(Forward(x, "gelu", outputs, None, y, 0.3, y=y).y, want.y)
        z = x.clone()
        a = Forward(z, "gelu", "z," + outputs, normal((1003,), 1, 1.0, dtype), residual, 0.3, z=z)
        b = Forward(x, "gelu", "z," + outputs, normal((1003,), 1, 1.0, dtype), residual, 0.3)
        assert torch.equal(z, b.z) and torch.equal(a.y, b.y)
    want = Backward(x, residual, "silu", "dz,turned", 0.3)
    dy = x.clone()
    assert torch.equal(Backward(dy, residual, "silu", "dz,turned", 0.3, dz=dy).dz, want.dz)
    z = residual.clone()
    assert torch.equal(Backward(x, z, "silu", "dz,turned", 0.3, dz=z).dz, want.dz)


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("dtype", HALF)
def test_backward_of_whole_numbers_is_exact(rows, cols, dtype):
    dy, z = _whole(rows, cols, 11, dtype), _whole(rows, cols, 12, dtype)
    for pad, offset in ((0, 0), (3, 1)):
        for drop in (0.0, 0.5):
            for activation in ("none", "relu"):
                dz, _ = backward(dy, z, activation, drop)
                for dbias, accumulate in ((torch.full((cols,), float("nan"), device="cuda:0"), False), (torch.full((cols,), 3.0, device="cuda:0"), True),
                                          (torch.full((cols,), 2.0, dtype=dtype, device="cuda:0"), True), (torch.empty(cols, dtype=dtype, device="cuda:0"), False)):
                    want = (dz.sum(0) + (dbias.double() if accumulate else 0)).to(dbias.dtype)
                    a = Backward(view_of(dy, pad, offset), view_of(z, pad), activation, "dz,dz8,turned", drop, dbias, accumulate, pad, offset)
                    assert torch.equal(a.dz.double(), dz) and _is_quantised(a.dz8, dz) and _is_quantised(a.turned, dz.t())
                    assert torch.equal(a.dbias, want)
    for outputs in ("dz", "dz8", "turned", "dz8,turned"):
        dz, _ = backward(dy, None, "none", 0.5)
        a = Backward(dy, None, "none", outputs, 0.5)
        assert a.dz is None or torch.equal(a.dz.double(), dz)
        assert (a.dz8 is None or _is_quantised(a.dz8, dz)) and (a.turned is None or _is_quantised(a.turned, dz.t()))


@pytest.mark.parametrize("rows,cols", [(1, 1000), (7, 129), (130, 1003), (2057, 264)])
@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("activation", list(ACTIVATIONS))
@pytest.mark.parametrize("drop", [0.0, 0.1])
def test_backward_of_normal_numbers(rows, cols, dtype, activation, drop):
    dy, z = normal((rows, cols), 13, 1e-3, dtype), normal((rows, cols), 14, 2.0, dtype)
    dz, off = backward(dy, z, activation, drop)
    dbias = torch.empty(cols, device="cuda:0")
    a = Backward(dy, z, activation, "dz,dz8,turned", drop, dbias)
    assert near(a.dz, dz, off) and near8(a.dz8, dz, off) and near8(a.turned, dz.t().contiguous(), off.t().contiguous())
    # each addition is off by half a step of its result, which the sum of magnitudes bounds; at most 8 + 2 + 4 + ceil(rows / 128) + 16 follow each other
    depth = 30 + -(-rows // 128)
    assert bool(((dbias.double() - dz.sum(0)).abs() <= off.sum(0) + dz.abs().sum(0) * depth * 2.0 ** -24).all())


@pytest.mark.parametrize("activation", list(ACTIVATIONS))
def test_gradient_against_differences(activation):
    """sum(y * dy) along a direction of signs: the forward call's own difference quotient, against the backward call's gradient.  Steps of 1/16 leave 2^-8 / 6 of the third
    derivative (below 0.8), and none of relu where they do not pass its corner."""
    rows, cols, p = 40, 300, 0.25
    step = 1.0 / 32 if activation == "relu" else 1.0 / 16
    x = (_whole(rows, cols, 15, torch.float16, 40) / 16 + 1.0 / 32).to(torch.float16)                 # odd multiples of 1/32: the steps are exact
    v, dy = torch.sign(_whole(rows, cols, 16, torch.float16) + 0.5), normal((rows, cols), 17, 1.0, torch.float16)
    more, less = Forward(x + step * v, activation, drop=p).y.double(), Forward(x - step * v, activation, drop=p).y.double()
    quotient = (dy.double() * (more - less)).sum() / (2 * step)
    gradient = (Backward(dy, x, activation, drop=p).dz.double() * v.double()).sum()
    # each y is rounded to 2^-11 of itself, each dz (1.13 factor(p) < 2 times dy at most) too; roundings are independent: five times the root of their squares' sum.  The curve's share adds
    # up at worst.
    rounded = (dy.double().square() * (more.square() + less.square())).sum().sqrt() * 2.0 ** -11 / (2 * step) + 2 * dy.double().norm() * 2.0 ** -11
    curve = 0.0 if activation in ("none", "relu") else float(dy.double().abs().sum()) * factor(p) * 0.8 * step * step / 6
    assert abs(float(quotient - gradient)) <= 5 * float(rounded) + curve


def test_same_bits_on_any_stream():
    x, residual = normal((700, 1003), 18, 1.0, torch.bfloat16), normal((700, 1003), 19, 1.0, torch.bfloat16)
    first = Forward(x, "gelu", "y,y8,turned", None, residual, 0.1)
    back = Backward(x, residual, "gelu", "dz,dz8,turned", 0.1, torch.empty(1003, device="cuda:0"))
    for _ in range(3):
        s = torch.cuda.Stream()
        a = Forward(x, "gelu", "y,y8,turned", None, residual, 0.1, stream=s)
        assert torch.equal(a.y, first.y) and same8(a.y8, first.y8) and same8(a.turned, first.turned)
        b = Backward(x, residual, "gelu", "dz,dz8,turned", 0.1, torch.empty(1003, device="cuda:0"), stream=s)
        assert torch.equal(b.dz, back.dz) and same8(b.dz8, back.dz8) and same8(b.turned, back.turned) and torch.equal(b.dbias, back.dbias)


def test_replays_count_their_offset():
    """A captured forward and backward call whose offset is counted on in device memory: each replay has the mask of its own offset, on both ways."""
    rows, cols, p = 150, 1003, 0.3
    x, dy = normal((rows, cols), 20, 1.0, torch.bfloat16), normal((rows, cols), 21, 1.0, torch.bfloat16)
    y, dz, dbias = torch.empty_like(x), torch.empty_like(x), torch.empty(cols, device="cuda:0")
    at = torch.tensor([(1 << 32) - 2], dtype=torch.int64, device="cuda:0")
    fwd = zi.make_epilogue(rows, cols, zi.ZI_BF16, y=y, activation=zi.ZI_ACT_SILU, drop=p, seed=SEED, offset=5, d_offset=at)
    bwd = zi.make_epilogue_backward(dy, x, dz, dbias, zi.ZI_BF16, activation=zi.ZI_ACT_SILU, drop=p, seed=SEED, offset=5, d_offset=at, dbias_dtype=zi.ZI_FP32)
    ws = torch.empty(zi.zi_epilogue_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda:0")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s = torch.cuda.current_stream()
        zi.zi_epilogue(x, rows, cols, cols, fwd, stream=s)
        zi.zi_epilogue_backward(bwd, None, None, ws, stream=s)
        at += 1
    for k in range(4):
        ws.fill_(0xFF)
        y.zero_()
        g.replay()
        torch.cuda.synchronize()
        offset = (1 << 32) - 2 + 5 + k
        a, b = Forward(x, "silu", drop=p, at=offset), Backward(dy, x, "silu", "dz", p, torch.empty(cols, device="cuda:0"), at=offset)
        assert torch.equal(y, a.y) and torch.equal(dz, b.dz) and torch.equal(dbias, b.dbias)
        mask = Forward(torch.ones_like(x), drop=p, at=offset).y != 0
        assert torch.equal(mask, kept(rows, cols, p, offset=offset, device="cuda:0"))


def test_no_rows():
    """The bias' gradient of nothing is 0, or what was there."""
    for dtype in (torch.float32, torch.bfloat16):
        dbias = torch.full((300,), 2.0, dtype=dtype, device="cuda:0")
        args = zi.zi_epilogue_backward_args(dbias=dbias.data_ptr(), rows=0, cols=300, dtype=zi.ZI_BF16, dbias_dtype=DT[dtype], accumulate=1)
        zi.zi_epilogue_backward(args)
        torch.cuda.synchronize()
        assert bool((dbias == 2.0).all())
        args.accumulate = 0
        zi.zi_epilogue_backward(args)
        torch.cuda.synchronize()
        assert not bool(dbias.any())


def test_without_the_library_of_its_kernels_a_call_is_an_error(tmp_path):
    """libzi.so by itself, in a folder of its own: everything else works, and these calls say what is missing."""
    alone = ctypes.CDLL(shutil.copy(zi.LIB_PATH, tmp_path))
    x = torch.zeros((3, 16), dtype=torch.bfloat16, device="cuda:0")
    args = zi.make_epilogue(3, 16, zi.ZI_BF16, y=x)
    alone.zi_last_error.restype = ctypes.c_char_p
    for _ in range(2):
        assert alone.zi_epilogue(ctypes.c_void_p(x.data_ptr()), *map(ctypes.c_int64, (3, 16, 16)), ctypes.byref(args), None, None, None) == ZI_ERR_HIP
        assert b"libzi_epilogue.so" in alone.zi_last_error()
    torch.cuda.synchronize()
    assert not bool(x.any())


def test_matrices_of_more_than_four_gib():
    """Offsets past 2^32 bytes and 2^31 elements, in rows (the last of 40000) and in tiles."""
    rows, cols = 40000, 65544
    x = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda:0")
    some = [0, 1, 16383, 32769, 39999]
    for i, r in enumerate(some):
        x[r] = _whole(1, cols, 30 + i, torch.bfloat16)[0]
    y = torch.empty_like(x)
    args = zi.make_epilogue(rows, cols, zi.ZI_BF16, y=y, activation=zi.ZI_ACT_RELU, drop=0.5, seed=SEED, offset=OFFSET)
    turned = Matrix(cols, rows)
    for t in (None, turned.struct):
        y.fill_(float("nan"))
        zi.zi_epilogue(x, rows, cols, cols, args, None, t)
        torch.cuda.synchronize()
        for r in some:
            assert torch.equal(y[r:r + 1].double(), forward(x[r:r + 1], "relu", 0.5, row0=r)[1])
        assert not bool(y[2:16383].any()) and not bool(y[32770:39999].any())
    for r in some:
        scale = torch.exp2(turned.scale[:, r // 128].double() - 127)
        from fp8_util import numbers
        want = forward(x[r:r + 1], "relu", 0.5, row0=r)[1][0]
        assert torch.equal(numbers(turned.data[:, r]) * scale, want)
    dz = Backward(x, x, "relu", "dz", 0.5, dbias := torch.empty(cols, device="cuda:0"), dz=y).dz
    total = torch.zeros(cols, dtype=torch.float64, device="cuda:0")
    for r in some:
        want = backward(x[r:r + 1], x[r:r + 1], "relu", 0.5, row0=r)[0]
        assert torch.equal(dz[r:r + 1].double(), want)
        total += want[0]
    assert torch.equal(dbias.double(), total)


@pytest.mark.parametrize("rows,cols", [(2 ** 25 + 37, 3), (2 ** 24 + 21, 136)])
def test_more_rows_than_are_under_way_at_a_time(rows, cols):
    """A launch has 2^20 workgroups at most, which then go on to further rows (of 32 and of 16 each)."""
    x = (torch.arange(rows, device="cuda:0", dtype=torch.int32)[:, None] * 7 + torch.arange(cols, device="cuda:0", dtype=torch.int32)).remainder_(255).sub_(127).to(torch.bfloat16)
    y = torch.full_like(x, float("nan"))
    zi.zi_epilogue(x, rows, cols, cols, zi.make_epilogue(rows, cols, zi.ZI_BF16, y=y, activation=zi.ZI_ACT_RELU))
    torch.cuda.synchronize()
    assert torch.equal(y, x.clamp_min(0))
    zi.zi_epilogue(x, rows, cols, cols, zi.make_epilogue(rows, cols, zi.ZI_BF16, y=y, drop=0.5, seed=SEED, offset=OFFSET))
    torch.cuda.synchronize()
    for r in (0, rows - 40, rows - 3):
        assert torch.equal(y[r:r + 3].double(), forward(x[r:r + 3], "none", 0.5, row0=r)[1])


@pytest.mark.parametrize("cols", [8200, 8203])
@pytest.mark.parametrize("activation", list(ACTIVATIONS))
def test_large_calls_are_like_small_ones(cols, activation):
    """What is read and written past the caches: the same bits as of its rows by 1280 at a time, whose calls are small.  (The mask goes by the row, so nothing is dropped.)"""
    rows, part = 16640, 1280                                              # 136 million elements, 546 MB and more
    dtype = torch.float16 if cols % 8 else torch.bfloat16
    x, residual, bias = normal((rows, cols), 40, 2.0, dtype), normal((rows, cols), 41, 1.0, dtype), normal((cols,), 42, 0.5, dtype)
    for outputs, r in (("z,y,y8", residual), ("y,y8,turned", None)):
        a = Forward(x, activation, outputs, bias, r)
        for at in range(0, rows, part):
            rest = slice(at, at + part)
            b = Forward(x[rest], activation, outputs, bias, None if r is None else r[rest])
            assert torch.equal(a.y[rest], b.y) and (a.z is None or torch.equal(a.z[rest], b.z))
            assert torch.equal(a.y8.codes()[rest], b.y8.codes()) and torch.equal(a.y8.scales()[rest], b.y8.scales())
            if a.turned:
                assert torch.equal(a.turned.codes()[:, rest], b.turned.codes()) and torch.equal(a.turned.scales()[:, at // 128:(at + part) // 128], b.turned.scales())
    dbias, total = torch.empty(cols, device="cuda:0"), torch.zeros(cols, dtype=torch.float64, device="cuda:0")
    a = Backward(residual, x, activation, "dz,dz8,turned", dbias=dbias)
    for at in range(0, rows, part):
        rest = slice(at, at + part)
        b = Backward(residual[rest], x[rest], activation, "dz,dz8,turned", dbias=torch.empty(cols, device="cuda:0"))
        assert torch.equal(a.dz[rest], b.dz) and torch.equal(a.dz8.codes()[rest], b.dz8.codes()) and torch.equal(a.turned.codes()[:, rest], b.turned.codes())
        total += b.dbias.double()
    # each of 13 sums and their total: 160 additions and less follow each other
    size = a.dz.double().abs().sum(0)
    assert bool(((dbias.double() - total).abs() <= size * 320 * 2.0 ** -24).all())
