"""zi_fp8_quantize against the definition in 64 bits: numbers and scales have to be equal, bit for bit."""
import pytest
import torch

import paper_2104_07857_amd as zi
from fp8_util import DT, Matrix, normal, numbers, powers, quantized, same, view_of

pytestmark = pytest.mark.gpu
FORMS = [(1, 0), (0, 1), (1, 1), (128, 0), (0, 128), (128, 128), (1, 128), (128, 1)]     # block_rows of out and of turned, 0: not wanted


def _check(x, out_blocks, turned_blocks, stream=None):
    rows, cols = x.shape
    out = Matrix(rows, cols, out_blocks) if out_blocks else None
    turned = Matrix(cols, rows, turned_blocks, more_ld=32, more_scale=4) if turned_blocks else None
    zi.zi_fp8_quantize(x, DT[x.dtype], rows, cols, x.stride(0) if rows > 1 else cols, out.struct if out else None,
                       turned.struct if turned else None, stream)
    torch.cuda.synchronize()
    for m, y in ((out, x), (turned, x.t())):
        if m is None:
            continue
        q, s = quantized(y.contiguous(), m.block_rows)
        assert torch.equal(m.scales(), s)
        assert same(numbers(m.codes()), q)
        assert bool((m.scale[:, s.shape[1]:] == 0xFF).all())                # nothing behind the last block
        assert bool((m.data[:, -(-m.cols // 16) * 16:] == 0xFF).all())      # nor behind the row's last 16 bytes


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 1000), (7, 8), (128, 128), (129, 127), (127, 129), (130, 1025), (1000, 260), (5, 4096), (4096, 5)])
@pytest.mark.parametrize("dtype", list(DT))
def test_every_form(rows, cols, dtype):
    x = normal((rows, cols), 1, dtype=dtype)
    for form in FORMS:
        _check(x, *form)


@pytest.mark.parametrize("pad,offset", [(1, 0), (3, 1), (8, 0), (0, 5), (24, 8)])
@pytest.mark.parametrize("dtype", list(DT))
def test_views_of_wider_rows(pad, offset, dtype):
    """Rows that start anywhere, with NaN between them."""
    _check(view_of(normal((140, 301), 2, dtype=dtype), pad, offset), 1, 1)
    _check(view_of(normal((140, 301), 2, dtype=dtype), pad, offset), 128, 128)


@pytest.mark.parametrize("form", [(1, 1), (128, 128)])
def test_values_that_scales_turn_on(form):
    """Blocks whose largest is just at, below and above 448 times a power of two, subnormals, the largest there are, zeros of
    both signs, ties between two numbers."""
    x = torch.zeros((256, 640), device="cuda:0")
    x[0, 0:128] = torch.linspace(-448, 448, 128, device="cuda:0")
    x[1, 128], x[1, 129] = 448.0, 17.0                                       # 17 is between 16 and 18
    x[2, 256], x[2, 257] = torch.nextafter(torch.tensor(448.0), torch.tensor(1e9)).item(), 19.0
    x[3, 384] = 3.4028234e38
    x[4, 512], x[4, 513] = 1e-45, -1e-45
    x[5, 0:8] = torch.tensor([1.0625, 1.1875, 2.125, -1.0625, 448.0, 2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -10], device="cuda:0")
    x[130, 0], x[131, 130], x[132, 300] = 2.0 ** -126, -(2.0 ** -149) * 12345, 1.17e-38
    x[200] = -0.0
    _check(x, *form)
    half = normal((256, 256), 3, 1e-7).half()                                # subnormals of fp16
    half[0, 0] = 65504.0
    _check(half, *form)


@pytest.mark.parametrize("dtype", list(DT))
def test_infinities_and_nan_keep_to_their_places(dtype):
    x = normal((256, 300), 4, dtype=dtype)
    x[3, 5], x[3, 140], x[200, 299] = float("inf"), float("-inf"), float("nan")
    x[10, :128] = float("nan")                                               # a block with nothing else in it
    for form in FORMS:
        _check(x, *form)
    m = Matrix(256, 300)
    zi.zi_fp8_quantize(x, DT[dtype], 256, 300, 300, m.struct)
    torch.cuda.synchronize()
    assert int(numbers(m.codes()).isnan().sum()) == 3 + 128 and int(m.scales()[10, 0]) == 127


def test_large_offsets():
    """Places past 2^32 bytes of a buffer."""
    wide = torch.zeros((3, 1 << 31), dtype=torch.bfloat16, device="cuda:0")
    x = wide[:, (1 << 31) - 200:]
    x.copy_(normal((3, 200), 5))
    _check(x, 1, 1)


@pytest.mark.parametrize("form,dtype", [((1, 1), torch.bfloat16), ((128, 128), torch.float32), ((0, 1), torch.float16)])
def test_outputs_larger_than_the_cache(form, dtype):
    rows, cols = 9001, 12001 if form[0] == 0 else 6007
    x = normal((rows, cols), 9, dtype=dtype)
    x[5, 7] = float("nan")
    _check(x, *form)


def test_another_stream_and_a_graph():
    x = normal((300, 700), 6, dtype=torch.bfloat16)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    _check(x, 1, 1, s)
    out = Matrix(300, 700)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        zi.zi_fp8_quantize(x, zi.ZI_BF16, 300, 700, 700, out.struct, None, torch.cuda.current_stream())
    for k in range(3):
        x.copy_(normal((300, 700), 7 + k, 10.0 ** k))
        g.replay()
        torch.cuda.synchronize()
        q, sc = quantized(x, 1)
        assert torch.equal(out.scales(), sc) and same(numbers(out.codes()), q)


def test_what_it_stands_for_is_near():
    """Half a step of three bits of fraction: 2^-4 of the value, or 2^-10 of the scale below the normal numbers."""
    x = normal((200, 333), 8).double()
    out = Matrix(200, 333)
    zi.zi_fp8_quantize(x.float(), zi.ZI_FP32, 200, 333, 333, out.struct)
    torch.cuda.synchronize()
    scale = powers(out.scales()).repeat_interleave(128, 1)[:, :333]
    assert bool(((out.values() - x).abs() <= torch.maximum(x.abs() * 2.0 ** -4, scale * 2.0 ** -10)).all())
