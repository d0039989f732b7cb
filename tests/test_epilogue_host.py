"""What follows a product, without a GPU: layouts, what the calls refuse and in which words, calls that have nothing to do, the generator's published values."""
import ctypes

import numpy as np
import pytest

import paper_2104_07857_amd as zi
from test_fp8_host import ALIGN, BF16, INVALID, UNSUPPORTED, _bytes, _half, _matrix, _refused

GIB = 1 << 30
ROWS, COLS = 4, 100


def _args(**over):
    y = _half(ROWS, COLS)
    if not isinstance(over.get("y", 0), (int, type(None))):
        y = over.pop("y")
    a = zi.make_epilogue(ROWS, COLS, BF16, y=y)
    a.keep = y
    for k, v in over.items():
        setattr(a, k, v)
    return a


def _back(**over):
    keep = [_half(ROWS, COLS) for _ in range(3)] + [_half(1, COLS)[0]]
    a = zi.make_epilogue_backward(*keep, BF16, activation=zi.ZI_ACT_GELU)
    a.keep = keep
    for k, v in over.items():
        setattr(a, k, v)
    return a


def _forward(args, y8=None, turned=None, x=None):
    return zi.zi_epilogue(_half(ROWS, COLS) if x is None else x, ROWS, COLS, COLS, args, y8, turned)


def _product(args, y8=None, turned=None, a=None, b=None):
    ws = _bytes(max(16, zi.zi_fp8_matmul_epilogue_workspace_bytes(ROWS, COLS, 200, 3)))
    return zi.zi_fp8_matmul_epilogue(a or _matrix(ROWS, 200), b or _matrix(COLS, 200, 128), args, y8, turned, ws, ws.nbytes)


def _backward(args, dz8=None, turned=None):
    ws = _bytes(zi.zi_epilogue_workspace_bytes(ROWS, COLS))
    return zi.zi_epilogue_backward(args, dz8, turned, ws, ws.nbytes)


def test_struct_sizes():
    assert ctypes.sizeof(zi.zi_epilogue_args) == 96 and ctypes.sizeof(zi.zi_epilogue_backward_args) == 120
    assert zi.zi_epilogue_workspace_bytes(0, 64) == 0 == zi.zi_epilogue_workspace_bytes(64, 0) == zi.zi_epilogue_workspace_bytes(-1, 5)
    assert zi.zi_epilogue_workspace_bytes(300, 64) >= 64 * 4
    assert zi.zi_fp8_matmul_epilogue_workspace_bytes(0, 5, 5) == 0 == zi.zi_fp8_matmul_epilogue_workspace_bytes(5, 5, -1)
    for outputs in range(4):
        assert zi.zi_fp8_matmul_epilogue_workspace_bytes(64, 128, 16384, outputs) >= 64 * 128 * 4       # k is shared out
    assert zi.zi_fp8_matmul_epilogue_workspace_bytes(1, 4096, 4096, zi.ZI_EPILOGUE_Y8) >= 4096 * 4


@pytest.mark.parametrize("call", [_forward, _product, lambda a, y8=None, turned=None: _backward(_back(**a.over), y8, turned)])
@pytest.mark.parametrize("over,status,word", [
    (dict(dtype=2), INVALID, "dtype"), (dict(activation=5), INVALID, "activation"), (dict(activation=-1), INVALID, "activation"),
    (dict(drop=1.0), INVALID, "drop"), (dict(drop=-0.1), INVALID, "drop"), (dict(drop=float("nan")), INVALID, "drop"), (dict(drop=float("inf")), INVALID, "drop"),
    (dict(d_offset=12), ALIGN, "d_offset"), (dict(reserved=1), INVALID, "reserved")])
def test_ways_are_checked(call, over, status, word):
    a = _args(**over)
    a.over = over
    _refused(status, word, call, a)


@pytest.mark.parametrize("call", [_forward, _product])
def test_forward_refuses(call):
    turned = lambda **kw: _matrix(COLS, ROWS, **kw)                                       # noqa: E731
    _refused(INVALID, "args", call, None)
    _refused(INVALID, "no output", call, _args(y=None))
    _refused(INVALID, "y8 is not", call, _args(), _matrix(ROWS, COLS + 1))
    _refused(INVALID, "turned is not", call, _args(), None, _matrix(ROWS, COLS))
    _refused(INVALID, "block_rows", call, _args(), _matrix(ROWS, COLS, 128))
    _refused(INVALID, "block_rows", call, _args(), None, turned(blocks=128))
    _refused(ALIGN, "multiple of 16", call, _args(), _matrix(ROWS, COLS, ld=COLS + 1))
    for name in ("residual", "z", "y"):
        x = _half(ROWS, COLS)
        _refused(INVALID, "pitch of " + name, call, _args(**{name: x.ctypes.data, name + "_ld": COLS - 1}))
        _refused(ALIGN, name + " must", call, _args(**{name: x.ctypes.data + 1, name + "_ld": COLS}))
        _refused(UNSUPPORTED, "2^40", call, _args(**{name: x.ctypes.data, name + "_ld": (1 << 38) + 1}))
    _refused(ALIGN, "bias", call, _args(bias=_half(1, COLS).ctypes.data + 1))
    y = _half(ROWS, COLS)
    at = y.ctypes.data
    _refused(INVALID, "overlap", call, _args(y=y, residual=at + 2, residual_ld=COLS))
    _refused(INVALID, "overlap", call, _args(y=y, residual=at, residual_ld=COLS + 1))     # the same place, but another pitch
    _refused(INVALID, "overlap", call, _args(y=y, z=at, z_ld=COLS))
    _refused(INVALID, "overlap", call, _args(y=y, bias=at + 10))
    _refused(INVALID, "overlap", call, _args(y=y, d_offset=at + 16, drop=0.5))
    _refused(INVALID, "overlap", call, _args(y=y), _matrix(ROWS, COLS, data=at))
    out = _matrix(ROWS, COLS)
    _refused(INVALID, "overlap", call, _args(y=y), out, turned(data=out.data))
    _refused(INVALID, "overlap", call, _args(y=y, z=_half(1, 8).ctypes.data, z_ld=COLS, residual=out.data, residual_ld=COLS), out)


def test_matrix_refuses():
    x = _half(ROWS, COLS)
    f = lambda *a, **k: zi.zi_epilogue(*a, **k)                                           # noqa: E731
    _refused(INVALID, "rows", f, x, -1, COLS, COLS, _args())
    _refused(INVALID, "cols", f, x, ROWS, -1, COLS, _args())
    _refused(INVALID, "x is NULL", f, None, ROWS, COLS, COLS, _args())
    _refused(INVALID, "pitch of x", f, x, ROWS, COLS, COLS - 1, _args())
    _refused(ALIGN, "x must", f, x.ctypes.data + 1, ROWS, COLS, COLS, _args())
    for rows, cols in ((1 << 31, 1), (1 << 30, 129), (1 << 19, 1 << 19)):
        a = _args(y=None)
        a.y, a.y_ld = 64 * GIB, cols
        _refused(UNSUPPORTED, "tiles", f, 16 * GIB, rows, cols, cols, a)
    both = _half(ROWS, COLS)
    _refused(INVALID, "overlap", f, both, ROWS, COLS, COLS, _args(y=both, z=both.ctypes.data, z_ld=COLS))      # only one of them can be x
    _refused(INVALID, "overlap", f, both, ROWS, COLS, COLS, _args(z=both.ctypes.data + 2, z_ld=COLS))


def test_product_refuses():
    f = zi.zi_fp8_matmul_epilogue
    _refused(INVALID, "NULL", f, None, _matrix(COLS, 200), _args())
    _refused(INVALID, "columns", f, _matrix(ROWS, 200), _matrix(COLS, 201), _args())
    _refused(UNSUPPORTED, "pitch", f, _matrix(ROWS, 200, ld=1 << 23), _matrix(COLS, 200), _args())
    a = _args()
    a.y_ld = 1 << 27
    _refused(UNSUPPORTED, "2^", f, _matrix(4, 16), _matrix(4, 16, rows=1 << 27), a)
    nbytes = zi.zi_fp8_matmul_epilogue_workspace_bytes(64, 128, 16384, 0)
    wide, ws = zi.make_epilogue(64, 128, BF16, y=_half(64, 128)), _bytes(nbytes)
    p, q = _matrix(64, 16384), _matrix(128, 16384)
    _refused(INVALID, "workspace", f, p, q, wide)
    _refused(INVALID, "workspace", f, p, q, wide, None, None, ws.ctypes.data, nbytes - 4)
    _refused(ALIGN, "d_workspace", f, p, q, wide, None, None, ws.ctypes.data + 4, nbytes)
    _refused(INVALID, "overlap", f, p, q, wide, None, None, p.data, nbytes)


def test_backward_refuses():
    _refused(INVALID, "args", _backward, None)
    _refused(INVALID, "no output", _backward, _back(dz=None, dbias=None))
    _refused(INVALID, "dbias_dtype", _backward, _back(dbias_dtype=zi.ZI_FP16))
    _refused(ALIGN, "dbias", _backward, _back(dbias_dtype=zi.ZI_FP32, dbias=_half(1, 2 * COLS + 2).ctypes.data + 2))
    _refused(INVALID, "dy is NULL", _backward, _back(dy=None))
    _refused(INVALID, "z is NULL", _backward, _back(z=None))
    _refused(INVALID, "dz8 is not", _backward, _back(), _matrix(ROWS, COLS + 1))
    _refused(INVALID, "turned is not", _backward, _back(), None, _matrix(ROWS, COLS))
    _refused(INVALID, "rows", _backward, _back(rows=-1))
    for name in ("dy", "z", "dz"):
        _refused(INVALID, "pitch of " + name, _backward, _back(**{name + "_ld": COLS - 1}))
        _refused(ALIGN, name + " must", _backward, _back(**{name: _half(ROWS, COLS).ctypes.data + 1}))
    a = _back()
    _refused(INVALID, "overlap", _backward, _back(dz=a.dy + 2, dy=a.dy))
    _refused(INVALID, "overlap", _backward, _back(dbias=a.z, z=a.z))
    _refused(UNSUPPORTED, "2^26", _backward, _back(cols=(1 << 26) + 1))
    ws = _bytes(zi.zi_epilogue_workspace_bytes(ROWS, COLS))
    f = zi.zi_epilogue_backward
    _refused(INVALID, "workspace", f, a)
    _refused(INVALID, "workspace", f, a, None, None, ws, ws.nbytes - 4)
    _refused(ALIGN, "d_workspace", f, a, None, None, ws.ctypes.data + 4, ws.nbytes)


def test_sizes_of_zero_do_nothing():
    """Also with no GPU: there is nothing to reach."""
    empty, none = zi.make_epilogue(0, COLS, BF16, y=_half(1, COLS)), zi.make_epilogue(ROWS, 0, BF16, y=_half(ROWS, 1))
    assert zi.zi_epilogue(None, 0, COLS, COLS, empty) == zi.ZI_OK
    assert zi.zi_epilogue(None, ROWS, 0, 0, none) == zi.ZI_OK
    assert zi.zi_fp8_matmul_epilogue(_matrix(0, 16), _matrix(COLS, 16), empty) == zi.ZI_OK
    assert zi.zi_epilogue_backward(_back(rows=0, dbias=None)) == zi.ZI_OK
    assert zi.zi_epilogue_backward(_back(cols=0)) == zi.ZI_OK


def test_ordinary_host_memory_is_an_error_and_no_fault():
    for call in (lambda: _forward(_args()), lambda: _product(_args()), lambda: _backward(_back())):
        with pytest.raises(zi.ZiError) as e:
            call()
        assert e.value.status in (zi.ZI_ERR_HIP, INVALID)


def test_in_place_and_beside_each_other():
    """What may coincide goes on to the query for its memory."""
    y = _half(ROWS, 4 * COLS)
    at = lambda i: y.ctypes.data + 2 * i * COLS                                           # noqa: E731
    columns = dict(y=None, z=at(1), z_ld=4 * COLS, residual=at(2), residual_ld=4 * COLS)
    for args, x, ld in ((_args(y=y[:, :COLS].copy()), None, COLS), (_args(**columns), at(0), 4 * COLS), (_args(**{**columns, "z": at(0)}), at(0), 4 * COLS)):
        for place in (None, at(2)):
            if place:
                args.y, args.y_ld = at(2), 4 * COLS
            with pytest.raises(zi.ZiError) as e:
                zi.zi_epilogue(_half(ROWS, COLS) if x is None else x, ROWS, COLS, ld, args)
            assert e.value.status in (zi.ZI_ERR_HIP, INVALID) and "overlap" not in e.value.message
    for name in ("dy", "z"):
        a = _back()
        a.dz = getattr(a, name)
        with pytest.raises(zi.ZiError) as e:
            _backward(a)
        assert "overlap" not in e.value.message


# ---- Python's side ---------------------------------------------------------------------------------------------

@pytest.fixture
def direct():
    from paper_2104_07857_amd import binding
    from paper_2104_07857_amd import build as zb
    if not zb.call_can_be_built():
        pytest.skip("no Python.h or no gcc: every call goes through ctypes")
    binding.lib()
    assert binding._call_epilogue is not binding._not_taken, zb.CALL_PATH + " is not built"
    return binding


def test_direct_calls_take_the_usual_forms(direct):
    a, args, back = _matrix(ROWS, COLS), _args(reserved=1), _back(reserved=1)
    for stream in (None, 0):
        assert direct._call_epilogue(16, ROWS, COLS, COLS, args, a, None, stream) == INVALID
        assert direct._call_matmul_epilogue(a, _matrix(5, COLS), args, None, a, None, None, stream) == INVALID
        assert direct._call_epilogue_backward(back, None, a, None, None, stream) == INVALID
    assert direct._call_epilogue(16, ROWS, 1.0, COLS, args, a, None, None) is None
    assert direct._call_epilogue(16, ROWS, COLS, COLS, a, a, None, None) is None          # another structure
    assert direct._call_epilogue(16, ROWS, COLS, COLS, args, args, None, None) is None
    assert direct._call_epilogue(16, ROWS, COLS, COLS, args, a, back, None) is None
    assert direct._call_matmul_epilogue(a, a, back, None, None, None, None, None) is None
    assert direct._call_matmul_epilogue(a, a, args, None, None, 16, None, None) is None   # an address without its bytes
    assert direct._call_epilogue_backward(args, None, None, None, None, None) is None
    assert direct._call_epilogue(args) is None and direct._call_epilogue_backward() is None


def test_both_ways_refuse_alike(direct, monkeypatch):
    calls = [lambda: _forward(_args(drop=2.0)), lambda: _product(_args(activation=9)), lambda: _backward(_back(drop=-1.0)), lambda: _forward(None)]

    def said():
        out = []
        for call in calls:
            with pytest.raises(zi.ZiError) as e:
                call()
            out.append((e.value.status, e.value.message))
        return out

    first = said()
    for name in ("_call_epilogue", "_call_matmul_epilogue", "_call_epilogue_backward"):
        monkeypatch.setattr(direct, name, direct._not_taken)
    assert said() == first


@pytest.mark.parametrize("name", ["residual", "z", "y", "bias", "d_offset"])
def test_arrays_that_do_not_hold_it_are_refused(name):
    torch = pytest.importorskip("torch")
    bf16 = torch.bfloat16
    wrong = {"bias": [torch.zeros(COLS - 1, dtype=bf16), torch.zeros(COLS), torch.zeros(2 * COLS, dtype=bf16)[::2]],
             "d_offset": [torch.zeros(1, dtype=torch.int32), torch.zeros(0, dtype=torch.int64), torch.zeros(1)]}
    for x in wrong.get(name, [_half(ROWS - 1, COLS), _half(ROWS, COLS - 1), _half(ROWS, 2 * COLS)[:, ::2], torch.zeros(ROWS, COLS)]):
        with pytest.raises(ValueError, match=name):
            zi.make_epilogue(ROWS, COLS, BF16, **{name: x})
    for x in wrong["bias"]:
        with pytest.raises(ValueError, match="dbias"):
            zi.make_epilogue_backward(_half(ROWS, COLS), None, None, x, BF16)
    with pytest.raises(ValueError, match="dbias"):
        zi.make_epilogue_backward(_half(ROWS, COLS), None, None, torch.zeros(COLS, dtype=bf16), BF16, dbias_dtype=zi.ZI_FP32)
    a = zi.make_epilogue(ROWS, COLS, BF16, d_offset=torch.zeros(1, dtype=torch.int64), bias=torch.zeros(COLS, dtype=bf16), seed=(1 << 64) - 1, offset=1 << 63)
    assert (a.seed, a.offset) == ((1 << 64) - 1, 1 << 63)


# ---- the generator ----------------------------------------------------------------------------------------------

@pytest.mark.parametrize("counter,key,want", [
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))])
def test_the_generators_published_values(counter, key, want):
    """The known answers that the generator's authors published with it pin the tests' own form of it."""
    from epilogue_util import philox
    assert tuple(int(w) for w in philox(counter, key)) == want


def test_share_of_what_is_dropped():
    from epilogue_util import kept, threshold
    for p in (0.1, 0.25, 0.5, 0.9):
        k = kept(64, 4096, p).double()
        n, q = k.numel(), threshold(p) / 65536
        assert abs(float(k.mean()) - (1 - q)) <= 5 * (q * (1 - q) / n) ** 0.5            # five standard deviations
        assert abs(float((k[:, 1:] * k[:, :-1]).mean()) - (1 - q) ** 2) <= 5 * (1 / n) ** 0.5
    assert threshold(0.0) == 0 == threshold(2.0 ** -18) and threshold(0.99999999) == 65535 and threshold(0.1) == 6554
    assert not np.array_equal(kept(8, 64, 0.5, offset=1).numpy(), kept(8, 64, 0.5, offset=2).numpy())
