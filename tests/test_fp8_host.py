"""The 8-bit operators without a GPU: layouts, what they refuse and in which words, calls that have nothing to do."""
import ctypes

import numpy as np
import pytest

import paper_2104_07857_amd as zi

BF16, INVALID, ALIGN, UNSUPPORTED = zi.ZI_BF16, zi.ZI_ERR_INVALID_ARG, zi.ZI_ERR_ALIGNMENT, zi.ZI_ERR_UNSUPPORTED


def _bytes(*shape):
    """Zeroed bytes, 64-byte aligned."""
    n = int(np.prod(shape))
    raw = np.zeros(n + 64, np.uint8)
    at = -raw.ctypes.data % 64
    return raw[at:at + n].reshape(shape)


def _matrix(n_rows, n_cols, blocks=1, **over):
    data, scale = (_bytes(*s) for s in zi.fp8_layout(n_rows, n_cols, blocks))
    x = zi.make_fp8_matrix(data, scale, n_rows, n_cols, blocks)
    x.keep = (data, scale)
    for k, v in over.items():
        setattr(x, k, v)
    return x


def _half(rows, cols):
    return _bytes(rows, 2 * cols).view(np.uint16)


def _refused(status, word, call, *args, **kw):
    with pytest.raises(zi.ZiError) as e:
        call(*args, **kw)
    assert e.value.status == status and word in e.value.message, (e.value.status, e.value.message)


def test_struct_sizes_and_layout():
    assert ctypes.sizeof(zi.zi_fp8_matrix) == 56
    assert ctypes.sizeof(zi.zi_rms_norm_args) == 104
    assert ctypes.sizeof(zi.zi_rms_norm_backward_args) == 120
    assert zi.fp8_layout(5, 129) == ((5, 256), (5, 4))
    assert zi.fp8_layout(129, 1000, 128) == ((129, 1024), (2, 8))
    assert zi.zi_rms_norm_workspace_bytes(0, 64) == 0 == zi.zi_rms_norm_workspace_bytes(4, 65537)
    assert zi.zi_rms_norm_workspace_bytes(10, 64) >= 64 * 4
    m = zi.make_fp8_matrix(_bytes(1, 48), _bytes(1, 4), 1, 40)
    assert (m.ld, m.scale_ld, m.cols) == (48, 4, 40)
    with pytest.raises(ValueError):
        zi.make_rms_norm(_half(4, 8)[:, ::2], _half(1, 4)[0], BF16, 1e-5)


@pytest.mark.parametrize("over,status,word", [
    (dict(block_rows=64), INVALID, "block_rows"), (dict(reserved=1), INVALID, "reserved"), (dict(rows=-1), INVALID, "< 0"),
    (dict(data=None), INVALID, "NULL"), (dict(scale=None), INVALID, "NULL"), (dict(ld=96), INVALID, "pitch"),
    (dict(ld=136), ALIGN, "multiple of 16"), (dict(scale_ld=0), INVALID, "pitch"), (dict(scale_ld=6), ALIGN, "scale_ld"),
    (dict(rows=(1 << 40) + 1), INVALID, "2^40")])
def test_matrices_are_checked(over, status, word):
    good, bad = _matrix(4, 100), _matrix(4, 100, **over)
    d = _half(4, 4)
    _refused(status, word, zi.zi_fp8_matmul, bad, good, d, BF16, 4)
    _refused(status, word, zi.zi_fp8_matmul, good, bad, d, BF16, 4)
    _refused(status, word, zi.zi_fp8_quantize, _half(4, 100), BF16, 4, 100, 100, bad)
    _refused(status, word, zi.zi_fp8_quantize, _half(100, 4), BF16, 100, 4, 4, None, bad)
    args = zi.make_rms_norm(_half(4, 100), _half(1, 100)[0], BF16, 1e-5)
    _refused(status, word, zi.zi_rms_norm, args, bad)


def test_addresses_have_to_be_aligned():
    for field, by in (("data", 8), ("scale", 1)):
        bad = _matrix(4, 100)
        setattr(bad, field, getattr(bad, field) + by)
        _refused(ALIGN, "aligned", zi.zi_fp8_matmul, bad, _matrix(4, 100), _half(4, 4), BF16, 4)
    x = _half(8, 100)
    _refused(ALIGN, "element", zi.zi_fp8_quantize, x.ctypes.data + 1, BF16, 4, 100, 100, _matrix(4, 100))
    _refused(ALIGN, "element", zi.zi_fp8_quantize, x.ctypes.data + 2, zi.ZI_FP32, 4, 50, 50, _matrix(4, 50))
    _refused(ALIGN, "2-byte", zi.zi_fp8_matmul, _matrix(4, 100), _matrix(4, 100), x.ctypes.data + 1, BF16, 4)


def test_quantize_refuses():
    x, out = _half(4, 100), _matrix(4, 100)
    q = zi.zi_fp8_quantize
    _refused(INVALID, "dtype", q, x, 3, 4, 100, 100, out)
    _refused(INVALID, "neither", q, x, BF16, 4, 100, 100)
    _refused(INVALID, "rows", q, x, BF16, -1, 100, 100, out)
    _refused(INVALID, "out is not", q, x, BF16, 3, 100, 100, out)
    _refused(INVALID, "turned is not", q, x, BF16, 4, 100, 100, None, out)
    _refused(INVALID, "pitch of x", q, x, BF16, 4, 100, 99, out)
    _refused(INVALID, "x is NULL", q, None, BF16, 4, 100, 100, out)
    _refused(INVALID, "overlap", q, out.data, BF16, 4, 100, 100, out)
    _refused(INVALID, "overlap", q, x, BF16, 4, 4, 100, _matrix(4, 4, data=out.data), _matrix(4, 4, data=out.data + 16))


def test_matmul_refuses():
    a, b, d = _matrix(4, 100), _matrix(6, 100), _half(4, 6)
    f = zi.zi_fp8_matmul
    _refused(INVALID, "dtype", f, a, b, d, zi.ZI_FP32, 6)
    _refused(INVALID, "NULL", f, None, b, d, BF16, 6)
    _refused(INVALID, "d is NULL", f, a, b, None, BF16, 6)
    _refused(INVALID, "columns", f, a, _matrix(6, 101), d, BF16, 6)
    _refused(INVALID, "pitch of d", f, a, b, d, BF16, 5)
    _refused(INVALID, "overlap", f, a, b, a.data, BF16, 6)
    _refused(INVALID, "overlap", f, a, b, d, BF16, 6, c=d.ctypes.data + 2)
    _refused(UNSUPPORTED, "pitch", f, _matrix(4, 100, ld=1 << 23), b, d, BF16, 6)
    _refused(UNSUPPORTED, "2^26", f, _matrix(4, 16), _matrix(4, 16, rows=1 << 27), d, BF16, 1 << 27)


def test_matmul_workspace():
    """What is asked for has to be there; where k is not shared out nothing is."""
    m, n, k = 64, 128, 16384
    nbytes = zi.zi_fp8_matmul_workspace_bytes(m, n, k)
    assert nbytes > 0 and nbytes % (m * n * 4) == 0
    assert zi.zi_fp8_matmul_workspace_bytes(4096, 4096, 4096) == 0 == zi.zi_fp8_matmul_workspace_bytes(0, n, k) == zi.zi_fp8_matmul_workspace_bytes(m, n, 0)
    a, b, d, ws = _matrix(m, k), _matrix(n, k, 128), _half(m, n), _bytes(nbytes)
    f = zi.zi_fp8_matmul
    _refused(INVALID, "workspace", f, a, b, d, BF16, n)
    _refused(INVALID, "workspace", f, a, b, d, BF16, n, None, ws.ctypes.data, nbytes - 4)
    _refused(ALIGN, "d_workspace", f, a, b, d, BF16, n, None, ws.ctypes.data + 4, nbytes)
    _refused(INVALID, "overlap", f, a, b, d, BF16, n, None, a.data, nbytes)


def test_norm_refuses():
    x, gamma, y = _half(4, 100), _half(1, 100)[0], _half(4, 100)
    make = lambda **kw: zi.make_rms_norm(x, gamma, BF16, kw.pop("eps", 1e-5), **{"y": y, **kw})       # noqa: E731

    def over(**kw):
        a = make()
        for k, v in kw.items():
            setattr(a, k, v)
        return a

    f = zi.zi_rms_norm
    _refused(INVALID, "args", f, None)
    _refused(INVALID, "dtype", f, over(dtype=2))
    for eps in (-1.0, float("nan"), float("inf")):
        _refused(INVALID, "eps", f, make(eps=eps))
    _refused(INVALID, "cols is 0", f, over(cols=0))
    _refused(UNSUPPORTED, "65536", f, over(cols=65537))
    _refused(INVALID, "no output", f, make(y=None))
    _refused(INVALID, "residual", f, make(sum=_half(4, 100)))
    _refused(INVALID, "y8 is not", f, make(), _matrix(3, 100))
    _refused(INVALID, "block_rows", f, make(), _matrix(4, 100, 128))
    _refused(INVALID, "x and gamma", f, over(gamma=None))
    _refused(INVALID, "pitch of x", f, over(x_ld=99))
    _refused(ALIGN, "rstd", f, over(rstd=gamma.ctypes.data + 2))
    _refused(ALIGN, "y must", f, over(y=y.ctypes.data + 1))
    _refused(INVALID, "overlap", f, over(y=x.ctypes.data + 2))
    _refused(INVALID, "overlap", f, over(y=gamma.ctypes.data))
    _refused(INVALID, "overlap", f, over(y=x.ctypes.data, y_ld=101))         # the same place, but another pitch


def test_backward_refuses():
    dy, h, gamma, rstd, dx, dgamma = _half(4, 100), _half(4, 100), _half(1, 100)[0], _bytes(16).view(np.float32), _half(4, 100), _half(1, 100)[0]
    ws = _bytes(zi.zi_rms_norm_workspace_bytes(4, 100))

    def over(**kw):
        a = zi.make_rms_norm_backward(dy, h, gamma, rstd, dx, dgamma, BF16)
        for k, v in kw.items():
            setattr(a, k, v)
        return a

    f = lambda a, w=ws, n=ws.nbytes: zi.zi_rms_norm_backward(a, w, n)                                # noqa: E731
    _refused(INVALID, "args", f, None)
    _refused(INVALID, "dtype", f, over(dtype=2))
    _refused(INVALID, "dgamma_dtype", f, over(dgamma_dtype=zi.ZI_FP16))
    _refused(INVALID, "reserved", f, over(reserved=3))
    _refused(INVALID, "no output", f, over(dx=None, dgamma=None))
    _refused(INVALID, "must not be NULL", f, over(rstd=None))
    _refused(INVALID, "cols is 0", f, over(cols=0))
    _refused(UNSUPPORTED, "65536", f, over(cols=70000))
    _refused(INVALID, "pitch of dx", f, over(dx_ld=7))
    _refused(INVALID, "workspace", f, over(), None, 0)
    _refused(INVALID, "workspace", f, over(), ws, ws.nbytes - 4)
    _refused(ALIGN, "d_workspace", f, over(), ws.ctypes.data + 4)
    _refused(ALIGN, "dgamma", f, over(dgamma_dtype=zi.ZI_FP32, dgamma=dgamma.ctypes.data + 2))
    _refused(INVALID, "overlap", f, over(dx=h.ctypes.data))
    _refused(INVALID, "overlap", f, over(dx=dy.ctypes.data + 2))
    _refused(INVALID, "overlap", f, over(dgamma=gamma.ctypes.data))


def test_sizes_of_zero_do_nothing():
    """Also with no GPU: there is nothing to reach."""
    empty, none = _matrix(0, 100), zi.zi_fp8_matrix(None, None, 4, 0, 0, 0, 1, 0)
    assert zi.zi_fp8_quantize(None, BF16, 0, 100, 100, empty) == zi.ZI_OK
    assert zi.zi_fp8_quantize(None, BF16, 4, 0, 0, none) == zi.ZI_OK
    assert zi.zi_fp8_matmul(empty, _matrix(4, 100), None, BF16, 4) == zi.ZI_OK
    args = zi.make_rms_norm(_half(4, 100), _half(1, 100)[0], BF16, 1e-5, y=_half(4, 100))
    args.rows = 0
    assert zi.zi_rms_norm(args) == zi.ZI_OK


def test_ordinary_host_memory_is_an_error_and_no_fault():
    """With a GPU ordinary memory is refused, without one there is no device to ask."""
    with pytest.raises(zi.ZiError) as e:
        zi.zi_fp8_matmul(_matrix(4, 100), _matrix(4, 100), _half(4, 4), BF16, 4)
    assert e.value.status in (zi.ZI_ERR_HIP, INVALID)
    with pytest.raises(zi.ZiError) as e:
        zi.zi_fp8_quantize(_half(4, 100), BF16, 4, 100, 100, _matrix(4, 100))
    assert e.value.status in (zi.ZI_ERR_HIP, INVALID)


@pytest.fixture
def direct():
    from paper_2104_07857_amd import binding
    from paper_2104_07857_amd import build as zb
    if not zb.call_can_be_built():
        pytest.skip("no Python.h or no gcc: every call goes through ctypes")
    binding.lib()
    assert binding._call_matmul is not binding._not_taken, zb.CALL_PATH + " is not built"
    return binding


def test_direct_calls_take_the_usual_forms(direct):
    """A status for them (these are all refused), None for what the general way has to look at."""
    a, args = _matrix(4, 100), zi.make_rms_norm(_half(4, 100), _half(1, 100)[0], BF16, 1e-5)
    back = zi.zi_rms_norm_backward_args()
    torch = pytest.importorskip("torch")
    ws = torch.zeros(64, dtype=torch.uint8)
    for stream in (None, 0):
        assert direct._call_quantize(None, 3, 4, 100, 100, a, None, stream) == INVALID
        assert direct._call_matmul(a, None, 16, 0, 4, None, ws, None, stream) == INVALID
        assert direct._call_rms_norm(args, None, stream) == INVALID
        assert direct._call_rms_norm_backward(back, None, None, stream) == INVALID
        assert direct._call_rms_norm_backward(back, ws, 64, stream) == INVALID
    x = _half(4, 100)
    assert direct._call_quantize(x, 0, 4, 100, 100, a, None, None) is None             # a numpy array's address
    assert direct._call_quantize(16, 0.0, 4, 100, 100, a, None, None) is None
    assert direct._call_matmul(args, a, 16, 0, 4, None, None, None, None) is None      # another structure
    assert direct._call_matmul(a, args, 16, 0, 4, None, None, None, None) is None
    assert direct._call_matmul(a, a, 16, 0, 4, None, 16, None, None) is None           # an address without its bytes
    assert direct._call_rms_norm(a, None, None) is None and direct._call_rms_norm(args, back, None) is None
    assert direct._call_rms_norm_backward(args, None, None, None) is None
    assert direct._call_rms_norm(args) is None and direct._call_matmul(a, a) is None


def test_both_ways_refuse_alike(direct, monkeypatch):
    a, args = _matrix(4, 100), zi.make_rms_norm(_half(4, 100), _half(1, 100)[0], BF16, 1e-5)
    calls = [lambda: zi.zi_fp8_quantize(16, 0, 4, 100, 99, a), lambda: zi.zi_fp8_matmul(a, _matrix(6, 101), 16, 0, 6), lambda: zi.zi_rms_norm(args),
             lambda: zi.zi_rms_norm_backward(zi.zi_rms_norm_backward_args())]

    def said():
        out = []
        for call in calls:
            with pytest.raises(zi.ZiError) as e:
                call()
            out.append((e.value.status, e.value.message))
        return out

    first = said()
    for name in ("_call_quantize", "_call_matmul", "_call_rms_norm", "_call_rms_norm_backward"):
        monkeypatch.setattr(direct, name, direct._not_taken)
    assert said() == first
