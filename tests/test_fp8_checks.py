"""What the 8-bit operators check of sizes and places before anything is launched (no GPU needed): the sizes themselves, not what
is left of them in 64 bits."""
import pytest

import paper_2104_07857_amd as zi
from test_fp8_host import BF16, INVALID, UNSUPPORTED, _half, _matrix, _refused

GIB = 1 << 30


def _at(rows, cols, block_rows=1, at=256 * GIB, **over):
    """A matrix in 8 bits at addresses that nothing is at: whatever passes the checks ends at the query for its memory."""
    m = zi.zi_fp8_matrix(at, at + 128 * GIB, rows, cols, -(-cols // 16) * 16, -(-cols // 512) * 4, block_rows, 0)
    for k, v in over.items():
        setattr(m, k, v)
    return m


# (rows - 1) * pitch + pitch is 0, or small, or less than nothing, in 64 bits
@pytest.mark.parametrize("rows,pitch", [(1 << 26, 1 << 38), (1 << 24, 1 << 40), (1 << 25, 1 << 38), ((1 << 26) + 1, 1 << 38), (1 << 30, 1 << 34)])
@pytest.mark.parametrize("field", ["ld", "scale_ld"])
def test_the_product_of_rows_and_pitch_is_bounded(rows, pitch, field):
    bad = _at(rows, 8, **{field: pitch})
    _refused(UNSUPPORTED, "2^40", zi.zi_fp8_quantize, 16 * GIB, BF16, rows, 8, 8, bad)
    _refused(UNSUPPORTED, "2^40", zi.zi_fp8_quantize, 16 * GIB, BF16, 8, rows, rows, None, bad)
    args = zi.zi_rms_norm_args(16 * GIB, None, 8 * GIB, None, None, None, rows, 8, 8, 0, 0, 0, 1e-5, BF16)
    _refused(UNSUPPORTED, "2^40", zi.zi_rms_norm, args, bad)
    _refused(UNSUPPORTED, "2^40", zi.zi_fp8_matmul, bad, _matrix(4, 8), _half(4, 4), BF16, 4)
    _refused(UNSUPPORTED, "2^40", zi.zi_fp8_matmul, _matrix(4, 8), bad, _half(4, 4), BF16, rows)


@pytest.mark.parametrize("field,pitch", [("ld", 1 << 40), ("scale_ld", 1 << 40)])
def test_rows_of_scales_are_what_counts_for_them(field, pitch):
    """One row of scales for 128 rows may have any pitch; rows of numbers may not."""
    x, m = _half(100, 8), _at(100, 8, 128, **{field: pitch})
    if field == "ld":
        _refused(UNSUPPORTED, "2^40", zi.zi_fp8_quantize, x, BF16, 100, 8, 8, m)
    else:
        with pytest.raises(zi.ZiError) as e:
            zi.zi_fp8_quantize(x, BF16, 100, 8, 8, m)
        assert e.value.status in (zi.ZI_ERR_HIP, INVALID) and "2^40" not in e.value.message


@pytest.mark.parametrize("rows,cols", [(1 << 31, 1), ((1 << 31) - 127, 1), (1 << 30, 129), (1 << 19, 1 << 19)])
def test_a_launch_of_two_to_the_32_threads_is_refused(rows, cols):
    """2^24 tiles of 256 threads are one thread more than a launch has."""
    _refused(UNSUPPORTED, "tiles", zi.zi_fp8_quantize, 16 * GIB, BF16, rows, cols, cols, None, _at(cols, rows))
    _refused(UNSUPPORTED, "tiles", zi.zi_fp8_quantize, 16 * GIB, BF16, rows, cols, cols, _at(rows, cols))


def test_one_tile_less_is_not():
    rows = (1 << 31) - 128
    x = _half(4, 4)
    with pytest.raises(zi.ZiError) as e:
        zi.zi_fp8_quantize(x, BF16, rows, 1, 1, None, _at(1, rows))
    assert e.value.status in (zi.ZI_ERR_HIP, INVALID) and "tiles" not in e.value.message


# ---- arrays that lie between each other's rows ------------------------------------------------------------------

def _said(call, *args):
    with pytest.raises(zi.ZiError) as e:
        call(*args)
    assert e.value.status in (zi.ZI_ERR_HIP, INVALID)
    return e.value.message


def _norm_at(x, x_ld, y, y_ld, rows, cols):
    """Of the addresses alone: rows x cols of x and y, pitches in elements."""
    return _said(zi.zi_rms_norm, zi.zi_rms_norm_args(x, None, 8 * GIB, None, y, None, rows, cols, x_ld, 0, 0, y_ld, 1e-5, BF16))


def test_overlap_is_bytes_that_are_shared():
    """Against all bytes of both, for rows of the same pitch, in any place."""
    shared = {False: 0, True: 0}
    for rows in (1, 2, 3):
        for ld in (3, 5, 8):
            for cols in (1, 2, 3):
                mine = {2 * (i * ld + j) + b for i in range(rows) for j in range(cols) for b in (0, 1)}
                for at in range(-2 * rows * ld - 4, 2 * rows * ld + 6, 2):
                    meet = any(b + at in mine for b in mine)
                    says = "overlap" in _norm_at(16 * GIB, ld, 16 * GIB + at, ld, rows, cols)
                    assert says == (meet and at != 0), (rows, ld, cols, at)          # (y may be x)
                    shared[meet] += 1
    assert min(shared.values()) > 100


def test_rows_of_two_pitches():
    """Bytes that are shared are always found; slices of one buffer whose rows are every one and every other are apart."""
    for rows in (2, 3):
        for p, q in ((4, 8), (8, 4), (6, 4), (5, 7), (3, 9)):
            for cols in (1, 2, 3):
                for at in range(-2 * rows * q - 2, 2 * rows * p + 4, 2):
                    x = {2 * (i * p + j) + b for i in range(rows) for j in range(cols) for b in (0, 1)}
                    y = {2 * (i * q + j) + b + at for i in range(rows) for j in range(cols) for b in (0, 1)}
                    if x & y:
                        assert "overlap" in _norm_at(16 * GIB, p, 16 * GIB + at, q, rows, cols), (rows, p, q, cols, at)
    assert "overlap" not in _norm_at(16 * GIB, 100, 16 * GIB + 100, 200, 4, 50)
    assert "overlap" in _norm_at(16 * GIB, 100, 16 * GIB + 98, 200, 4, 50)


def test_columns_and_rows_of_one_buffer_are_apart():
    wide = _half(8, 400)
    at = lambda col, row=0: wide.ctypes.data + 2 * (row * 400 + col)                     # noqa: E731
    q, k = at(0), at(100)
    assert "overlap" not in _norm_at(q, 400, k, 400, 8, 100)
    assert "overlap" in _norm_at(q, 400, at(99), 400, 8, 100)
    assert "overlap" not in _norm_at(at(0), 800, at(0, 1), 800, 4, 400)                  # even rows, odd rows
    a, b = _matrix(8, 100), _matrix(100, 100)
    f = zi.zi_fp8_matmul
    assert "overlap" not in _said(f, a, b, q, BF16, 400, k)                              # D and C side by side
    assert "overlap" in _said(f, a, b, q, BF16, 400, at(99))
    assert "overlap" in _said(zi.zi_fp8_quantize, wide, BF16, 8, 100, 400, _matrix(8, 100, data=at(104), ld=800))      # an output in 8 bits
    args = zi.zi_rms_norm_backward_args(at(0), at(100), 8 * GIB, 9 * GIB, None, at(200), at(300), 8, 100, 400, 400, 0, 400, BF16, BF16, 0, 0)
    assert "overlap" not in _said(zi.zi_rms_norm_backward, args, 10 * GIB, 1 << 20)      # one row, of dgamma, beside them too


def test_8_bit_operands_are_columns_of_one_buffer():
    """A matrix holds the bytes of its columns, up to a multiple of 16 (of its scales, of 4): none behind them in its last row, and, where it is
    an input, none between its rows."""
    wide, scales = _matrix(6, 256), _matrix(6, 4096)
    one = lambda col, at=0: _matrix(6, 100, data=wide.data + col, ld=256, scale=scales.scale + at, scale_ld=32)           # noqa: E731
    f = lambda d, ldd=128: _said(zi.zi_fp8_matmul, one(0), one(128, 4), d, BF16, ldd)                                    # noqa: E731
    assert "overlap" not in f(wide.data + 112) and "overlap" not in f(wide.data + 240)       # D between the operands' columns, and behind them
    assert "a's data" in f(wide.data + 110) and "b's data" in f(wide.data + 128 - 10)
    assert "overlap" not in f(scales.scale + 8, 16) and "scale" in f(scales.scale + 6, 16)
    end = wide.data + 5 * 256 + 128 + 112
    x = _half(6, 100)
    args = lambda rstd: zi.zi_rms_norm_args(x.ctypes.data, None, 8 * GIB, None, None, rstd, 6, 100, 100, 0, 0, 0, 1e-5, BF16)      # noqa: E731
    assert "overlap" not in _said(zi.zi_rms_norm, args(end), one(128))                   # right behind the last column slice
    assert "y8's data" in _said(zi.zi_rms_norm, args(end - 4), one(128))                 # in what its columns are rounded up to
    assert "y8's data" in _said(zi.zi_rms_norm, args(end - 40 - 256), one(128))          # between rows of an output
