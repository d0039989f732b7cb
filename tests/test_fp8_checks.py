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
