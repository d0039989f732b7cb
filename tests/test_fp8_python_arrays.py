"""The structures that Python makes of arrays: arrays that do not hold what the call would read or write there are refused."""
import numpy as np
import pytest

import paper_2104_07857_amd as zi
from test_fp8_host import BF16, _bytes, _half

torch = pytest.importorskip("torch")
ROWS, COLS = 4, 100


def _norm(x=None, gamma=None, **kw):
    return zi.make_rms_norm(_half(ROWS, COLS) if x is None else x, _half(1, COLS)[0] if gamma is None else gamma, BF16, 1e-5, **kw)


def _f32(n):
    return _bytes(4 * n).view(np.float32)


def _backward(**kw):
    given = dict(dy=_half(ROWS, COLS), h=_half(ROWS, COLS), gamma=_half(1, COLS)[0], rstd=_f32(ROWS), dx=_half(ROWS, COLS), dgamma=_half(1, COLS)[0])
    given.update(kw)
    return zi.make_rms_norm_backward(dtype=BF16, **given)


WRONG_MATRIX = [lambda: _half(ROWS - 1, COLS), lambda: _half(ROWS, COLS - 1), lambda: _half(ROWS, 2 * COLS)[:, ::2], lambda: _half(1, ROWS * COLS)[0],
                lambda: _f32(ROWS * COLS).reshape(ROWS, COLS), lambda: torch.zeros(ROWS, COLS), lambda: torch.zeros(COLS, ROWS, dtype=torch.bfloat16).t()]
WRONG_VECTOR = [lambda: _half(1, 2 * COLS)[0][::2], lambda: _half(1, COLS - 1)[0], lambda: _f32(COLS), lambda: torch.zeros(2 * COLS, dtype=torch.bfloat16)[::2],
                lambda: torch.zeros(COLS), lambda: torch.zeros(1, dtype=torch.bfloat16).expand(COLS)]


@pytest.mark.parametrize("wrong", WRONG_MATRIX)
def test_matrices_of_another_shape_type_or_order(wrong):
    for name in ("residual", "sum", "y"):
        with pytest.raises(ValueError, match=name):
            _norm(**{name: wrong()})
    for name in ("h", "dsum", "dx"):
        with pytest.raises(ValueError, match=name):
            _backward(**{name: wrong()})


@pytest.mark.parametrize("wrong", WRONG_VECTOR)
def test_vectors_that_are_short_strided_or_of_another_type(wrong):
    with pytest.raises(ValueError, match="gamma"):
        _norm(gamma=wrong())
    for name in ("gamma", "dgamma"):
        with pytest.raises(ValueError, match=name):
            _backward(**{name: wrong()})


@pytest.mark.parametrize("wrong", [lambda: _f32(ROWS - 1), lambda: _f32(2 * ROWS)[::2], lambda: np.zeros(ROWS), lambda: _half(1, ROWS)[0]])
def test_rstd(wrong):
    for make in (_norm, _backward):
        with pytest.raises(ValueError, match="rstd"):
            make(rstd=wrong())


def test_dgamma_is_of_its_own_type():
    assert _backward(dgamma=_f32(COLS), dgamma_dtype=zi.ZI_FP32).dgamma_dtype == zi.ZI_FP32
    for given, dtype in ((_f32(COLS), None), (_half(1, COLS)[0], zi.ZI_FP32)):
        with pytest.raises(ValueError, match="dgamma"):
            _backward(dgamma=given, dgamma_dtype=dtype)


def test_what_holds_it_is_taken():
    """Views, longer and larger ones, a row or a column as a vector, addresses."""
    wide = torch.zeros((ROWS + 2, COLS + 20), dtype=torch.bfloat16)
    a = _norm(wide[:ROWS, 3:3 + COLS], wide[0], residual=wide, sum=wide[1:], y=wide[:, 20:], rstd=torch.zeros(ROWS + 1))
    assert (a.rows, a.cols, a.x_ld, a.residual_ld, a.gamma) == (ROWS, COLS, COLS + 20, COLS + 20, wide.data_ptr())
    b = _backward(gamma=wide.data_ptr(), rstd=16, dgamma=None, dx=None, dsum=wide)
    assert (b.gamma, b.rstd, b.dgamma, b.dx, b.dsum_ld) == (wide.data_ptr(), 16, None, None, COLS + 20)
    one = torch.zeros((7, 1), dtype=torch.bfloat16)
    assert zi.make_rms_norm(one, one[0], BF16, 1e-5, y=one, rstd=torch.zeros((7, 1))).rows == 7
    assert zi.make_rms_norm(wide[:0], wide[0], BF16, 1e-5, y=wide[:0], rstd=torch.zeros(0)).rows == 0


def test_8_bit_matrices():
    data, scale = (_bytes(*s) for s in zi.fp8_layout(ROWS, 300))
    assert zi.make_fp8_matrix(data, scale, ROWS, 300).ld == 384
    assert zi.make_fp8_matrix(data, scale, ROWS - 1, 200).cols == 200
    assert zi.make_fp8_matrix(data.ctypes.data, scale.ctypes.data, 99, 300, ld=384, scale_ld=4).rows == 99       # addresses: the caller's word
    wrong = [(data, scale, ROWS + 1, 300), (data, scale, ROWS, 385), (data[:, :256], scale, ROWS, 300), (data, scale[:2], ROWS, 300),
             (data, scale[:, :2], ROWS, 300), (data[:, ::2], scale, ROWS, 100), (data.view(np.uint16), scale, ROWS, 100),
             (torch.zeros(ROWS, 384), scale, ROWS, 300), (data[0], scale, 1, 300)]
    for args in wrong:
        with pytest.raises(ValueError):
            zi.make_fp8_matrix(*args)
    squares = _bytes(1, 4)
    assert zi.make_fp8_matrix(data, squares, ROWS, 300, 128).block_rows == 128
