"""The epilogues' kernels are a library of their own, which the first call that launches one loads: from the same folder and of the same build."""
import ctypes
import shutil
import subprocess

import pytest
import torch

import paper_2104_07857_amd as zi
from paper_2104_07857_amd import build as zb

pytestmark = pytest.mark.gpu
OK, ZI_ERR_HIP = 0, -4


def _relu(library, x):
    """zi_epilogue of another copy of libzi.so: its status, what it said, y."""
    rows, cols = x.shape
    y = torch.full_like(x, 7.0)
    args = zi.make_epilogue(rows, cols, zi.ZI_BF16, y=y, activation=zi.ZI_ACT_RELU)
    library.zi_last_error.restype = ctypes.c_char_p
    status = library.zi_epilogue(ctypes.c_void_p(x.data_ptr()), *map(ctypes.c_int64, (rows, cols, cols)), ctypes.byref(args), None, None, None)
    torch.cuda.synchronize()
    return status, library.zi_last_error().decode(), y


def _x():
    return (torch.arange(48, device="cuda:0") - 20).to(torch.bfloat16).view(3, 16)


# Another build's library: its table begins with what a call would go to.
STAND_IN = """
static int nothing(void) { return 0; }
static int (*const kernels[8])(void) = {nothing, nothing, nothing, nothing, nothing, nothing, nothing, nothing};
const void* zi_epilogue_kernels(void) { return kernels; }
"""


@pytest.mark.skipif(shutil.which("gcc") is None, reason="no gcc here")
def test_a_library_of_another_build_is_refused(tmp_path):
    (tmp_path / "stand_in.c").write_text(STAND_IN)
    subprocess.run(["gcc", "-shared", "-fPIC", "-o", str(tmp_path / "libzi_epilogue.so"), str(tmp_path / "stand_in.c")], check=True)
    other = ctypes.CDLL(shutil.copy(zi.LIB_PATH, tmp_path))
    for _ in range(2):
        status, said, y = _relu(other, _x())
        assert status == ZI_ERR_HIP and "libzi_epilogue.so" in said and "another build" in said, (status, said)
        assert bool((y == 7.0).all())


def test_a_load_that_failed_is_tried_again(tmp_path):
    """And it says what the loader said."""
    other = ctypes.CDLL(shutil.copy(zi.LIB_PATH, tmp_path))
    status, said, _ = _relu(other, _x())
    assert status == ZI_ERR_HIP and str(tmp_path / "libzi_epilogue.so") in said and "No such file" in said, (status, said)
    shutil.copy(zb.EPILOGUE_PATH, tmp_path)
    status, said, y = _relu(other, _x())
    assert status == OK, said
    assert torch.equal(y, _x().clamp_min(0))


def test_a_build_of_another_name_has_a_library_of_its_own(tmp_path):
    """libzi_more.so loads libzi_more_epilogue.so, and not the one of libzi.so beside it."""
    other = ctypes.CDLL(shutil.copy(zi.LIB_PATH, tmp_path / "libzi_more.so"))
    shutil.copy(zb.EPILOGUE_PATH, tmp_path)
    status, said, _ = _relu(other, _x())
    assert status == ZI_ERR_HIP and "libzi_more_epilogue.so" in said, (status, said)
    shutil.copy(zb.EPILOGUE_PATH, tmp_path / "libzi_more_epilogue.so")
    status, said, y = _relu(other, _x())
    assert status == OK and torch.equal(y, _x().clamp_min(0)), said
