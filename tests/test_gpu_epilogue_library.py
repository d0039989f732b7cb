"""The epilogues' kernels are a library of their own, which the first call that launches one loads: from the same folder and of the same build, also
while a graph is captured."""
import ctypes
import os
import shutil
import subprocess
import sys

import pytest
import torch

import paper_2104_07857_amd as zi
from conftest import ROOT
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


# The first call of a process, made while a graph is captured: nothing of the kernels was loaded before.
CODE = """
import sys
sys.path[:0] = [{root!r}, {tests!r}]
import torch
import paper_2104_07857_amd as zi
from fp8_util import Matrix, normal

def loaded():
    return any("libzi_epilogue.so" in line for line in open("/proc/self/maps"))

call = {call!r}
m, n, k = 40, 200, 16384                        # a product in parts of k: two kernels
x, dy = normal((m, n), 1, 1.0, torch.bfloat16), normal((m, n), 2, 1.0, torch.bfloat16)
a, b = Matrix(m, k), Matrix(n, k, 128)
for q in (a, b):
    q.data.fill_(0x30)
    q.scale.fill_(120)
y, dbias = torch.empty_like(x), torch.empty(n, device="cuda:0")
y8, turned = Matrix(m, n), Matrix(n, m)
forward = zi.make_epilogue(m, n, zi.ZI_BF16, residual=dy, y=y, activation=zi.ZI_ACT_GELU, drop=0.1, seed=1)
backward = zi.make_epilogue_backward(dy, x, y, dbias, zi.ZI_BF16, activation=zi.ZI_ACT_GELU, drop=0.1, seed=1, dbias_dtype=zi.ZI_FP32)
ws = torch.empty(max(zi.zi_epilogue_workspace_bytes(m, n), zi.zi_fp8_matmul_epilogue_workspace_bytes(m, n, k, 3)), dtype=torch.uint8, device="cuda:0")

def go(stream):
    if call == "epilogue":
        zi.zi_epilogue(x, m, n, n, forward, y8.struct, turned.struct, stream)
    elif call == "matmul":
        zi.zi_fp8_matmul_epilogue(a.struct, b.struct, forward, y8.struct, turned.struct, ws, stream=stream)
    else:
        zi.zi_epilogue_backward(backward, y8.struct, turned.struct, ws, stream=stream)

def outputs():
    torch.cuda.synchronize()
    return [t.clone() for t in (y, y8.codes(), y8.scales(), turned.codes(), turned.scales())] + ([dbias.clone()] if call == "backward" else [])

def clear():
    for t in (y, y8.data, y8.scale, turned.data, turned.scale, dbias):
        t.zero_()

torch.cuda.synchronize()
assert not loaded()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    go(torch.cuda.current_stream())
assert loaded()
go(None)
want = outputs()
assert bool(want[0].any()) and bool(want[1].any()) and bool(want[3].any())
for _ in range(3):
    clear()
    g.replay()
    assert all(torch.equal(p, q) for p, q in zip(outputs(), want))
    clear()
    go(None)
    assert all(torch.equal(p, q) for p, q in zip(outputs(), want))
print("as they should be", flush=True)
"""


@pytest.mark.parametrize("call", ["epilogue", "matmul", "backward"])
def test_the_first_call_may_be_captured(call):
    code = CODE.format(root=ROOT, tests=os.path.join(ROOT, "tests"), call=call)
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0 and "as they should be" in r.stdout, r.stdout + r.stderr
