"""What test_epilogue_codegen.py says of the product's tiles with an epilogue, of the sources of all three kinds of activation (no GPU needed)."""
import os
import shutil
import subprocess

import pytest

import test_epilogue_codegen as codegen
from paper_2104_07857_amd import build as zb
from test_fp8_codegen import _directive

KINDS = ["zi_fp8_matmul_floor.hip", "zi_fp8_matmul_sigmoid.hip", "zi_fp8_matmul_normal.hip"]


@pytest.fixture(scope="module")
def texts(tmp_path_factory):
    if shutil.which(zb.hipcc()) is None and not os.path.exists(zb.hipcc()):
        pytest.skip("no hipcc here")
    at = tmp_path_factory.mktemp("isa")
    flags = [f for f in zb.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    runs = [subprocess.Popen([zb.hipcc(), *flags, "-I", os.path.join(zb.ROOT, "include"), "-I", zb.CSRC, "-S", "--cuda-device-only", "-o", str(at / (s + ".s")),
                              os.path.join(zb.CSRC, s)], stdout=subprocess.DEVNULL, stderr=subprocess.DEVNULL) for s in KINDS]
    assert all(r.wait() == 0 for r in runs)
    return {s: (at / (s + ".s")).read_text() for s in KINDS}


@pytest.mark.parametrize("kind", KINDS)
def test_tiles_of_each_kind(texts, kind):
    codegen.test_tiles({"zi_fp8_matmul_sigmoid.hip": texts[kind]})
    codegen.test_no_atomics_and_no_packed_arithmetic({kind: texts[kind]})


def test_scratch_memory_of_the_largest_tiles(texts):
    """Of 256 x 256 with 8-bit outputs 40 bytes a thread at most, as the comment at the kernel says, and of no others any."""
    for text in texts.values():
        for key, body in codegen._kernels(text, "fp8_matmul_epilogue_kernel").items():
            assert _directive(body, "private_segment_fixed_size") <= (40 if key[1:3] == (4, 4) and key[4] > 0 else 0), key
