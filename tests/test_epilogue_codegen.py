"""Properties of the compiled kernels of what follows a product that their speed or their safety depends on, read from the assembly hipcc emits for the library's own sources (no GPU
needed): no scratch memory but little of it in the largest tiles with 8-bit outputs, and none where k is gone through; a step of the product as test_fp8_codegen.py has it; no atomics and no
packed fp32 arithmetic; registers for as many workgroups on a compute unit as the kernels are made for."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2104_07857_amd import build as zb
from test_fp8_codegen import LDS_OF_A_COMPUTE_UNIT, _directive, _instructions, _stretches

SOURCES = ["zi_fp8_matmul_sigmoid.hip", "zi_fp8_matmul_epilogue.hip", "zi_epilogue_rows.hip", "zi_epilogue_tiles.hip", "zi_epilogue_backward.hip"]


@pytest.fixture(scope="module")
def texts(tmp_path_factory):
    if shutil.which(zb.hipcc()) is None and not os.path.exists(zb.hipcc()):
        pytest.skip("no hipcc here")
    at = tmp_path_factory.mktemp("isa")
    flags = [f for f in zb.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    runs = [subprocess.Popen([zb.hipcc(), *flags, "-I", os.path.join(zb.ROOT, "include"), "-I", zb.CSRC, "-S", "--cuda-device-only", "-o", str(at / (s + ".s")),
                              os.path.join(zb.CSRC, s)], stdout=subprocess.DEVNULL, stderr=subprocess.DEVNULL) for s in SOURCES]
    assert all(r.wait() == 0 for r in runs)
    return {s: (at / (s + ".s")).read_text() for s in SOURCES}


def _kernels(text, name):
    """Bodies by the numbers among their template arguments."""
    found = {}
    for mt in re.finditer(r"^_ZN2zi\d+%sI(\S+?)EE?v\S+:" % name, text, re.M):
        key = tuple(-int(x[1:]) if x[0] == "n" else int(x) for x in re.findall(r"L(?:[ib]|NS_\d+[A-Z]\w+?E)(n?\d+)E", mt.group(1) + "E"))
        found[key] = text[mt.end():text.index(".end_amdhsa_kernel", mt.end())]
    return found


def test_tiles(texts):
    kernels = _kernels(texts["zi_fp8_matmul_sigmoid.hip"], "fp8_matmul_epilogue_kernel")
    assert len(kernels) == 32, sorted(kernels)      # {bf16, fp16} x (six tiles, five of them with 8-bit outputs too, with z and without)
    for key, body in kernels.items():
        _, fm, fn, ring, outputs = key[:5]
        together = 1 if ring * (fm + fn) > 8 else 2
        assert _directive(body, "private_segment_fixed_size") <= (64 if (fm, fn) == (4, 4) and outputs > 0 else 0), key
        assert _directive(body, "group_segment_fixed_size") * together <= LDS_OF_A_COMPUTE_UNIT, key
        assert _directive(body, "next_free_vgpr") <= 512 // together, key
        multiply = [s for s in _stretches(body) if any(x.startswith("v_mfma") for x in s)]
        steps = [s for s in multiply if any(x.endswith(" lds") for x in s)]
        assert len(steps) == 1, key
        count = lambda start: sum(x.startswith(start) for x in steps[0])                 # noqa: E731
        assert count("v_mfma_scale_f32_32x32x64_f8f6f4") == 2 * fm * fn and count("ds_read_b128") == 4 * (fm + fn), key
        assert not any("vmcnt" in x or x.startswith(("s_barrier", "scratch_", "v_accvgpr")) for x in steps[0]), key
        code = _instructions(body)
        for i, x in enumerate(code):
            if re.search(r"\bm0\b", x):
                assert x.startswith(("s_mov_b32 m0, s", "s_mov_b32 m0, vcc")) and code[i + 1] == "s_nop 0" and code[i + 2].endswith("offen lds"), (key, code[i:i + 3])


def test_rows_and_tiles_by_themselves(texts):
    rows, tiles, backward = (_kernels(texts[f], n) for f, n in (("zi_epilogue_rows.hip", "epilogue_rows_kernel"), ("zi_epilogue_tiles.hip", "epilogue_tiles_kernel"),
                                                              ("zi_epilogue_backward.hip", "epilogue_backward_kernel")))
    # {bf16, fp16} x {five activations x whole octets or not x large or not, rows of less than eight}, rows of up to 128 columns besides; sums
    assert [len(x) for x in (rows, tiles, backward)] == [2 * (5 * 2 * (2 + 1) + 1 + 5), 2 * (5 * 2 * 2 + 1 + 3), 2 * (5 * 2 * 2 + 1)]
    for kernels in (rows, tiles, backward):
        for key, body in kernels.items():
            assert _directive(body, "private_segment_fixed_size") == 0, key
            sums = key[2] == 1 and kernels is not backward
            assert _directive(body, "next_free_vgpr") <= (512 if sums else 128), key      # four wavefronts on a SIMD


def test_few_rows(texts):
    kernels = _kernels(texts["zi_fp8_matmul_epilogue.hip"], "fp8_matmul_few_epilogue_kernel")
    assert len(kernels) == 4
    for key, body in kernels.items():
        assert _directive(body, "private_segment_fixed_size") == 0, key
        wide = max(sum(x.startswith("global_load_dwordx4") for x in s) for s in _stretches(body) if any(x.startswith("v_mfma") for x in s))
        assert wide == 8 * (1 + key[1]), (key, wide)


def test_no_atomics_and_no_packed_arithmetic(texts):
    for text in texts.values():
        assert not re.search(r"^\s*\w*atomic", text, re.M)
        assert not re.search(r"^\s*v_pk_(add|mul|fma)_f32", text, re.M)
