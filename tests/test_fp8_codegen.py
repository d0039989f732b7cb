"""Properties of the compiled 8-bit and norm kernels that their speed or their safety depends on, read from the assembly hipcc
emits for the library's own sources (no GPU needed):

  * no scratch memory, but for the few kernels of very long rows that are known to have some;
  * a step of the product over tiles is one stretch of code with all of its multiplications, its loads from memory to LDS and its
    reads of LDS, and no wait for memory in it: that stands in front, once a step, with the barrier;
  * m0 is written only right in front of a load to LDS, which takes the place to write to from there;
  * the kernel for few rows has all loads of a run in flight before it multiplies;
  * no atomics (results would depend on the order of workgroups) and no packed fp32 arithmetic.
"""
import os
import re
import shutil
import subprocess

import pytest

from paper_2104_07857_amd import build as zb

LDS_OF_A_COMPUTE_UNIT = 160 * 1024


def _assembly(source, out):
    if shutil.which(zb.hipcc()) is None and not os.path.exists(zb.hipcc()):
        pytest.skip("no hipcc here")
    flags = [f for f in zb.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    cmd = [zb.hipcc(), *flags, "-I", os.path.join(zb.ROOT, "include"), "-I", zb.CSRC, "-S", "--cuda-device-only",
           "-o", str(out), os.path.join(zb.CSRC, source)]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    return out.read_text()


@pytest.fixture(scope="module")
def matmul(tmp_path_factory):
    return _assembly("zi_fp8_matmul.hip", tmp_path_factory.mktemp("isa") / "matmul.s")


@pytest.fixture(scope="module")
def rows(tmp_path_factory):
    return _assembly("zi_fp8_rows.hip", tmp_path_factory.mktemp("isa") / "rows.s")


def _kernels(text, name):
    """Bodies by the integers of their template arguments."""
    found = {}
    for mt in re.finditer(r"^_ZN2zi\d+%sI((?:L(?:[ib]|NS_4EndsE)\d+E)+)E\w+:" % name, text, re.M):
        key = tuple(int(x) for x in re.findall(r"L(?:[ib]|NS_4EndsE)(\d+)E", mt.group(1)))
        found[key] = text[mt.end():text.index(".end_amdhsa_kernel", mt.end())]
    return found


def _directive(body, name):
    m = re.search(r"\.amdhsa_" + name + r"\s+(\d+)", body)
    assert m, name
    return int(m.group(1))


def _instructions(body):
    lines = (line.split(";")[0].strip() for line in body.splitlines())
    return [x for x in lines if x and not x.startswith(".") and not x.endswith(":")]


def _stretches(body):
    """Instructions between labels."""
    return [_instructions(x) for x in re.split(r"^\.LBB\w+:.*$", body.split(".amdhsa_kernel")[0], flags=re.M)]


def test_tiles_have_no_scratch_and_fit(matmul):
    kernels = _kernels(matmul, "fp8_matmul_kernel")
    assert len(kernels) == 13, sorted(kernels)     # {bf16, fp16} x six tiles, and parts of k in the smallest
    for key, body in kernels.items():
        assert _directive(body, "private_segment_fixed_size") == 0, key
        _, fm, fn, ring = key
        together = 1 if ring * (fm + fn) > 8 else 2
        assert _directive(body, "group_segment_fixed_size") * together <= LDS_OF_A_COMPUTE_UNIT, key
        assert _directive(body, "next_free_vgpr") <= 512 // together, key      # of a wavefront for each SIMD and workgroup


def test_a_step_is_one_stretch_that_waits_for_no_memory(matmul):
    for key, body in _kernels(matmul, "fp8_matmul_kernel").items():
        _, fm, fn, _ = key
        steps = [s for s in _stretches(body) if any(x.startswith("v_mfma") for x in s) and any(x.endswith(" lds") for x in s)]
        assert len(steps) == 1, key
        step = steps[0]
        count = lambda start: sum(x.startswith(start) for x in step)
        assert count("v_mfma_scale_f32_32x32x64_f8f6f4") == 2 * fm * fn, key
        assert sum(x.startswith("buffer_load_dwordx4") and x.endswith("offen lds") for x in step) == 2 * (fm + fn), key
        assert count("ds_read_b128") == 4 * (fm + fn), key
        assert not any("vmcnt" in x or x.startswith(("s_barrier", "scratch_", "v_accvgpr")) for x in step), key
        # reads and multiplications take turns: at most two pieces, of two reads each, in a row
        if fm * fn > 1:
            kinds = "".join("m" if x.startswith("v_mfma") else "r" if x.startswith("ds_read_b128") else "" for x in step)
            assert max(len(x) for x in kinds.split("m")) <= 4 and max(len(x) for x in kinds.split("r")) <= fm * fn, (key, kinds)


def test_m0_is_that_of_loads_to_lds(matmul):
    for key, body in _kernels(matmul, "fp8_matmul_kernel").items():
        code = _instructions(body)
        at = [i for i, x in enumerate(code) if re.search(r"\bm0\b", x)]
        assert at, key
        for i in at:
            assert code[i].startswith("s_mov_b32 m0, s"), (key, code[i])
            assert code[i + 1] == "s_nop 0" and code[i + 2].startswith("buffer_load_dword") and code[i + 2].endswith("offen lds"), (key, code[i:i + 3])
        assert sum(x.endswith(" lds") for x in code) == len(at), key


def test_few_rows_have_a_run_in_flight(matmul):
    kernels = _kernels(matmul, "fp8_matmul_few_kernel")
    assert len(kernels) == 4, sorted(kernels)      # {bf16, fp16} x {16, 32} rows
    for key, body in kernels.items():
        assert _directive(body, "private_segment_fixed_size") == 0, key
        code = _instructions(body)
        first = min(i for i, x in enumerate(code) if x.startswith("v_mfma"))
        wide = max(sum(x.startswith("global_load_dwordx4") for x in s) for s in _stretches(body) if any(x.startswith("v_mfma") for x in s))
        assert wide == 8 * (1 + key[1]) and first > 0, (key, wide)


def test_rows_have_no_scratch(rows):
    quantize, norm, backward, means, dgamma = (_kernels(rows, n) for n in ("fp8_quantize_kernel", "rms_norm_kernel", "rms_norm_backward_kernel",
                                                                         "rms_norm_means_kernel", "rms_norm_dgamma_kernel"))
    assert [len(k) for k in (quantize, norm, backward, means, dgamma)] == [6, 42, 28, 4, 6]
    for key, body in [*quantize.items(), *means.items(), *dgamma.items()]:
        assert _directive(body, "private_segment_fixed_size") == 0, key
    for key, body in norm.items():                 # (type, threads, octets, how rows end)
        assert _directive(body, "private_segment_fixed_size") <= (96 if key[2] == 8 else 0), key
    for key, body in backward.items():
        assert _directive(body, "private_segment_fixed_size") <= (64 if key[1] == 1024 else 0), key


def test_no_atomics_and_no_packed_arithmetic(matmul, rows):
    for text in (matmul, rows):
        assert not re.search(r"^\s*\w*atomic", text, re.M)
        assert not re.search(r"^\s*v_pk_(add|mul|fma)_f32", text, re.M)
