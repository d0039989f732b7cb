"""Builds libzi.so (HIP kernels + C ABI) for gfx950 with hipcc and the module _zi_call (argument marshalling) with gcc, in-tree."""
from __future__ import annotations

import concurrent.futures
import hashlib
import importlib.machinery
import os
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB_PATH = os.path.join(HERE, "libzi.so")
# (it uses more than the limited API, so its name has this interpreter's version in it)
CALL_PATH = os.path.join(HERE, "_zi_call" + importlib.machinery.EXTENSION_SUFFIXES[0])
SOURCES = ["zi_kernels.hip", "zi_api.hip", "zi_plan.hip", "zi_engine.hip", "zi_offload.hip", "zi_probe.hip",
           "zi_fp8_api.hip", "zi_fp8_rows.hip", "zi_fp8_matmul.hip",
           "zi_epilogue_api.hip", "zi_epilogue_plan.hip"]
# The kernels of zi_epilogue.h, which libzi.so loads from its own folder when they are first called; a library of another name those of its own name.
def epilogue_path(lib: str) -> str:
    stem, end = os.path.splitext(lib)
    return stem + "_epilogue" + end


EPILOGUE_PATH = epilogue_path(LIB_PATH)
EPILOGUE_SOURCES = ["zi_epilogue_rows.hip", "zi_epilogue_tiles.hip", "zi_epilogue_backward.hip", "zi_fp8_matmul_epilogue.hip",
                    "zi_fp8_matmul_floor.hip", "zi_fp8_matmul_sigmoid.hip", "zi_fp8_matmul_normal.hip"]

# -ffp-contract=off: the only fused multiply-adds are the ones the kernels write as fma.
# Packed fp32 instructions are switched off for the device code.
HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    "-ffp-contract=off", "-fhip-fp32-correctly-rounded-divide-sqrt", "-fno-fast-math",
    "-fno-gpu-flush-denormals-to-zero",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wextra", "-Wno-unused-parameter",
]


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", "hipcc"):
        if cand and (os.path.sep not in cand or os.path.exists(cand)):
            return cand
    return "hipcc"


def has_python_headers() -> bool:
    return os.path.exists(os.path.join(sysconfig.get_paths()["include"], "Python.h"))


def call_can_be_built() -> bool:
    return has_python_headers() and shutil.which("gcc") is not None


def needs_build() -> bool:
    built = [LIB_PATH, EPILOGUE_PATH, CALL_PATH] if call_can_be_built() else [LIB_PATH, EPILOGUE_PATH]
    if not all(os.path.exists(f) for f in built):
        return True
    t = min(os.path.getmtime(f) for f in built)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + \
           [os.path.join(ROOT, "include", f) for f in ("zi.h", "zi_fp8.h", "zi_epilogue.h", "zi_probe.h")]
    return any(os.path.getmtime(d) > t for d in deps)


# The host-CPU step is plain C++ with AVX2 / FMA / F16C intrinsics, built by the host compiler.
HOST_SOURCES = ["zi_cpu_step.cpp"]
HOST_FLAGS = ["-O3", "-std=c++17", "-fPIC", "-mavx2", "-mfma", "-mf16c", "-ffp-contract=off", "-fno-fast-math",
              "-Wall", "-Wextra", "-pthread"]


def build_call() -> str | None:
    """The Python side of the calls made once per step (csrc/zi_python.c).  Where it cannot be built there is none, and
    binding.py takes every call through ctypes."""
    for old in (CALL_PATH, os.path.join(HERE, "_zi_call.so")):      # the second is any Python's to import
        if os.path.exists(old):
            os.remove(old)
    if not call_can_be_built():
        sys.stderr.write("no Python.h or no gcc: calls go through ctypes\n")
        return None
    try:
        r = subprocess.run(["gcc", "-O2", "-std=c99", "-fPIC", "-shared", "-Wall", "-Wextra", "-Wno-unused-parameter",
                            "-Wno-missing-field-initializers", "-I", sysconfig.get_paths()["include"], "-I", os.path.join(ROOT, "include"),
                            os.path.join(CSRC, "zi_python.c"), "-o", CALL_PATH], capture_output=True, text=True)
        failed, said = r.returncode != 0, r.stderr
    except OSError as e:
        failed, said = True, str(e)
    if said.strip():
        sys.stderr.write(said.rstrip() + "\n")
    if failed:
        sys.stderr.write("_zi_call was not built: calls go through ctypes\n")
        return None
    return CALL_PATH


def _run_hipcc(cmd):
    r = subprocess.run(cmd, capture_output=True, text=True)
    noise = "packed-fp32-ops' is not a recognized feature"
    err = "\n".join(l for l in r.stderr.splitlines() if noise not in l)
    if r.returncode != 0:
        sys.stderr.write(err + "\n")
        raise RuntimeError("hipcc failed: " + " ".join(cmd))
    if err.strip():
        sys.stderr.write(err + "\n")


def build_number(flags) -> int:
    """64 bits of all sources and flags: two libraries that have the same are of one build."""
    h = hashlib.sha256("\0".join(flags).encode())
    for folder in (CSRC, os.path.join(ROOT, "include")):
        for name in sorted(n for n in os.listdir(folder) if n.endswith((".h", ".hip", ".c", ".cpp"))):
            with open(os.path.join(folder, name), "rb") as f:
                h.update(name.encode() + b"\0" + f.read() + b"\0")
    return int.from_bytes(h.digest()[:8], "little")


def build(force: bool = True, extra_flags=(), out: str | None = None) -> str:
    out = out or LIB_PATH
    if not force and out == LIB_PATH and not needs_build():
        return out
    if out == LIB_PATH:
        build_call()
    objs = []
    for src in HOST_SOURCES:
        obj = os.path.join(HERE, "_" + os.path.splitext(src)[0] + ".o")
        subprocess.run(["g++", *HOST_FLAGS, "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-c", os.path.join(CSRC, src),
                        "-o", obj], check=True)
        objs.append(obj)
    # A source a process, as many as there are CPUs (16 at most); each leaves an object of its own next to the libraries that are made of them.
    flags = [*HIPCC_FLAGS, *extra_flags, f"-DZI_BUILD={build_number([*HIPCC_FLAGS, *extra_flags])}ull", "-I", os.path.join(ROOT, "include"), "-I", CSRC]
    stem = os.path.splitext(out)[0]
    obj_of = {src: f"{stem}_{os.path.splitext(src)[0]}.o" for src in EPILOGUE_SOURCES + SOURCES}
    compiles = [[hipcc(), *(f for f in flags if f != "-shared"), "-c", os.path.join(CSRC, src), "-o", obj] for src, obj in obj_of.items()]
    with concurrent.futures.ThreadPoolExecutor(max(1, min(16, os.cpu_count() or 1))) as pool:
        list(pool.map(_run_hipcc, compiles))
    link = [hipcc(), "--offload-arch=gfx950", "-shared", "-pthread", "-o"]
    _run_hipcc([*link, out, *(obj_of[s] for s in SOURCES), *objs])
    # (both libraries have some kernels of the product: each takes its own)
    _run_hipcc([*link, epilogue_path(out), "-Wl,-Bsymbolic", *(obj_of[s] for s in EPILOGUE_SOURCES)])
    for obj in obj_of.values():
        os.remove(obj)
    return out


if __name__ == "__main__":
    print(build(True))
