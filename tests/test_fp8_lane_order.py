"""The product's epilogue turns a tile in LDS, in a place of each wavefront's own and without a barrier: what other lanes of the wavefront wrote is
read there, and read again from places that they wrote before.  The order of the two has to be stated, or the compiler may
take a lane's reads for independent of its writes.  Read from the compiler's intermediate form (no GPU needed)."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2104_07857_amd import build as zb

FENCE = re.compile(r'^\s*fence syncscope\("wavefront[^"]*"\) (release|acquire)', re.M)


@pytest.fixture(scope="module")
def bodies(tmp_path_factory):
    if shutil.which(zb.hipcc()) is None and not os.path.exists(zb.hipcc()):
        pytest.skip("no hipcc here")
    out = tmp_path_factory.mktemp("ir") / "matmul.ll"
    flags = [f for f in zb.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    cmd = [zb.hipcc(), *flags, "-I", os.path.join(zb.ROOT, "include"), "-I", zb.CSRC, "-S", "-emit-llvm", "--cuda-device-only",
           "-o", str(out), os.path.join(zb.CSRC, "zi_fp8_matmul.hip")]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    found = {}
    for part in out.read_text().split("\ndefine ")[1:]:
        m = re.match(r".*?@_ZN2zi17fp8_matmul_kernelILi(\d)ELi(\d)ELi(\d)ELi(\d)E", part)
        if m:
            found[tuple(int(x) for x in m.groups())] = part[:part.index("\n}")]
    return found


def test_lanes_meet_between_writes_and_reads(bodies):
    assert len(bodies) == 13
    for key, body in bodies.items():
        kinds = [m.group(1) for m in FENCE.finditer(body)]
        if key[0] == 2:                       # parts of k: sums go out as they are
            assert not kinds, key
            continue
        # behind C's rows (a copy of that path for whole tiles and one for ends may have been made), and behind the sums
        assert len(kinds) >= 4 and kinds.count("release") == kinds.count("acquire"), (key, kinds)
        assert body.count("call void @llvm.amdgcn.wave.barrier()") == kinds.count("release"), key
