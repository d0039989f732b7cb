"""How the two libraries are built, without compiling their kernels: the number that says that they are of one build, and where they go."""
import ctypes
import os

from paper_2104_07857_amd import build as zb


def test_the_builds_number(tmp_path, monkeypatch):
    """Of all sources and flags; the built library of the epilogues' kernels has one."""
    first = zb.build_number(zb.HIPCC_FLAGS)
    assert 0 < first < 1 << 64 and first == zb.build_number(zb.HIPCC_FLAGS) != zb.build_number([*zb.HIPCC_FLAGS, "-g"])
    (tmp_path / "a.hip").write_text("1")
    (tmp_path / "notes.txt").write_text("1")
    monkeypatch.setattr(zb, "CSRC", str(tmp_path))
    other = zb.build_number(zb.HIPCC_FLAGS)
    (tmp_path / "notes.txt").write_text("2")
    assert zb.build_number(zb.HIPCC_FLAGS) == other != first
    (tmp_path / "a.hip").write_text("2")
    assert zb.build_number(zb.HIPCC_FLAGS) != other
    kernels = ctypes.CDLL(zb.EPILOGUE_PATH).zi_epilogue_kernels
    kernels.restype = ctypes.POINTER(ctypes.c_uint64)
    assert kernels()[0] != 0


def test_a_build_of_another_name_touches_no_other(monkeypatch):
    """In the package's own folder too: both libraries have the name that was asked for."""
    made = []

    def hipcc(cmd):
        made.append(cmd[cmd.index("-o") + 1])
        open(made[-1], "ab").close()

    before = [os.stat(f).st_mtime_ns for f in (zb.LIB_PATH, zb.EPILOGUE_PATH)]
    monkeypatch.setattr(zb, "_run_hipcc", hipcc)
    out = os.path.join(zb.HERE, "libzi_more.so")
    try:
        assert zb.build(out=out) == out
        assert [f for f in made if f.endswith(".so")] == [out, os.path.join(zb.HERE, "libzi_more_epilogue.so")]
        assert all(os.path.basename(f).startswith("libzi_more_") and not os.path.exists(f) for f in made if not f.endswith(".so"))
    finally:
        for f in made:
            if os.path.exists(f) and os.path.basename(f).startswith("libzi_more"):
                os.remove(f)
    assert [os.stat(f).st_mtime_ns for f in (zb.LIB_PATH, zb.EPILOGUE_PATH)] == before
