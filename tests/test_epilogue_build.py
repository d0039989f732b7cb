"""How the two libraries are built, without compiling anything: the number that says that they are of one build."""
import ctypes

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
