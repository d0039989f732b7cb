"""The sizes that the GPU tests of the product in 8 bits go through reach every kernel that it has, with ends in every place (no GPU
needed): if the choice among the kernels changes, sizes have to follow."""
import pytest

import paper_2104_07857_amd as zi
from fp8_plans import FEW, FEW_16, FEW_32, PARTS, SHAPES, TILES, plan


@pytest.mark.parametrize("sizes,rows", [(FEW_16, range(1, 17)), (FEW_32, range(17, 33))])
def test_few_rows(sizes, rows):
    assert all(m in rows and plan(m, n, k).shape == FEW for m, n, k in sizes)
    last = {(k % 512 + 127) // 128 if k % 512 else 4 for _, _, k in sizes if k > 4096}     # blocks of the last run, behind a first turn
    assert {1, 2, 4} <= last or {1, 3, 4} <= last, last
    assert any(k % 128 for _, _, k in sizes) and any(k < 512 or k % 512 for _, _, k in sizes if k <= 4096)
    assert any(n % 16 for _, n, _ in sizes) and any(m == rows[-1] for m, _, _ in sizes) and any(m < rows[-1] for m, _, _ in sizes)


def test_parts_of_k():
    plans = [plan(*s) for s in PARTS]
    assert all(p.shape == 0 and p.parts > 1 for p in plans) and len({p.parts for p in plans}) >= 4
    assert all(zi.zi_fp8_matmul_workspace_bytes(*s) == 4 * s[0] * s[1] * p.parts for s, p in zip(PARTS, plans))
    steps = [-(-k // 128) for _, _, k in PARTS]
    assert any(s % p.part_steps for s, p in zip(steps, plans)) and any(s % p.part_steps == 0 for s, p in zip(steps, plans))
    assert any(k % 128 for _, _, k in PARTS) and any(n % 4 for _, n, _ in PARTS) and any(n > 1024 and n % 1024 for _, n, _ in PARTS)


def test_tiles():
    seen = {i: [] for i in range(len(SHAPES))}
    for s in TILES:
        p = plan(*s)
        assert p.shape >= 0 and p.parts == 1, s
        seen[p.shape].append(s)
    for i, (rows, cols) in enumerate(SHAPES):
        assert seen[i], i
        assert any(m % rows and n % cols and n % 8 for m, n, _ in seen[i]), (i, seen[i])
        assert any(k % 128 for _, _, k in seen[i]), (i, seen[i])
