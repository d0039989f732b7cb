"""The sizes that the GPU tests of the product with an epilogue go through reach every way that it is made, with ends in every place (no GPU needed): if the choice changes, sizes
have to follow."""
import random

import pytest

import paper_2104_07857_amd as zi
from epilogue_plans import ALONE, BOTH, SUMS, TURNED, Y8, plan
from fp8_plans import FEW, FEW_16, FEW_32, PARTS, SHAPES, TILES
from fp8_plans import plan as product_plan

ALL = FEW_16 + FEW_32 + PARTS + TILES + SUMS + ALONE


@pytest.mark.parametrize("outputs8", [0, Y8, TURNED, BOTH])
def test_every_way_is_gone(outputs8):
    seen = {}
    for s in ALL:
        p = plan(*s, outputs8)
        seen.setdefault((p.whole, p.shape, p.parts > 1), []).append(s)
    least = 2 if outputs8 & TURNED else 1 if outputs8 & Y8 else 0
    want = {(1, i, False) for i in range(least, len(SHAPES))} | {(0, 0, True)}
    want |= {(0, FEW, False), (0, 0, False)} if outputs8 else {(1, FEW, False)}
    want |= {(0, 1, False)} if outputs8 & TURNED else set()
    assert set(seen) == want
    for (whole, shape, _), sizes in seen.items():
        if whole and shape >= 0:
            rows, cols = SHAPES[shape]
            assert any(m % rows and n % cols and n % 8 for m, n, _ in sizes), (shape, sizes)


def test_no_other_way_is_ever_gone():
    r = random.Random(3)
    for _ in range(20000):
        s = tuple(int(2 ** r.uniform(lo, 15)) for lo in (0, 4, 4))
        for outputs8 in (0, Y8, TURNED, BOTH):
            p = plan(*s, outputs8)
            least = 2 if outputs8 & TURNED else 1 if outputs8 & Y8 else FEW
            if p.whole:
                assert p.parts == 1 and p.shape >= least, (s, outputs8)
            else:
                assert p.shape in (FEW, 0, 1) and (p.parts == 1 or p.shape == 0), (s, outputs8)
                assert zi.zi_fp8_matmul_epilogue_workspace_bytes(*s, outputs8) == 4 * p.parts * s[0] * s[1]
            assert p.whole == 0 or zi.zi_fp8_matmul_epilogue_workspace_bytes(*s, outputs8) == 0


def test_without_8_bit_outputs_it_is_the_products_own_way():
    for s in ALL:
        p, q = plan(*s, 0), product_plan(*s)
        assert (p.shape, p.parts, p.part_steps) == (q.shape, q.parts, q.part_steps)
