"""The product in 8 bits through each of its kernels (test_fp8_plans.py says that these sizes reach them), with and without C, against 64 bits:
whole numbers bit for bit, as test_gpu_fp8_matmul.py explains, and normal numbers within the matrix cores' bound that it derives."""
import pytest
import torch

import paper_2104_07857_amd as zi
from fp8_plans import FEW_16, FEW_32, PARTS, TILES
from fp8_util import DT, HALF_ULP, LEAST
from test_gpu_fp8_matmul import _call, _exact, _normal, _whole

pytestmark = pytest.mark.gpu
HALF = [torch.bfloat16, torch.float16]


def _c(m, n, dtype):
    return torch.randint(-64, 65, (m, n), generator=torch.Generator(device="cuda:0").manual_seed(90), device="cuda:0").to(dtype)


@pytest.mark.parametrize("m,n,k", FEW_16 + FEW_32 + PARTS + TILES)
@pytest.mark.parametrize("dtype", HALF)
def test_whole_numbers_with_and_without_c(m, n, k, dtype):
    a, b = _whole(m, k, 1, 91), _whole(n, k, 128, 92)
    exact, c = _exact(a, b), _c(m, n, dtype)
    want = (exact + c.double()).to(dtype)
    assert torch.equal(_call(a, b, dtype, pad=5), exact.to(dtype))
    assert torch.equal(_call(a, b, dtype, c), want)
    assert torch.equal(_call(a, b, dtype, c, pad=3), want)
    assert torch.equal(_call(a, b, dtype, c, pad=8, inplace=True), want)


@pytest.mark.parametrize("m,n,k", FEW_16[:4] + FEW_32[:5] + PARTS[:4])
@pytest.mark.parametrize("dtype", HALF)
def test_normal_numbers_and_normal_c(m, n, k, dtype):
    a, b = _normal(m, k, 1, 93, outliers=True), _normal(n, k, 1, 94)
    c = (torch.randn((m, n), generator=torch.Generator(device="cuda:0").manual_seed(95), device="cuda:0") * k ** 0.5).to(dtype)
    d, e = _call(a, b, dtype, c).double(), _exact(a, b, c)
    size = a.values().abs() @ b.values().abs().t().contiguous()
    # sums of up to 2^4 * 2^12 terms in 2^-20 (see there); C is one term more
    assert bool(((d - e).abs() <= size * (2.0 ** -9 + 2.0 ** -20) + c.double().abs() * 2.0 ** -20 + e.abs() * HALF_ULP[dtype] * 1.01 + LEAST[dtype]).all())
    assert float((d - e).norm() / e.norm()) <= HALF_ULP[dtype] + 2e-4


@pytest.mark.parametrize("m,n,k", [FEW_16[2], FEW_32[0], FEW_32[4], PARTS[1], PARTS[5]])
def test_nan_keeps_to_its_row_and_column(m, n, k):
    a, b = _whole(m, k, 1, 96), _whole(n, k, 1, 97)
    a.data[m - 1, k - 1], b.data[n - 1, k // 2] = 0x7F, 0xFF
    c = _c(m, n, torch.bfloat16)
    c[0, 0] = float("nan")
    d, e = _call(a, b, torch.bfloat16, c), _exact(a, b, c)
    assert torch.equal(d.isnan(), e.isnan()) and int(e.isnan().sum()) == n + m
    assert torch.equal(d[~d.isnan()], e.to(torch.bfloat16)[~d.isnan()])


@pytest.mark.parametrize("m,n,k", [FEW_16[3], FEW_32[2], PARTS[1], PARTS[5]])
def test_replays_with_c(m, n, k):
    """A captured call with C: every replay's result is that of a call by itself, whatever the workspace held."""
    a, b, c = _normal(m, k, 1, 98), _normal(n, k, 128, 99), _c(m, n, torch.float16)
    want = _call(a, b, torch.float16, c)
    out = torch.zeros_like(want)
    ws = torch.empty(max(16, zi.zi_fp8_matmul_workspace_bytes(m, n, k)), dtype=torch.uint8, device="cuda:0")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        zi.zi_fp8_matmul(a.struct, b.struct, out, DT[torch.float16], n, c, ws, stream=torch.cuda.current_stream())
    for _ in range(4):
        out.fill_(float("nan"))
        ws.fill_(0xFF)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        assert torch.equal(_call(a, b, torch.float16, c), want)
