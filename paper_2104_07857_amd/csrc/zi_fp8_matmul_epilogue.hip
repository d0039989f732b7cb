// The product in 8 bits with an epilogue (include/zi_epilogue.h): which kernel makes it.
#include <hip/hip_runtime.h>

#include "zi_fp8_matmul_epilogue_kernels.h"

namespace zi {

template <>
hipError_t launch_fp8_matmul_epilogue_tiles<ActivationKind::kFloor>(const MatmulArgs&, const MatmulPlan&, const EpilogueArgs&, int, hipStream_t);
template <>
hipError_t launch_fp8_matmul_epilogue_tiles<ActivationKind::kSigmoid>(const MatmulArgs&, const MatmulPlan&, const EpilogueArgs&, int, hipStream_t);
template <>
hipError_t launch_fp8_matmul_epilogue_tiles<ActivationKind::kNormal>(const MatmulArgs&, const MatmulPlan&, const EpilogueArgs&, int, hipStream_t);

// Few rows, whose sums become 16-bit outputs here, element by element.  (Of eight numbers that dropout's generator makes at a time one is used; blocks of 128 columns are eight
// workgroups', so that outputs in 8 bits are left to a second kernel.)  Bound by B's bytes; bias and residual come while they do.  us, fp8_matmul_few_kernel with C / this with bias, dropout
// and residual: 1 x 4096 x 4096 4.9 / 5.5, 8 x 4096 x 4096 5.5 / 5.8, 24 x 4096 x 2048 7.4 / 8.3.
template <int DT, int FA, int W>
__global__ __launch_bounds__(64 * W) void fp8_matmul_few_epilogue_kernel(const MatmulArgs p, const EpilogueArgs e)
{
    __shared__ float s_sum[W][FA][16][17];
    const int64_t n0 = (int64_t)blockIdx.x * 16;
    const auto of = [](const void* base, int64_t at) {
        Octet<DT> x;
        x.w[0] = static_cast<const uint16_t*>(base)[at];
        return x.get(0);
    };
    const auto put = [](void* base, int64_t at, float x) { static_cast<uint16_t*>(base)[at] = (uint16_t)Octet<DT>::pair(x, 0.0f); };
    const Dropout drop(e.drop);
    constexpr int kEach = FA * 256 > 64 * W ? FA * 256 / (64 * W) : 1;
    float bias[kEach], residual[kEach];                 // (under way while the product is made)
    const auto place = [&](int i, int& f, int& m, int& n) {
        const int t = threadIdx.x + i * 64 * W;
        f = t >> 8;
        m = (t >> 4) & 15;
        n = t & 15;
        return f < FA && 16 * f + m < p.m && n0 + n < p.n;
    };
    int f, m, n;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        bias[i] = residual[i] = 0.0f;
        if (!place(i, f, m, n)) continue;
        if (e.bias) bias[i] = of(e.bias, n0 + n);
        if (e.residual) residual[i] = of(e.residual, (16 * f + m) * e.residual_ld + n0 + n);
    }
    multiply_few<FA, W>(p, n0, s_sum);
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        if (!place(i, f, m, n)) continue;
        const int64_t row = 16 * f + m, col = n0 + n;
        float x = sum_of_few<FA, W>(s_sum, f, m, n);
        if (e.bias) x += bias[i];
        if (e.z) put(e.z, row * e.z_ld + col, x);
        if (!e.y) continue;
        with_activation(e.activation, [&](auto act) { x = activated<decltype(act)::value>(x); });
        if (drop.active()) {
            const u32x4 w = drop.numbers((uint32_t)(col >> 3), (uint32_t)row);
            const int j = (int)(col & 7);
            const uint32_t word = j < 4 ? (j < 2 ? w[0] : w[1]) : (j < 6 ? w[2] : w[3]);
            x = (j & 1 ? word >> 16 : word & 0xFFFFu) >= drop.threshold ? x * drop.scale : 0.0f;
        }
        if (e.residual) x += residual[i];
        put(e.y, row * e.y_ld + col, x);
    }
}
namespace {

template <int DT>
hipError_t launch_few_epilogue(const MatmulArgs& a, const EpilogueArgs& e, hipStream_t s)
{
    const dim3 grid((unsigned)((a.n + 15) / 16)), block(512);
    if (a.m <= 16) hipLaunchKernelGGL((fp8_matmul_few_epilogue_kernel<DT, 1, 8>), grid, block, 0, s, a, e);
    else hipLaunchKernelGGL((fp8_matmul_few_epilogue_kernel<DT, 2, 8>), grid, block, 0, s, a, e);
    return hipGetLastError();
}

// Sums in a workspace, for a kernel over rows or tiles to go on with.
template <int FM, int FN, int RING>
hipError_t launch_sums_of_tiles(const MatmulArgs& a, const MatmulPlan& plan, float* sums, hipStream_t s)
{
    const TileOrder order = order_of(a, plan, 64 * FM, 64 * FN);
    hipLaunchKernelGGL((fp8_matmul_kernel<ZI_FP32, FM, FN, RING>), dim3(order.count), dim3(256), 0, s, a, order, sums);
    return hipGetLastError();
}
template <int FA>
hipError_t launch_sums_of_few(MatmulArgs a, float* sums, hipStream_t s)
{
    a.d = sums;
    a.d_ld = a.n;
    hipLaunchKernelGGL((fp8_matmul_few_kernel<ZI_FP32, FA, 8>), dim3((unsigned)((a.n + 15) / 16)), dim3(512), 0, s, a);
    return hipGetLastError();
}
hipError_t launch_sums(const MatmulArgs& a, const MatmulPlan& plan, float* sums, hipStream_t s)
{
    if (plan.shape == 0) return launch_sums_of_tiles<1, 1, 4>(a, plan, sums, s);
    if (plan.shape == 1) return launch_sums_of_tiles<1, 2, 3>(a, plan, sums, s);
    return a.m <= 16 ? launch_sums_of_few<1>(a, sums, s) : launch_sums_of_few<2>(a, sums, s);
}

}  // namespace

// How a product is made, and whether all of its outputs come from there: tiles put out blocks of 128 rows or columns that are a workgroup's own.  Where the fastest way to the sums is none
// to the outputs, a second kernel that reads the sums again stands against the fastest way that is.
//
// Tiles of 256 rows have a compute unit to themselves, and nothing hides what becomes of their sums; of 128 x 128 there are two, one of which multiplies meanwhile.  So they are the faster ones for
// outputs in 8 bits up to k of 4000 or so.  us, 256 x 256 / 128 x 128: 8191 x 8192 x 2048 with gelu to 8 bits 201 / 160, both ways 223 / 178, 4096 x 16384 x 4096 285 / 265 and 308 / 278,
// 8192 x 32768 x 8192 1830 / 1967 and 1920 / 2055.  kAlone are fitted to 90 products (m of 64 to 16384, n of 128 to 32768, k of 181 to 16384, drawn evenly on a logarithmic scale) with outputs one way and both, without
// an activation, with gelu and silu, in each tile: the choice is 0.2 % slower than the fastest tile for one way along the rows and 0.3 % for the others; without them 2.6 and 3.3 to 3.9 %.
static constexpr float kSecond = 2.5f, kSecondStream = 4.5e6f, kWhole = 1.5f;      // us of the second kernel; bytes a us; us of blocks made in tiles
static constexpr MatmulAlone kAloneRows = {8.0f, 8.0f}, kAloneTurned = {8.0f, 14.0f};      // us a round: outputs along the rows, and transposed
static MatmulPlan plan_whole(int64_t m, int64_t n, int64_t k, int outputs8, float& estimate)
{
    const int first = outputs8 & ZI_EPILOGUE_TURNED ? 2 : outputs8 & ZI_EPILOGUE_Y8 ? 1 : 0;
    return plan_fp8_matmul_from(m, n, k, first, outputs8 & ZI_EPILOGUE_TURNED ? kAloneTurned : outputs8 ? kAloneRows : MatmulAlone{}, estimate);
}
EpiloguePlan plan_fp8_matmul_epilogue(int64_t m, int64_t n, int64_t k, int outputs8)
{
    const int first = outputs8 & ZI_EPILOGUE_TURNED ? 2 : outputs8 & ZI_EPILOGUE_Y8 ? 1 : kFewRows;
    float any, whole;
    const MatmulPlan plan = plan_fp8_matmul_from(m, n, k, kFewRows, MatmulAlone{}, any);
    if (outputs8 == 0 && plan.parts == 1) return {plan, 1};
    const MatmulPlan other = plan_whole(m, n, k, outputs8, whole);
    if (plan.parts == 1 && plan.shape >= first) return {other, 1};
    // (The estimate for parts has their sum in it already.)  1 x 16384 x 4096 to 8 bits: in two kernels 15.0 us, whole in tiles of 64 x 128 17.3; 2048 x 2048 x 2048 transposed 22 and 14.
    const float second = plan.parts > 1 ? 0.0f : kSecond + 8.0f * (float)m * (float)n / kSecondStream;
    if (other.parts == 1 && whole + kWhole <= any + second) return {other, 1};
    return {plan, 0};
}

size_t fp8_matmul_epilogue_workspace_floats(int64_t m, int64_t n, int64_t k, int outputs8)
{
    const EpiloguePlan p = plan_fp8_matmul_epilogue(m, n, k, outputs8);
    return p.whole ? 0 : p.plan.parts * (size_t)m * (size_t)n;
}

hipError_t launch_fp8_matmul_epilogue(const MatmulArgs& a, const EpilogueArgs& e, int dtype, float* workspace, hipStream_t s)
{
    const EpiloguePlan p = plan_fp8_matmul_epilogue(a.m, a.n, a.k, (e.y8.out ? ZI_EPILOGUE_Y8 : 0) | (e.y8.turned ? ZI_EPILOGUE_TURNED : 0));
    if (!p.whole) {
        const hipError_t err = launch_sums(a, p.plan, workspace, s);
        if (err != hipSuccess) return err;
        return launch_epilogue(e, EpilogueSource{nullptr, 0, workspace, p.plan.parts}, dtype, s);
    }
    if (p.plan.shape == kFewRows) return dtype == ZI_BF16 ? launch_few_epilogue<ZI_BF16>(a, e, s) : launch_few_epilogue<ZI_FP16>(a, e, s);
    switch (kind_of(e.activation)) {
    case ActivationKind::kFloor: return launch_fp8_matmul_epilogue_tiles<ActivationKind::kFloor>(a, p.plan, e, dtype, s);
    case ActivationKind::kSigmoid: return launch_fp8_matmul_epilogue_tiles<ActivationKind::kSigmoid>(a, p.plan, e, dtype, s);
    case ActivationKind::kNormal: break;
    }
    return launch_fp8_matmul_epilogue_tiles<ActivationKind::kNormal>(a, p.plan, e, dtype, s);
}

}  // namespace zi
