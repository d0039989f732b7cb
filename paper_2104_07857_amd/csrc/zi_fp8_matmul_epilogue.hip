// The product in 8 bits with an epilogue (include/zi_epilogue.h): few rows, sums, and the kernel that a plan names.
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

hipError_t launch_fp8_matmul_epilogue(const MatmulArgs& a, const EpiloguePlan& p, const EpilogueArgs& e, int dtype, float* workspace, hipStream_t s)
{
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

// What libzi.so takes this library's kernels by.
extern "C" __attribute__((visibility("default"))) const zi::EpilogueKernels* zi_epilogue_kernels()
{
    static const zi::EpilogueKernels kernels = {ZI_BUILD, zi::launch_epilogue, zi::launch_fp8_matmul_epilogue, zi::launch_epilogue_backward};
    return &kernels;
}
