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

namespace {

// What the tiles of a plan can put out themselves: blocks of 128 rows or columns have to be a workgroup's own.
bool makes_all(const MatmulPlan& plan, int outputs8)
{
    if (plan.shape < 0 || plan.parts > 1) return false;
    return !(outputs8 & ZI_EPILOGUE_TURNED ? plan.shape < 2 : outputs8 & ZI_EPILOGUE_Y8 ? plan.shape < 1 : false);
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

size_t fp8_matmul_epilogue_workspace_floats(int64_t m, int64_t n, int64_t k, int outputs8)
{
    const MatmulPlan plan = plan_fp8_matmul(m, n, k);
    return makes_all(plan, outputs8) ? 0 : plan.parts * (size_t)m * (size_t)n;
}

hipError_t launch_fp8_matmul_epilogue(const MatmulArgs& a, const EpilogueArgs& e, int dtype, float* workspace, hipStream_t s)
{
    const MatmulPlan plan = plan_fp8_matmul(a.m, a.n, a.k);
    const int outputs8 = (e.y8.out ? ZI_EPILOGUE_Y8 : 0) | (e.y8.turned ? ZI_EPILOGUE_TURNED : 0);
    if (makes_all(plan, outputs8)) {
        switch (kind_of(e.activation)) {
        case ActivationKind::kFloor: return launch_fp8_matmul_epilogue_tiles<ActivationKind::kFloor>(a, plan, e, dtype, s);
        case ActivationKind::kSigmoid: return launch_fp8_matmul_epilogue_tiles<ActivationKind::kSigmoid>(a, plan, e, dtype, s);
        case ActivationKind::kNormal: return launch_fp8_matmul_epilogue_tiles<ActivationKind::kNormal>(a, plan, e, dtype, s);
        }
    }
    const hipError_t err = launch_sums(a, plan, workspace, s);
    if (err != hipSuccess) return err;
    return launch_epilogue(e, EpilogueSource{nullptr, 0, workspace, plan.parts}, dtype, s);
}

}  // namespace zi
