// The product in 8 bits with an epilogue (include/zi_epilogue.h).
#include <hip/hip_runtime.h>

#include "zi_epilogue_internal.h"
#include "zi_fp8_matmul_kernels.h"

namespace zi {

namespace {

template <int FM, int FN, int RING>
hipError_t launch_sums_of_tiles(const MatmulArgs& a, const MatmulPlan& plan, float* sums, hipStream_t s)
{
    TileOrder order;
    order.across = (uint32_t)((a.n + 64 * FN - 1) / (64 * FN));
    order.down = (uint32_t)((a.m + 64 * FM - 1) / (64 * FM));
    order.count = order.across * order.down * plan.parts;
    order.part_steps = plan.part_steps;
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
    switch (plan.shape) {
    case 0: return launch_sums_of_tiles<1, 1, 4>(a, plan, sums, s);
    case 1: return launch_sums_of_tiles<1, 2, 3>(a, plan, sums, s);
    case 2: return launch_sums_of_tiles<2, 2, 4>(a, plan, sums, s);
    case 3: return launch_sums_of_tiles<2, 2, 2>(a, plan, sums, s);
    case 4: return launch_sums_of_tiles<4, 2, 3>(a, plan, sums, s);
    case 5: return launch_sums_of_tiles<4, 4, 2>(a, plan, sums, s);
    }
    return a.m <= 16 ? launch_sums_of_few<1>(a, sums, s) : launch_sums_of_few<2>(a, sums, s);
}

}  // namespace

size_t fp8_matmul_epilogue_workspace_floats(int64_t m, int64_t n, int64_t k, int outputs8)
{
    return plan_fp8_matmul(m, n, k).parts * (size_t)m * (size_t)n;
}

hipError_t launch_fp8_matmul_epilogue(const MatmulArgs& a, const EpilogueArgs& e, int dtype, float* workspace, hipStream_t s)
{
    const MatmulPlan plan = plan_fp8_matmul(a.m, a.n, a.k);
    const hipError_t err = launch_sums(a, plan, workspace, s);
    if (err != hipSuccess) return err;
    return launch_epilogue(e, EpilogueSource{nullptr, 0, workspace, plan.parts}, dtype, s);
}

}  // namespace zi
