// Kernels of the product in 8 bits, D = A B^T + C (include/zi_fp8.h), on the matrix cores' scaled e4m3 instructions: a
// block's scale goes in with its numbers, so the sum over k stays in fp32 registers from the first block to the last.
// (An instruction adds 16 products at a time before that, in fewer bits: the header says how many.)
#include <hip/hip_runtime.h>

#include <cmath>

#include "zi_fp8_matmul_kernels.h"

namespace zi {

template <int DT, int FA, int W>
static hipError_t launch_few(const MatmulArgs& a, hipStream_t s)
{
    hipLaunchKernelGGL((fp8_matmul_few_kernel<DT, FA, W>), dim3((unsigned)((a.n + 15) / 16)), dim3(64 * W), 0, s, a);
    return hipGetLastError();
}

// The sums of all parts in their order, and C, in fp32, rounded once.  Bound by the launch: 13 x 4096 in four parts 3.5 to 3.9 us.
template <int DT>
__global__ __launch_bounds__(256) void fp8_matmul_join_kernel(const MatmulArgs p, const float* partials, uint32_t parts, uint32_t across)
{
    const int64_t row = blockIdx.x / across, col = ((int64_t)(blockIdx.x % across) * 256 + threadIdx.x) * 4;
    const int64_t left = p.n - col;
    if (left <= 0) return;
    const float* from = partials + row * p.n + col;
    float x[4] = {};
    for (uint32_t i = 0; i < parts; ++i, from += p.m * p.n) {
        if (left >= 4) {
            const u32x4_of_4 y = *reinterpret_cast<const u32x4_of_4*>(from);
#pragma unroll
            for (int w = 0; w < 4; ++w) x[w] += __uint_as_float(y[w]);
        } else {
#pragma unroll
            for (int w = 0; w < 3; ++w)
                if (w < left) x[w] += from[w];
        }
    }
    const int64_t at = row * p.d_ld + col;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        if (w >= left) break;
        if (p.c) {
            Octet<DT> c;
            c.w[0] = static_cast<const uint16_t*>(p.c)[at + w];
            x[w] += c.get(0);
        }
        static_cast<uint16_t*>(p.d)[at + w] = (uint16_t)Octet<DT>::pair(x[w], 0.0f);
    }
}

// ---- which kernel ---------------------------------------------------------------------------------------------

// Tiles, steps of k in LDS, workgroups that share a compute unit, and what a round of them takes: so much a step and so much besides, in us,
// measured on the products below, with one workgroup on a compute unit and with two (256 x 128 and 256 x 256: on up to half of the compute units, and
// on all of them, where the power the card may draw holds the clock down).  By tile, us:
//                           64 x 64   64 x 128  128 x 128 (4 steps)  128 x 128 (2)  256 x 128  256 x 256
//     64 x  4096 x  4096     11.1      12.1         17                 24             -          -
//    512 x  4096 x  4096     17.0      15.0         16.0               23.8          24         35
//   2048 x  2048 x  2048     17.6      13.3         12.2               15.0          16.1       24.5
//   1001 x  8192 x  2048     32.0      24.7         23.3               19.6          19.8       27.2
//   1024 x  8192 x  8192      -         -           74.9               70.6          60.6        -
//   3000 x  5000 x  4096     99        80           73                 64            62.3       53.0
//   8192 x  8192 x  8192    881       650          549                507           487        406
struct TileShape {
    int rows, cols, together;
    float step, step_together, besides;
};
constexpr int kShapes = 6;
constexpr TileShape kShape[kShapes] = {{64, 64, 2, 0.268f, 0.373f, 3.26f},
                                       {64, 128, 2, 0.34f, 0.55f, 4.5f},
                                       {128, 128, 1, 0.40f, 0.53f, 5.0f},
                                       {128, 128, 2, 0.565f, 0.93f, 4.65f},
                                       {256, 128, 1, 0.65f, 0.755f, 8.75f},
                                       {256, 256, 1, 1.04f, 1.28f, 14.2f}};
constexpr int64_t kUnits = 256;                  // compute units
constexpr float kStream = 4.8e6f, kOutput = 5.4f, kJoinStream = 5.2e6f, kJoin = 1.4f, kJoinPart = 0.6f;     // bytes a us; an element of D in bytes; us
constexpr float kFewStream = 6.3e6f, kFewOfA = 0.22f, kFewTurn = 2.5f, kFewTurn2 = 3.85f, kFewBesides = 1.3f;

// The kernel for few rows of A, against tiles: B's bytes with a charge for each row of A, or the turns that a wavefront takes to its loads (longer
// ones with more than 16 rows of A) where few workgroups share a compute unit.  The charge is what makes the choice come out right, and no rate of
// anything: 13 x 4096 x 16384 takes 18 us in this kernel and is put at 42; tiles take 15.
static float few_rows_estimate(int64_t m, int64_t n, int64_t k)
{
    const float stream = (float)n * (float)k * (1.0f + kFewOfA * (float)m) / kFewStream;
    const int64_t turns = ((k + 32 * kStep - 1) / (32 * kStep)) * ((n + 16 * 512 - 1) / (16 * 512));
    const float wait = (float)turns * (m > 16 ? kFewTurn2 : kFewTurn);
    return (stream > wait ? stream : wait) + kFewBesides;
}

// The least of these estimates: the kernel for few rows of A, or tiles, and of the smallest as many parts of k as pay for adding them (13 x 4096 x
// 16384 in one, two, four, eight parts 35.1, 22.0, 15.3, 16.8).  The constants are those with which this finds the fastest of all that were timed on 386
// products, m of 1 to 16384, n of 128 to 32768 and k of 128 to 16384 drawn evenly on a logarithmic scale (with up to 64 rows of A, B from memory): on
// these same products it is 0.4 % slower than that on the average; on others it was not measured.
MatmulPlan plan_fp8_matmul(int64_t m, int64_t n, int64_t k)
{
    float estimate;
    return plan_fp8_matmul_from(m, n, k, kFewRows, MatmulAlone{}, estimate);
}
MatmulPlan plan_fp8_matmul_from(int64_t m, int64_t n, int64_t k, int first, const MatmulAlone& alone, float& least)
{
    const int64_t steps = (k + kStep - 1) / kStep;
    const float stream = ((float)m + (float)n) * (float)k + kOutput * (float)m * (float)n;
    MatmulPlan best{kFewRows, 1, (uint32_t)((steps + 3) / 4 * 4)};
    least = INFINITY;
    if (m <= 32 && first == kFewRows) least = few_rows_estimate(m, n, k);
    for (int i = first > 0 ? first : 0; i < kShapes; ++i) {
        const TileShape& t = kShape[i];
        const float besides = t.besides + (i == kAloneShape ? alone.rows_256_128 : i == kAloneShape + 1 ? alone.rows_256_256 : 0.0f);
        const int64_t tiles = ((m + t.rows - 1) / t.rows) * ((n + t.cols - 1) / t.cols);
        for (int64_t parts = 1; parts <= (i == 0 ? 16 : 1); parts *= 2) {
            const int64_t each = ((steps + parts - 1) / parts + 3) / 4 * 4;       // a part begins with a word of scales
            const int64_t really = each ? (steps + each - 1) / each : 1;
            const int64_t groups = tiles * really, rounds = groups / (kUnits * t.together), rest = groups % (kUnits * t.together);
            const auto round = [&](float step) { return (float)(really > 1 ? each : steps) * step + besides; };
            const bool apart = t.together == 2 ? rest <= kUnits : rounds == 0 && rest <= kUnits / 2;
            const float work = (float)rounds * round(t.step_together) + (rest ? round(apart ? t.step : t.step_together) : 0.0f);
            float all = 0.01f * work + (work > stream / kStream ? work : stream / kStream);
            if (really > 1) all += kJoin + (float)really * kJoinPart + 8.0f * (float)really * (float)m * (float)n / kJoinStream;
            if (all < least) {
                least = all;
                best = {i, (uint32_t)really, (uint32_t)each};
            }
        }
    }
    return best;
}

template <int DT, int FM, int FN, int RING>
static hipError_t launch_tiles(const MatmulArgs& a, const MatmulPlan& plan, float* partials, hipStream_t s)
{
    TileOrder order;
    order.across = (uint32_t)((a.n + 64 * FN - 1) / (64 * FN));
    order.down = (uint32_t)((a.m + 64 * FM - 1) / (64 * FM));
    order.count = order.across * order.down * plan.parts;
    order.part_steps = plan.part_steps;
    if constexpr (FM == 1 && FN == 1) {
        if (plan.parts > 1) {
            hipLaunchKernelGGL((fp8_matmul_kernel<ZI_FP32, FM, FN, RING>), dim3(order.count), dim3(256), 0, s, a, order, partials);
            const uint32_t across = (uint32_t)((a.n + 1023) / 1024);
            hipLaunchKernelGGL(fp8_matmul_join_kernel<DT>, dim3((unsigned)(across * a.m)), dim3(256), 0, s, a, (const float*)partials, plan.parts, across);
            return hipGetLastError();
        }
    }
    hipLaunchKernelGGL((fp8_matmul_kernel<DT, FM, FN, RING>), dim3(order.count), dim3(256), 0, s, a, order, (float*)nullptr);
    return hipGetLastError();
}

template <int DT>
static hipError_t launch_of(const MatmulArgs& a, float* partials, hipStream_t s)
{
    const MatmulPlan plan = plan_fp8_matmul(a.m, a.n, a.k);
    switch (plan.shape) {
    case 0: return launch_tiles<DT, 1, 1, 4>(a, plan, partials, s);
    case 1: return launch_tiles<DT, 1, 2, 3>(a, plan, partials, s);
    case 2: return launch_tiles<DT, 2, 2, 4>(a, plan, partials, s);
    case 3: return launch_tiles<DT, 2, 2, 2>(a, plan, partials, s);
    case 4: return launch_tiles<DT, 4, 2, 3>(a, plan, partials, s);
    case 5: return launch_tiles<DT, 4, 4, 2>(a, plan, partials, s);
    }
    return a.m <= 16 ? launch_few<DT, 1, 8>(a, s) : launch_few<DT, 2, 8>(a, s);
}

hipError_t launch_fp8_matmul(const MatmulArgs& a, int dtype, float* partials, hipStream_t s)
{
    return dtype == ZI_BF16 ? launch_of<ZI_BF16>(a, partials, s) : launch_of<ZI_FP16>(a, partials, s);
}

}  // namespace zi
