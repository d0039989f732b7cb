// Internal interface between the C-ABI layer of the 8-bit operators (zi_fp8_api.hip) and their kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "zi_fp8.h"

namespace zi {

constexpr int kFp8Block = ZI_FP8_BLOCK;

struct QuantizeArgs {
    const void* x;
    int64_t rows, cols, ld;
    uint8_t* out;            // NULL: not wanted
    uint8_t* out_scale;
    int64_t out_ld, out_scale_ld;
    uint8_t* turned;         // NULL: not wanted
    uint8_t* turned_scale;
    int64_t turned_ld, turned_scale_ld;
    uint32_t tiles_across;   // tiles of 128 columns
    int32_t out_square, turned_square;   // blocks of 128 x 128 (else of 1 x 128)
};
hipError_t launch_fp8_quantize(const QuantizeArgs& a, int dtype, hipStream_t s);

struct RmsNormArgs {
    zi_rms_norm_args a;
    uint8_t* y8;             // NULL: not wanted
    uint8_t* y8_scale;
    int64_t y8_ld, y8_scale_ld;
};
hipError_t launch_rms_norm(const RmsNormArgs& a, hipStream_t s);

size_t rms_norm_workspace_floats(int64_t rows, int64_t cols);     // of the backward pass
bool rms_norm_needs_means(int64_t cols);                          // it needs them without dgamma too
hipError_t launch_rms_norm_backward(const zi_rms_norm_backward_args& a, float* workspace, hipStream_t s);

// out (cols elements; with accumulate added to) of `count` rows of cols sums, added in a fixed order.
hipError_t launch_column_sums(const float* partials, int count, int64_t cols, void* out, int dtype, int accumulate, hipStream_t s);

struct MatmulArgs {
    const uint8_t* a;
    const uint8_t* b;
    const uint8_t* a_scale;
    const uint8_t* b_scale;
    void* d;
    const void* c;
    int64_t m, n, k;
    int64_t a_ld, b_ld, a_scale_ld, b_scale_ld, d_ld;
    int32_t a_shift, b_shift;     // row >> shift is its row of scales: 0 or 7
};
struct MatmulPlan {
    int shape;               // of the tiles, or kFewRows: the kernel for few rows
    uint32_t parts, part_steps;      // workgroups that share out k, and their steps of 128
};
constexpr int kFewRows = -1;
MatmulPlan plan_fp8_matmul(int64_t m, int64_t n, int64_t k);
// The same among shapes from `first` on, of which more than the smallest come in one part; and the time that it is expected to take, in us.  `alone`: what an epilogue adds to a round of tiles of
// 256 x 128 and of 256 x 256, which have a compute unit to themselves.
struct MatmulAlone {
    float rows_256_128, rows_256_256;
};
constexpr int kAloneShape = 4;       // the first of the two
MatmulPlan plan_fp8_matmul_from(int64_t m, int64_t n, int64_t k, int first, const MatmulAlone& alone, float& estimate);
hipError_t launch_fp8_matmul(const MatmulArgs& a, int dtype, float* partials, hipStream_t s);

}  // namespace zi
