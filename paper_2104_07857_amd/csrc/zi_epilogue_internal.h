// Internal interface between the C-ABI layer of the epilogues (zi_epilogue_api.hip) and their kernels.
#pragma once

#include "zi_epilogue.h"
#include "zi_fp8_internal.h"

namespace zi {

struct DropoutArgs {
    const uint64_t* d_offset;     // NULL: 0
    uint64_t seed, offset;
    uint32_t threshold;           // of numbers of 16 bits; 0: nothing is dropped
    float scale;
};

// What becomes of a matrix x (include/zi_epilogue.h).
struct EpilogueArgs {
    int64_t rows, cols;
    const void* bias;
    const void* residual;
    void* z;
    void* y;
    int64_t residual_ld, z_ld, y_ld;
    DropoutArgs drop;
    int32_t activation;
    QuantizeArgs y8;              // its out and turned; x and ld are not used
    bool large_out;               // outputs alone are more than what is worth keeping in the caches
};
// Where x comes from: 16 bits, or the sums that a product left in parts of rows x cols.
struct EpilogueSource {
    const void* x;                // NULL: sums
    int64_t ld;
    const float* sums;
    uint32_t parts;
};
hipError_t launch_epilogue_tiles(const EpilogueArgs& e, const EpilogueSource& x, int dtype, hipStream_t s);     // also where `turned` is wanted
hipError_t launch_epilogue(const EpilogueArgs& e, const EpilogueSource& x, int dtype, hipStream_t s);

struct EpiloguePlan {
    MatmulPlan plan;
    int32_t whole;                // all outputs come from the product's kernel; else a second one makes them of its sums
};
EpiloguePlan plan_fp8_matmul_epilogue(int64_t m, int64_t n, int64_t k, int outputs8);
size_t fp8_matmul_epilogue_workspace_floats(int64_t m, int64_t n, int64_t k, int outputs8);
hipError_t launch_fp8_matmul_epilogue(const MatmulArgs& a, const EpiloguePlan& p, const EpilogueArgs& e, int dtype, float* workspace, hipStream_t s);

struct EpilogueBackwardArgs {
    int64_t rows, cols;
    const void* dy;
    const void* z;
    void* dz;
    int64_t dy_ld, z_ld, dz_ld;
    void* dbias;
    int32_t dbias_dtype, accumulate;
    DropoutArgs drop;
    int32_t activation;
    QuantizeArgs dz8;
    bool large_out;
};
// dz in all its forms, and dbias where there is but one row of tiles; of more of them their sums, in `partials`.
hipError_t launch_epilogue_backward(const EpilogueBackwardArgs& a, int dtype, float* partials, hipStream_t s);

// The kernels (266 of them) are a library of their own, libzi_epilogue.so beside libzi.so, which the first call that launches one loads: programs that only step do without.  Both have to be of
// one build, which a number made of all sources and flags says (build.py), since they hand each other the structures above as they are.
#ifndef ZI_BUILD
#define ZI_BUILD 0
#endif
struct EpilogueKernels {
    uint64_t build;
    decltype(&launch_epilogue) epilogue;
    decltype(&launch_fp8_matmul_epilogue) matmul;
    decltype(&launch_epilogue_backward) backward;
};

}  // namespace zi
