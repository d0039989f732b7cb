// Which way a product with an epilogue is made (include/zi_epilogue.h).
#include "zi_epilogue_internal.h"

namespace zi {

// How a product is made, and whether all of its outputs come from there: tiles put out blocks of 128 rows or columns that are a workgroup's own.  Where the fastest way to the sums is none
// to the outputs, a second kernel that reads the sums again stands against the fastest way that is.
//
// Tiles of 256 rows have a compute unit to themselves, and nothing hides what becomes of their sums; of 128 x 128 there are two, one of which multiplies meanwhile.  So they are the faster ones for
// outputs in 8 bits up to k of 4000 or so.  us, 256 x 256 / 128 x 128: 8191 x 8192 x 2048 with gelu to 8 bits 201 / 160, both ways 223 / 178, 4096 x 16384 x 4096 285 / 265 and 308 / 278,
// 8192 x 32768 x 8192 1830 / 1967 and 1920 / 2055.  kAlone are fitted to 90 products (m of 64 to 16384, n of 128 to 32768, k of 181 to 16384, drawn evenly on a logarithmic scale) with outputs one way and both, without
// an activation, with gelu and silu, in each tile: on these same products the choice is 0.2 % slower than the fastest tile for one way along the rows and 0.3 % for the others (on other products it was not measured);
// without them 2.6 and 3.3 to 3.9 %.
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
    // (The estimate for parts has their sum in it already.)  1 x 16384 x 4096 to 8 bits: in two kernels 15.0 us, whole in tiles of 64 x 128 17.3 (rows of whole blocks in the kernel for few rows were not tried); 2048 x 2048 x 2048 transposed 22 and 14.
    const float second = plan.parts > 1 ? 0.0f : kSecond + 8.0f * (float)m * (float)n / kSecondStream;
    if (other.parts == 1 && whole + kWhole <= any + second) return {other, 1};
    return {plan, 0};
}

size_t fp8_matmul_epilogue_workspace_floats(int64_t m, int64_t n, int64_t k, int outputs8)
{
    const EpiloguePlan p = plan_fp8_matmul_epilogue(m, n, k, outputs8);
    return p.whole ? 0 : p.plan.parts * (size_t)m * (size_t)n;
}

}  // namespace zi
