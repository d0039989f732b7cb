// What the kernels of what follows a product, by itself, share (include/zi_epilogue.h).  All are bound by memory, with dropout or an activation close to what the vector units do meanwhile, so
// every kernel is made for one activation (but those of sums and of rows of less than eight).  LARGE: what is read and written is more than the memory-side cache holds, and passes the caches
// by.  us, without / with: dropout and residual of 16384 x 4096 (403 MB) 69.6 / 63.5, of 4096 x 8192 (201 MB) 31.7 / 35.2.  Compile with -ffp-contract=off.
#pragma once

#include <hip/hip_runtime.h>

#include "zi_epilogue_device.h"
#include "zi_fp8_tile.h"

namespace zi {

// ---- octets ---------------------------------------------------------------------------------------------------

// `valid` columns of an octet, of which there are eight or (ENDS kWhole) none.
template <Ends ENDS, bool LARGE, typename T>
__device__ __forceinline__ void put_octet(const T& x, void* base, int64_t at, int left)
{
    if constexpr (ENDS == Ends::kWhole) {
        if (left <= 0) return;
        left = 8;
    }
    if (left <= 0) return;
    x.template store<LARGE>(base, at, left);
}

// An octet's x (16 bits, or sums of a product's parts in their order) and how it becomes y.
template <int DT, int ACT, bool SUMS, Ends ENDS, bool LARGE>
struct EpilogueOctet {
    Octet<SUMS ? ZI_FP32 : DT> x;
    Octet<DT> residual;

    __device__ __forceinline__ void load(const EpilogueArgs& e, const EpilogueSource& from, int64_t row, int64_t col, int left)
    {
        if constexpr (SUMS) x.template load<ENDS, LARGE>(from.sums, row * e.cols + col, left);
        else x.template load<ENDS, LARGE>(from.x, row * from.ld + col, left);
        if (e.residual) residual.template load<ENDS, LARGE>(e.residual, row * e.residual_ld + col, left);
    }
    // y, zeros behind the row's end; z goes out on the way.
    __device__ __forceinline__ void finish(const EpilogueArgs& e, const EpilogueSource& from, const Dropout& drop, const float (&bias)[8], int64_t row, int64_t col, int left,
                                           float (&y)[8])
    {
        if constexpr (!SUMS) x.template settle<ENDS>(left);
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = x.get(j);
        if (e.bias) {
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] += bias[j];
        }
        if (e.z) {
            Octet<DT> w;
            w.set(y);
            put_octet<ENDS, LARGE>(w, e.z, row * e.z_ld + col, left);
        }
        activate<ACT>(y, e.activation);
        drop.apply(y, (uint32_t)(col >> 3), (uint32_t)row);
        if (e.residual) {
            residual.template settle<ENDS>(left);
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] += residual.get(j);
        }
    }
};
// The other parts' sums, in their order, for octets of R rows: with few rows three parts at a time are under way (there may be any number from 1 to 16), with more two.
template <int R, int APART, int DT, int ACT, Ends ENDS>
__device__ __forceinline__ void add_parts(EpilogueOctet<DT, ACT, true, ENDS, false> (&x)[R], const EpilogueArgs& e, const EpilogueSource& from, int64_t row0, int64_t col, int left)
{
    constexpr int kParts = R <= 2 ? 3 : 2;
#pragma unroll
    for (int r = 0; r < R; ++r)
        if (row0 + r * APART < e.rows) x[r].x.template settle<ENDS>(left);
    for (uint32_t first = 1; first < from.parts; first += kParts) {
        Octet<ZI_FP32> more[kParts][R];
#pragma unroll
        for (int i = 0; i < kParts; ++i)
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (first + i < from.parts && row0 + r * APART < e.rows)
                    more[i][r].template load<ENDS>(from.sums, ((int64_t)(first + i) * e.rows + row0 + r * APART) * e.cols + col, left);
#pragma unroll
        for (int i = 0; i < kParts; ++i)
#pragma unroll
            for (int r = 0; r < R; ++r) {
                if (first + i >= from.parts || row0 + r * APART >= e.rows) continue;
                more[i][r].template settle<ENDS>(left);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[r].x.w[j] = __float_as_uint(x[r].x.get(j) + more[i][r].get(j));
            }
    }
}
template <int DT, Ends ENDS>
__device__ __forceinline__ void load_bias(const void* bias, int64_t col, int left, float (&x)[8])
{
    Octet<DT> b;
    b.clear();
    if (bias) {
        b.template load<ENDS>(bias, col, left);
        b.template settle<ENDS>(left);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = b.get(j);
}

// What holds for a thread's octets of a tile of 128 x 128 (zi_fp8_tile.h).
struct TileThread {
    int64_t tile_row, tile_col, row0, col;
    int left;
    __device__ __forceinline__ TileThread(int64_t cols, uint32_t across)
    {
        place_of_tile(blockIdx.x, gridDim.x, across, tile_row, tile_col);
        row0 = tile_row * kTile + (threadIdx.x >> 4) * 8;
        col = tile_col * kTile + (threadIdx.x & 15) * 8;
        left = cols - col < 8 ? (int)(cols - col) : 8;
    }
};

// ---- which kernel ---------------------------------------------------------------------------------------------

// Large outputs in 8 bits pass the caches by for less: 8191 x 8192 in 16 bits to 8 bits both ways 58.2 us without, 54.9 with.
constexpr int64_t kLargeBytes = (int64_t)256 << 20, kLargeOutBytes = (int64_t)96 << 20;

// f with what kernels of 16-bit matrices are made for: the activation, how rows end, and whether they are large (rows of less than eight are not).
template <typename F>
void with_kind(int activation, int64_t cols, bool large, const F& f)
{
    const auto of = [&](auto act) {
        if (cols % 8 == 0) {
            if (large) f(act, std::integral_constant<Ends, Ends::kWhole>(), std::true_type());
            else f(act, std::integral_constant<Ends, Ends::kWhole>(), std::false_type());
        } else {
            if (large) f(act, std::integral_constant<Ends, Ends::kMoved>(), std::true_type());
            else f(act, std::integral_constant<Ends, Ends::kMoved>(), std::false_type());
        }
    };
    if (cols < 8) return f(std::integral_constant<int, kAnyActivation>(), std::integral_constant<Ends, Ends::kApart>(), std::false_type());
    switch (activation) {
    case ZI_ACT_NONE: return of(std::integral_constant<int, ZI_ACT_NONE>());
    case ZI_ACT_RELU: return of(std::integral_constant<int, ZI_ACT_RELU>());
    case ZI_ACT_GELU: return of(std::integral_constant<int, ZI_ACT_GELU>());
    case ZI_ACT_GELU_TANH: return of(std::integral_constant<int, ZI_ACT_GELU_TANH>());
    case ZI_ACT_SILU: return of(std::integral_constant<int, ZI_ACT_SILU>());
    }
}
// The same of sums, of an activation that is not known.
template <typename F>
void with_ends(int64_t cols, const F& f)
{
    if (cols % 8 == 0) f(std::integral_constant<Ends, Ends::kWhole>());
    else if (cols > 8) f(std::integral_constant<Ends, Ends::kMoved>());
    else f(std::integral_constant<Ends, Ends::kApart>());
}
inline int64_t bytes_out(const EpilogueArgs& e) { return e.rows * e.cols * ((e.z ? 2 : 0) + (e.y ? 2 : 0) + (e.y8.out ? 1 : 0) + (e.y8.turned ? 1 : 0)); }
inline bool is_large(const EpilogueArgs& e) { return e.rows * e.cols * (e.residual ? 4 : 2) + bytes_out(e) >= kLargeBytes; }

}  // namespace zi
