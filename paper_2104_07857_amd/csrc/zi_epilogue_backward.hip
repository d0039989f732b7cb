// The gradient of what follows a product.
#include "zi_epilogue_octets.h"

namespace zi {

// dz of a tile, in all its forms, and the sums over the tile's rows, which a second kernel adds in their order.  Bound by memory as the tiles of the forward pass: 8191 x 16384, gelu_tanh to 8 bits both ways
// and dbias 150 us (810 MB, 5.4 TB/s) and 5 for the sums; dropout's of 16384 x 4096 58 (269 MB, 4.6 TB/s: ten rounds of the generator are 9 of its 18 instructions an element) and 5.  Where there is but one row of tiles they are dbias: 100 x 4096 in one
// kernel 5.1 us, in two 6.9; with two rows of tiles one after the other in a workgroup it is 6.8 against 6.7 (and, with 8-bit outputs, 12.2 against 9.8).
template <int DT, int ACT, Ends ENDS, bool LARGE>
__global__ __launch_bounds__(256) void epilogue_backward_kernel(const EpilogueBackwardArgs a, float* partials)
{
    __shared__ ResultSpace s_space;
    __shared__ float s_sum[4][kTile];
    const TileThread at(a.cols, a.dz8.tiles_across);
    const int t = threadIdx.x;
    float dz[8][8], sum[8] = {};
    const auto make = [&](auto whole) {
        Octet<DT> dy[8], z[ACT == ZI_ACT_NONE ? 1 : 8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (decltype(whole)::value || at.row0 + i < a.rows) {
                dy[i].template load<ENDS, LARGE>(a.dy, (at.row0 + i) * a.dy_ld + at.col, at.left);
                if constexpr (ACT != ZI_ACT_NONE)
                    if (ACT != kAnyActivation || a.z) z[i].template load<ENDS, LARGE>(a.z, (at.row0 + i) * a.z_ld + at.col, at.left);
            }
        const Dropout drop(a.drop);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int64_t row = at.row0 + i;
            if (!decltype(whole)::value && row >= a.rows) {
#pragma unroll
                for (int j = 0; j < 8; ++j) dz[i][j] = 0.0f;
                continue;
            }
            dy[i].template settle<ENDS>(at.left);
#pragma unroll
            for (int j = 0; j < 8; ++j) dz[i][j] = dy[i].get(j);
            if constexpr (ACT == ZI_ACT_NONE) {
                drop.apply(dz[i], (uint32_t)(at.col >> 3), (uint32_t)row);
            } else {
                float f[8] = {};
                if (ACT != kAnyActivation || a.z) {
                    z[i].template settle<ENDS>(at.left);
#pragma unroll
                    for (int j = 0; j < 8; ++j) f[j] = z[i].get(j);
                }
                if constexpr (ACT == ZI_ACT_RELU) drop.apply(dz[i], (uint32_t)(at.col >> 3), (uint32_t)row);       // (it leaves 0 at 0, whatever z is)
                else drop.apply(dz[i], f, (uint32_t)(at.col >> 3), (uint32_t)row);
                derive<ACT>(dz[i], f, a.activation);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[j] += dz[i][j];
            if (a.dz) {
                Octet<DT> w;
                w.set(dz[i]);
                put_octet<ENDS, LARGE>(w, a.dz, row * a.dz_ld + at.col, at.left);
            }
        }
    };
    if ((at.tile_row + 1) * kTile <= a.rows) make(std::true_type());
    else make(std::false_type());
    if (a.dbias) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            sum[j] += __shfl_xor(sum[j], 16);
            sum[j] += __shfl_xor(sum[j], 32);
            if ((t & 63) < 16) s_sum[t >> 6][(t & 15) * 8 + j] = sum[j];
        }
        __syncthreads();
        const int64_t col = at.tile_col * kTile + t;
        if (t < kTile && col < a.cols) {
            const float x = s_sum[0][t] + s_sum[1][t] + s_sum[2][t] + s_sum[3][t];
            if (a.rows > kTile) {
                partials[at.tile_row * a.cols + col] = x;
            } else if (a.dbias_dtype == ZI_FP32) {
                float* to = static_cast<float*>(a.dbias) + col;
                *to = a.accumulate ? *to + x : x;
            } else {
                uint16_t* to = static_cast<uint16_t*>(a.dbias) + col;
                Octet<DT> old;
                old.w[0] = *to;
                *to = (uint16_t)Octet<DT>::pair(a.accumulate ? old.get(0) + x : x, 0.0f);
            }
        }
    }
    if (a.dz8.out || a.dz8.turned) {
        if (LARGE || a.large_out) quantize_results<true>(a.dz8, dz, at.tile_row, at.tile_col, s_space);
        else quantize_results<false>(a.dz8, dz, at.tile_row, at.tile_col, s_space);
    }
}

namespace {

template <int DT>
void launch_backward_of(const EpilogueBackwardArgs& a, bool large, float* partials, hipStream_t s)
{
    const dim3 grid((unsigned)(a.dz8.tiles_across * ((a.rows + kTile - 1) / kTile))), block(256);
    with_kind(a.activation, a.cols, large, [&](auto act, auto ends, auto stream) {
        hipLaunchKernelGGL((epilogue_backward_kernel<DT, decltype(act)::value, decltype(ends)::value, decltype(stream)::value>), grid, block, 0, s, a, partials);
    });
}

}  // namespace

hipError_t launch_epilogue_backward(const EpilogueBackwardArgs& given, int dtype, float* partials, hipStream_t s)
{
    EpilogueBackwardArgs a = given;
    const int64_t out = a.rows * a.cols * ((a.dz ? 2 : 0) + (a.dz8.out ? 1 : 0) + (a.dz8.turned ? 1 : 0));
    const bool large = a.rows * a.cols * (a.z ? 4 : 2) + out >= kLargeBytes;
    a.large_out = out >= kLargeOutBytes;
    if (dtype == ZI_BF16) launch_backward_of<ZI_BF16>(a, large, partials, s);
    else launch_backward_of<ZI_FP16>(a, large, partials, s);
    return hipGetLastError();
}

}  // namespace zi
