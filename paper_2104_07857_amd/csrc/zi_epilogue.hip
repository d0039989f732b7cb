// Kernels of what follows a product, by itself, and of its gradients (include/zi_epilogue.h).  All are bound by memory, with dropout or an activation close to what the vector units do
// meanwhile.  Compile with -ffp-contract=off.
#include <hip/hip_runtime.h>

#include "zi_epilogue_device.h"
#include "zi_fp8_tile.h"

namespace zi {

// ---- forward --------------------------------------------------------------------------------------------------

// An octet's x (16 bits, or sums of a product's parts in their order) and how it becomes y.
template <int DT, bool SUMS, Ends ENDS>
struct EpilogueOctet {
    Octet<SUMS ? ZI_FP32 : DT> x;
    Octet<DT> residual;

    __device__ __forceinline__ void clear()
    {
        x.clear();
        residual.clear();
    }
    __device__ __forceinline__ void load(const EpilogueArgs& e, const EpilogueSource& from, int64_t row, int64_t col, int left)
    {
        if constexpr (SUMS) x.template load<ENDS>(from.sums, row * e.cols + col, left);
        else x.template load<ENDS>(from.x, row * from.ld + col, left);
        if (e.residual) residual.template load<ENDS>(e.residual, row * e.residual_ld + col, left);
    }
    // y of `valid` columns (zeros behind them); z goes out on the way.
    __device__ __forceinline__ void finish(const EpilogueArgs& e, const EpilogueSource& from, const Dropout& drop, const float (&bias)[8], int64_t row, int64_t col, int left,
                                           float (&y)[8])
    {
        x.template settle<ENDS>(left);
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = x.get(j);
        if constexpr (SUMS) {
            for (uint32_t i = 1; i < from.parts; ++i) {
                Octet<ZI_FP32> more;
                more.template load<ENDS>(from.sums, ((int64_t)i * e.rows + row) * e.cols + col, left);
                more.template settle<ENDS>(left);
#pragma unroll
                for (int j = 0; j < 8; ++j) y[j] += more.get(j);
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] += bias[j];
        if (e.z && left > 0) {
            Octet<DT> w;
            w.set(y);
            w.store(e.z, row * e.z_ld + col, left);
        }
        activate(y, e.activation);
        drop.apply(y, (uint32_t)(col >> 3), (uint32_t)row);
        if (e.residual) {
            residual.template settle<ENDS>(left);
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] += residual.get(j);
        }
    }
};
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

// Rows as they are.  L lanes have a strip of 8 L columns, whose bias stays in registers, and kRows rows each at a time, whose loads go out together.
template <int DT, bool SUMS, int L, Ends ENDS>
__global__ __launch_bounds__(256) void epilogue_rows_kernel(const EpilogueArgs e, const EpilogueSource from, uint32_t strips)
{
    constexpr int kRows = 4, kApartBy = 64 / L, kGroup = 4 * kRows * kApartBy;
    const Dropout drop(e.drop);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t col = ((int64_t)(blockIdx.x % strips) * L + lane % L) * 8;
    const int64_t behind = e.cols - col;
    const int left = behind < 8 ? (int)behind : 8;
    float bias[8];
    load_bias<DT, ENDS>(e.bias, col, left, bias);
    for (int64_t first = (int64_t)(blockIdx.x / strips) * kGroup; first < e.rows; first += (int64_t)(gridDim.x / strips) * kGroup) {
        const int64_t row0 = first + wave * (kRows * kApartBy) + lane / L;
        EpilogueOctet<DT, SUMS, ENDS> x[kRows];
#pragma unroll
        for (int i = 0; i < kRows; ++i)
            if (row0 + i * kApartBy < e.rows) x[i].load(e, from, row0 + i * kApartBy, col, left);
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const int64_t row = row0 + i * kApartBy;
            if (row >= e.rows) continue;                  // (all 16 lanes of a block)
            float y[8];
            x[i].finish(e, from, drop, bias, row, col, left, y);
            if (e.y && left > 0) {
                Octet<DT> w;
                w.set(y);
                w.store(e.y, row * e.y_ld + col, left);
            }
            if (e.y8.out) {
                uint32_t most = 0;
#pragma unroll
                for (int j = 0; j < 8; ++j) most = max_of(most, magnitudes<ZI_FP32, false>(__float_as_uint(y[j])));
                if (most >= kInfinity<ZI_FP32>) {
                    most = 0;
#pragma unroll
                    for (int j = 0; j < 8; ++j) most = max_of(most, magnitudes<ZI_FP32, true>(__float_as_uint(y[j])));
                }
                const uint32_t byte = scale_byte(max_16(most));
                if (left > 0) {
                    const float scale = scale_of(byte);
                    *reinterpret_cast<u32x2*>(e.y8.out + row * e.y8.out_ld + col) =
                        u32x2{four_e4m3(y[0], y[1], y[2], y[3], scale), four_e4m3(y[4], y[5], y[6], y[7], scale)};
                    if ((lane & 15) == 0) e.y8.out_scale[row * e.y8.out_scale_ld + col / kFp8Block] = (uint8_t)byte;
                }
            }
        }
    }
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

// Tiles, whose transposed numbers are wanted.
template <int DT, bool SUMS, Ends ENDS>
__global__ __launch_bounds__(256) void epilogue_tiles_kernel(const EpilogueArgs e, const EpilogueSource from)
{
    __shared__ TileSpace<ZI_FP32> s_space;
    const Dropout drop(e.drop);
    const TileThread at(e.cols, e.y8.tiles_across);
    float bias[8];
    load_bias<DT, ENDS>(e.bias, at.col, at.left, bias);
    EpilogueOctet<DT, SUMS, ENDS> x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (at.row0 + i < e.rows) x[i].load(e, from, at.row0 + i, at.col, at.left);
    Octet<ZI_FP32> y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        y[i].clear();
        if (at.row0 + i >= e.rows) continue;
        float f[8];
        x[i].finish(e, from, drop, bias, at.row0 + i, at.col, at.left, f);
        y[i].set(f);
        if (e.y && at.left > 0) {
            Octet<DT> w;
            w.set(f);
            w.store(e.y, (at.row0 + i) * e.y_ld + at.col, at.left);
        }
    }
    quantize_tile<ZI_FP32, false>(e.y8, y, at.tile_row, at.tile_col, s_space);
}

// ---- backward -------------------------------------------------------------------------------------------------

// dz of a tile, in all its forms, and the sums over the tile's rows, which a second kernel adds in their order.
template <int DT, Ends ENDS>
__global__ __launch_bounds__(256) void epilogue_backward_kernel(const EpilogueBackwardArgs a, float* partials)
{
    __shared__ TileSpace<ZI_FP32> s_space;
    __shared__ float s_sum[4][kTile];
    const Dropout drop(a.drop);
    const TileThread at(a.cols, a.dz8.tiles_across);
    const int t = threadIdx.x;
    const bool with_z = a.activation != ZI_ACT_NONE;
    Octet<DT> dy[8], z[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (at.row0 + i >= a.rows) continue;
        dy[i].template load<ENDS>(a.dy, (at.row0 + i) * a.dy_ld + at.col, at.left);
        if (with_z) z[i].template load<ENDS>(a.z, (at.row0 + i) * a.z_ld + at.col, at.left);
    }
    Octet<ZI_FP32> dz[8];
    float sum[8] = {};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        dz[i].clear();
        const int64_t row = at.row0 + i;
        if (row >= a.rows) continue;
        dy[i].template settle<ENDS>(at.left);
        float f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = dy[i].get(j);
        drop.apply(f, (uint32_t)(at.col >> 3), (uint32_t)row);
        if (with_z) {
            z[i].template settle<ENDS>(at.left);
            with_activation(a.activation, [&](auto act) {
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] = with_derivative<decltype(act)::value>(f[j], z[i].get(j));
            });
        }
        dz[i].set(f);
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] += f[j];
        if (a.dz && at.left > 0) {
            Octet<DT> w;
            w.set(f);
            w.store(a.dz, row * a.dz_ld + at.col, at.left);
        }
    }
    if (a.dbias) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            sum[j] += __shfl_xor(sum[j], 16);
            sum[j] += __shfl_xor(sum[j], 32);
            if ((t & 63) < 16) s_sum[t >> 6][(t & 15) * 8 + j] = sum[j];
        }
        __syncthreads();
        const int64_t col = at.tile_col * kTile + t;
        if (t < kTile && col < a.cols) partials[at.tile_row * a.cols + col] = s_sum[0][t] + s_sum[1][t] + s_sum[2][t] + s_sum[3][t];
    }
    if (a.dz8.out || a.dz8.turned) quantize_tile<ZI_FP32, false>(a.dz8, dz, at.tile_row, at.tile_col, s_space);
}

// ---- which kernel ---------------------------------------------------------------------------------------------

namespace {

constexpr int64_t kMostGroups = (int64_t)1 << 20;     // workgroups over rows

template <int DT, bool SUMS, Ends ENDS>
void launch_forward(const EpilogueArgs& e, const EpilogueSource& from, hipStream_t s)
{
    const int64_t down = (e.rows + kTile - 1) / kTile;
    if (e.y8.turned) {
        hipLaunchKernelGGL((epilogue_tiles_kernel<DT, SUMS, ENDS>), dim3((unsigned)(e.y8.tiles_across * down)), dim3(256), 0, s, e, from);
        return;
    }
    const auto rows = [&](auto lanes, auto kernel) {
        constexpr int kLanes = decltype(lanes)::value;
        const int64_t strips = (e.cols + 8 * kLanes - 1) / (8 * kLanes), groups = (e.rows + 1024 / kLanes - 1) / (1024 / kLanes);
        const int64_t most = strips < kMostGroups ? kMostGroups / strips : 1;
        hipLaunchKernelGGL(kernel, dim3((unsigned)(strips * (groups < most ? groups : most))), dim3(256), 0, s, e, from, (uint32_t)strips);
    };
    if (e.cols <= 128) rows(std::integral_constant<int, 16>(), epilogue_rows_kernel<DT, SUMS, 16, ENDS>);
    else rows(std::integral_constant<int, 64>(), epilogue_rows_kernel<DT, SUMS, 64, ENDS>);
}
template <int DT, bool SUMS>
void launch_forward_of(const EpilogueArgs& e, const EpilogueSource& from, hipStream_t s)
{
    if (e.cols % 8 == 0) launch_forward<DT, SUMS, Ends::kWhole>(e, from, s);
    else if (e.cols > 8) launch_forward<DT, SUMS, Ends::kMoved>(e, from, s);
    else launch_forward<DT, SUMS, Ends::kApart>(e, from, s);
}
template <int DT>
void launch_backward_of(const EpilogueBackwardArgs& a, float* partials, hipStream_t s)
{
    const dim3 grid((unsigned)(a.dz8.tiles_across * ((a.rows + kTile - 1) / kTile))), block(256);
    if (a.cols % 8 == 0) hipLaunchKernelGGL((epilogue_backward_kernel<DT, Ends::kWhole>), grid, block, 0, s, a, partials);
    else if (a.cols > 8) hipLaunchKernelGGL((epilogue_backward_kernel<DT, Ends::kMoved>), grid, block, 0, s, a, partials);
    else hipLaunchKernelGGL((epilogue_backward_kernel<DT, Ends::kApart>), grid, block, 0, s, a, partials);
}

}  // namespace

hipError_t launch_epilogue(const EpilogueArgs& e, const EpilogueSource& from, int dtype, hipStream_t s)
{
    if (dtype == ZI_BF16) from.x ? launch_forward_of<ZI_BF16, false>(e, from, s) : launch_forward_of<ZI_BF16, true>(e, from, s);
    else from.x ? launch_forward_of<ZI_FP16, false>(e, from, s) : launch_forward_of<ZI_FP16, true>(e, from, s);
    return hipGetLastError();
}

hipError_t launch_epilogue_backward(const EpilogueBackwardArgs& a, int dtype, float* partials, hipStream_t s)
{
    const int64_t down = (a.rows + kTile - 1) / kTile;
    if (a.rows > 0) {
        if (dtype == ZI_BF16) launch_backward_of<ZI_BF16>(a, partials, s);
        else launch_backward_of<ZI_FP16>(a, partials, s);
        const hipError_t err = hipGetLastError();
        if (err != hipSuccess) return err;
    }
    return a.dbias ? launch_column_sums(partials, (int)down, a.cols, a.dbias, a.dbias_dtype, a.accumulate, s) : hipSuccess;
}

}  // namespace zi
