// Kernels of what follows a product, by itself, and of its gradients (include/zi_epilogue.h).  All are bound by memory, with dropout or an activation close to what the vector units do
// meanwhile, so every kernel is made for one activation (but those of sums and of rows of less than eight).  Compile with -ffp-contract=off.
#include <hip/hip_runtime.h>

#include "zi_epilogue_device.h"
#include "zi_fp8_tile.h"

namespace zi {

// ---- octets ---------------------------------------------------------------------------------------------------

// `valid` columns of an octet, of which there are eight or (ENDS kWhole) none.
template <Ends ENDS, typename T>
__device__ __forceinline__ void put_octet(const T& x, void* base, int64_t at, int left, bool stream)
{
    if constexpr (ENDS == Ends::kWhole) {
        if (left <= 0) return;
        left = 8;
    }
    if (left <= 0) return;
    if (stream) x.template store<true>(base, at, left);
    else x.store(base, at, left);
}

// An octet's x (16 bits, or sums of a product's parts in their order) and how it becomes y.
template <int DT, int ACT, bool SUMS, Ends ENDS>
struct EpilogueOctet {
    Octet<SUMS ? ZI_FP32 : DT> x;
    Octet<DT> residual;

    __device__ __forceinline__ void load(const EpilogueArgs& e, const EpilogueSource& from, int64_t row, int64_t col, int left)
    {
        if constexpr (SUMS) x.template load<ENDS>(from.sums, row * e.cols + col, left);
        else x.template load<ENDS>(from.x, row * from.ld + col, left);
        if (e.residual) residual.template load<ENDS>(e.residual, row * e.residual_ld + col, left);
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
            put_octet<ENDS>(w, e.z, row * e.z_ld + col, left, e.large);
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
// The other parts' sums, in their order, for octets of R rows: with few rows three parts at a time are under way (there are 2, 4, 8 or 16), with more two.
template <int R, int APART, int DT, int ACT, Ends ENDS>
__device__ __forceinline__ void add_parts(EpilogueOctet<DT, ACT, true, ENDS> (&x)[R], const EpilogueArgs& e, const EpilogueSource& from, int64_t row0, int64_t col, int left)
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

// ---- forward --------------------------------------------------------------------------------------------------

// Rows as they are.  L lanes have a strip of 8 L columns, whose bias stays in registers, and R rows each at a time, whose loads go out together.
template <int DT, int ACT, bool SUMS, int L, int R, Ends ENDS>
__global__ __launch_bounds__(256) void epilogue_rows_kernel(const EpilogueArgs e, const EpilogueSource from, uint32_t strips)
{
    constexpr int kApartBy = 64 / L, kGroup = 4 * R * kApartBy;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t col = ((int64_t)(blockIdx.x % strips) * L + lane % L) * 8;
    const int64_t behind = e.cols - col;
    const int left = behind < 8 ? (int)behind : 8;
    for (int64_t first = (int64_t)(blockIdx.x / strips) * kGroup; first < e.rows; first += (int64_t)(gridDim.x / strips) * kGroup) {
        const int64_t row0 = first + wave * (R * kApartBy) + lane / L;
        EpilogueOctet<DT, ACT, SUMS, ENDS> x[R];
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (row0 + i * kApartBy < e.rows) x[i].load(e, from, row0 + i * kApartBy, col, left);
        float bias[8];
        load_bias<DT, ENDS>(e.bias, col, left, bias);
        const Dropout drop(e.drop);
        if constexpr (SUMS) add_parts<R, kApartBy>(x, e, from, row0, col, left);
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int64_t row = row0 + i * kApartBy;
            if (row >= e.rows) continue;                  // (all 16 lanes of a block)
            float y[8];
            x[i].finish(e, from, drop, bias, row, col, left, y);
            if (e.y) {
                Octet<DT> w;
                w.set(y);
                put_octet<ENDS>(w, e.y, row * e.y_ld + col, left, e.large);
            }
            if (e.y8.out) {
                const uint32_t byte = scale_byte(max_16(most_of(y)));
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
template <int DT, int ACT, bool SUMS, Ends ENDS>
__global__ __launch_bounds__(256) void epilogue_tiles_kernel(const EpilogueArgs e, const EpilogueSource from)
{
    __shared__ ResultSpace s_space;
    const TileThread at(e.cols, e.y8.tiles_across);
    float y[8][8];
    const auto make = [&](auto whole) {               // (a tile with all its rows needs no look at them)
        EpilogueOctet<DT, ACT, SUMS, ENDS> x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (decltype(whole)::value || at.row0 + i < e.rows) x[i].load(e, from, at.row0 + i, at.col, at.left);
        float bias[8];
        load_bias<DT, ENDS>(e.bias, at.col, at.left, bias);
        const Dropout drop(e.drop);
        if constexpr (SUMS) add_parts<8, 1>(x, e, from, at.row0, at.col, at.left);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (!decltype(whole)::value && at.row0 + i >= e.rows) {
#pragma unroll
                for (int j = 0; j < 8; ++j) y[i][j] = 0.0f;
                continue;
            }
            x[i].finish(e, from, drop, bias, at.row0 + i, at.col, at.left, y[i]);
            if (e.y) {
                Octet<DT> w;
                w.set(y[i]);
                put_octet<ENDS>(w, e.y, (at.row0 + i) * e.y_ld + at.col, at.left, e.large);
            }
        }
    };
    if ((at.tile_row + 1) * kTile <= e.rows) make(std::true_type());
    else make(std::false_type());
    if (e.large) quantize_results<true>(e.y8, y, at.tile_row, at.tile_col, s_space);
    else quantize_results<false>(e.y8, y, at.tile_row, at.tile_col, s_space);
}

// ---- backward -------------------------------------------------------------------------------------------------

// dz of a tile, in all its forms, and the sums over the tile's rows, which a second kernel adds in their order.  Where there is but one row of tiles they are dbias: 100 x 4096 in one
// kernel 5.1 us, in two 6.9; with two rows of tiles one after the other in a workgroup it is 6.8 against 6.7 (and, with 8-bit outputs, 12.2 against 9.8).
template <int DT, int ACT, Ends ENDS>
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
                dy[i].template load<ENDS>(a.dy, (at.row0 + i) * a.dy_ld + at.col, at.left);
                if constexpr (ACT != ZI_ACT_NONE)
                    if (ACT != kAnyActivation || a.z) z[i].template load<ENDS>(a.z, (at.row0 + i) * a.z_ld + at.col, at.left);
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
            drop.apply(dz[i], (uint32_t)(at.col >> 3), (uint32_t)row);
            if constexpr (ACT != ZI_ACT_NONE) {
                if (ACT != kAnyActivation || a.z) {
                    float f[8];
                    z[i].template settle<ENDS>(at.left);
#pragma unroll
                    for (int j = 0; j < 8; ++j) f[j] = z[i].get(j);
                    derive<ACT>(dz[i], f, a.activation);
                }
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[j] += dz[i][j];
            if (a.dz) {
                Octet<DT> w;
                w.set(dz[i]);
                put_octet<ENDS>(w, a.dz, row * a.dz_ld + at.col, at.left, a.large);
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
        if (a.large) quantize_results<true>(a.dz8, dz, at.tile_row, at.tile_col, s_space);
        else quantize_results<false>(a.dz8, dz, at.tile_row, at.tile_col, s_space);
    }
}

// ---- which kernel ---------------------------------------------------------------------------------------------

namespace {

constexpr int64_t kMostGroups = (int64_t)1 << 20;     // workgroups over rows
constexpr int kRowsAtATime = 4;
// Outputs of more do not stay in the memory-side cache for whoever reads them next, and pass it by.
constexpr int64_t kLargeBytes = (int64_t)96 << 20;

template <int N>
using int_type = std::integral_constant<int, N>;

// f with what kernels of 16-bit matrices are made for: the activation and how rows end.
template <typename F>
void with_kind(int activation, int64_t cols, const F& f)
{
    const auto of = [&](auto act) {
        if (cols % 8 == 0) f(act, std::integral_constant<Ends, Ends::kWhole>());
        else f(act, std::integral_constant<Ends, Ends::kMoved>());
    };
    if (cols < 8) return f(int_type<kAnyActivation>(), std::integral_constant<Ends, Ends::kApart>());
    switch (activation) {
    case ZI_ACT_NONE: return of(int_type<ZI_ACT_NONE>());
    case ZI_ACT_RELU: return of(int_type<ZI_ACT_RELU>());
    case ZI_ACT_GELU: return of(int_type<ZI_ACT_GELU>());
    case ZI_ACT_GELU_TANH: return of(int_type<ZI_ACT_GELU_TANH>());
    case ZI_ACT_SILU: return of(int_type<ZI_ACT_SILU>());
    }
}

template <int DT, int ACT, bool SUMS, Ends ENDS>
void launch_forward(const EpilogueArgs& e, const EpilogueSource& from, hipStream_t s)
{
    const int64_t down = (e.rows + kTile - 1) / kTile;
    if (e.y8.turned) {
        hipLaunchKernelGGL((epilogue_tiles_kernel<DT, ACT, SUMS, ENDS>), dim3((unsigned)(e.y8.tiles_across * down)), dim3(256), 0, s, e, from);
        return;
    }
    const auto rows = [&](int lanes, int at_a_time, auto kernel) {
        const int64_t strips = (e.cols + 8 * lanes - 1) / (8 * lanes), each = 4 * (64 / lanes) * at_a_time, groups = (e.rows + each - 1) / each;
        const int64_t most = strips < kMostGroups ? kMostGroups / strips : 1;
        hipLaunchKernelGGL(kernel, dim3((unsigned)(strips * (groups < most ? groups : most))), dim3(256), 0, s, e, from, (uint32_t)strips);
    };
    constexpr int kEach = SUMS ? 1 : kRowsAtATime;
    if (ENDS == Ends::kApart || e.cols <= 128) rows(16, 2, epilogue_rows_kernel<DT, ACT, SUMS, 16, 2, ENDS>);
    else if constexpr (ENDS != Ends::kApart) rows(64, kEach, epilogue_rows_kernel<DT, ACT, SUMS, 64, kEach, ENDS>);
}

template <int DT>
void launch_forward_of(const EpilogueArgs& e, const EpilogueSource& from, hipStream_t s)
{
    if (!from.x) {
        if (e.cols % 8 == 0) launch_forward<DT, kAnyActivation, true, Ends::kWhole>(e, from, s);
        else if (e.cols > 8) launch_forward<DT, kAnyActivation, true, Ends::kMoved>(e, from, s);
        else launch_forward<DT, kAnyActivation, true, Ends::kApart>(e, from, s);
        return;
    }
    with_kind(e.activation, e.cols, [&](auto act, auto ends) { launch_forward<DT, decltype(act)::value, false, decltype(ends)::value>(e, from, s); });
}
template <int DT>
void launch_backward_of(const EpilogueBackwardArgs& a, float* partials, hipStream_t s)
{
    const dim3 grid((unsigned)(a.dz8.tiles_across * ((a.rows + kTile - 1) / kTile))), block(256);
    with_kind(a.activation, a.cols, [&](auto act, auto ends) {
        hipLaunchKernelGGL((epilogue_backward_kernel<DT, decltype(act)::value, decltype(ends)::value>), grid, block, 0, s, a, partials);
    });
}

}  // namespace

hipError_t launch_epilogue(const EpilogueArgs& given, const EpilogueSource& from, int dtype, hipStream_t s)
{
    EpilogueArgs e = given;
    e.large = e.rows * e.cols * ((e.z ? 2 : 0) + (e.y ? 2 : 0) + (e.y8.out ? 1 : 0) + (e.y8.turned ? 1 : 0)) >= kLargeBytes;
    if (dtype == ZI_BF16) launch_forward_of<ZI_BF16>(e, from, s);
    else launch_forward_of<ZI_FP16>(e, from, s);
    return hipGetLastError();
}

hipError_t launch_epilogue_backward(const EpilogueBackwardArgs& given, int dtype, float* partials, hipStream_t s)
{
    EpilogueBackwardArgs a = given;
    a.large = a.rows * a.cols * ((a.dz ? 2 : 0) + (a.dz8.out ? 1 : 0) + (a.dz8.turned ? 1 : 0)) >= kLargeBytes;
    const int64_t down = (a.rows + kTile - 1) / kTile;
    if (a.rows > 0) {
        if (dtype == ZI_BF16) launch_backward_of<ZI_BF16>(a, partials, s);
        else launch_backward_of<ZI_FP16>(a, partials, s);
        const hipError_t err = hipGetLastError();
        if (err != hipSuccess || down == 1) return err;
    }
    return a.dbias ? launch_column_sums(partials, (int)down, a.cols, a.dbias, a.dbias_dtype, a.accumulate, s) : hipSuccess;
}

}  // namespace zi
