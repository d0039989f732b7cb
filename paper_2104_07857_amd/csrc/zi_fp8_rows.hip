// Kernels of the 8-bit operators that go over rows once: quantisation, the root-mean-square norm and its backward pass.
// All are bound by memory; see include/zi_fp8.h for the formulas.  Compile with -ffp-contract=off.
#include <hip/hip_runtime.h>

#include "zi_fp8_tile.h"

namespace zi {

// ---- quantisation ---------------------------------------------------------------------------------------------

// A workgroup takes a tile of 128 x 128, which holds whole blocks of every kind, so x is read once whatever is wanted.
// A thread has 8 x 8 elements in registers; 16 threads (a row of lanes) have a tile's row, so the largest of a row's
// block comes from its lanes and that of a column's block from the thread's own rows, two steps over lanes and four
// wavefronts.  The transposed numbers pass through LDS, which makes rows of 128 bytes of them.  16384 x 4096 fp32 in squares, both 73 us (403 MB, 5.5 TB/s);
// 8191 x 8192 bf16, blocks of rows, both 55 us (269 MB, 4.9 TB/s, with 6 MB more of scales that were written in pieces); one row of 1000 3.7 us.
// LARGE: the outputs do not stay in the memory-side cache for whoever reads them next.  Their stores pass it by then.  us, ordinary / so: 32768 x 8192
// fp32 in squares, both 316 / 287, 16384 x 8192 bf16 114 / 102; but quantisation and product of 4096 x 4096 (x 4096) 70 / 75.
// Large outputs of fp32 keep to two workgroups on a compute unit, three where registers allow them: 16384 x 4096 in squares 72.8 / 77.1, 32768 x 8192 280 /
// 296, but 8192 x 8192 in blocks of rows 76.4 / 73.3, and with small outputs 4096 x 4096 20.5 / 20.0.
constexpr int64_t kLargeBytes = (int64_t)96 << 20;
template <int DT, bool LARGE>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1, LARGE && DT == ZI_FP32 ? 2 : 8))) void fp8_quantize_kernel(const QuantizeArgs a)
{
    __shared__ uint32_t s_col[4][kTile / 8 * Octet<DT>::kWords];
    __shared__ uint32_t s_all[4];
    __shared__ __align__(16) uint8_t s_turned[kTile * kTile];

    const int t = threadIdx.x, o = t & 15, g = t >> 4, wave = t >> 6;
    int64_t tile_row, tile_col;
    place_of_tile(blockIdx.x, gridDim.x, a.tiles_across, tile_row, tile_col);
    const auto put = [](auto x, auto* at) {
        if constexpr (LARGE) __builtin_nontemporal_store(x, at);
        else *at = x;
    };
    const int64_t row0 = tile_row * kTile + g * 8, col0 = tile_col * kTile + o * 8;
    const int64_t left = a.cols - col0;
    const int in_row = left >= 8 ? 8 : left > 0 ? (int)left : 0, in_row_or_less = left >= 8 ? 8 : (int)left;

    Octet<DT> x[8];
    const auto load_rows = [&](auto ends) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[i].clear();
            if (row0 + i < a.rows) x[i].template load<decltype(ends)::value>(a.x, (row0 + i) * a.ld + col0, in_row_or_less);
        }
    };
    if (a.cols < 8) {
        load_rows(std::integral_constant<Ends, Ends::kApart>());
    } else {
        load_rows(std::integral_constant<Ends, Ends::kMoved>());
        if (in_row < 8) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i].template settle<Ends::kMoved>(in_row_or_less);
        }
    }

    constexpr int kWords = Octet<DT>::kWords;
    uint32_t row_most[8], col_most[kWords], most;
    const auto look = [&](auto finite) {
        most = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint32_t m[kWords];
#pragma unroll
            for (int w = 0; w < kWords; ++w) {
                m[w] = magnitudes<DT, decltype(finite)::value>(x[i].w[w]);
                col_most[w] = i == 0 ? m[w] : max_of_words<DT>(col_most[w], m[w]);
            }
#pragma unroll
            for (int w = 1; w < kWords; ++w) m[0] = max_of_words<DT>(m[0], m[w]);
            row_most[i] = larger<DT>(m[0]);
            most = max_of(most, row_most[i]);
        }
    };
    look(std::false_type());
    if (most >= kInfinity<DT>) look(std::true_type());
    const bool square = a.out_square || a.turned_square, columns = a.turned && !a.turned_square;
    if (square) {
        most = max_of_rows<ZI_FP32>(max_16(most));
        if ((t & 63) == 0) s_all[wave] = most;
    }
    if (columns) {
#pragma unroll
        for (int w = 0; w < kWords; ++w) {
            const uint32_t m = max_of_rows<DT>(col_most[w]);
            if ((t & 63) < 16) s_col[wave][o * kWords + w] = m;
        }
    }
    if (square || columns) __syncthreads();
    uint32_t all = 127;
    if (square) all = scale_byte(as_fp32<DT>(max_of(max_of(s_all[0], s_all[1]), max_of(s_all[2], s_all[3]))));

    if (a.out) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t byte = a.out_square ? all : scale_byte(as_fp32<DT>(max_16(row_most[i])));
            if (row0 + i >= a.rows || in_row == 0) continue;
            put(eight_e4m3<DT>(x[i], scale_of(byte)), reinterpret_cast<u32x2*>(a.out + (row0 + i) * a.out_ld + col0));
            if (!a.out_square && o == 0) a.out_scale[(row0 + i) * a.out_scale_ld + tile_col] = (uint8_t)byte;
        }
        if (a.out_square && t == 0) a.out_scale[tile_row * a.out_scale_ld + tile_col] = (uint8_t)all;
    }
    if (!a.turned) return;

    // A column's 128 numbers are eight chunks of 16 bytes; chunk p of column c lies at p ^ (c / 8 % 8), so that the 16
    // threads that write one row's octets reach different banks.
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int c = o * 8 + j;
        uint32_t byte = all;
        if (!a.turned_square) {
            const int w = c * kWords / 8;
            const uint32_t m = max_of_words<DT>(max_of_words<DT>(s_col[0][w], s_col[1][w]), max_of_words<DT>(s_col[2][w], s_col[3][w]));
            byte = scale_byte(as_fp32<DT>(DT == ZI_FP32 ? m : c % 2 ? m >> 16 : m & 0xFFFFu));
        }
        *reinterpret_cast<u32x2*>(s_turned + c * kTile + (((g >> 1) ^ (o & 7)) << 4) + (g & 1) * 8) = eight_e4m3_down<DT>(x, j, scale_of(byte));
        if (!a.turned_square && g == 0 && j < in_row) a.turned_scale[(col0 + j) * a.turned_scale_ld + tile_row] = (uint8_t)byte;
    }
    if (a.turned_square && t == 0) a.turned_scale[tile_col * a.turned_scale_ld + tile_row] = (uint8_t)all;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int c = i * 32 + (t >> 3), part = t & 7;
        const int64_t col = tile_col * kTile + c, row = tile_row * kTile + part * 16;
        if (col >= a.cols || row >= a.rows) continue;
        put(*reinterpret_cast<const u32x4*>(s_turned + c * kTile + ((part ^ ((c >> 3) & 7)) << 4)),
            reinterpret_cast<u32x4*>(a.turned + col * a.turned_ld + row));
    }
}

template <int DT>
static hipError_t launch_quantize(const QuantizeArgs& a, hipStream_t s)
{
    const int64_t tiles = (int64_t)a.tiles_across * ((a.rows + kTile - 1) / kTile);
    const bool large = a.rows * a.cols * ((a.out ? 1 : 0) + (a.turned ? 1 : 0)) >= kLargeBytes;
    const dim3 grid((unsigned)tiles), block(256);
    if (large) hipLaunchKernelGGL((fp8_quantize_kernel<DT, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((fp8_quantize_kernel<DT, false>), grid, block, 0, s, a);
    return hipGetLastError();
}
hipError_t launch_fp8_quantize(const QuantizeArgs& a, int dtype, hipStream_t s)
{
    return dtype == ZI_BF16 ? launch_quantize<ZI_BF16>(a, s) : dtype == ZI_FP16 ? launch_quantize<ZI_FP16>(a, s) : launch_quantize<ZI_FP32>(a, s);
}

// ---- root-mean-square norm ------------------------------------------------------------------------------------

// One pass: h stays in registers while its squares are summed in fp32 (lanes, then wavefronts in their order), so x and the residual are read once and
// every output is written once.  T threads have a row, V octets each: octet v * T + t.  16 lanes have a block of 128 columns; its scale is that of the
// unrounded y, which is rounded to 8 bits directly.  Bound by memory: 16384 x 8192 bf16 with everything 202 us (1209 MB, 6.0 TB/s, a plain copy 6.7); one
// row of 4096 3.3 to 4.0 us, most of it the way to memory and back twice.
template <int DT, int T, int V, Ends ENDS>
__global__ __launch_bounds__(T) void rms_norm_kernel(const RmsNormArgs k)
{
    __shared__ float s_sum[T / 64];
    constexpr bool kAllFirst = V <= 2;          // all loads in front of what uses them, while there are registers for them
    const zi_rms_norm_args& a = k.a;
    const int cols = (int)a.cols, own = (int)threadIdx.x * 8;                    // (columns are at most 65536)
    const auto column = [&](int v) { return own + v * T * 8; };
    const auto valid = [&](int v) { return cols - column(v) < 8 ? cols - column(v) : 8; };
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        Octet<DT> h[V], gammas[kAllFirst ? V : 1];
        float sum = 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int col = column(v);
            h[v].template load<ENDS>(a.x, row * a.x_ld + col, valid(v));
            if constexpr (kAllFirst) gammas[v].template load<ENDS>(a.gamma, col, valid(v));
        }
        Octet<DT> residual[kAllFirst ? V : 1];
        if (kAllFirst && a.residual) {
#pragma unroll
            for (int v = 0; v < V; ++v) residual[kAllFirst ? v : 0].template load<ENDS>(a.residual, row * a.residual_ld + column(v), valid(v));
        }
#pragma unroll
        for (int v = 0; v < V; ++v) h[v].template settle<ENDS>(valid(v));
        if (a.residual) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int col = column(v);
                Octet<DT>& r = residual[kAllFirst ? v : 0];
                if constexpr (!kAllFirst) r.template load<ENDS>(a.residual, row * a.residual_ld + col, valid(v));
                r.template settle<ENDS>(valid(v));
                float f[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] = h[v].get(j) + r.get(j);
                h[v].set(f);
                if (a.sum && valid(v) > 0) h[v].template store<true>(a.sum, row * a.sum_ld + col, valid(v));
            }
        }
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int j = 0; j < 8; ++j) sum = __builtin_fmaf(h[v].get(j), h[v].get(j), sum);
        sum = sum_of_group<T>(sum, s_sum);
        const float rstd = 1.0f / sqrtf(sum / (float)a.cols + a.eps);
        if (a.rstd && threadIdx.x == 0) a.rstd[row] = rstd;
        if (a.y || k.y8) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int col = column(v);
                Octet<DT>& gamma = gammas[kAllFirst ? v : 0];
                if constexpr (!kAllFirst) gamma.template load<ENDS>(a.gamma, col, valid(v));
                gamma.template settle<ENDS>(valid(v));
                float y[8];
                uint32_t most = 0;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    y[j] = h[v].get(j) * rstd * gamma.get(j);
                    if (j >= valid(v)) y[j] = 0.0f;                 // (0 times an infinite rstd would be NaN)
                    most = max_of(most, magnitudes<ZI_FP32, false>(__float_as_uint(y[j])));
                }
                if (a.y && valid(v) > 0) {
                    Octet<DT> w;
                    w.set(y);
                    w.template store<true>(a.y, row * a.y_ld + col, valid(v));
                }
                if (k.y8) {
                    if (most >= kInfinity<ZI_FP32>) {
                        most = 0;
#pragma unroll
                        for (int j = 0; j < 8; ++j) most = max_of(most, magnitudes<ZI_FP32, true>(__float_as_uint(y[j])));
                    }
                    const uint32_t byte = scale_byte(max_16(most));
                    if (valid(v) > 0) {
                        const float scale = scale_of(byte);
                        *reinterpret_cast<u32x2*>(k.y8 + row * k.y8_ld + col) =
                            u32x2{four_e4m3(y[0], y[1], y[2], y[3], scale), four_e4m3(y[4], y[5], y[6], y[7], scale)};
                        if ((threadIdx.x & 15) == 0) k.y8_scale[row * k.y8_scale_ld + col / kFp8Block] = (uint8_t)byte;
                    }
                }
            }
        }
        if constexpr (T > 64) __syncthreads();                  // s_sum is written again
    }
}

// ---- its backward pass ----------------------------------------------------------------------------------------

// What a thread has of a row: V octets T threads apart, from column `first` on.
template <int DT, int T, int V, Ends ENDS>
struct BackwardRow {
    Octet<DT> dy[V], h[V], add[V];
    float rstd;
    static __device__ __forceinline__ int column(int first, int v) { return first + (v * T + (int)threadIdx.x) * 8; }
    static __device__ __forceinline__ int valid(const zi_rms_norm_backward_args& a, int first, int v)
    {
        const int left = (int)a.cols - column(first, v);
        return left < 8 ? left : 8;
    }
    __device__ __forceinline__ void load(const zi_rms_norm_backward_args& a, int64_t row, int first)
    {
        rstd = a.rstd[row];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            dy[v].template load<ENDS>(a.dy, row * a.dy_ld + column(first, v), valid(a, first, v));
            h[v].template load<ENDS>(a.h, row * a.h_ld + column(first, v), valid(a, first, v));
        }
    }
    __device__ __forceinline__ void load_dsum(const zi_rms_norm_backward_args& a, int64_t row, int first)
    {
        if (!a.dsum) return;
#pragma unroll
        for (int v = 0; v < V; ++v) add[v].template load<ENDS>(a.dsum, row * a.dsum_ld + column(first, v), valid(a, first, v));
    }
    __device__ __forceinline__ void settle(const zi_rms_norm_backward_args& a, int first)
    {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            dy[v].template settle<ENDS>(valid(a, first, v));
            h[v].template settle<ENDS>(valid(a, first, v));
            if (a.dsum) add[v].template settle<ENDS>(valid(a, first, v));
        }
    }
    __device__ __forceinline__ float dot(const Octet<DT> (&gamma)[V]) const
    {
        float sum = 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int j = 0; j < 8; ++j) sum = __builtin_fmaf(dy[v].get(j) * gamma[v].get(j), h[v].get(j) * rstd, sum);
        return sum;
    }
    // dx of the row, whose mean of u * n this is, and its share of dgamma
    __device__ __forceinline__ void finish(const zi_rms_norm_backward_args& a, int64_t row, int first, float mean, const Octet<DT> (&gamma)[V],
                                           float (&share)[V][8]) const
    {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int in = valid(a, first, v);
            if (in <= 0) continue;
            float dx[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float n = h[v].get(j) * rstd;
                dx[j] = rstd * (dy[v].get(j) * gamma[v].get(j) - n * mean);
                if (a.dsum) dx[j] += add[v].get(j);
                share[v][j] = __builtin_fmaf(dy[v].get(j), n, share[v][j]);
            }
            if (a.dx) {
                Octet<DT> w;
                w.set(dx);
                w.template store<true>(a.dx, row * a.dx_ld + column(first, v), in);
            }
        }
    }
};

// Bound by memory: 16384 x 4096 bf16 with dsum 92 us (537 MB, 5.8 TB/s) and 4.9 us for the shares of dgamma.
// A workgroup goes over rows a grid apart and keeps its columns' share of dgamma in registers; the shares of all
// workgroups are added by a second kernel in their order.  The next row's loads go out before this row's sum is known (16384 x 4096
// with dsum 123 -> 97 us).  MEANS: rows that do not fit one workgroup's registers (is_cut) are cut, and means of whole rows come from a kernel in
// front (rms_norm_means_kernel), so that dy and h are read twice.
template <int DT, int T, int V, bool MEANS, Ends ENDS>
__global__ __launch_bounds__(T) void rms_norm_backward_kernel(const zi_rms_norm_backward_args a, float* partials, const float* means, uint32_t cuts)
{
    using Row = BackwardRow<DT, T, V, ENDS>;
    constexpr bool kAhead = T < 1024;          // dsum too; 1024 threads have 128 registers each, and no room for it
    __shared__ float s_sum[2][T / 64];
    const uint32_t group = MEANS ? blockIdx.x / cuts : blockIdx.x, groups = MEANS ? gridDim.x / cuts : gridDim.x;
    const int first = MEANS ? (int)(blockIdx.x % cuts) * (T * V * 8) : 0;
    float share[V][8] = {};
    Octet<DT> gamma[V];
    Row now, next;
    now.load(a, group, first);
    if constexpr (kAhead) now.load_dsum(a, group, first);
#pragma unroll
    for (int v = 0; v < V; ++v) {
        gamma[v].template load<ENDS>(a.gamma, Row::column(first, v), Row::valid(a, first, v));
        gamma[v].template settle<ENDS>(Row::valid(a, first, v));
    }
    int turn = 0;
    for (int64_t row = group; row < a.rows; row += groups, turn ^= 1) {
        if constexpr (!kAhead) now.load_dsum(a, row, first);
        if (row + groups < a.rows) {
            next.load(a, row + groups, first);
            if constexpr (kAhead) next.load_dsum(a, row + groups, first);
        }
        now.settle(a, first);
        float mean;
        if constexpr (MEANS) mean = means[row];
        else mean = sum_of_group<T>(now.dot(gamma), s_sum[turn]) / (float)a.cols;
        now.finish(a, row, first, mean, gamma, share);
        now = next;
    }
    if (!a.dgamma) return;
    float* mine = partials + (int64_t)group * a.cols;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < Row::valid(a, first, v)) mine[Row::column(first, v) + j] = share[v][j];
}

// The mean of u * n of each row.
template <int DT, Ends ENDS>
__global__ __launch_bounds__(1024) void rms_norm_means_kernel(const zi_rms_norm_backward_args a, float* means)
{
    using Row = BackwardRow<DT, 1024, 2, ENDS>;
    __shared__ float s_sum[16];
    zi_rms_norm_backward_args b = a;             // without dsum, which is not loaded
    b.dsum = nullptr;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        float sum = 0.0f;
        for (int first = 0; first < (int)a.cols; first += 1024 * 16) {
            Row r;
            Octet<DT> gamma[2];
            r.load(a, row, first);
#pragma unroll
            for (int v = 0; v < 2; ++v) gamma[v].template load<ENDS>(a.gamma, Row::column(first, v), Row::valid(a, first, v));
            r.settle(b, first);
#pragma unroll
            for (int v = 0; v < 2; ++v) gamma[v].template settle<ENDS>(Row::valid(a, first, v));
            sum += r.dot(gamma);
        }
        sum = sum_of_group<1024>(sum, s_sum);
        if (threadIdx.x == 0) means[row] = sum / (float)a.cols;
        __syncthreads();                                        // s_sum is written again
    }
}

// dgamma (or other sums over rows) of 16 columns: P rows of threads take every Pth share each, and are added in a fixed order.  Bound by latency: 256 shares of 4096 columns
// 4.9 us (4.2 MB).  Eight shares' loads go out at a time (backward pass of 13683 x 152 18.4 -> 14.3, 8192 x 1024 21.3 -> 18.8).
template <int DT, int P>
__global__ __launch_bounds__(16 * P) void rms_norm_dgamma_kernel(const float* partials, int count, int64_t cols, void* dgamma, int accumulate)
{
    constexpr int kAtOnce = 8;
    __shared__ float s_sum[P][16];
    const int in = threadIdx.x & 15, part = threadIdx.x >> 4;
    const int64_t col = (int64_t)blockIdx.x * 16 + in;
    float sum = 0.0f;
    if (col < cols)
        for (int first = part; first < count; first += kAtOnce * P) {
            float x[kAtOnce];
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) {
                const int at = first + i * P;
                x[i] = partials[(int64_t)(at < count ? at : part) * cols + col];
            }
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i)
                if (first + i * P < count) sum += x[i];
        }
    s_sum[part][in] = sum;
    __syncthreads();
    if (part != 0 || col >= cols) return;
#pragma unroll
    for (int i = 1; i < P; ++i) sum += s_sum[i][in];
    if constexpr (DT == ZI_FP32) {
        float* p = static_cast<float*>(dgamma) + col;
        *p = accumulate ? *p + sum : sum;
    } else {
        uint16_t* p = static_cast<uint16_t*>(dgamma) + col;
        Octet<DT> old;
        old.w[0] = *p;
        *p = (uint16_t)Octet<DT>::pair(accumulate ? old.get(0) + sum : sum, 0.0f);
    }
}

// Calls f with the threads and octets a thread that hold a row of up to 16384 columns: two octets each where that makes at least a wavefront.
// 16384 x 8192 with everything, us: 256 threads with four octets 217, 512 with two 206, 1024 with one 250.
template <int DT, typename F>
static void with_row_shape(int64_t cols, const F& f)
{
    if (cols <= 64 * 8) f.template operator()<DT, 64, 1>();
    else if (cols <= 64 * 16) f.template operator()<DT, 64, 2>();
    else if (cols <= 128 * 16) f.template operator()<DT, 128, 2>();
    else if (cols <= 256 * 16) f.template operator()<DT, 256, 2>();
    else if (cols <= 512 * 16) f.template operator()<DT, 512, 2>();
    else f.template operator()<DT, 1024, 2>();
}

namespace {
// Whether one workgroup of the backward pass has a row in registers: up to 16384 columns, or 8192 where they are not whole octets, which takes more
// registers than 1024 threads have.
bool is_cut(int64_t cols) { return cols > (cols % 8 ? 512 * 16 : 1024 * 16); }
constexpr int kCutThreads = 256, kCutCols = kCutThreads * 16;

struct LaunchNorm {
    const RmsNormArgs& a;
    hipStream_t s;
    template <int DT, int T, int V>
    void operator()() const
    {
        const int64_t most = (int64_t)1 << 20;
        const dim3 grid((unsigned)(a.a.rows < most ? a.a.rows : most)), block(T);
        constexpr Ends kRagged = V <= 4 ? Ends::kMoved : Ends::kApart;       // (eight octets leave no registers for moving)
        if (a.a.cols % 8 == 0) hipLaunchKernelGGL((rms_norm_kernel<DT, T, V, Ends::kWhole>), grid, block, 0, s, a);
        else if (a.a.cols > 8) hipLaunchKernelGGL((rms_norm_kernel<DT, T, V, kRagged>), grid, block, 0, s, a);
        else if constexpr (T == 64 && V == 1) hipLaunchKernelGGL((rms_norm_kernel<DT, T, V, Ends::kApart>), grid, block, 0, s, a);
    }
};
struct LaunchBackward {
    const zi_rms_norm_backward_args& a;
    float* partials;
    unsigned groups;
    hipStream_t s;
    template <int DT, int T, int V>
    void operator()() const
    {
        launch<DT, T, V, false>(groups, nullptr, 1);
    }
    template <int DT, int T, int V, bool MEANS>
    void launch(unsigned grid, const float* means, unsigned cuts) const
    {
        if (a.cols % 8 == 0) return launch_ends<DT, T, V, MEANS, Ends::kWhole>(grid, means, cuts);
        if constexpr (T == 64 && V == 1)
            if (a.cols < 8) return launch_ends<DT, T, V, MEANS, Ends::kApart>(grid, means, cuts);
        if constexpr (T < 1024) launch_ends<DT, T, V, MEANS, Ends::kMoved>(grid, means, cuts);
    }
    template <int DT, int T, int V, bool MEANS, Ends ENDS>
    void launch_ends(unsigned grid, const float* means, unsigned cuts) const
    {
        hipLaunchKernelGGL((rms_norm_backward_kernel<DT, T, V, MEANS, ENDS>), dim3(grid), dim3(T), 0, s, a, partials, means, cuts);
    }
    template <int DT>
    void cut() const
    {
        float* means = partials + (int64_t)groups * a.cols;
        const unsigned cuts = (unsigned)((a.cols + kCutCols - 1) / kCutCols);
        const dim3 grid((unsigned)(a.rows < 4096 ? a.rows : 4096)), block(1024);
        if (a.cols % 8) hipLaunchKernelGGL((rms_norm_means_kernel<DT, Ends::kMoved>), grid, block, 0, s, a, means);
        else hipLaunchKernelGGL((rms_norm_means_kernel<DT, Ends::kWhole>), grid, block, 0, s, a, means);
        launch<DT, kCutThreads, 2, true>(groups * cuts, means, cuts);
    }
    template <int DT>
    void of() const
    {
        if (is_cut(a.cols)) cut<DT>();
        else with_row_shape<DT>(a.cols, *this);
    }
};
template <int DT>
void launch_norm_of(const RmsNormArgs& a, hipStream_t s)
{
    const LaunchNorm f{a, s};
    // Of 8193 to 16384 columns, 1024 threads with two octets leave room for one workgroup on a compute unit, 512 with three or four for two; they need more
    // turns for a row, which counts where each unit has one row at most.  us, 1024 / 512: 16351 x 8208 fp16 260 / 182, 12000 x 11000 219 / 175, 10483 x 12803
    // 330 / 282, 8192 x 16384 220 / 219; but 1 x 16000 4.8 / 6.1.
    const bool many = a.a.rows > 256;
    if (many && a.a.cols > 512 * 16 && a.a.cols <= 512 * 24) f.template operator()<DT, 512, 3>();
    else if (many && a.a.cols > 512 * 24 && a.a.cols <= 512 * 32) f.template operator()<DT, 512, 4>();
    else if (a.a.cols <= 1024 * 16) with_row_shape<DT>(a.a.cols, f);
    else if (a.a.cols <= 1024 * 32) f.template operator()<DT, 1024, 4>();
    else f.template operator()<DT, 1024, 8>();
}
}  // namespace

hipError_t launch_rms_norm(const RmsNormArgs& a, hipStream_t s)
{
    if (a.a.dtype == ZI_BF16) launch_norm_of<ZI_BF16>(a, s);
    else launch_norm_of<ZI_FP16>(a, s);
    return hipGetLastError();
}

// Workgroups that go over the rows of the backward pass: few, as each has a row and the next under way.  us with
// 256 / 512 / 1024 / 1536: 16384 x 4096 97 / 101 / 113 / 112, 4096 x 2048 24.1 / 20.9 / 24.4 / 29.0, 16384 x 1024 63 / 39 / 30 / 30, 65536 x 512
// 166 / 98 / 68 / 60.
static int64_t backward_groups(int64_t rows, int64_t cols)
{
    const int64_t cuts = (cols + kCutCols - 1) / kCutCols;
    const int64_t most = cols <= 512 ? 1536 : cols <= 1024 ? 1024 : cols <= 2048 ? 512 : !is_cut(cols) ? 256 : 768 / cuts;
    return rows < most ? rows : most;
}

template <int DT>
static void launch_sums(const float* partials, int count, int64_t cols, void* out, int accumulate, hipStream_t s)
{
    const dim3 grid((unsigned)((cols + 15) / 16));
    if (count <= 64) hipLaunchKernelGGL((rms_norm_dgamma_kernel<DT, 16>), grid, dim3(256), 0, s, partials, count, cols, out, accumulate);
    else hipLaunchKernelGGL((rms_norm_dgamma_kernel<DT, 64>), grid, dim3(1024), 0, s, partials, count, cols, out, accumulate);
}
hipError_t launch_column_sums(const float* partials, int count, int64_t cols, void* out, int dtype, int accumulate, hipStream_t s)
{
    if (dtype == ZI_BF16) launch_sums<ZI_BF16>(partials, count, cols, out, accumulate, s);
    else if (dtype == ZI_FP16) launch_sums<ZI_FP16>(partials, count, cols, out, accumulate, s);
    else launch_sums<ZI_FP32>(partials, count, cols, out, accumulate, s);
    return hipGetLastError();
}

size_t rms_norm_workspace_floats(int64_t rows, int64_t cols)
{
    return (size_t)(backward_groups(rows, cols) * cols + (is_cut(cols) ? rows : 0));
}
bool rms_norm_needs_means(int64_t cols) { return is_cut(cols); }

hipError_t launch_rms_norm_backward(const zi_rms_norm_backward_args& a, float* partials, hipStream_t s)
{
    const unsigned groups = (unsigned)backward_groups(a.rows, a.cols);
    if (groups > 0) {
        const LaunchBackward f{a, partials, groups, s};
        if (a.dtype == ZI_BF16) f.of<ZI_BF16>();
        else f.of<ZI_FP16>();
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return a.dgamma ? launch_column_sums(partials, (int)groups, a.cols, a.dgamma, a.dgamma_dtype, a.accumulate, s) : hipSuccess;
}

}  // namespace zi
