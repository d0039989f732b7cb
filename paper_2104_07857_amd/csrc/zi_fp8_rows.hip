// Kernels of the 8-bit operators that go over rows once: quantisation, the root-mean-square norm and its backward pass.
// All are bound by memory; see include/zi_fp8.h for the formulas.  Compile with -ffp-contract=off.
#include <hip/hip_runtime.h>

#include "zi_fp8_device.h"
#include "zi_fp8_internal.h"

namespace zi {

// ---- quantisation ---------------------------------------------------------------------------------------------

// A workgroup takes a tile of 128 x 128, which holds whole blocks of every kind, so x is read once whatever is wanted.
// A thread has 8 x 8 elements in registers; 16 threads (a row of lanes) have a tile's row, so the largest of a row's
// block comes from its lanes and that of a column's block from the thread's own rows, two steps over lanes and four
// wavefronts.  The transposed numbers pass through LDS, which makes rows of 128 bytes of them.
constexpr int kTile = kFp8Block;

template <int DT>
__global__ __launch_bounds__(256) void fp8_quantize_kernel(const QuantizeArgs a)
{
    __shared__ uint32_t s_col[4][kTile];
    __shared__ uint32_t s_all[4];
    __shared__ __align__(16) uint8_t s_turned[kTile * kTile];

    const int t = threadIdx.x, o = t & 15, g = t >> 4, wave = t >> 6;
    const int64_t tile_row = blockIdx.x / a.tiles_across, tile_col = blockIdx.x % a.tiles_across;
    const int64_t row0 = tile_row * kTile + g * 8, col0 = tile_col * kTile + o * 8;
    const int64_t left = a.cols - col0;
    const int in_row = left >= 8 ? 8 : left > 0 ? (int)left : 0;

    Octet<DT> x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i].load(a.x, (row0 + i) * a.ld + col0, row0 + i < a.rows ? in_row : 0);

    uint32_t row_most[8], col_most[8], most = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) col_most[j] = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        row_most[i] = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t v = magnitude(x[i].get(j));
            row_most[i] = max_of(row_most[i], v);
            col_most[j] = max_of(col_most[j], v);
        }
        most = max_of(most, row_most[i]);
    }
    const bool square = a.out_square || a.turned_square, columns = a.turned && !a.turned_square;
    if (square) {
        most = max_of_rows(max_16(most));
        if ((t & 63) == 0) s_all[wave] = most;
    }
    if (columns) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t m = max_of_rows(col_most[j]);
            if ((t & 63) < 16) s_col[wave][o * 8 + j] = m;
        }
    }
    if (square || columns) __syncthreads();
    uint32_t all = 127;
    if (square) all = scale_byte(max_of(max_of(s_all[0], s_all[1]), max_of(s_all[2], s_all[3])));

    if (a.out) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t byte = a.out_square ? all : scale_byte(max_16(row_most[i]));
            if (row0 + i >= a.rows || in_row == 0) continue;
            const float inv = inverse_scale(byte);
            u32x2 q;
            q[0] = four_e4m3(x[i].get(0) * inv, x[i].get(1) * inv, x[i].get(2) * inv, x[i].get(3) * inv);
            q[1] = four_e4m3(x[i].get(4) * inv, x[i].get(5) * inv, x[i].get(6) * inv, x[i].get(7) * inv);
            *reinterpret_cast<u32x2*>(a.out + (row0 + i) * a.out_ld + col0) = q;
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
        if (!a.turned_square) byte = scale_byte(max_of(max_of(s_col[0][c], s_col[1][c]), max_of(s_col[2][c], s_col[3][c])));
        const float inv = inverse_scale(byte);
        u32x2 q;
        q[0] = four_e4m3(x[0].get(j) * inv, x[1].get(j) * inv, x[2].get(j) * inv, x[3].get(j) * inv);
        q[1] = four_e4m3(x[4].get(j) * inv, x[5].get(j) * inv, x[6].get(j) * inv, x[7].get(j) * inv);
        *reinterpret_cast<u32x2*>(s_turned + c * kTile + (((g >> 1) ^ (o & 7)) << 4) + (g & 1) * 8) = q;
        if (!a.turned_square && g == 0 && j < in_row) a.turned_scale[(col0 + j) * a.turned_scale_ld + tile_row] = (uint8_t)byte;
    }
    if (a.turned_square && t == 0) a.turned_scale[tile_col * a.turned_scale_ld + tile_row] = (uint8_t)all;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int c = i * 32 + (t >> 3), part = t & 7;
        const int64_t col = tile_col * kTile + c, row = tile_row * kTile + part * 16;
        if (col >= a.cols || row >= a.rows) continue;
        *reinterpret_cast<u32x4*>(a.turned + col * a.turned_ld + row) =
            *reinterpret_cast<const u32x4*>(s_turned + c * kTile + ((part ^ ((c >> 3) & 7)) << 4));
    }
}

hipError_t launch_fp8_quantize(const QuantizeArgs& a, int dtype, hipStream_t s)
{
    const int64_t tiles = (int64_t)a.tiles_across * ((a.rows + kTile - 1) / kTile);
    const dim3 grid((unsigned)tiles), block(256);
    if (dtype == ZI_BF16) hipLaunchKernelGGL(fp8_quantize_kernel<ZI_BF16>, grid, block, 0, s, a);
    else if (dtype == ZI_FP16) hipLaunchKernelGGL(fp8_quantize_kernel<ZI_FP16>, grid, block, 0, s, a);
    else hipLaunchKernelGGL(fp8_quantize_kernel<ZI_FP32>, grid, block, 0, s, a);
    return hipGetLastError();
}

// ---- root-mean-square norm ------------------------------------------------------------------------------------

// T threads have a row, V octets each: octet v * T + t.  16 lanes have a block of 128 columns.
template <int DT, int T, int V>
__global__ __launch_bounds__(T) void rms_norm_kernel(const RmsNormArgs k)
{
    __shared__ float s_sum[T / 64];
    const zi_rms_norm_args& a = k.a;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        Octet<DT> h[V];
        int in[V];
        float sum = 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int64_t col = (int64_t)(v * T + threadIdx.x) * 8;
            in[v] = (int)(a.cols - col < 8 ? a.cols - col : 8);
            h[v].load(a.x, row * a.x_ld + col, in[v]);
        }
        if (a.residual) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int64_t col = (int64_t)(v * T + threadIdx.x) * 8;
                Octet<DT> r;
                r.load(a.residual, row * a.residual_ld + col, in[v]);
                float f[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] = h[v].get(j) + r.get(j);
                h[v].set(f);
                if (a.sum && in[v] > 0) h[v].store(a.sum, row * a.sum_ld + col, in[v]);
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
                const int64_t col = (int64_t)(v * T + threadIdx.x) * 8;
                Octet<DT> gamma;
                gamma.load(a.gamma, col, in[v]);
                float y[8];
                uint32_t most = 0;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    y[j] = h[v].get(j) * rstd * gamma.get(j);
                    if (j >= in[v]) y[j] = 0.0f;                 // (0 times an infinite rstd would be NaN)
                    most = max_of(most, magnitude(y[j]));
                }
                if (a.y && in[v] > 0) {
                    Octet<DT> w;
                    w.set(y);
                    w.store(a.y, row * a.y_ld + col, in[v]);
                }
                if (k.y8) {
                    const uint32_t byte = scale_byte(max_16(most));
                    const float inv = inverse_scale(byte);
                    if (in[v] > 0) {
                        u32x2 q;
                        q[0] = four_e4m3(y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv);
                        q[1] = four_e4m3(y[4] * inv, y[5] * inv, y[6] * inv, y[7] * inv);
                        *reinterpret_cast<u32x2*>(k.y8 + row * k.y8_ld + col) = q;
                        if ((threadIdx.x & 15) == 0) k.y8_scale[row * k.y8_scale_ld + col / kFp8Block] = (uint8_t)byte;
                    }
                }
            }
        }
        if constexpr (T > 64) __syncthreads();                  // s_sum is written again
    }
}

// ---- its backward pass ----------------------------------------------------------------------------------------

// A workgroup goes over rows a grid apart and keeps its columns' share of dgamma in registers; the shares of all
// workgroups are added by a second kernel in their order.  Rows of up to 32768 columns stay in registers between the
// sum over the row and what needs it; longer ones are read again.
template <int DT, int T, int V>
__global__ __launch_bounds__(T) void rms_norm_backward_kernel(const zi_rms_norm_backward_args a, float* partials)
{
    constexpr bool kKeep = V < 8;
    __shared__ float s_sum[T / 64];
    float share[V][8];
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
        for (int j = 0; j < 8; ++j) share[v][j] = 0.0f;
    const auto column = [](int v) { return (int64_t)(v * T + threadIdx.x) * 8; };
    const auto valid = [&](int v) { const int64_t left = a.cols - column(v); return (int)(left < 8 ? left : 8); };

    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const float rstd = a.rstd[row];
        Octet<DT> dy[kKeep ? V : 1], h[kKeep ? V : 1], gamma[kKeep ? V : 1];
        float dot = 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int i = kKeep ? v : 0, in = valid(v);
            dy[i].load(a.dy, row * a.dy_ld + column(v), in);
            h[i].load(a.h, row * a.h_ld + column(v), in);
            gamma[i].load(a.gamma, column(v), in);
#pragma unroll
            for (int j = 0; j < 8; ++j) dot = __builtin_fmaf(dy[i].get(j) * gamma[i].get(j), h[i].get(j) * rstd, dot);
        }
        dot = sum_of_group<T>(dot, s_sum) / (float)a.cols;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int i = kKeep ? v : 0, in = valid(v);
            if (in <= 0) continue;
            if constexpr (!kKeep) {
                dy[0].load(a.dy, row * a.dy_ld + column(v), in);
                h[0].load(a.h, row * a.h_ld + column(v), in);
                gamma[0].load(a.gamma, column(v), in);
            }
            Octet<DT> add;
            if (a.dsum) add.load(a.dsum, row * a.dsum_ld + column(v), in);
            float dx[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float n = h[i].get(j) * rstd;
                dx[j] = rstd * (dy[i].get(j) * gamma[i].get(j) - n * dot);
                if (a.dsum) dx[j] += add.get(j);
                share[v][j] = __builtin_fmaf(dy[i].get(j), n, share[v][j]);
            }
            if (a.dx) {
                Octet<DT> w;
                w.set(dx);
                w.store(a.dx, row * a.dx_ld + column(v), in);
            }
        }
        if constexpr (T > 64) __syncthreads();                  // s_sum is written again
    }
    if (!a.dgamma) return;
    float* mine = partials + (int64_t)blockIdx.x * a.cols;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < valid(v)) mine[column(v) + j] = share[v][j];
}

// dgamma of 64 columns: 16 wavefronts take every sixteenth share each.
template <int DT>
__global__ __launch_bounds__(1024) void rms_norm_dgamma_kernel(const float* partials, int count, int64_t cols, void* dgamma, int accumulate)
{
    __shared__ float s_sum[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t col = (int64_t)blockIdx.x * 64 + lane;
    float sum = 0.0f;
    if (col < cols)
        for (int i = wave; i < count; i += 16) sum += partials[(int64_t)i * cols + col];
    s_sum[wave][lane] = sum;
    __syncthreads();
    if (wave != 0 || col >= cols) return;
#pragma unroll
    for (int i = 1; i < 16; ++i) sum += s_sum[i][lane];
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

// Calls f(type, threads, octets) with the shape that holds a row: 64 threads up to 512 columns, 256 up to 8192, 1024 up to 65536.
template <int DT, typename F>
static void with_row_shape(int64_t cols, const F& f)
{
    if (cols <= 64 * 8) f.template operator()<DT, 64, 1>();
    else if (cols <= 256 * 8) f.template operator()<DT, 256, 1>();
    else if (cols <= 256 * 16) f.template operator()<DT, 256, 2>();
    else if (cols <= 256 * 32) f.template operator()<DT, 256, 4>();
    else if (cols <= 1024 * 16) f.template operator()<DT, 1024, 2>();
    else if (cols <= 1024 * 32) f.template operator()<DT, 1024, 4>();
    else f.template operator()<DT, 1024, 8>();
}

namespace {
struct LaunchNorm {
    const RmsNormArgs& a;
    hipStream_t s;
    template <int DT, int T, int V>
    void operator()() const
    {
        const int64_t most = (int64_t)1 << 20;
        const dim3 grid((unsigned)(a.a.rows < most ? a.a.rows : most)), block(T);
        hipLaunchKernelGGL((rms_norm_kernel<DT, T, V>), grid, block, 0, s, a);
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
        hipLaunchKernelGGL((rms_norm_backward_kernel<DT, T, V>), dim3(groups), dim3(T), 0, s, a, partials);
    }
};
}  // namespace

hipError_t launch_rms_norm(const RmsNormArgs& a, hipStream_t s)
{
    if (a.a.dtype == ZI_BF16) with_row_shape<ZI_BF16>(a.a.cols, LaunchNorm{a, s});
    else with_row_shape<ZI_FP16>(a.a.cols, LaunchNorm{a, s});
    return hipGetLastError();
}

size_t rms_norm_partials(int64_t rows, int64_t cols)
{
    const int64_t most = cols <= 8192 ? 1024 : 512;
    return (size_t)(rows < most ? rows : most);
}

hipError_t launch_rms_norm_backward(const zi_rms_norm_backward_args& a, float* partials, hipStream_t s)
{
    const unsigned groups = (unsigned)rms_norm_partials(a.rows, a.cols);
    if (groups > 0) {
        if (a.dtype == ZI_BF16) with_row_shape<ZI_BF16>(a.cols, LaunchBackward{a, partials, groups, s});
        else with_row_shape<ZI_FP16>(a.cols, LaunchBackward{a, partials, groups, s});
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (!a.dgamma) return hipSuccess;
    const dim3 grid((unsigned)((a.cols + 63) / 64)), block(1024);
    if (a.dgamma_dtype == ZI_BF16)
        hipLaunchKernelGGL(rms_norm_dgamma_kernel<ZI_BF16>, grid, block, 0, s, partials, (int)groups, a.cols, a.dgamma, a.accumulate);
    else if (a.dgamma_dtype == ZI_FP16)
        hipLaunchKernelGGL(rms_norm_dgamma_kernel<ZI_FP16>, grid, block, 0, s, partials, (int)groups, a.cols, a.dgamma, a.accumulate);
    else
        hipLaunchKernelGGL(rms_norm_dgamma_kernel<ZI_FP32>, grid, block, 0, s, partials, (int)groups, a.cols, a.dgamma, a.accumulate);
    return hipGetLastError();
}

}  // namespace zi
