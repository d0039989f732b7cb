// Kernels of the product in 8 bits, D = A B^T + C (include/zi_fp8.h), on the matrix cores' scaled e4m3 instructions: a
// block's scale goes in with its numbers, so the sum over k stays in fp32 registers from the first block to the last.
#include <hip/hip_runtime.h>

#include "zi_fp8_device.h"
#include "zi_fp8_internal.h"

namespace zi {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// A lane's 32 numbers of a row times those of another, added to what 32 x 32 such pairs have: rows of the first operand are
// D's columns here, so that a lane's registers hold neighbours of a row of D.
__device__ __forceinline__ f32x16 multiply_add(i32x8 b, i32x8 a, f32x16 sum, uint32_t b_scale, uint32_t a_scale)
{
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(b, a, sum, 0, 0, 0, (int)b_scale, 0, (int)a_scale);
}

// Tiles of 128 x 128 and steps of 128 in k, four wavefronts with 64 x 64 each.
constexpr int kSide = 128, kStep = kFp8Block;

// 16 bytes of a matrix in 8 bits, zeros where it ends.
__device__ __forceinline__ u32x4 chunk_of(const uint8_t* data, int64_t ld, int64_t rows, int64_t cols, int64_t row, int64_t col)
{
    u32x4 x = {0, 0, 0, 0};
    if (row >= rows || col >= cols) return x;
    x = *reinterpret_cast<const u32x4*>(data + row * ld + col);
    if (cols - col < 16) {
        const int valid = (int)(cols - col);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int left = valid - 4 * i;
            x[i] &= left >= 4 ? 0xFFFFFFFFu : left > 0 ? (1u << (8 * left)) - 1u : 0u;
        }
    }
    return x;
}

// Chunk p of a row of 128 bytes lies at p ^ (row % 8): lanes that read the same chunk of eight rows reach all banks.
__device__ __forceinline__ int chunk_at(int row, int p) { return row * kStep + ((p ^ (row & 7)) << 4); }

template <int DT>
__global__ __launch_bounds__(256) void fp8_matmul_kernel(const MatmulArgs p, uint32_t tiles_across)
{
    __shared__ __align__(16) uint8_t s_a[kSide * kStep], s_b[kSide * kStep];
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const int64_t m0 = (int64_t)(blockIdx.x / tiles_across) * kSide, n0 = (int64_t)(blockIdx.x % tiles_across) * kSide;
    const int wave_m = (wave >> 1) * 64, wave_n = (wave & 1) * 64, in = lane & 31, half = lane >> 5;

    f32x16 sum[2][2] = {};
    const auto scale_row = [](int64_t row, int64_t rows, int shift) { return (row < rows ? row : rows - 1) >> shift; };
    const uint8_t *scale_a[2], *scale_b[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        scale_a[i] = p.a_scale + scale_row(m0 + wave_m + 32 * i + in, p.m, p.a_shift) * p.a_scale_ld;
        scale_b[i] = p.b_scale + scale_row(n0 + wave_n + 32 * i + in, p.n, p.b_shift) * p.b_scale_ld;
    }
    for (int64_t k0 = 0; k0 < p.k; k0 += kStep) {
        const int64_t block = k0 / kStep;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = i * 32 + (t >> 3), part = t & 7;
            *reinterpret_cast<u32x4*>(s_a + chunk_at(row, part)) = chunk_of(p.a, p.a_ld, p.m, p.k, m0 + row, k0 + part * 16);
            *reinterpret_cast<u32x4*>(s_b + chunk_at(row, part)) = chunk_of(p.b, p.b_ld, p.n, p.k, n0 + row, k0 + part * 16);
        }
        __syncthreads();
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            i32x8 a[2], b[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const u32x4 x = *reinterpret_cast<const u32x4*>(s_a + chunk_at(wave_m + 32 * i + in, 4 * h + 2 * half + j));
                    const u32x4 y = *reinterpret_cast<const u32x4*>(s_b + chunk_at(wave_n + 32 * i + in, 4 * h + 2 * half + j));
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        a[i][4 * j + w] = (int)x[w];
                        b[i][4 * j + w] = (int)y[w];
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) sum[i][j] = multiply_add(b[j], a[i], sum[i][j], scale_b[j][block], scale_a[i][block]);
        }
    }
    // Of 32 x 32, a lane has row `in` of A and, of B, rows 8 q + 4 half + 0..3 in registers 4 q..4 q + 3.
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int64_t row = m0 + wave_m + 32 * i + in;
        if (row >= p.m) continue;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int64_t col = n0 + wave_n + 32 * j + 8 * (r >> 2) + 4 * half + (r & 3);
                if (col >= p.n) continue;
                float x = sum[i][j][r];
                if (p.c) {
                    Octet<DT> c;
                    c.w[0] = static_cast<const uint16_t*>(p.c)[row * p.d_ld + col];
                    x += c.get(0);
                }
                static_cast<uint16_t*>(p.d)[row * p.d_ld + col] = (uint16_t)Octet<DT>::pair(x, 0.0f);
            }
    }
}

hipError_t launch_fp8_matmul(const MatmulArgs& a, int dtype, float*, hipStream_t s)
{
    const uint32_t across = (uint32_t)((a.n + kSide - 1) / kSide);
    const dim3 grid((unsigned)(across * ((a.m + kSide - 1) / kSide))), block(256);
    if (dtype == ZI_BF16) hipLaunchKernelGGL(fp8_matmul_kernel<ZI_BF16>, grid, block, 0, s, a, across);
    else hipLaunchKernelGGL(fp8_matmul_kernel<ZI_FP16>, grid, block, 0, s, a, across);
    return hipGetLastError();
}

}  // namespace zi
