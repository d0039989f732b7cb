// What the kernels of the 8-bit operators share: octets of 16- and 32-bit elements, the scale of a block, and sums and
// maxima over lanes.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "zi_fp8.h"

namespace zi {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

typedef uint32_t u32x4_of_2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x4_of_4 __attribute__((ext_vector_type(4), aligned(4)));

// Eight elements of a row.  Rows need only be aligned to their element: the hardware takes such vectors as they are.
template <int DT>
struct Octet {
    static constexpr int kWords = DT == ZI_FP32 ? 8 : 4;
    static constexpr int kBytes = DT == ZI_FP32 ? 4 : 2;
    using vec = std::conditional_t<DT == ZI_FP32, u32x4_of_4, u32x4_of_2>;
    uint32_t w[kWords];

    // `valid` leading elements of eight, zeros behind them.
    __device__ __forceinline__ void load(const void* base, int64_t at, int valid)
    {
        const char* p = static_cast<const char*>(base) + at * kBytes;
        if (valid >= 8) {
#pragma unroll
            for (int i = 0; i < kWords / 4; ++i) {
                const vec v = reinterpret_cast<const vec*>(p)[i];
#pragma unroll
                for (int j = 0; j < 4; ++j) w[4 * i + j] = v[j];
            }
            return;
        }
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = 0;
        if (valid <= 0) return;
#pragma unroll
        for (int j = 0; j < 7; ++j) {
            if (j < valid) {
                if constexpr (DT == ZI_FP32) w[j] = reinterpret_cast<const uint32_t*>(p)[j];
                else w[j / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[j] << (16 * (j % 2));
            }
        }
    }
    // STREAM: past the caches, for what the kernels that follow do not read at once.
    template <bool STREAM = false>
    __device__ __forceinline__ void store(void* base, int64_t at, int valid) const
    {
        char* p = static_cast<char*>(base) + at * kBytes;
        if (valid >= 8) {
#pragma unroll
            for (int i = 0; i < kWords / 4; ++i) {
                vec v;
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = w[4 * i + j];
                if constexpr (STREAM) __builtin_nontemporal_store(v, reinterpret_cast<vec*>(p) + i);
                else reinterpret_cast<vec*>(p)[i] = v;
            }
            return;
        }
#pragma unroll
        for (int j = 0; j < 7; ++j) {
            if (j < valid) {
                if constexpr (DT == ZI_FP32) reinterpret_cast<uint32_t*>(p)[j] = w[j];
                else reinterpret_cast<uint16_t*>(p)[j] = (uint16_t)(w[j / 2] >> (16 * (j % 2)));
            }
        }
    }
    __device__ __forceinline__ float get(int j) const
    {
        if constexpr (DT == ZI_FP32) return __uint_as_float(w[j]);
        else if constexpr (DT == ZI_BF16) return __uint_as_float(j % 2 ? w[j / 2] & 0xFFFF0000u : w[j / 2] << 16);
        else return (float)__builtin_bit_cast(_Float16, (uint16_t)(w[j / 2] >> (16 * (j % 2))));
    }
    __device__ __forceinline__ void set(const float (&x)[8])     // rounded to nearest even
    {
#pragma unroll
        for (int i = 0; i < kWords; ++i) {
            if constexpr (DT == ZI_FP32) w[i] = __float_as_uint(x[i]);
            else w[i] = pair(x[2 * i], x[2 * i + 1]);
        }
    }
    static __device__ __forceinline__ uint32_t pair(float lo, float hi)
    {
        if constexpr (DT == ZI_BF16)
            return (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)lo) | (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)hi) << 16;
        else
            return (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)lo) | (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)hi) << 16;
    }
};

// ---- the scale of a block -------------------------------------------------------------------------------------

// Magnitudes are compared by their bits, which order as they do; an infinity or NaN counts as zero.
__device__ __forceinline__ uint32_t magnitude(float x)
{
    const uint32_t b = __float_as_uint(x) & 0x7FFFFFFFu;
    return b < 0x7F800000u ? b : 0u;
}
// The e8m0 byte of the smallest power of two s with `most` <= 448 s; 448 is 1.75 * 2^8.  (The bits of an fp32
// subnormal have no exponent; its scale is the least there is.)
__device__ __forceinline__ uint32_t scale_byte(uint32_t most)
{
    const int b = (int)(most >> 23) - 8 + ((most & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return most == 0 ? 127u : (uint32_t)(b > 0 ? b : 0);
}
// 1 / scale: a power of two from 2^-120 to 2^127, so that the product with it is exact but for numbers that round to
// zero anyway.
__device__ __forceinline__ float inverse_scale(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }

// Four e4m3 numbers, rounded to nearest even.  None is above 448 but infinities, which become NaN.
__device__ __forceinline__ uint32_t four_e4m3(float a, float b, float c, float d)
{
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
    return (uint32_t)w;
}

// ---- over lanes -----------------------------------------------------------------------------------------------

template <int CONTROL>
__device__ __forceinline__ uint32_t dpp(uint32_t x)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CONTROL, 0xF, 0xF, true);
}
constexpr int kDppXor1 = 0xB1, kDppXor2 = 0x4E, kDppHalfMirror = 0x141, kDppMirror = 0x140;

__device__ __forceinline__ uint32_t max_of(uint32_t a, uint32_t b) { return a > b ? a : b; }

// Largest over the 16 lanes of a row, in each of them.
__device__ __forceinline__ uint32_t max_16(uint32_t x)
{
    x = max_of(x, dpp<kDppXor1>(x));
    x = max_of(x, dpp<kDppXor2>(x));
    x = max_of(x, dpp<kDppHalfMirror>(x));
    return max_of(x, dpp<kDppMirror>(x));
}
// Largest over the four rows of 16 lanes, in each lane for its place in the row.
__device__ __forceinline__ uint32_t max_of_rows(uint32_t x)
{
    x = max_of(x, (uint32_t)__shfl_xor((int)x, 16));
    return max_of(x, (uint32_t)__shfl_xor((int)x, 32));
}
__device__ __forceinline__ float sum_64(float x)
{
    x += __uint_as_float(dpp<kDppXor1>(__float_as_uint(x)));
    x += __uint_as_float(dpp<kDppXor2>(__float_as_uint(x)));
    x += __uint_as_float(dpp<kDppHalfMirror>(__float_as_uint(x)));
    x += __uint_as_float(dpp<kDppMirror>(__float_as_uint(x)));
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}
// Over a workgroup of T threads, in each of them.  `space` is not used again before the next barrier.
template <int T>
__device__ __forceinline__ float sum_of_group(float x, float* space)
{
    x = sum_64(x);
    if constexpr (T == 64) return x;
    if ((threadIdx.x & 63) == 0) space[threadIdx.x >> 6] = x;
    __syncthreads();
    float sum = space[0];
#pragma unroll
    for (int i = 1; i < T / 64; ++i) sum += space[i];
    return sum;
}

}  // namespace zi
