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

// How an octet comes that a row ends in: there is none; it is the row's last eight elements (of eight at least), one load for all lanes alike, which settle()
// moves down where they are used (where they are loaded it would wait for them: backward pass of 10743 x 2509 154 us against 102); its elements one by one.
enum class Ends { kWhole, kMoved, kApart };

// Eight elements of a row.  Rows need only be aligned to their element: the hardware takes such vectors as they are.
template <int DT>
struct Octet {
    static constexpr int kWords = DT == ZI_FP32 ? 8 : 4;
    static constexpr int kBytes = DT == ZI_FP32 ? 4 : 2;
    using vec = std::conditional_t<DT == ZI_FP32, u32x4_of_4, u32x4_of_2>;
    uint32_t w[kWords];

    // The octet at `at`, of which a row of `cols` has `left` more elements (none or less than none: zeros); zeros behind its end.
    // STREAM: past the caches, of what is more than they hold.
    template <Ends ENDS, bool STREAM = false>
    __device__ __forceinline__ void load(const void* base, int64_t at, int left)
    {
        int past = 0;
        if constexpr (ENDS == Ends::kMoved) {
            past = left >= 8 ? 0 : 8 - left;
        } else if (left < 8) {
            if (ENDS == Ends::kApart) load_short(base, at, left);
            else clear();
            return;
        }
        const char* p = static_cast<const char*>(base) + (at - past) * kBytes;
#pragma unroll
        for (int i = 0; i < kWords / 4; ++i) {
            vec v;
            if constexpr (STREAM) v = __builtin_nontemporal_load(reinterpret_cast<const vec*>(p) + i);
            else v = reinterpret_cast<const vec*>(p)[i];
#pragma unroll
            for (int j = 0; j < 4; ++j) w[4 * i + j] = v[j];
        }
    }
    template <Ends ENDS>
    __device__ __forceinline__ void settle(int left)
    {
        if constexpr (ENDS == Ends::kMoved)
            if (left < 8) {
                if (left > 0) drop(8 - left);
                else clear();
            }
    }
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = 0;
    }
    // Without its first `count` elements, with zeros behind the others.
    __device__ __forceinline__ void drop(int count)
    {
        constexpr int kEach = 4 / kBytes;           // elements of a word
        if constexpr (kEach == 2)
            if (count & 1) {
#pragma unroll
                for (int i = 0; i < kWords; ++i) w[i] = (w[i] >> 16) | (i + 1 < kWords ? w[i + 1] << 16 : 0u);
            }
#pragma unroll
        for (int by = 1; by < kWords; by *= 2)
            if (count & (by * kEach)) {
#pragma unroll
                for (int i = 0; i < kWords; ++i) w[i] = i + by < kWords ? w[i + by] : 0u;
            }
    }
    // Less than eight elements, one by one.
    __device__ __forceinline__ void load_short(const void* base, int64_t at, int left)
    {
        const char* p = static_cast<const char*>(base) + at * kBytes;
        clear();
#pragma unroll
        for (int j = 0; j < 7; ++j) {
            if (j < left) {
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

// Magnitudes are compared by their bits, which order as they do: one fp32 or two 16-bit elements of a word at a time.
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
template <int DT>
constexpr uint32_t kInfinity = DT == ZI_FP32 ? 0x7F800000u : DT == ZI_BF16 ? 0x7F80u : 0x7C00u;

// FINITE: an infinity or NaN counts as zero.
template <int DT, bool FINITE>
__device__ __forceinline__ uint32_t magnitudes(uint32_t w)
{
    if constexpr (DT == ZI_FP32) {
        w &= 0x7FFFFFFFu;
        return FINITE && w >= kInfinity<DT> ? 0u : w;
    } else {
        w &= 0x7FFF7FFFu;
        if constexpr (FINITE) {
            if ((w & 0xFFFFu) >= kInfinity<DT>) w &= 0xFFFF0000u;
            if (w >> 16 >= kInfinity<DT>) w &= 0xFFFFu;
        }
        return w;
    }
}
__device__ __forceinline__ uint32_t max_of(uint32_t a, uint32_t b) { return a > b ? a : b; }
template <int DT>
__device__ __forceinline__ uint32_t max_of_words(uint32_t a, uint32_t b)
{
    if constexpr (DT == ZI_FP32) return max_of(a, b);
    else return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}
// The larger element of a word, and its fp32 bits.
template <int DT>
__device__ __forceinline__ uint32_t larger(uint32_t w)
{
    return DT == ZI_FP32 ? w : max_of(w & 0xFFFFu, w >> 16);
}
template <int DT>
__device__ __forceinline__ uint32_t as_fp32(uint32_t m)
{
    if constexpr (DT == ZI_FP32) return m;
    else if constexpr (DT == ZI_BF16) return m << 16;
    else return __float_as_uint((float)__builtin_bit_cast(_Float16, (uint16_t)m));
}
// The e8m0 byte of the smallest power of two s with `most` <= 448 s; 448 is 1.75 * 2^8.  (The bits of an fp32
// subnormal have no exponent; its scale is the least there is.)
__device__ __forceinline__ uint32_t scale_byte(uint32_t most)
{
    const int b = (int)(most >> 23) - 8 + ((most & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return most == 0 ? 127u : (uint32_t)(b > 0 ? b : 0);
}
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte > 0 ? byte << 23 : 1u << 22); }

// Two e4m3 numbers into half of a word: elements divided by the scale, rounded to nearest even.  None is above 448 then
// but infinities, which become NaN.
typedef short i16x2 __attribute__((ext_vector_type(2)));
template <int HALF>
__device__ __forceinline__ i16x2 two_e4m3(i16x2 w, float a, float b, float scale)
{
    return __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, a, b, scale, HALF);
}
template <int DT, int HALF>
__device__ __forceinline__ i16x2 two_e4m3(i16x2 w, uint32_t ab, float scale)
{
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
    if constexpr (DT == ZI_BF16) return __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, __builtin_bit_cast(bf16x2, ab), scale, HALF);
    else return __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(w, __builtin_bit_cast(f16x2, ab), scale, HALF);
}
__device__ __forceinline__ uint32_t four_e4m3(float a, float b, float c, float d, float scale)
{
    return __builtin_bit_cast(uint32_t, two_e4m3<1>(two_e4m3<0>(i16x2{0, 0}, a, b, scale), c, d, scale));
}
// Eight of a row, and eight that stand below each other.
template <int DT>
__device__ __forceinline__ u32x2 eight_e4m3(const Octet<DT>& x, float scale)
{
    u32x2 q;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if constexpr (DT == ZI_FP32)
            q[i] = four_e4m3(x.get(4 * i), x.get(4 * i + 1), x.get(4 * i + 2), x.get(4 * i + 3), scale);
        else
            q[i] = __builtin_bit_cast(uint32_t, two_e4m3<DT, 1>(two_e4m3<DT, 0>(i16x2{0, 0}, x.w[2 * i], scale), x.w[2 * i + 1], scale));
    }
    return q;
}
template <int DT>
__device__ __forceinline__ u32x2 eight_e4m3_down(const Octet<DT> (&x)[8], int j, float scale)
{
    u32x2 q;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if constexpr (DT == ZI_FP32) {
            q[i] = four_e4m3(x[4 * i].get(j), x[4 * i + 1].get(j), x[4 * i + 2].get(j), x[4 * i + 3].get(j), scale);
        } else {
            const uint32_t halves = j % 2 ? 0x07060302u : 0x05040100u;       // the upper or the lower halves of two words
            const uint32_t ab = __builtin_amdgcn_perm(x[4 * i + 1].w[j / 2], x[4 * i].w[j / 2], halves);
            const uint32_t cd = __builtin_amdgcn_perm(x[4 * i + 3].w[j / 2], x[4 * i + 2].w[j / 2], halves);
            q[i] = __builtin_bit_cast(uint32_t, two_e4m3<DT, 1>(two_e4m3<DT, 0>(i16x2{0, 0}, ab, scale), cd, scale));
        }
    }
    return q;
}

// ---- over lanes -----------------------------------------------------------------------------------------------

template <int CONTROL>
__device__ __forceinline__ uint32_t dpp(uint32_t x)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CONTROL, 0xF, 0xF, true);
}
constexpr int kDppXor1 = 0xB1, kDppXor2 = 0x4E, kDppHalfMirror = 0x141, kDppMirror = 0x140;

// Largest over the 16 lanes of a row, in each of them.
__device__ __forceinline__ uint32_t max_16(uint32_t x)
{
    x = max_of(x, dpp<kDppXor1>(x));
    x = max_of(x, dpp<kDppXor2>(x));
    x = max_of(x, dpp<kDppHalfMirror>(x));
    return max_of(x, dpp<kDppMirror>(x));
}
// Largest (of a word's elements each) over the four rows of 16 lanes, in each lane for its place in the row.
template <int DT>
__device__ __forceinline__ uint32_t max_of_rows(uint32_t x)
{
    x = max_of_words<DT>(x, (uint32_t)__shfl_xor((int)x, 16));
    return max_of_words<DT>(x, (uint32_t)__shfl_xor((int)x, 32));
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
