// Activations, their derivatives and dropout's generator, as the kernels of the epilogues use them (include/zi_epilogue.h has the formulas).
#pragma once

#include "zi_epilogue_internal.h"
#include "zi_fp8_device.h"

namespace zi {

// ---- activations ----------------------------------------------------------------------------------------------

// exp and 1 / x are the hardware's (one step off at most; results below 2^-126 are zero): what is made of them is rounded to 16 or 8 bits.
__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float inverse(float x) { return __builtin_amdgcn_rcpf(x); }
constexpr float kLog2E = 1.44269504f;

// 1 / (1 + exp(-z)) for z = -x / log2 e
__device__ __forceinline__ float sigmoid_of_exponent(float x) { return inverse(1.0f + exp2_of(x)); }

// Phi(-t) = exp(-t^2 / 2) R(t) for t >= 0, where R falls slowly from 1/2: a polynomial in 1 / (1 + 0.3 t), fitted to the smallest largest relative error on [0, 14.5]
// (6e-8; 4.2e-7 as it is computed here).  `e` is exp(-t^2 / 2), which the derivative needs too.
__device__ __forceinline__ float normal_cdf(float z, float& e)
{
    const float t = __builtin_fabsf(z), w = inverse(__builtin_fmaf(0.3f, t, 1.0f));
    float r = 0.038407549262046814f;
    r = __builtin_fmaf(r, w, -0.16930820047855377f);
    r = __builtin_fmaf(r, w, 0.2289532572031021f);
    r = __builtin_fmaf(r, w, -0.07684128731489182f);
    r = __builtin_fmaf(r, w, 0.1427663415670395f);
    r = __builtin_fmaf(r, w, 0.09458543360233307f);
    r = __builtin_fmaf(r, w, 0.12194536626338959f);
    r = __builtin_fmaf(r, w, 0.11948419362306595f);
    r = __builtin_fmaf(r, w, 7.373110292974161e-06f);
    e = exp2_of(z * z * (-0.5f * kLog2E));
    r *= e;
    return z < 0.0f ? r : 1.0f - r;
}

constexpr float kTanh = 1.5957691216f, kTanhCube = 0.0713548163f;        // 2 sqrt(2 / pi), and that times 0.044715

template <int ACT>
__device__ __forceinline__ float activated(float z)
{
    if constexpr (ACT == ZI_ACT_RELU) return z < 0.0f ? 0.0f : z;
    else if constexpr (ACT == ZI_ACT_GELU) {
        float e;
        return z * normal_cdf(z, e);
    } else if constexpr (ACT == ZI_ACT_GELU_TANH) {
        return z * sigmoid_of_exponent(z * __builtin_fmaf(z * z, -kLog2E * kTanhCube, -kLog2E * kTanh));
    } else if constexpr (ACT == ZI_ACT_SILU) return z * sigmoid_of_exponent(-kLog2E * z);
    else return z;
}
// dy times the derivative.  (Where a sigmoid s is 0 or 1, s (1 - s) is 0, which its large factors are multiplied to one after the other; z counts as FAR there at most, so that
// infinities have the limits 0 and 1 and not 0 times infinity.  A NaN comes back through exp.)  It is one instruction an element.  us, without / with, to 8 bits both ways and dbias: gelu_tanh of
// 8191 x 16384 155.9 / 156.0, gelu of 8192 x 16384 159.0 / 160.1, silu 154.0 / 154.2.
template <int FAR>
__device__ __forceinline__ float not_beyond(float z) { return __builtin_amdgcn_fmed3f(z, -(float)FAR, (float)FAR); }
template <int ACT>
__device__ __forceinline__ float with_derivative(float dy, float z)
{
    if constexpr (ACT == ZI_ACT_RELU) return z <= 0.0f ? 0.0f : dy;
    else if constexpr (ACT == ZI_ACT_GELU) {
        float e;
        const float phi = normal_cdf(z, e);
        return dy * __builtin_fmaf(not_beyond<64>(z) * e, 0.398942280f, phi);                                   // (beyond 15, e is 0)
    } else if constexpr (ACT == ZI_ACT_GELU_TANH) {
        // 1 - s is exp(..) s, without the rounding of s near 1, which the slope of the cube (up to 50) would make much of; 1 where exp is infinite.
        const float z2 = z * z, e = exp2_of(z * __builtin_fmaf(z2, -kLog2E * kTanhCube, -kLog2E * kTanh)), s = inverse(1.0f + e), rest = __builtin_fminf(e * s, 1.0f);
        const float slope = __builtin_fmaf(__builtin_fminf(z2, 256.0f), 3.0f * kTanhCube, kTanh);                // (beyond 16, s (1 - s) is 0)
        return dy * __builtin_fmaf(s * rest * not_beyond<16>(z), slope, s);
    } else if constexpr (ACT == ZI_ACT_SILU) {
        const float s = sigmoid_of_exponent(-kLog2E * z);
        return dy * __builtin_fmaf(__builtin_fmaf(-s, s, s), not_beyond<128>(z), s);                            // (beyond 89, s is 0 or 1)
    } else return dy;
}
// f(activation as a type), for an activation that is the same in all lanes.
template <typename F>
__device__ __forceinline__ void with_activation(int activation, const F& f)
{
    switch (activation) {
    case ZI_ACT_RELU: return f(std::integral_constant<int, ZI_ACT_RELU>());
    case ZI_ACT_GELU: return f(std::integral_constant<int, ZI_ACT_GELU>());
    case ZI_ACT_GELU_TANH: return f(std::integral_constant<int, ZI_ACT_GELU_TANH>());
    case ZI_ACT_SILU: return f(std::integral_constant<int, ZI_ACT_SILU>());
    }
}
// Eight elements, of an activation that is known or (ACT kAnyActivation) is not.
constexpr int kAnyActivation = -1;
template <int ACT>
__device__ __forceinline__ void activate(float (&x)[8], int activation)
{
    if constexpr (ACT != kAnyActivation) {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = activated<ACT>(x[j]);
    } else {
        with_activation(activation, [&](auto act) { activate<decltype(act)::value>(x, activation); });
    }
}
template <int ACT>
__device__ __forceinline__ void derive(float (&dy)[8], const float (&z)[8], int activation)
{
    if constexpr (ACT != kAnyActivation) {
#pragma unroll
        for (int j = 0; j < 8; ++j) dy[j] = with_derivative<ACT>(dy[j], z[j]);
    } else {
        with_activation(activation, [&](auto act) { derive<decltype(act)::value>(dy, z, activation); });
    }
}

// The product's kernels know less of the activation, as each is made for several sizes of tile too (and a branch among all of them, with a tile's sums in registers, costs registers that
// there are not): its kind, with numbers that are the same in all lanes.
enum class ActivationKind { kFloor, kSigmoid, kNormal };       // none and relu; gelu_tanh and silu; gelu
struct ActivationForm {
    float a, b;
    __device__ __forceinline__ explicit ActivationForm(int activation)
        : a(activation == ZI_ACT_GELU_TANH ? -kLog2E * kTanh : activation == ZI_ACT_SILU ? -kLog2E : activation == ZI_ACT_RELU ? 0.0f : -__builtin_inff()),
          b(activation == ZI_ACT_GELU_TANH ? -kLog2E * kTanhCube : 0.0f)
    {
    }
};
template <ActivationKind KIND>
__device__ __forceinline__ float activated_as(const ActivationForm& f, float z)
{
    if constexpr (KIND == ActivationKind::kFloor) return z < f.a ? 0.0f : z;
    else if constexpr (KIND == ActivationKind::kSigmoid) return z * sigmoid_of_exponent(z * __builtin_fmaf(__builtin_fminf(z * z, 0x1p100f), f.b, f.a));      // (0 times infinity would be NaN)
    else return activated<ZI_ACT_GELU>(z);
}
inline ActivationKind kind_of(int activation)
{
    return activation == ZI_ACT_GELU ? ActivationKind::kNormal : activation == ZI_ACT_GELU_TANH || activation == ZI_ACT_SILU ? ActivationKind::kSigmoid : ActivationKind::kFloor;
}

// Largest finite magnitude of N numbers, its fp32 bits.  (A NaN has no part in a maximum; only where an infinity is found they are looked through again.)
template <int N>
__device__ __forceinline__ uint32_t most_of(const float (&x)[N])
{
    float most = 0.0f;
#pragma unroll
    for (int j = 0; j < N; j += 2) most = __builtin_fmaxf(__builtin_fmaxf(__builtin_fabsf(x[j]), __builtin_fabsf(x[j + 1])), most);
    if (most == __builtin_inff()) {
        most = 0.0f;
#pragma unroll
        for (int j = 0; j < N; ++j) most = __builtin_fabsf(x[j]) < __builtin_inff() ? __builtin_fmaxf(most, __builtin_fabsf(x[j])) : most;
    }
    return __float_as_uint(most);
}

// ---- dropout --------------------------------------------------------------------------------------------------

__device__ __forceinline__ uint32_t xor_of(uint32_t a, uint32_t b, uint32_t c) { return __builtin_amdgcn_bitop3_b32(a, b, c, 0x96); }

// Philox4x32-10: ten rounds, of two 32 x 32 -> 64 multiplications each, on a counter of four words.  One call is eight columns' numbers.
struct Dropout {
    uint32_t key0, key1, offset0, offset1, threshold;
    float scale;

    __device__ __forceinline__ explicit Dropout(const DropoutArgs& a) : key0((uint32_t)a.seed), key1((uint32_t)(a.seed >> 32)), threshold(a.threshold), scale(a.scale)
    {
        const uint64_t offset = a.offset + (a.threshold && a.d_offset ? *a.d_offset : 0);
        offset0 = (uint32_t)offset;
        offset1 = (uint32_t)(offset >> 32);
    }
    __device__ __forceinline__ u32x4 numbers(uint32_t octet, uint32_t row) const
    {
        uint32_t x0 = octet, x1 = row, x2 = offset0, x3 = offset1, k0 = key0, k1 = key1;
#pragma unroll
        for (int i = 0; i < 10; ++i) {
            const uint64_t a = (uint64_t)x0 * 0xD2511F53u, b = (uint64_t)x2 * 0xCD9E8D57u;
            x0 = xor_of((uint32_t)(b >> 32), x1, k0);
            x1 = (uint32_t)b;
            x2 = xor_of((uint32_t)(a >> 32), x3, k1);
            x3 = (uint32_t)a;
            k0 += 0x9E3779B9u;
            k1 += 0xBB67AE85u;
        }
        return u32x4{x0, x1, x2, x3};
    }
    __device__ __forceinline__ bool active() const { return threshold != 0; }
    __device__ __forceinline__ static bool is_kept(const u32x4& w, int j, uint32_t threshold)
    {
        return (uint16_t)(w[j / 2] >> (16 * (j % 2))) >= (uint16_t)threshold;
    }
    // Eight columns of a row, from 8 * octet on.
    __device__ __forceinline__ void apply(float (&x)[8], uint32_t octet, uint32_t row) const
    {
        if (!active()) return;
        const u32x4 w = numbers(octet, row);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = is_kept(w, j, threshold) ? x[j] * scale : 0.0f;
    }
    // The same of a gradient that a derivative at z follows: what is dropped is made of z = 0, since 0 times the derivative at an infinity or NaN would not be 0.
    __device__ __forceinline__ void apply(float (&x)[8], float (&z)[8], uint32_t octet, uint32_t row) const
    {
        if (!active()) return;
        const u32x4 w = numbers(octet, row);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const bool keep = is_kept(w, j, threshold);
            x[j] = keep ? x[j] * scale : 0.0f;
            z[j] = keep ? z[j] : 0.0f;
        }
    }
};

}  // namespace zi
