// Arithmetic shared by the kernels of the client's training step: activations and their
// slopes, the 8-bit group form of activations, conversions.
#pragma once

#include <cstdint>
#include <type_traits>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "../../include/eden.h"

namespace eden {

constexpr int kGroup = (int)EDEN_CHECKPOINT_GROUP;

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }

template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// ---- activations --------------------------------------------------------------------
// sigmoid(u) = 1 / (1 + exp(-u)); exp overflows to infinity for u < -88, which gives 0
__device__ __forceinline__ float sigmoid(float u) { return __fdividef(1.f, 1.f + __expf(-u)); }

constexpr float kTanhScale = 0.7978845608028654f;      // sqrt(2 / pi)
constexpr float kTanhCubic = 0.044715f;

template <int ACT>
__device__ __forceinline__ float act_value(float z)
{
    if constexpr (ACT == EDEN_ACT_RELU) return z < 0.f ? 0.f : z;          // NaN stays NaN
    if constexpr (ACT == EDEN_ACT_GELU) return 0.5f * z * (1.f + erff(z * 0.7071067811865476f));
    // (1 + tanh(u)) / 2 = sigmoid(2u)
    if constexpr (ACT == EDEN_ACT_GELU_TANH) return z * sigmoid(2.f * kTanhScale * (z + kTanhCubic * z * z * z));
    if constexpr (ACT == EDEN_ACT_SILU) return z * sigmoid(z);
    return z;
}

// Beyond |z| = 100 every slope is 0 or 1 to fp32; the clamp keeps z * z * z and z * p * (1 - p)
// from meeting as infinity times zero.  A NaN compares false and passes through.
template <int ACT>
__device__ __forceinline__ float act_slope(float z)
{
    if constexpr (ACT == EDEN_ACT_NONE) return 1.f;
    if constexpr (ACT == EDEN_ACT_RELU) return z > 0.f ? 1.f : (z <= 0.f ? 0.f : z);
    if (fabsf(z) > 100.f) z = copysignf(100.f, z);
    if constexpr (ACT == EDEN_ACT_GELU)
        return 0.5f * (1.f + erff(z * 0.7071067811865476f)) + z * 0.3989422804014327f * __expf(-0.5f * z * z);
    if constexpr (ACT == EDEN_ACT_GELU_TANH) {
        const float p = sigmoid(2.f * kTanhScale * (z + kTanhCubic * z * z * z));
        return p + z * p * (1.f - p) * 2.f * kTanhScale * (1.f + 3.f * kTanhCubic * z * z);
    }
    if constexpr (ACT == EDEN_ACT_SILU) {
        const float p = sigmoid(z);
        return p * (1.f + z * (1.f - p));
    }
    return 1.f;
}

// f(std::integral_constant<int, act>): one branch around a block of values
template <typename F>
__device__ __forceinline__ void with_act(int act, F&& f)
{
    switch (act) {
        case EDEN_ACT_RELU: f(std::integral_constant<int, EDEN_ACT_RELU>()); break;
        case EDEN_ACT_GELU: f(std::integral_constant<int, EDEN_ACT_GELU>()); break;
        case EDEN_ACT_GELU_TANH: f(std::integral_constant<int, EDEN_ACT_GELU_TANH>()); break;
        case EDEN_ACT_SILU: f(std::integral_constant<int, EDEN_ACT_SILU>()); break;
        default: f(std::integral_constant<int, EDEN_ACT_NONE>()); break;
    }
}

// ---- 8-bit groups -------------------------------------------------------------------
__device__ __forceinline__ uint32_t magnitude_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// Exponent byte of a group from the largest magnitude's bits.  max = 1.f * 2^E; 127 * 2^(E-6)
// is 1.984375 * 2^E, so e = E - 6, or E - 5 where the fraction is above 0x7E0000: adding
// 0x1FFFF carries into the exponent exactly then.  Infinity and NaN have the largest bits.
__device__ __forceinline__ uint32_t group_exponent(uint32_t max_bits)
{
    if (max_bits >= 0x7F800000u) return 255u;
    const int e = (int)((max_bits + 0x1FFFFu) >> 23) - 6;
    return (uint32_t)(e < 1 ? 1 : e);
}

// 2^-e; 0 for the byte 255, so that finite members of a NaN group code as 0
__device__ __forceinline__ float group_inverse(uint32_t exp_byte)
{
    return exp_byte == 255u ? 0.f : __uint_as_float((254u - exp_byte) << 23);
}

// 2^e, NaN for the byte 255
__device__ __forceinline__ float group_scale(uint32_t exp_byte)
{
    return __uint_as_float(exp_byte == 255u ? 0x7FC00000u : exp_byte << 23);
}

// v * 2^-e as a whole number in the low byte: the sum with 1.5 * 2^23 rounds to nearest even.
// In a NaN group the product can be NaN: its code is 0 as well.
__device__ __forceinline__ uint32_t group_code(float v, float inverse)
{
    const uint32_t bits = __float_as_uint(__fmaf_rn(v, inverse, 12582912.f));
    return inverse == 0.f ? 0u : bits & 0xFFu;
}

__device__ __forceinline__ float code_value(int8_t code, float scale) { return (float)code * scale; }

// four codes in a word: the byte c + 128 under the exponent of 2^23 is 2^23 + 128 + c
__device__ __forceinline__ void code_values(uint32_t w, float scale, float& v0, float& v1, float& v2, float& v3)
{
    w ^= 0x80808080u;
    v0 = (__uint_as_float(__byte_perm(w, 0x4B000000u, 0x7440)) - 8388736.f) * scale;
    v1 = (__uint_as_float(__byte_perm(w, 0x4B000000u, 0x7441)) - 8388736.f) * scale;
    v2 = (__uint_as_float(__byte_perm(w, 0x4B000000u, 0x7442)) - 8388736.f) * scale;
    v3 = (__uint_as_float(__byte_perm(w, 0x4B000000u, 0x7443)) - 8388736.f) * scale;
}

__device__ __forceinline__ uint32_t group_codes(float v0, float v1, float v2, float v3, float inverse)
{
    const uint32_t b0 = __float_as_uint(__fmaf_rn(v0, inverse, 12582912.f)), b1 = __float_as_uint(__fmaf_rn(v1, inverse, 12582912.f));
    const uint32_t b2 = __float_as_uint(__fmaf_rn(v2, inverse, 12582912.f)), b3 = __float_as_uint(__fmaf_rn(v3, inverse, 12582912.f));
    const uint32_t w = __byte_perm(__byte_perm(b0, b1, 0x0040), __byte_perm(b2, b3, 0x0040), 0x5410);
    return inverse == 0.f ? 0u : w;
}

// A restored value in the type of its activations.  A maximum close to the type's largest
// number can round up to a code past it (64 * 2^122, 64 * 2^10): that saturates.
template <typename T> struct Largest;
template <> struct Largest<float> { static constexpr float value = 3.4028234663852886e38f; };
template <> struct Largest<__nv_bfloat16> { static constexpr float value = 3.3895313892515355e38f; };
template <> struct Largest<__half> { static constexpr float value = 65504.f; };

template <typename T>
__device__ __forceinline__ float saturated(float v)
{
    return fabsf(v) > Largest<T>::value ? copysignf(Largest<T>::value, v) : v;      // NaN compares false
}

// groups whose exponent byte is below this cannot pass the largest number: 128 * 2^e
template <typename T> constexpr uint32_t kSaturates = std::is_same_v<T, __half> ? 127 + 9 : 127 + 121;

// ---- 32-byte accesses ---------------------------------------------------------------
__device__ __forceinline__ void load_32b(const void* p, uint32_t (&w)[8])
{
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                 : "l"(p) : "memory");
}

__device__ __forceinline__ void store_32b(void* p, const uint32_t (&w)[8])
{
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                 : "memory");
}

template <typename T>
__device__ __forceinline__ void unpack(uint32_t w, float& lo, float& hi)
{
    if constexpr (std::is_same_v<T, __nv_bfloat16>) {
        lo = __uint_as_float(w << 16);
        hi = __uint_as_float(w & 0xFFFF0000u);
    } else {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
        lo = f.x;
        hi = f.y;
    }
}

template <typename T>
__device__ __forceinline__ uint32_t pack(float lo, float hi)
{
    if constexpr (std::is_same_v<T, __nv_bfloat16>) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&h);
    } else {
        const __half2 h = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
}

struct CheckpointView {
    int8_t* codes;
    uint64_t codes_stride;
    uint8_t* exps;
    uint64_t exps_stride;
};

// ---- launches that overlap ----------------------------------------------------------
// These kernels are launched before the stream's previous kernel has ended.  Each one waits
// for it (and for its memory) before it touches global memory, and lets the next one start.
// What they read may be written while they already run, so no pointer is __restrict__: that
// would allow loads through the read-only path, which assumes constant data.
__device__ __forceinline__ void dependency_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void dependency_release() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

}  // namespace eden
