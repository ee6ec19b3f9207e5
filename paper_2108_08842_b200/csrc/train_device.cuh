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

// ---- pairs of fp32 values: one packed instruction does both ---------------------------
struct Pair {
    uint64_t bits;
    __device__ __forceinline__ Pair() {}
    __device__ __forceinline__ Pair(float x, float y) { asm("mov.b64 %0, {%1, %2};" : "=l"(bits) : "f"(x), "f"(y)); }
    explicit __device__ __forceinline__ Pair(float x) : Pair(x, x) {}
    __device__ __forceinline__ void get(float& x, float& y) const { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(bits)); }
};

__device__ __forceinline__ Pair operator*(Pair a, Pair b)
{
    Pair r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.bits) : "l"(a.bits), "l"(b.bits));
    return r;
}

__device__ __forceinline__ Pair operator+(Pair a, Pair b)
{
    Pair r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.bits) : "l"(a.bits), "l"(b.bits));
    return r;
}

// a * b + c
__device__ __forceinline__ Pair fma(Pair a, Pair b, Pair c)
{
    Pair r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.bits) : "l"(a.bits), "l"(b.bits), "l"(c.bits));
    return r;
}

__device__ __forceinline__ float exp2_fast(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

__device__ __forceinline__ float reciprocal_fast(float x)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

__device__ __forceinline__ Pair exp2_fast(Pair a)
{
    float x, y;
    a.get(x, y);
    return {exp2_fast(x), exp2_fast(y)};
}

__device__ __forceinline__ Pair reciprocal_fast(Pair a)
{
    float x, y;
    a.get(x, y);
    return {reciprocal_fast(x), reciprocal_fast(y)};
}

__device__ __forceinline__ Pair magnitude(Pair a)
{
    float x, y;
    a.get(x, y);
    return {fabsf(x), fabsf(y)};
}

// ---- activations --------------------------------------------------------------------
// Two values at a time.  2^x and 1/x come from the special function unit, good to a unit or two in
// the last place of fp32, which the 16-bit types of the results do not show; it takes numbers below
// 2^-126 for 0, so results below about 2^-119 (silu under -87, gelu under -13) may be 0 too.  Two
// results a value: at 16 a cycle that is 4096 cycles for the 128 x 256 values of a product's epilogue
// and bounds the smooth activations there; one reciprocal shared by a pair cost more in
// multiplications and selections than it saved.  An erff and an expf for each value made the
// activation gradient of 8192 x 16384 take 257 us against 180, all else as it was.
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kTanhScale = 0.7978845608028654f;      // sqrt(2 / pi)
constexpr float kTanhCubic = 0.044715f;

// sigmoid(u) = 1 / (1 + 2^w) for w = -u * log2(e); 2^w overflows to infinity, which gives 0
__device__ __forceinline__ Pair sigmoid_of(Pair w) { return reciprocal_fast(Pair(1.f) + exp2_fast(w)); }

// 1 - Phi(|z|) = erfc(|z| / sqrt(2)) / 2 = t P(t) exp(-z^2 / 2) with t = 1 / (1 + p |z|), and
// exp(-z^2 / 2).  That form is Hastings' for erfc; P is the polynomial of degree 6 whose largest
// relative error for |z| up to 14.5 is the least (7.9e-7; a linear programme over 4000 points, p by
// search).  A fit of erfc's absolute error, with two terms less, was 5e-5 off at z = -3 and 9e-4 at
// -4.5, past fp16's half unit.
__device__ __forceinline__ Pair upper_tail(Pair z, Pair& bell)
{
    const Pair t = reciprocal_fast(fma(magnitude(z), Pair(0.3625f), Pair(1.f)));
    bell = exp2_fast(z * z * Pair(-0.5f * kLog2e));
    Pair q = fma(t, Pair(0.047876328f), Pair(-0.17912251f));
    q = fma(t, q, Pair(0.17428418f));
    q = fma(t, q, Pair(0.030232456f));
    q = fma(t, q, Pair(0.13906018f));
    q = fma(t, q, Pair(0.14297165f));
    q = fma(t, q, Pair(0.14469792f));
    return q * t * bell;
}

template <int ACT>
__device__ __forceinline__ Pair act_value(Pair z)
{
    if constexpr (ACT == EDEN_ACT_RELU) {
        float x, y;
        z.get(x, y);
        return {x < 0.f ? 0.f : x, y < 0.f ? 0.f : y};                     // NaN stays NaN
    }
    if constexpr (ACT == EDEN_ACT_GELU) {
        // z Phi(z) = max(z, 0) - |z| (1 - Phi(|z|)); the minimum keeps infinity from meeting its tail of 0
        Pair bell;
        const Pair tail = upper_tail(z, bell);
        float x, y;
        z.get(x, y);
        return fma(tail, Pair(-fminf(fabsf(x), 3.0e38f), -fminf(fabsf(y), 3.0e38f)), Pair(fmaxf(x, 0.f), fmaxf(y, 0.f)));
    }
    // (1 + tanh(u)) / 2 = sigmoid(2u)
    if constexpr (ACT == EDEN_ACT_GELU_TANH)
        return z * sigmoid_of(z * fma(z * z, Pair(-2.f * kLog2e * kTanhScale * kTanhCubic), Pair(-2.f * kLog2e * kTanhScale)));
    if constexpr (ACT == EDEN_ACT_SILU) return z * sigmoid_of(z * Pair(-kLog2e));
    return z;
}

// For |z| below 2^28 (see slope_scale), so that z * z * z stays finite where p * (1 - p) is 0.
template <int ACT>
__device__ __forceinline__ Pair act_slope(Pair z)
{
    if constexpr (ACT == EDEN_ACT_NONE) return Pair(1.f);
    float x, y;
    z.get(x, y);
    if constexpr (ACT == EDEN_ACT_RELU) return {x > 0.f ? 1.f : (x <= 0.f ? 0.f : x), y > 0.f ? 1.f : (y <= 0.f ? 0.f : y)};
    if constexpr (ACT == EDEN_ACT_GELU) {
        // Phi(z) + z exp(-z^2 / 2) / sqrt(2 pi): g = tail - |z| exp(-z^2 / 2) / sqrt(2 pi) below 0 and 1 - g
        // from 0 on, so that no difference of nearly equal numbers makes a small one
        Pair bell;
        const Pair tail = upper_tail(z, bell), g = fma(magnitude(z) * Pair(-0.3989422804014327f), bell, tail);
        float a, b, c, d;
        g.get(a, b);
        fma(g, Pair(-1.f), Pair(1.f)).get(c, d);
        return {x < 0.f ? a : c, y < 0.f ? b : d};
    }
    if constexpr (ACT == EDEN_ACT_GELU_TANH) {
        const Pair zz = z * z;
        const Pair p = sigmoid_of(z * fma(zz, Pair(-2.f * kLog2e * kTanhScale * kTanhCubic), Pair(-2.f * kLog2e * kTanhScale)));
        const Pair du = z * fma(zz, Pair(6.f * kTanhScale * kTanhCubic), Pair(2.f * kTanhScale));        // z * d(2u)/dz
        return fma(p * fma(p, Pair(-1.f), Pair(1.f)), du, p);
    }
    if constexpr (ACT == EDEN_ACT_SILU) {
        const Pair p = sigmoid_of(z * Pair(-kLog2e));
        return fma(p * fma(p, Pair(-1.f), Pair(1.f)), z, p);
    }
    return Pair(1.f);
}

template <int ACT>
__device__ __forceinline__ float act_value(float z)
{
    float x, y;
    act_value<ACT>(Pair(z, z)).get(x, y);
    return x;
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

// The scale for slopes: at most 2^20.  Beyond |z| = 100 every slope is 0 or 1 to fp32, so codes
// other than 0 have the same slopes under any larger scale.  NaN compares false and stays.
__device__ __forceinline__ float slope_scale(uint32_t exp_byte)
{
    const float s = group_scale(exp_byte);
    return s > 1048576.f ? 1048576.f : s;
}

// v * 2^-e as a whole number in the low byte: the sum with 1.5 * 2^23 rounds to nearest even.
// In a NaN group the product can be NaN: its code is 0 as well.
__device__ __forceinline__ uint32_t group_code(float v, float inverse)
{
    const uint32_t bits = __float_as_uint(__fmaf_rn(v, inverse, 12582912.f));
    return inverse == 0.f ? 0u : bits & 0xFFu;
}

// four codes in a word: the byte c + 128 under the exponent of 2^23 is 2^23 + 128 + c
__device__ __forceinline__ void code_values(uint32_t w, Pair scale, Pair& v01, Pair& v23)
{
    w ^= 0x80808080u;
    const Pair offset(-8388736.f);
    v01 = (Pair(__uint_as_float(__byte_perm(w, 0x4B000000u, 0x7440)), __uint_as_float(__byte_perm(w, 0x4B000000u, 0x7441))) + offset) * scale;
    v23 = (Pair(__uint_as_float(__byte_perm(w, 0x4B000000u, 0x7442)), __uint_as_float(__byte_perm(w, 0x4B000000u, 0x7443))) + offset) * scale;
}

__device__ __forceinline__ uint32_t group_codes(float v0, float v1, float v2, float v3, float inverse)
{
    float c0, c1, c2, c3;
    fma(Pair(v0, v1), Pair(inverse), Pair(12582912.f)).get(c0, c1);
    fma(Pair(v2, v3), Pair(inverse), Pair(12582912.f)).get(c2, c3);
    const uint32_t w = __byte_perm(__byte_perm(__float_as_uint(c0), __float_as_uint(c1), 0x0040),
                                   __byte_perm(__float_as_uint(c2), __float_as_uint(c3), 0x0040), 0x5410);
    return inverse == 0.f ? 0u : w;
}

// max(m, |a|, |b|), NaN if one is
__device__ __forceinline__ float max_magnitude(float m, float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(m), "f"(fabsf(a)), "f"(fabsf(b)));
    return r;
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

// ---- accesses at any address ----------------------------------------------------------
// WORDS words from p on, of which the first `bytes` bytes exist (zeros after them): the aligned
// 16-byte chunks that hold them, shifted.  Chunks without a byte of theirs are not touched.
template <int WORDS>
__device__ __forceinline__ void load_shifted(const void* p, int bytes, uint32_t (&v)[WORDS])
{
    const uintptr_t address = (uintptr_t)p;
    const int off = (int)(address & 15u);
    const uint4* chunk = (const uint4*)(address - off);
    uint32_t w[WORDS + 4];
#pragma unroll
    for (int i = 0; i <= WORDS / 4; ++i) {
        uint4 q = make_uint4(0, 0, 0, 0);
        if (bytes > 0 && off + bytes > 16 * i) q = chunk[i];
        w[4 * i] = q.x; w[4 * i + 1] = q.y; w[4 * i + 2] = q.z; w[4 * i + 3] = q.w;
    }
    if (off & 8) {
#pragma unroll
        for (int i = 0; i < WORDS + 2; ++i) w[i] = w[i + 2];
    }
    if (off & 4) {
#pragma unroll
        for (int i = 0; i < WORDS + 1; ++i) w[i] = w[i + 1];
    }
    const uint32_t bits = (off & 3) * 8;
#pragma unroll
    for (int j = 0; j < WORDS; ++j) v[j] = __funnelshift_r(w[j], w[j + 1], bits);
    if (bytes < 4 * WORDS) {
#pragma unroll
        for (int j = 0; j < WORDS; ++j) {
            const int left = bytes - 4 * j;
            v[j] = left >= 4 ? v[j] : left > 0 ? v[j] & (0xFFFFFFFFu >> (32 - 8 * left)) : 0u;
        }
    }
}

// The first `bytes` bytes of v to p, in words where they are whole, in bytes at the ends.
template <int WORDS>
__device__ __forceinline__ void store_shifted(void* p, int bytes, const uint32_t (&v)[WORDS])
{
    const int off = (int)((uintptr_t)p & 3u);
    char* base = (char*)p - off;
#pragma unroll
    for (int j = 0; j <= WORDS; ++j) {
        const uint32_t w = __funnelshift_l(j > 0 ? v[j - 1] : 0u, j < WORDS ? v[j] : 0u, 8 * off);
        const int first = 4 * j - off;                       // byte of v at the word's start
        if (first >= 0 && first + 4 <= bytes) {
            *(uint32_t*)(base + 4 * j) = w;
        } else if (first + 4 > 0 && first < bytes) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (first + i >= 0 && first + i < bytes) base[4 * j + i] = (char)(w >> 8 * i);
        }
    }
}

// The same for 8 values of 16 bits, of which `count` exist, without a branch: several calls' loads
// are on their way together (94 us for 4 x 12544 x 6046 through load_shifted, 67 through this).
__device__ __forceinline__ uint4 load_shifted_8(const void* p, int count)
{
    const uintptr_t address = (uintptr_t)p;
    const uint32_t off = (uint32_t)address & 15u;
    const uint4* chunk = (const uint4*)(address - off);
    uint4 lo = make_uint4(0, 0, 0, 0), hi = lo;
    if (count > 0) lo = chunk[0];
    if ((int)off + 2 * count > 16) hi = chunk[1];
    uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
    for (int i = 0; i < 6; ++i) w[i] = off & 8u ? w[i + 2] : w[i];
#pragma unroll
    for (int i = 0; i < 5; ++i) w[i] = off & 4u ? w[i + 1] : w[i];
    const uint32_t bits = (off & 2u) * 8;
    uint32_t v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int left = count - 2 * j;                      // values from this word on
        v[j] = __funnelshift_r(w[j], w[j + 1], bits) & (left >= 2 ? 0xFFFFFFFFu : left == 1 ? 0xFFFFu : 0u);
    }
    return make_uint4(v[0], v[1], v[2], v[3]);
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
