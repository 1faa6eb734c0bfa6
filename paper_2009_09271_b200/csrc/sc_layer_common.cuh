// Definitions shared by the layer operators: 16-bit types, activations and their slopes, the 8-bit checkpoint's rounding.
#pragma once
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <type_traits>

#include "../../include/sparsecomm.h"

namespace sc {

constexpr uint32_t CKPT_GROUP = 32;           // features that share one scale

__host__ __device__ inline uint64_t ckpt_groups(uint64_t cols) { return (cols + CKPT_GROUP - 1) / CKPT_GROUP; }

// ---------------------------------------------------------------------------
// types
// ---------------------------------------------------------------------------
template <typename T> struct Elem;
template <> struct Elem<__nv_bfloat16> {
    static constexpr int EMIN = -126, EMAX = 122;              // q 2^e is a bf16 for |q| <= 127 and e in this range
    static constexpr uint32_t ABS = 0x7FFF7FFFu, INF16 = 0x7F80u;
    __device__ static float2 unpack(uint32_t v) { return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xFFFF0000u)); }
    __device__ static uint32_t pack(float lo, float hi) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
    __device__ static float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
    __device__ static __nv_bfloat16 from_float(float v) { return __float2bfloat16_rn(v); }
};
template <> struct Elem<__half> {
    static constexpr int EMIN = -24, EMAX = 10;                // multiples of 2^-24 up to 63 * 2^10
    static constexpr uint32_t ABS = 0x7FFF7FFFu, INF16 = 0x7C00u;
    __device__ static float2 unpack(uint32_t v) { return __half22float2(*reinterpret_cast<const __half2*>(&v)); }
    __device__ static uint32_t pack(float lo, float hi) {
        const __half2 h = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
    __device__ static float to_float(__half v) { return __half2float(v); }
    __device__ static __half from_float(float v) { return __float2half_rn(v); }
};
template <> struct Elem<float> {
    static constexpr int EMIN = -126, EMAX = 122;
    __device__ static float to_float(float v) { return v; }
    __device__ static float from_float(float v) { return v; }
};

// ---------------------------------------------------------------------------
// activations, in 32 bits
// ---------------------------------------------------------------------------
constexpr float SQRT_HALF = 0.70710678118654752f, INV_SQRT_2PI = 0.39894228040143268f;
constexpr float GELU_C = 1.5957691216057308f, GELU_A = 0.044715f;      // 2 sqrt(2 / pi), cubic coefficient

// 1 / (1 + 2^v): one exponential and one reciprocal, both within a few units of the last place.
__device__ __forceinline__ float inv_1p_exp2(float v) {
    float e, r;
    asm("ex2.approx.f32 %0, %1;" : "=f"(e) : "f"(v));
    asm("rcp.approx.f32 %0, %1;" : "=f"(r) : "f"(1.0f + e));
    return r;
}
constexpr float LOG2E = 1.4426950408889634f;

// Runs f(std::integral_constant<int, ACT>) for the activation `act`: the choice is made once for many elements.
template <typename F>
__device__ __forceinline__ void with_activation(int act, F&& f) {
    switch (act) {
        case SC_ACT_RELU: f(std::integral_constant<int, SC_ACT_RELU>()); break;
        case SC_ACT_GELU: f(std::integral_constant<int, SC_ACT_GELU>()); break;
        case SC_ACT_GELU_TANH: f(std::integral_constant<int, SC_ACT_GELU_TANH>()); break;
        case SC_ACT_SILU: f(std::integral_constant<int, SC_ACT_SILU>()); break;
        default: f(std::integral_constant<int, SC_ACT_NONE>()); break;
    }
}

// (1 + tanh(u)) / 2 is the logistic function of 2 u, so the tanh form of gelu is z logistic(2 u).
template <int ACT>
__device__ __forceinline__ float activation(float z) {
    if constexpr (ACT == SC_ACT_RELU) return z < 0.0f ? 0.0f : z;                  // NaN passes
    else if constexpr (ACT == SC_ACT_GELU) return 0.5f * z * (1.0f + erff(z * SQRT_HALF));
    else if constexpr (ACT == SC_ACT_GELU_TANH) return z * inv_1p_exp2(z * fmaf(-LOG2E * GELU_C * GELU_A, z * z, -LOG2E * GELU_C));
    else if constexpr (ACT == SC_ACT_SILU) return z * inv_1p_exp2(-LOG2E * z);
    else return z;
}

// Products with a logistic that has reached 0 or 1 take a bounded z: the limit is 0, never 0 * inf.
template <int ACT>
__device__ __forceinline__ float activation_slope(float z) {
    if constexpr (ACT == SC_ACT_RELU) return z > 0.0f ? 1.0f : (z <= 0.0f ? 0.0f : z);
    else if constexpr (ACT == SC_ACT_GELU) {
        float e;
        asm("ex2.approx.f32 %0, %1;" : "=f"(e) : "f"(-0.5f * LOG2E * z * z));
        return fmaf(z * INV_SQRT_2PI, e, 0.5f * (1.0f + erff(z * SQRT_HALF)));
    } else if constexpr (ACT == SC_ACT_GELU_TANH) {
        z = z > 64.0f ? 64.0f : (z < -64.0f ? -64.0f : z);                         // NaN passes
        const float zz = z * z, s = inv_1p_exp2(z * fmaf(-LOG2E * GELU_C * GELU_A, zz, -LOG2E * GELU_C));
        return fmaf(s * z, (1.0f - s) * fmaf(3.0f * GELU_C * GELU_A, zz, GELU_C), s);
    } else if constexpr (ACT == SC_ACT_SILU) {
        const float s = inv_1p_exp2(-LOG2E * z), b = z > 128.0f ? 128.0f : z;
        return fmaf(s * b, 1.0f - s, s);
    } else return 1.0f;
}

// ---------------------------------------------------------------------------
// the checkpoint's numbers
// ---------------------------------------------------------------------------
// Least e with m <= 127 2^e, clamped to the type's range; m >= 0 finite, by its bits: m = f 2^x with 1 <= f < 2 needs
// e = x - 6 while f <= 127 / 64 (mantissa <= 0x7E0000) and x - 5 beyond, which the carry of an addition decides.
template <typename T>
__device__ __forceinline__ int ckpt_exponent(uint32_t m_bits) {
    const int e = (int)((m_bits + 0x1FFFFu) >> 23) - 127 - 6;
    return min(max(e, Elem<T>::EMIN), Elem<T>::EMAX);
}

__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // -126 <= e <= 127

// Byte of rint(v 2^-e): adding 1.5 2^23 rounds to the integer in the low mantissa bits (the product is exact).
// |v| 2^-e <= 127 except where e has reached the type's largest, whose caller clamps.
__device__ __forceinline__ uint32_t ckpt_byte(float v, float inv) { return __float_as_uint(fmaf(v, inv, 12582912.0f)) & 0xFFu; }

// Bytes b[0..7] side by side.
__device__ __forceinline__ uint2 ckpt_join8(const uint32_t b[8]) {
    return make_uint2(__byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410),
                      __byte_perm(__byte_perm(b[4], b[5], 0x0040), __byte_perm(b[6], b[7], 0x0040), 0x5410));
}

// The same for any v: not finite -> -128, which stands for NaN; |q| <= most.
__device__ __forceinline__ uint32_t ckpt_byte_any(float v, float inv, float most) {
    if ((__float_as_uint(v) & 0x7FFFFFFFu) >= 0x7F800000u) return 0x80u;
    return ckpt_byte(fminf(fmaxf(rintf(v * inv), -most), most), 1.0f);
}

// Four stored bytes to their values: byte u = q + 128 as the low mantissa byte of 2^23; the difference and the product
// are exact (one multiply-add would overflow for the largest scales).
__device__ __forceinline__ void ckpt_values4(uint32_t q4, float scale, float v[4]) {
    const uint32_t u = q4 ^ 0x80808080u;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (__uint_as_float(__byte_perm(u, 0x4B000000u, 0x7440 + i)) - 8388736.0f) * scale;
    if (__vcmpeq4(u, 0u)) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (((u >> (8 * i)) & 0xFFu) == 0u) v[i] = __uint_as_float(0x7FFFFFFFu);
    }
}

// Eight elements of a group that four neighbouring lanes hold, `m` the largest magnitude of them all by its bits (values that
// are not finite order above the others): their bytes and the group's exponent.  The four lanes call it together.
template <typename T>
__device__ __forceinline__ int ckpt_encode8(const float f[8], uint32_t m, uint32_t b[8]) {
    int e = ckpt_exponent<T>(m);
    if (m < 0x7F800000u && e != Elem<T>::EMAX) {
        const float inv = pow2(-e);
#pragma unroll
        for (int i = 0; i < 8; ++i) b[i] = ckpt_byte(f[i], inv);
    } else {
        const uint32_t mask = 0xFu << (threadIdx.x & 28u);
        m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t a = __float_as_uint(f[i]) & 0x7FFFFFFFu;
            if (a < 0x7F800000u) m = max(m, a);
        }
        m = max(m, __shfl_xor_sync(mask, m, 1));
        m = max(m, __shfl_xor_sync(mask, m, 2));
        e = ckpt_exponent<T>(m);
        const float inv = pow2(-e), most = e == Elem<T>::EMAX ? 63.0f : 127.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) b[i] = ckpt_byte_any(f[i], inv, most);
    }
    return e;
}

__device__ __forceinline__ float ckpt_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

}  // namespace sc
