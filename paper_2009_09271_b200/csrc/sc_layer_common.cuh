// Definitions shared by the layer operators: 16-bit types, activations and their slopes, the 8-bit checkpoint's rounding.
#pragma once
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

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

__device__ __forceinline__ float logistic(float v) { return __fdividef(1.0f, 1.0f + __expf(-v)); }

// (1 + tanh(u)) / 2 is the logistic function of 2 u, so the tanh form of gelu is z logistic(2 u).
__device__ __forceinline__ float activation(int act, float z) {
    switch (act) {
        case SC_ACT_RELU: return z < 0.0f ? 0.0f : z;                  // NaN passes
        case SC_ACT_GELU: return 0.5f * z * (1.0f + erff(z * SQRT_HALF));
        case SC_ACT_GELU_TANH: return z * logistic(GELU_C * (z + GELU_A * z * z * z));
        case SC_ACT_SILU: return z * logistic(z);
        default: return z;
    }
}

// Products with a logistic that has reached 0 or 1 take a bounded z: the limit is 0, never 0 * inf.
__device__ __forceinline__ float activation_slope(int act, float z) {
    switch (act) {
        case SC_ACT_RELU: return z > 0.0f ? 1.0f : (z <= 0.0f ? 0.0f : z);
        case SC_ACT_GELU: return 0.5f * (1.0f + erff(z * SQRT_HALF)) + z * __expf(-0.5f * z * z) * INV_SQRT_2PI;
        case SC_ACT_GELU_TANH: {
            z = z > 64.0f ? 64.0f : (z < -64.0f ? -64.0f : z);         // NaN passes
            const float s = logistic(GELU_C * (z + GELU_A * z * z * z));
            return s + z * s * (1.0f - s) * (GELU_C + 3.0f * GELU_C * GELU_A * z * z);
        }
        case SC_ACT_SILU: {
            const float s = logistic(z), b = z > 128.0f ? 128.0f : z;
            return s + b * s * (1.0f - s);
        }
        default: return 1.0f;
    }
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

__device__ __forceinline__ float ckpt_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

}  // namespace sc
