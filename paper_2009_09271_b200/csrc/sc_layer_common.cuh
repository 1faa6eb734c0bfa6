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

// Layer kernels are launched so that they may begin while their predecessor on the stream ends: what precedes
// wait_for_predecessor() touches nothing in HBM, and release_successor() lets the next such kernel begin likewise.  Every
// kernel that is launched that way waits, so a kernel's end implies the end of all before it.
__device__ __forceinline__ void wait_for_predecessor() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void release_successor() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
// What a predecessor may have written is therefore not read-only for the kernel's whole life: no pointer of these kernels is declared
// __restrict__, which would allow loads ahead of the wait and through the path for constant data, and loads with a cache hint are
// the ones below, whose volatile statements keep their place behind the wait and behind fences.
__device__ __forceinline__ uint4 load_stream16(const void* p) {
    uint4 r;
    asm volatile("ld.global.cs.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p));
    return r;
}
__device__ __forceinline__ uint2 load_stream8(const void* p) {
    uint2 r;
    asm volatile("ld.global.cs.v2.b32 {%0, %1}, [%2];" : "=r"(r.x), "=r"(r.y) : "l"(p));
    return r;
}
// From L2, where other CTAs of the same kernel, or the one before it, have left their sums.
__device__ __forceinline__ float load_l2(const float* p) {
    float r;
    asm volatile("ld.global.cg.f32 %0, [%1];" : "=f"(r) : "l"(p) : "memory");
    return r;
}
__device__ __forceinline__ float4 load_l2(const float4* p) {
    float4 r;
    asm volatile("ld.global.cg.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(r.x), "=f"(r.y), "=f"(r.z), "=f"(r.w) : "l"(p));
    return r;
}

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
constexpr float INV_SQRT_2PI = 0.39894228040143268f;
constexpr float GELU_C = 1.5957691216057308f, GELU_A = 0.044715f;      // 2 sqrt(2 / pi), cubic coefficient

// Two fp32 numbers in one register pair, and the instructions that work on both at once.
struct Pair { unsigned long long v; };
__device__ __forceinline__ Pair pair(float lo, float hi) {
    Pair r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ Pair pair(float v) { return pair(v, v); }
__device__ __forceinline__ float2 both(Pair a) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(a.v));
    return r;
}
__device__ __forceinline__ Pair operator*(Pair a, Pair b) {
    Pair r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ Pair operator+(Pair a, Pair b) {
    Pair r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
    Pair r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}
// The exponential and the reciprocal flush what is below 2^-126 to zero: that far out the activations are 0 or z.
__device__ __forceinline__ float exp2_approx(float v) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float rcp_approx(float v) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ Pair exp2_approx(Pair a) { const float2 f = both(a); return pair(exp2_approx(f.x), exp2_approx(f.y)); }
__device__ __forceinline__ Pair rcp_approx(Pair a) { const float2 f = both(a); return pair(rcp_approx(f.x), rcp_approx(f.y)); }

constexpr float LOG2E = 1.4426950408889634f;
// 1 / (1 + 2^v)
__device__ __forceinline__ Pair inv_1p_exp2(Pair v) { return rcp_approx(exp2_approx(v) + pair(1.0f)); }

// Phi(-|z|), the normal distribution's tail, with e = exp(-z^2 / 2) given: e t P(t), t = 1 / (1 + 0.3 |z|).  That form of an
// approximation to erfc is Hastings'; P is a least-squares fit, reweighted towards equal errors, to Phi(-z) / (e t) on
// [0, 14] (1.5e-7 of the value).  The exponential is shared with the density, which the slope needs as well.
__device__ __forceinline__ Pair normal_tail(Pair z, Pair e) {
    const float2 f = both(z);
    const Pair t = rcp_approx(fma2(pair(fabsf(f.x), fabsf(f.y)), pair(0.3f), pair(1.0f)));
    Pair p = fma2(t, pair(0.0356747428f), pair(-0.1572029058f));
    p = fma2(t, p, pair(0.2063531245f));
    p = fma2(t, p, pair(-0.05368322389f));
    p = fma2(t, p, pair(0.1285613688f));
    p = fma2(t, p, pair(0.09991358065f));
    p = fma2(t, p, pair(0.1207539403f));
    p = fma2(t, p, pair(0.1196293f));
    return e * (t * p);
}
__device__ __forceinline__ Pair exp_half_square(Pair z) { return exp2_approx(z * z * pair(-0.5f * LOG2E)); }

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
__device__ __forceinline__ Pair activation(Pair z) {
    if constexpr (ACT == SC_ACT_RELU) {
        const float2 f = both(z);
        return pair(f.x < 0.0f ? 0.0f : f.x, f.y < 0.0f ? 0.0f : f.y);              // NaN passes
    } else if constexpr (ACT == SC_ACT_GELU) {                                       // max(z, 0) - |z| Phi(-|z|)
        const float2 f = both(z);
        const Pair h = normal_tail(z, exp_half_square(z));                          // NaN passes through here
        return fma2(pair(-fminf(fabsf(f.x), 64.0f), -fminf(fabsf(f.y), 64.0f)), h, pair(fmaxf(f.x, 0.0f), fmaxf(f.y, 0.0f)));
    } else if constexpr (ACT == SC_ACT_GELU_TANH)
        return z * inv_1p_exp2(z * fma2(z * z, pair(-LOG2E * GELU_C * GELU_A), pair(-LOG2E * GELU_C)));
    else if constexpr (ACT == SC_ACT_SILU) return z * inv_1p_exp2(z * pair(-LOG2E));
    else return z;
}

// z is a checkpoint's value, read through slope_scale(): |z| < 2^48, so that no product below overflows.  NaN passes.  gelu takes
// Phi(z) for z < 0 as the tail itself: through 1/2 - tail it would be off by 3e-8, at z = -5.5 three per cent of the slope.
template <int ACT>
__device__ __forceinline__ Pair activation_slope(Pair z) {
    if constexpr (ACT == SC_ACT_RELU) {                                              // 0 z keeps NaN
        const float2 f = both(z), n = both(z * pair(0.0f));
        return pair(f.x > 0.0f ? 1.0f : n.x, f.y > 0.0f ? 1.0f : n.y);
    } else if constexpr (ACT == SC_ACT_GELU) {                                       // Phi(z) + z phi(z)
        const Pair e = exp_half_square(z), tail = normal_tail(z, e);
        const float2 f = both(z), below = both(tail), above = both(fma2(tail, pair(-1.0f), pair(1.0f)));
        return fma2(z * pair(INV_SQRT_2PI), e, pair(f.x < 0.0f ? below.x : above.x, f.y < 0.0f ? below.y : above.y));
    } else if constexpr (ACT == SC_ACT_GELU_TANH) {
        const Pair zz = z * z, s = inv_1p_exp2(z * fma2(zz, pair(-LOG2E * GELU_C * GELU_A), pair(-LOG2E * GELU_C)));
        return fma2(s * z, fma2(s, pair(-1.0f), pair(1.0f)) * fma2(zz, pair(3.0f * GELU_C * GELU_A), pair(GELU_C)), s);
    } else if constexpr (ACT == SC_ACT_SILU) {
        const Pair s = inv_1p_exp2(z * pair(-LOG2E));
        return fma2(s * z, fma2(s, pair(-1.0f), pair(1.0f)), s);
    } else return pair(1.0f);
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

// The bytes of 8 elements side by side.
__device__ __forceinline__ uint2 ckpt_join8(const uint32_t b[8]) {
    return make_uint2(__byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410),
                      __byte_perm(__byte_perm(b[4], b[5], 0x0040), __byte_perm(b[6], b[7], 0x0040), 0x5410));
}
__device__ __forceinline__ uint2 ckpt_bytes8(const float f[8], int e) {
    const float inv = pow2(-e);
    uint32_t b[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) b[i] = ckpt_byte(f[i], inv);
    return ckpt_join8(b);
}
template <typename T>
__device__ __forceinline__ uint2 ckpt_bytes8_any(const float f[8], int e) {
    const float inv = pow2(-e), most = e == Elem<T>::EMAX ? 63.0f : 127.0f;
    uint32_t b[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) b[i] = ckpt_byte_any(f[i], inv, most);
    return ckpt_join8(b);
}
// Bits of the largest finite magnitude.
__device__ __forceinline__ uint32_t finite_max8(const float f[8]) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t a = __float_as_uint(f[i]) & 0x7FFFFFFFu;
        if (a < 0x7F800000u) m = max(m, a);
    }
    return m;
}

// Stored bytes to their values: byte u = q + 128 as the low mantissa byte of 2^23, then one exact multiply-add.  Scales above
// 2^100, where its constant would overflow, take the difference first.
struct Scale { float s, off; };
__device__ __forceinline__ Scale ckpt_scale(uint32_t byte) {
    Scale k;
    k.s = __uint_as_float(byte << 23);
    k.off = -8388736.0f * k.s;
    return k;
}
// For the activations' slopes: every one of them has reached its limit long before 2^40, so a larger scale reads as 2^40.
__device__ __forceinline__ Scale slope_scale(uint32_t byte) { return ckpt_scale(min(byte, 127u + 40u)); }

template <bool LARGE>
__device__ __forceinline__ void ckpt_values8(uint2 q8, Scale k, Pair v[4]) {
    const uint32_t u[2] = {q8.x ^ 0x80808080u, q8.y ^ 0x80808080u};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const Pair f = pair(__uint_as_float(__byte_perm(u[i >> 1], 0x4B000000u, 0x7440 + 2 * (i & 1))),
                            __uint_as_float(__byte_perm(u[i >> 1], 0x4B000000u, 0x7441 + 2 * (i & 1))));
        v[i] = LARGE ? (f + pair(-8388736.0f)) * pair(k.s) : fma2(f, pair(k.s), pair(k.off));
    }
    // some byte of u is zero: q = -128, not finite
    if ((((u[0] - 0x01010101u) & ~u[0]) | ((u[1] - 0x01010101u) & ~u[1])) & 0x80808080u) {
        const float nan = __uint_as_float(0x7FFFFFFFu);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t two = u[i >> 1] >> (16 * (i & 1));
            const float2 f = both(v[i]);
            v[i] = pair((two & 0xFFu) ? f.x : nan, (two & 0xFF00u) ? f.y : nan);
        }
    }
}
constexpr uint32_t LARGE_SCALE = 127 + 100;

// Eight elements of a group that four neighbouring lanes hold, `m` the largest magnitude of them all by its bits (values that
// are not finite order above the others): their bytes, and the group's exponent.  The four lanes call it together.
template <typename T>
__device__ __forceinline__ uint2 ckpt_encode8(const float f[8], uint32_t m, int& e) {
    e = ckpt_exponent<T>(m);
    if (m < 0x7F800000u && e != Elem<T>::EMAX) return ckpt_bytes8(f, e);
    const uint32_t mask = 0xFu << (threadIdx.x & 28u);
    m = finite_max8(f);
    m = max(m, __shfl_xor_sync(mask, m, 1));
    m = max(m, __shfl_xor_sync(mask, m, 2));
    e = ckpt_exponent<T>(m);
    return ckpt_bytes8_any<T>(f, e);
}

}  // namespace sc
