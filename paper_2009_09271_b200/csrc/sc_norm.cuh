// Rows in 8 bits with one scale each, and the root-mean-square norm with the residual's addition, forward and backward.
//
//   8-bit rows   m = max |v|, s = m / 127, q = rint(v i), i = 127 (1 / m), every product and quotient rounded to fp32
//   forward      h = residual + dropout(x),  r = (mean(h^2) + eps)^(-1/2),  y = h r gamma, in 16 bits or as 8-bit rows
//   backward     g = gamma dy,  u = h r,  dh = residual + r (g - u mean(g u)),  dx = dropout(dh),  dgamma = column sums of dy u
// A row's sums and its largest magnitude are fp32; y is made from the fp32 h, before that is rounded to its type.
#pragma once
#include "sc_checkpoint.cuh"
#include "sc_dropout.cuh"

namespace sc {

constexpr int NORM_THREADS = 256;

// ---------------------------------------------------------------------------
// 8-bit rows
// ---------------------------------------------------------------------------
struct RowScale { float scale, inv; };        // inv = 0: every byte is 0
// From the bits of the largest magnitude, where infinities and NaN order above every number: such a row's scale is NaN, so that
// whatever reads it is NaN.  Below 2^-100 the reciprocal would leave fp32's range soon: such a row counts as zero.  At the
// range's other end 127 scales must stay a number, whichever way the quotient was rounded.
constexpr float LARGEST_SCALE = 2.6793883890187504e+36f;
__device__ __forceinline__ RowScale row_scale(uint32_t m_bits) {
    const float m = __uint_as_float(m_bits);
    if (m_bits >= 0x7F800000u) return {__uint_as_float(0x7FFFFFFFu), 0.0f};
    if (m < 7.8886090522101181e-31f) return {0.0f, 0.0f};
    return {fminf(m / 127.0f, LARGEST_SCALE), 127.0f * (1.0f / m)};
}
// The bytes of 8 values: the product is rounded before the integer is taken, so that any IEEE fp32 arithmetic gives the same ones.
__device__ __forceinline__ uint2 row_bytes8(const float v[8], float inv) {
    if (inv == 0.0f) return make_uint2(0u, 0u);
    uint32_t b[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) b[i] = __float_as_uint(__fadd_rn(__fmul_rn(v[i], inv), 12582912.0f)) & 0xFFu;
    return ckpt_join8(b);
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    return v;
}
// Sum of `v` over the CTA's threads and the largest `m`, in every thread; `slots` are free again after the next call's barrier.
__device__ __forceinline__ void block_reduce(float& v, uint32_t& m, float (*slots)[2]) {
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u, warps = blockDim.x >> 5;
    v = warp_sum(v);
    m = __reduce_max_sync(0xFFFFFFFFu, m);
    __syncthreads();
    if (lane == 0) { slots[warp][0] = v; slots[warp][1] = __uint_as_float(m); }
    __syncthreads();
    v = 0.0f;
    m = 0u;
    for (uint32_t w = 0; w < warps; ++w) { v += slots[w][0]; m = max(m, __float_as_uint(slots[w][1])); }
}
__device__ __forceinline__ void block_reduce(float& v, float& u, float (*slots)[2]) {
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u, warps = blockDim.x >> 5;
    v = warp_sum(v);
    u = warp_sum(u);
    __syncthreads();
    if (lane == 0) { slots[warp][0] = v; slots[warp][1] = u; }
    __syncthreads();
    v = u = 0.0f;
    for (uint32_t w = 0; w < warps; ++w) { v += slots[w][0]; u += slots[w][1]; }
}

struct QuantizeArgs {
    uint64_t rows, ldx, ldq;
    uint32_t cols, grain_x, grain_q;
};

// A CTA a row, read twice: once for its largest magnitude, once for its bytes.
template <typename T>
__global__ void __launch_bounds__(NORM_THREADS) quantize_kernel(const T* x, QuantizeArgs a, uint8_t* q, float* scales) {
    __shared__ float slots[NORM_THREADS / 32][2];
    wait_for_predecessor();
    release_successor();
    for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T* from = x + row * a.ldx;
        uint32_t m = 0u;
        float none = 0.0f;
        for (uint32_t c0 = threadIdx.x * 8; c0 < a.cols; c0 += NORM_THREADS * 8) m = max(m, abs_max8(load8(from, c0, a.cols, a.grain_x)));
        block_reduce(none, m, slots);
        const RowScale s = row_scale(m);
        for (uint32_t c0 = threadIdx.x * 8; c0 < a.cols; c0 += NORM_THREADS * 8) {
            float f[8];
            to_floats(load8(from, c0, a.cols, a.grain_x), f);
            store_q8(q + row * a.ldq + c0, c0, a.cols, a.grain_q, row_bytes8(f, s.inv));
        }
        if (threadIdx.x == 0) scales[row] = s.scale;
    }
}

// The values of 8-bit rows, eight elements a thread and item.
template <typename T>
__global__ void __launch_bounds__(CKPT_THREADS) dequantize_kernel(const uint8_t* q, uint64_t ldq, const float* scales, ItemWalk w, T* out, uint64_t ldo) {
    wait_for_predecessor();
    release_successor();
    const uint64_t first = (uint64_t)blockIdx.x * CKPT_THREADS + threadIdx.x, stride = (uint64_t)gridDim.x * CKPT_THREADS;
    ItemAt at(w, first);
    for (uint64_t i = first; i < w.total; i += stride, at.next(w)) {
        const uint32_t c0 = at.item * 8;
        const uint2 b = load_q8(q + at.row * ldq, c0, w.cols, w.grain_q);
        const float s = scales[at.row];
        float f[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] = (float)(int8_t)((k < 4 ? b.x : b.y) >> (8 * (k & 3))) * s;
        store8(out + at.row * ldo, c0, w.cols, w.grain_x, f);
    }
}

// ---------------------------------------------------------------------------
// the norm
// ---------------------------------------------------------------------------
struct NormArgs {
    uint64_t rows, ldx, ldr, ldh, ldy, ldq;
    uint32_t cols, grain_x, grain_r, grain_g, grain_h, grain_y, grain_q;
    float eps, mean;           // mean: 1 / cols
    Drop drop;
};

// (mean of squares + eps)^(-1/2).  Squares that leave fp32's range make it NaN rather than 0: the row is lost and says so.
__device__ __forceinline__ float rms_inverse(float sum, float mean, float eps) {
    return sum <= 3.402823466e38f ? 1.0f / sqrtf(fmaf(sum, mean, eps)) : __uint_as_float(0x7FFFFFFFu);
}

// h of 8 columns in fp32; zero past the end.
template <typename T>
__device__ __forceinline__ void norm_input8(const T* x, const T* residual, const NormArgs& a, uint64_t row, uint32_t c0, float f[8]) {
    to_floats(load8(x + row * a.ldx, c0, a.cols, a.grain_x), f);
    if (a.drop.cut) drop8(a.drop, row, c0, f);
    if (residual) {
        float r[8];
        to_floats(load8(residual + row * a.ldr, c0, a.cols, a.grain_r), r);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] += r[i];
    }
}

// A CTA a row, its inputs read twice.  max |h gamma| times r is max |y|, so one pass gives both statistics.
template <typename T>
__global__ void __launch_bounds__(NORM_THREADS) rms_norm_kernel(const T* x, const T* residual, const T* gamma, NormArgs a, T* h, T* y, uint8_t* q,
                                                                float* scales) {
    __shared__ float slots[NORM_THREADS / 32][2];
    wait_for_predecessor();
    release_successor();
    for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        float sum = 0.0f;
        uint32_t m = 0u;
        for (uint32_t c0 = threadIdx.x * 8; c0 < a.cols; c0 += NORM_THREADS * 8) {
            float f[8], g[8];
            norm_input8(x, residual, a, row, c0, f);
            to_floats(load8(gamma, c0, a.cols, a.grain_g), g);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                sum = fmaf(f[i], f[i], sum);
                m = max(m, __float_as_uint(f[i] * g[i]) & 0x7FFFFFFFu);
            }
        }
        block_reduce(sum, m, slots);
        const float r = rms_inverse(sum, a.mean, a.eps);
        const RowScale s = row_scale(__float_as_uint(__uint_as_float(m) * r) & 0x7FFFFFFFu);
        for (uint32_t c0 = threadIdx.x * 8; c0 < a.cols; c0 += NORM_THREADS * 8) {
            float f[8], g[8];
            norm_input8(x, residual, a, row, c0, f);
            to_floats(load8(gamma, c0, a.cols, a.grain_g), g);
            if (h) store8(h + row * a.ldh, c0, a.cols, a.grain_h, f);
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = f[i] * r * g[i];
            if (y) store8(y + row * a.ldy, c0, a.cols, a.grain_y, f);
            if (q) store_q8(q + row * a.ldq + c0, c0, a.cols, a.grain_q, row_bytes8(f, s.inv));
        }
        if (q && threadIdx.x == 0) scales[row] = s.scale;
    }
}

struct NormGradArgs {
    uint64_t rows, lddy, ldh, ldr, lddh, lddx;
    uint32_t cols, grain_y, grain_h, grain_g, grain_r, grain_dh, grain_dx;
    uint32_t runs, run_rows, accumulate;
    float eps, mean;
    Drop drop;
};

// Each row's r and mean(g u).
template <typename T>
__global__ void __launch_bounds__(NORM_THREADS) norm_stats_kernel(const T* dy, const T* h, const T* gamma, NormGradArgs a, float2* stats) {
    __shared__ float slots[NORM_THREADS / 32][2];
    wait_for_predecessor();
    release_successor();
    for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        float sum = 0.0f, dot = 0.0f;
        for (uint32_t c0 = threadIdx.x * 8; c0 < a.cols; c0 += NORM_THREADS * 8) {
            float d[8], f[8], g[8];
            to_floats(load8(dy + row * a.lddy, c0, a.cols, a.grain_y), d);
            to_floats(load8(h + row * a.ldh, c0, a.cols, a.grain_h), f);
            to_floats(load8(gamma, c0, a.cols, a.grain_g), g);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                sum = fmaf(f[i], f[i], sum);
                dot = fmaf(d[i] * g[i], f[i], dot);
            }
        }
        block_reduce(sum, dot, slots);
        const float r = rms_inverse(sum, a.mean, a.eps);
        if (threadIdx.x == 0) stats[row] = make_float2(r, dot * r * a.mean);
    }
}

// The rest, element by element: a CTA owns a strip of 256 columns and a run of rows, as the activation's gradient does, and leaves the
// column sums the same way: over its row lanes in shared memory, over the runs by the strip's last CTA, in order.
template <typename T>
__global__ void __launch_bounds__(CKPT_THREADS) norm_strips_kernel(const T* dy, const T* h, const T* gamma, const T* residual, NormGradArgs a,
                                                                   const float2* stats, T* dh, T* dx, float* partial, uint32_t* tickets, float* dgamma) {
    wait_for_predecessor();
    release_successor();
    const uint32_t tx = threadIdx.x & 31u, ty = threadIdx.x >> 5;
    const uint32_t c0 = blockIdx.x * GRAD_COLS + tx * 8;
    const uint64_t first = (uint64_t)blockIdx.y * a.run_rows, end = min(first + a.run_rows, a.rows);
    float sum[8] = {}, g[8] = {};
    if (c0 < a.cols) {
        to_floats(load8(gamma, c0, a.cols, a.grain_g), g);
        for (uint64_t row = first + ty; row < end; row += GRAD_LANES) {
            float d[8], f[8], e[8] = {};
            to_floats(load8(dy + row * a.lddy, c0, a.cols, a.grain_y), d);
            to_floats(load8(h + row * a.ldh, c0, a.cols, a.grain_h), f);
            if (residual) to_floats(load8(residual + row * a.ldr, c0, a.cols, a.grain_r), e);
            const float2 s = stats[row];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float u = f[i] * s.x;
                sum[i] = fmaf(d[i], u, sum[i]);
                e[i] = fmaf(s.x, fmaf(-u, s.y, d[i] * g[i]), e[i]);
            }
            if (dh) store8(dh + row * a.lddh, c0, a.cols, a.grain_dh, e);
            if (dx) {
                if (a.drop.cut) drop8(a.drop, row, c0, e);
                store8(dx + row * a.lddx, c0, a.cols, a.grain_dx, e);
            }
        }
    }
    if (!dgamma) return;
    __shared__ float join[GRAD_LANES][GRAD_COLS];
    __shared__ uint32_t last;
#pragma unroll
    for (int i = 0; i < 8; ++i) join[ty][tx * 8 + i] = sum[i];
    __syncthreads();
    const uint32_t c = blockIdx.x * GRAD_COLS + threadIdx.x;
    float total = 0.0f;
#pragma unroll
    for (int j = 0; j < GRAD_LANES; ++j) total += join[j][threadIdx.x];
    if (a.runs > 1) {
        if (c < a.cols) partial[(uint64_t)blockIdx.y * a.cols + c] = total;
        __threadfence();
        __syncthreads();
        if (threadIdx.x == 0) last = atomicAdd(&tickets[blockIdx.x], 1u);
        __syncthreads();
        if (last != a.runs - 1) return;
        __threadfence();
        total = 0.0f;
        if (c < a.cols)
            for (uint32_t j = 0; j < a.runs; ++j) total += load_l2(&partial[(uint64_t)j * a.cols + c]);
        if (threadIdx.x == 0) tickets[blockIdx.x] = 0u;               // zero again for the next call
    }
    if (c < a.cols) dgamma[c] = a.accumulate ? dgamma[c] + total : total;
}

}  // namespace sc
