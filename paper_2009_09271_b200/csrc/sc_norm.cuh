// Rows in 8 bits with one scale each, and the root-mean-square norm with the residual's addition, forward and backward.
//
//   8-bit rows   m = max |v|, s = m / 127, q = rint(v i), i = 127 (1 / m), every product and quotient rounded to fp32
//   forward      h = residual + dropout(x),  r = (mean(h^2) + eps)^(-1/2),  y = (h gamma) r, in 16 bits or as 8-bit rows
//   backward     g = gamma dy,  u = h r,  dh = residual + r (g - u mean(g u)),  dx = dropout(dh),  dgamma = column sums of dy u
// A row's sums and its largest magnitude are fp32; y is made from the fp32 h, before that is rounded to its type, and the 8-bit rows are
// those of the fp32 y.
#pragma once
#include "sc_checkpoint.cuh"
#include "sc_dropout.cuh"
#include "sc_tcgen05.cuh"

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

// The largest of three magnitudes; NaN if one of them is.
__device__ __forceinline__ float abs_max(float a, float b, float c) {
    float r;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
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

// The same over a team, the threads that share a row: a warp, or a whole CTA that makes one reduction.
template <int TEAM>
__device__ __forceinline__ void team_reduce(float& v, uint32_t& m, float2* slots) {
    v = warp_sum(v);
    m = __reduce_max_sync(0xFFFFFFFFu, m);
    if constexpr (TEAM > 32) {
        if ((threadIdx.x & 31u) == 0) slots[threadIdx.x >> 5] = make_float2(v, __uint_as_float(m));
        __syncthreads();
        v = 0.0f;
        m = 0u;
#pragma unroll
        for (int w = 0; w < TEAM / 32; ++w) { v += slots[w].x; m = max(m, __float_as_uint(slots[w].y)); }
    }
}

__device__ __forceinline__ uint2 row_bytes8(const Pair v[4], float inv) {
    if (inv == 0.0f) return make_uint2(0u, 0u);
    uint32_t b[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = both(v[i] * pair(inv));          // a paired addition here would be joined with it, without the rounding between
        b[2 * i] = __float_as_uint(__fadd_rn(f.x, 12582912.0f));             // its low byte
        b[2 * i + 1] = __float_as_uint(__fadd_rn(f.y, 12582912.0f));
    }
    return ckpt_join8(b);
}
__device__ __forceinline__ uint8_t row_byte(float v, float inv) { return inv == 0.0f ? 0 : (uint8_t)__float_as_uint(__fadd_rn(__fmul_rn(v, inv), 12582912.0f)); }
struct QuantizeArgs {
    uint64_t rows;
    InRows x;
    OutRows q;
    uint32_t cols, grain_x, grain_q;
    Phase phase;
};

// A CTA a row, read twice: once for its largest magnitude, once for its bytes.
template <typename T>
__global__ void __launch_bounds__(NORM_THREADS) quantize_kernel(QuantizeArgs a, float* scales) {
    __shared__ float slots[NORM_THREADS / 32][2];
    wait_for_predecessor();
    release_successor();
    for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T* from = static_cast<const T*>(a.x.p) + row * a.x.ld;
        uint8_t* to = static_cast<uint8_t*>(a.q.p) + row * a.q.ld;
        uint32_t m = 0u;
        float none = 0.0f;
        for (uint32_t c0 = threadIdx.x * 8; c0 < a.cols; c0 += NORM_THREADS * 8) m = max(m, abs_max8(load8(from, c0, a.cols, a.grain_x)));
        block_reduce(none, m, slots);
        const RowScale s = row_scale(m);
        for (uint32_t c0 = threadIdx.x * 8; c0 < a.cols; c0 += NORM_THREADS * 8) {
            float f[8];
            to_floats(load8(from, c0, a.cols, a.grain_x), f);
            store_q8(to + c0, c0, a.cols, a.grain_q, row_bytes8(f, s.inv));
        }
        if (threadIdx.x == 0) scales[row] = s.scale;
    }
}

// The same with the row in registers, V times eight elements a thread, read once.  Bound by HBM: 16384 x 4096 bf16 in 31 to 33 us (6.1 to
// 6.5 TB/s, 0.93 to 0.99 of the measured copy rate), 65536 x 1024 31 us; read twice by a CTA a row it took 44.
template <typename T, int TEAM, int V, bool WIDE>
__global__ void __launch_bounds__(TEAM == 32 ? 256 : TEAM) quantize_rows_kernel(QuantizeArgs a, float* scales) {
    constexpr int TEAMS = TEAM == 32 ? 8 : 1;
    __shared__ float2 slots[TEAM / 32];
    wait_for_predecessor();
    release_successor();
    const uint32_t t = TEAM == 32 ? threadIdx.x & 31u : threadIdx.x;
    const uint64_t row = (uint64_t)blockIdx.x * TEAMS + (TEAM == 32 ? threadIdx.x >> 5 : 0u);
    if (row >= a.rows) return;
    const RowCut cut = row_cut<WIDE>(a.phase, row, a.cols);
    const T* from = row_of<T>(a.x, row);
    uint8_t* to = row_of<uint8_t>(a.q, row);
    const int ec = !WIDE && last_warp<TEAM>(t) ? end_col(cut, a.cols, t & 31u) : -1;        // the ends are the last warp's
    Raw8<T> raw[V];
#pragma unroll
    for (int j = 0; j < V; ++j) raw[j] = j * TEAM + t < cut.whole ? chunk_load8<T, WIDE>(a.x, from, cut.lead + (int)(j * TEAM + t) * 8) : Raw8<T>{};
    const float end = ec >= 0 ? element(from[ec]) : 0.0f;
    uint32_t m = WIDE ? 0u : __float_as_uint(end) & 0x7FFFFFFFu;
    float none = 0.0f;
#pragma unroll
    for (int j = 0; j < V; ++j) m = max(m, abs_max8(raw[j]));
    team_reduce<TEAM>(none, m, slots);
    const RowScale s = row_scale(m);
#pragma unroll
    for (int j = 0; j < V; ++j)
        if (j * TEAM + t < cut.whole) {
            Pair v[4];
            to_pairs(raw[j], v);
            chunk_store_bytes8<WIDE>(a.q, to, cut.lead + (int)(j * TEAM + t) * 8, row_bytes8(v, s.inv));
        }
    if (ec >= 0) to[ec] = row_byte(end, s.inv);
    if (t == 0) scales[row] = s.scale;
}

// The values of 8-bit rows, sixteen elements a thread and item, several items in flight.  For rows a multiple of 16 long whose bytes
// take 16-byte accesses and whose values take 32-byte ones.  Bound by HBM: 16384 x 8192 to bf16 in 62 us (6.5 TB/s, 0.99 of the copy rate).
constexpr int DEQUANTIZE_UNROLL = 4;
template <typename T>
__global__ void __launch_bounds__(CKPT_THREADS) dequantize_kernel(const uint8_t* q, uint64_t ldq, const float* scales, ItemWalk w, T* out, uint64_t ldo) {
    wait_for_predecessor();
    release_successor();
    const uint64_t first = (uint64_t)blockIdx.x * CKPT_THREADS + threadIdx.x, stride = (uint64_t)gridDim.x * CKPT_THREADS;
    ItemAt at(w, first);
    for (uint64_t base = first; base < w.total; base += stride * DEQUANTIZE_UNROLL) {
        uint4 raw[DEQUANTIZE_UNROLL];
        float s[DEQUANTIZE_UNROLL];
        ItemAt from = at;
#pragma unroll
        for (int u = 0; u < DEQUANTIZE_UNROLL; ++u) {
            if (base + u * stride < w.total) {
                raw[u] = load_stream16(q + at.row * ldq + at.item * 16);
                s[u] = scales[at.row];
            }
            at.next(w);
        }
#pragma unroll
        for (int u = 0; u < DEQUANTIZE_UNROLL; ++u) {
            if (base + u * stride < w.total) {
                const uint32_t b[4] = {raw[u].x, raw[u].y, raw[u].z, raw[u].w};
                T* to = out + from.row * ldo + from.item * 16;
                uint4 o[sizeof(T)];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    // a byte's value plus 128 as the low mantissa byte of 2^23; the difference and the product are exact but for the last rounding
                    const uint32_t v = b[k] ^ 0x80808080u;
                    float f[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) f[i] = (__uint_as_float(__byte_perm(v, 0x4B000000u, 0x7440 + i)) - 8388736.0f) * s[u];
                    if constexpr (sizeof(T) == 4) {
                        o[k] = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
                    } else {
                        uint32_t* p = reinterpret_cast<uint32_t*>(o) + 2 * k;
                        p[0] = Elem<T>::pack(f[0], f[1]);
                        p[1] = Elem<T>::pack(f[2], f[3]);
                    }
                }
                store32(to, o[0], o[1]);
                if constexpr (sizeof(T) == 4) store32(to + 8, o[2], o[3]);
            }
            from.next(w);
        }
    }
}

// The same for other rows: a team of threads a row, or with blockIdx.y a part of one, V times eight elements a thread at a time.
struct DequantizeArgs {
    uint64_t rows;
    InRows q;
    OutRows out;
    const float* scales;
    uint32_t cols;
    Phase phase;
};
template <typename T, int TEAM, int V>
__global__ void __launch_bounds__(TEAM == 32 ? 256 : TEAM) dequantize_rows_kernel(DequantizeArgs a) {
    constexpr int TEAMS = TEAM == 32 ? 8 : 1;
    wait_for_predecessor();
    release_successor();
    const uint32_t t = TEAM == 32 ? threadIdx.x & 31u : threadIdx.x;
    const uint64_t row = (uint64_t)blockIdx.x * TEAMS + (TEAM == 32 ? threadIdx.x >> 5 : 0u);
    if (row >= a.rows) return;
    const RowCut cut = row_cut<false>(a.phase, row, a.cols);
    const uint8_t* q = row_of<uint8_t>(a.q, row);
    T* out = row_of<T>(a.out, row);
    const float s = a.scales[row];
    if (blockIdx.y == 0 && last_warp<TEAM>(t)) {                           // the ends
        const int c = end_col(cut, a.cols, t & 31u);
        if (c >= 0) out[c] = rounded<T>((float)(int8_t)q[c] * s);
    }
    for (uint32_t first = blockIdx.y * (TEAM * V) + t; first < cut.whole; first += gridDim.y * (TEAM * V)) {
        uint2 raw[V];
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (first + j * TEAM < cut.whole) raw[j] = chunk_load_bytes8(a.q, q, cut.lead + (int)(first + j * TEAM) * 8);
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (first + j * TEAM < cut.whole) {
                const int c = cut.lead + (int)(first + j * TEAM) * 8;
                float f[8];
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    f[i] = (__uint_as_float(__byte_perm((i < 4 ? raw[j].x : raw[j].y) ^ 0x80808080u, 0x4B000000u, 0x7440 + (i & 3))) - 8388736.0f) * s;
                if constexpr (sizeof(T) == 2) {
                    const Pair v[4] = {pair(f[0], f[1]), pair(f[2], f[3]), pair(f[4], f[5]), pair(f[6], f[7])};
                    chunk_store8<T, false>(a.out, out, c, v);
                } else {
                    *reinterpret_cast<float4*>(out + c) = make_float4(f[0], f[1], f[2], f[3]);
                    *reinterpret_cast<float4*>(out + c + 4) = make_float4(f[4], f[5], f[6], f[7]);
                }
            }
    }
}

// ---------------------------------------------------------------------------
// the norm
// ---------------------------------------------------------------------------
struct NormArgs {
    uint64_t rows;
    InRows x, residual, gamma;
    OutRows h, y, q;
    uint32_t cols, grain_x, grain_r, grain_g, grain_h, grain_y, grain_q;
    float eps, mean;           // mean: 1 / cols
    Phase phase;
    Drop drop;
};

// (mean of squares + eps)^(-1/2), the approximate root after one step of Newton's method.  Squares that leave fp32's range make it NaN rather
// than 0: the row is lost and says so.
__device__ __forceinline__ float rms_inverse(float sum, float mean, float eps) {
    const float v = fmaf(sum, mean, eps), r = rsqrtf(v);
    return sum <= 3.402823466e38f ? r * fmaf(-0.5f * v * r, r, 1.5f) : __uint_as_float(0x7FFFFFFFu);
}

// h of 8 columns in fp32; zero past the end.
template <typename T>
__device__ __forceinline__ void norm_input8(const NormArgs& a, uint64_t row, uint32_t c0, float f[8]) {
    to_floats(load8(static_cast<const T*>(a.x.p) + row * a.x.ld, c0, a.cols, a.grain_x), f);
    if (a.drop.cut) drop8(a.drop, row, c0, f);
    if (a.residual.p) {
        float r[8];
        to_floats(load8(static_cast<const T*>(a.residual.p) + row * a.residual.ld, c0, a.cols, a.grain_r), r);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] += r[i];
    }
}

// A CTA a row, its inputs read twice, for rows of any length.  max |h gamma| times r is max |y|, so one pass gives both statistics.
template <typename T>
__global__ void __launch_bounds__(NORM_THREADS) rms_norm_kernel(NormArgs a, float* scales) {
    __shared__ float slots[NORM_THREADS / 32][2];
    wait_for_predecessor();
    release_successor();
    const T* gamma = static_cast<const T*>(a.gamma.p);
    for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        float sum = 0.0f;
        uint32_t m = 0u;
        for (uint32_t c0 = threadIdx.x * 8; c0 < a.cols; c0 += NORM_THREADS * 8) {
            float f[8], g[8];
            norm_input8<T>(a, row, c0, f);
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
            norm_input8<T>(a, row, c0, f);
            to_floats(load8(gamma, c0, a.cols, a.grain_g), g);
            if (a.h.p) store8(static_cast<T*>(a.h.p) + row * a.h.ld, c0, a.cols, a.grain_h, f);
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = f[i] * g[i] * r;
            if (a.y.p) store8(static_cast<T*>(a.y.p) + row * a.y.ld, c0, a.cols, a.grain_y, f);
            if (a.q.p) store_q8(static_cast<uint8_t*>(a.q.p) + row * a.q.ld + c0, c0, a.cols, a.grain_q, row_bytes8(f, s.inv));
        }
        if (a.q.p && threadIdx.x == 0) scales[row] = s.scale;
    }
}

// The same with the row in registers, V times eight elements a thread, and its inputs read once.  h leaves before the reduction; what stays
// for after it is h gamma, which becomes y, and y the bytes.  Bound by HBM: 16384 x 8192 bf16 with residual in 158 us (6.8 TB/s, 1.04 of the copy
// rate), to 8 bits 139 us, with dropout 166 and 156 (0.99, 0.92).  A row of 8192 in 256 threads: what is kept decides how many rows an SM
// has in flight, and to 8 bits without residual and h they are too few (16384 x 8192 77 us, 0.80; 16384 x 4096 44, 0.70).  With gamma kept in its own
// type and h stored after the reduction the 8-bit form took 212 us.  Rows of 16384 and more leave room for two CTAs an SM and one (8192 x 16384
// 165 us, 2000 x 20000 68).  Held to 40 registers rows of 4096 without a residual take 46.6 us instead of 48.4.  Rows with ends: 16384 x 4097
// 97 us (0.85), 16384 x 1001 26 (0.77); to 8 bits without residual 75 (0.41) and 23 (0.33).  One token of 4096 takes 1.9 us.
template <typename T, int TEAM, int V, bool DROP, bool WIDE>
__global__ void __launch_bounds__(TEAM == 32 ? 256 : TEAM, TEAM == 32 ? 3 : TEAM == 1024 ? 1 : TEAM >= 256 && V == 4 ? 1024 / TEAM - (DROP && TEAM == 256) : V == 2 && WIDE && !DROP ? 1536 / TEAM : 1024 / TEAM)
rms_norm_rows_kernel(NormArgs a, float* scales) {
    constexpr int TEAMS = TEAM == 32 ? 8 : 1;
    __shared__ float2 slots[TEAM / 32];
    wait_for_predecessor();
    release_successor();
    const uint32_t t = TEAM == 32 ? threadIdx.x & 31u : threadIdx.x;
    const uint64_t row = (uint64_t)blockIdx.x * TEAMS + (TEAM == 32 ? threadIdx.x >> 5 : 0u);
    if (row >= a.rows) return;
    const RowCut cut = row_cut<WIDE>(a.phase, row, a.cols);
    const int first = cut.lead + (int)t * 8, cols = (int)a.cols;
    const int ec = !WIDE && last_warp<TEAM>(t) ? end_col(cut, a.cols, t & 31u) : -1;        // the ends are the last warp's
    const T *x = row_of<T>(a.x, row), *add = row_of<T>(a.residual, row);
    Raw8<T> in[V], res[V], g[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        in[j] = j * TEAM + t < cut.whole ? chunk_load8<T, WIDE>(a.x, x, first + j * TEAM * 8) : Raw8<T>{};
        if (a.residual.p) res[j] = j * TEAM + t < cut.whole ? chunk_load8<T, WIDE>(a.residual, add, first + j * TEAM * 8) : Raw8<T>{};
    }
    T ends[3] = {};
    if (ec >= 0) {
        ends[0] = x[ec];
        if (a.residual.p) ends[1] = add[ec];
        ends[2] = static_cast<const T*>(a.gamma.p)[ec];
    }
#pragma unroll
    for (int j = 0; j < V; ++j) g[j] = j * TEAM + t < cut.whole ? across_load8<T, WIDE>(a.gamma, first + j * TEAM * 8, cols) : Raw8<T>{};
    Pair v[V][4], sums = pair(0.0f);
    float top = 0.0f;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int c0 = first + j * TEAM * 8;
        const bool own = j * TEAM + t < cut.whole;
        to_pairs(in[j], v[j]);
        if constexpr (DROP) drop_pairs<WIDE>(a.drop, drop_row(a.drop, row), c0, v[j]);
        if (a.residual.p) {
            Pair r[4];
            to_pairs(res[j], r);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[j][i] = v[j][i] + r[i];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) sums = fma2(v[j][i], v[j][i], sums);       // zeros outside the row, dropped or not
        if (a.h.p && own) chunk_store8<T, WIDE>(a.h, row_of<T>(a.h, row), c0, v[j]);
        Pair w[4];
        if (WIDE || own) to_pairs(across_join8<T, WIDE>(a.gamma, g[j], c0, cols), w);
        else
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = pair(0.0f);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[j][i] = v[j][i] * w[i];
        if (a.q.p) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 f = both(v[j][i]);
                top = abs_max(top, f.x, f.y);
            }
        }
    }
    const float2 two = both(sums);
    float sum = two.x + two.y, end = 0.0f;
    if (!WIDE && ec >= 0) {
        end = element(ends[0]);
        if constexpr (DROP) end = drop1(a.drop, drop_row(a.drop, row), ec, end);
        if (a.residual.p) end += element(ends[1]);
        sum = fmaf(end, end, sum);
        if (a.h.p) row_of<T>(a.h, row)[ec] = rounded<T>(end);
        end *= element(ends[2]);
        top = abs_max(top, end, end);
    }
    uint32_t m = __float_as_uint(top);
    team_reduce<TEAM>(sum, m, slots);
    // y, in place of h gamma: rounding keeps the order of magnitudes, so the largest h gamma times r is the largest y
    const float r = rms_inverse(sum, a.mean, a.eps);
#pragma unroll
    for (int j = 0; j < V; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) v[j][i] = v[j][i] * pair(r);
    end *= r;
    if (a.q.p) {
        const RowScale s = row_scale(__float_as_uint(__uint_as_float(m) * r) & 0x7FFFFFFFu);
        uint8_t* q = row_of<uint8_t>(a.q, row);
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (j * TEAM + t < cut.whole) chunk_store_bytes8<WIDE>(a.q, q, first + j * TEAM * 8, row_bytes8(v[j], s.inv));
        if (ec >= 0) q[ec] = row_byte(end, s.inv);
        if (t == 0) scales[row] = s.scale;
    }
    if (a.y.p) {
        T* y = row_of<T>(a.y, row);
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (j * TEAM + t < cut.whole) chunk_store8<T, WIDE>(a.y, y, first + j * TEAM * 8, v[j]);
        if (ec >= 0) y[ec] = rounded<T>(end);
    }
}

struct NormGradArgs {
    uint64_t rows;
    InRows dy, h, gamma, residual;
    OutRows dh, dx;
    uint32_t cols, grain_y, grain_h, grain_g, grain_r, grain_dh, grain_dx;
    uint32_t runs, run_rows, accumulate;
    uint64_t part_ld;          // floats between two partial rows of column sums
    float eps, mean;
    Phase phase;
    Drop drop;
};

// What a team of threads makes of eight columns of a row once its statistics are known: dh and dx, and the column sums' terms.
template <typename T, bool DROP, bool WIDE>
__device__ __forceinline__ void norm_grad8(const NormGradArgs& a, uint64_t row, int c, float r, float mean_gu, const Pair d[4], const Pair f[4],
                                           const Pair g[4], Pair e[4], Pair sum[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const Pair u = f[i] * pair(r);
        sum[i] = fma2(d[i], u, sum[i]);
        e[i] = fma2(pair(r), fma2(u, pair(-mean_gu), d[i] * g[i]), e[i]);
    }
    if (a.dh.p) chunk_store8<T, WIDE>(a.dh, row_of<T>(a.dh, row), c, e);
    if (!a.dx.p) return;
    if constexpr (DROP) drop_pairs<WIDE>(a.drop, drop_row(a.drop, row), c, e);
    chunk_store8<T, WIDE>(a.dx, row_of<T>(a.dx, row), c, e);
}

// Sums of h^2 and g h over eight columns.
__device__ __forceinline__ void norm_grad_stats8(const Pair d[4], const Pair f[4], const Pair g[4], Pair& sum, Pair& dot) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        sum = fma2(f[i], f[i], sum);
        dot = fma2(d[i] * g[i], f[i], dot);
    }
}
// A team's column sums to `to`: its threads' chunks, and the ends.
template <int TEAM, int V>
__device__ __forceinline__ void norm_leave_sums(const Pair (&sum)[V][4], float end, int ec, uint32_t t, const RowCut& cut, float* to) {
#pragma unroll
    for (int j = 0; j < V; ++j) {
        if (j * TEAM + t >= cut.whole) break;
        float* at = to + cut.lead + (j * TEAM + t) * 8;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = both(sum[j][i]);
            at[2 * i] = f.x;
            at[2 * i + 1] = f.y;
        }
    }
    if (ec >= 0) to[ec] = end;
}

// A team a row, V times eight elements a thread, for inputs of one phase, from a ring of shared-memory stages that bulk copies fill
// ahead of use: loads are in flight while a row is reduced and written, and its operands are read from there twice instead of being
// kept in registers.  Teams walk the rows with their columns' sums in registers and leave one partial row of sums a CTA; their steps are
// multiples of 8 rows, so that all of a team's rows have the same cut and the same columns.  A warp has a ring of its own; a larger team
// fills a stage again after the next row's barrier, which every thread reaches done with it.
// Bound by HBM at 2048 columns and more: 16384 x 8192 bf16 with residual in 168 us (6.4 TB/s, 0.98 of the copy rate), with dx through dropout
// 225 (0.91: the generator's products, at half the multiply-add rate).  Narrower rows spend issue slots instead: 65536 x 1024 0.89, 262144 x
// 256 0.71.  Read twice from HBM by two kernels, statistics and strips, 16384 x 8192 with dropout took 316 us.
// 16384 x 4097 takes 89 us (0.92), 16384 x 1001 31 (0.64).
// row_bytes: of a stage's place for one operand, a row's chunks and, where rows have ends, sixteen more
struct NormRing { uint32_t stages, row_bytes, operands; };
constexpr uint32_t RING_MOST_STAGES = 8;
// Teams a CTA, and CTAs an SM: 16 warps of up to 128 registers a thread.
__host__ __device__ constexpr int ring_teams(int team, int v) { return team == 32 ? 8 : team == 128 && v == 1 ? 4 : 1; }
__host__ __device__ constexpr int ring_ctas(int team, int v) { return 512 / (team * ring_teams(team, v)); }
// A team's barrier; whether all of its threads say yes.
template <int TEAM>
__device__ __forceinline__ bool team_and(bool yes, uint32_t team) {
    uint32_t all;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.and.pred.aligned q, %2, %3, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(all) : "r"((uint32_t)yes), "r"(team + 1), "n"(TEAM) : "memory");
    return all != 0;
}
template <typename T, int TEAM, int V, bool DROP, bool WIDE>
__global__ void __launch_bounds__(ring_teams(TEAM, V) * TEAM, ring_ctas(TEAM, V)) norm_grad_ring_kernel(NormGradArgs a, NormRing ring, float* partial, int* status) {
    constexpr int TEAMS = ring_teams(TEAM, V);
    extern __shared__ __align__(128) uint8_t raw[];
    __shared__ __align__(8) unsigned long long bars[TEAMS * RING_MOST_STAGES];
    __shared__ float2 slots[2][TEAMS][TEAM / 32];
    const uint32_t t = threadIdx.x % TEAM, team = threadIdx.x / TEAM;
    const uint32_t stage_bytes = ring.operands * ring.row_bytes;
    const uint8_t* own = raw + team * ring.stages * stage_bytes;
    const uint32_t base = smem_addr(own), full = smem_addr(bars + team * RING_MOST_STAGES);
    if (t == 0) {
        for (uint32_t s = 0; s < ring.stages; ++s) mbar_init(full + 8 * s, 1);
        mbar_init_fence();
    }
    __syncthreads();
    wait_for_predecessor();
    release_successor();
    const uint64_t first = (uint64_t)blockIdx.x * TEAMS + team, step = (uint64_t)gridDim.x * TEAMS;
    const uint32_t mine = first < a.rows ? (uint32_t)((a.rows - first + step - 1) / step) : 0u;
    uint32_t filled = 0, fill_stage = 0;
    const RowCut cut = row_cut<WIDE>(a.phase, first, a.cols);
    const int cols = (int)a.cols;
    const auto fill = [&] {                                            // this team's next row
        const uint64_t row = first + filled * step;
        const uint32_t bar = full + 8 * fill_stage, bytes = 16 * cut.whole, to = base + fill_stage * stage_bytes;
        mbar_expect_tx(bar, bytes * ring.operands);
        if (bytes) {
            bulk_load(to, row_of<T>(a.dy, row) + cut.lead, bytes, bar);
            bulk_load(to + ring.row_bytes, row_of<T>(a.h, row) + cut.lead, bytes, bar);
            if (a.residual.p) bulk_load(to + 2 * ring.row_bytes, row_of<T>(a.residual, row) + cut.lead, bytes, bar);
        }
        ++filled;
        if (++fill_stage == ring.stages) fill_stage = 0;
    };
    if (t == 0)
        while (filled < mine && filled < ring.stages) fill();
    // the ends are the last warp's, loaded a row ahead
    const int ec = !WIDE && last_warp<TEAM>(t) ? end_col(cut, a.cols, t & 31u) : -1;
    T ends[3] = {};
    const auto ahead = [&](uint64_t row) {
        ends[0] = row_of<T>(a.dy, row)[ec];
        ends[1] = row_of<T>(a.h, row)[ec];
        if (a.residual.p) ends[2] = row_of<T>(a.residual, row)[ec];
    };
    float end_gamma = 0.0f, end_sum = 0.0f;
    if (ec >= 0) {
        end_gamma = element(static_cast<const T*>(a.gamma.p)[ec]);
        if (mine) ahead(first);
    }
    Raw8<T> gr[V];
    Pair sum[V][4];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        gr[j] = j * TEAM + t < cut.whole ? across_load8<T, WIDE>(a.gamma, cut.lead + (int)(j * TEAM + t) * 8, cols) : Raw8<T>{};
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[j][i] = pair(0.0f);
    }
#pragma unroll
    for (int j = 0; j < V; ++j)
        if (j * TEAM + t < cut.whole) gr[j] = across_join8<T, WIDE>(a.gamma, gr[j], cut.lead + (int)(j * TEAM + t) * 8, cols);
    uint32_t stage = 0, phase = 0;
    bool ok = true;
    for (uint32_t n = 0; n < mine; ++n) {
        const uint64_t row = first + n * step;
        const uint8_t* at = own + stage * stage_bytes;
        const auto operand = [&](int which, uint32_t chunk) {
            Raw8<T> x;
            x.v = *reinterpret_cast<const uint4*>(at + which * ring.row_bytes + chunk * 16);
            return x;
        };
        const float end_d = element(ends[0]), end_f = element(ends[1]), end_e = element(ends[2]);
        if (ec >= 0 && n + 1 < mine) ahead(row + step);
        ok = mbar_wait(full + 8 * stage, phase);
        Pair ss = pair(0.0f), dd = pair(0.0f);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            if (j * TEAM + t >= cut.whole) break;
            Pair d[4], f[4], g[4];
            to_pairs(operand(0, j * TEAM + t), d); to_pairs(operand(1, j * TEAM + t), f);
            to_pairs(gr[j], g);
            norm_grad_stats8(d, f, g, ss, dd);
        }
        const float2 s2 = both(ss), d2 = both(dd);
        float square = s2.x + s2.y, dot = d2.x + d2.y;
        if constexpr (!WIDE) {                                         // zeros where there is none
            square = fmaf(end_f, end_f, square);
            dot = fmaf(end_d * end_gamma, end_f, dot);
        }
        square = warp_sum(square);
        dot = warp_sum(dot);
        if constexpr (TEAM == 32) {
            if (!(ok = __all_sync(0xFFFFFFFFu, ok))) break;            // the wait ran out: the team leaves together
        } else {
            float2* slot = slots[n & 1u][team];
            if ((t & 31u) == 0) slot[t >> 5] = make_float2(square, dot);
            if (!(ok = team_and<TEAM>(ok, team))) break;
            if (t == 0 && n > 0 && filled < mine) fill();
            square = dot = 0.0f;
#pragma unroll
            for (int w = 0; w < TEAM / 32; ++w) { square += slot[w].x; dot += slot[w].y; }
        }
        const float r = rms_inverse(square, a.mean, a.eps), mean_gu = dot * r * a.mean;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const uint32_t chunk = j * TEAM + t;
            if (chunk >= cut.whole) break;
            Pair d[4], f[4], g[4], e[4];
            to_pairs(operand(0, chunk), d); to_pairs(operand(1, chunk), f); to_pairs(gr[j], g);
            if (a.residual.p) to_pairs(operand(2, chunk), e);
            else
#pragma unroll
                for (int i = 0; i < 4; ++i) e[i] = pair(0.0f);
            norm_grad8<T, DROP, WIDE>(a, row, cut.lead + (int)chunk * 8, r, mean_gu, d, f, g, e, sum[j]);
        }
        if (!WIDE && ec >= 0) {
            const float u = end_f * r;
            end_sum = fmaf(end_d, u, end_sum);
            float e = fmaf(r, fmaf(u, -mean_gu, end_d * end_gamma), end_e);
            if (a.dh.p) row_of<T>(a.dh, row)[ec] = rounded<T>(e);
            if (a.dx.p) {
                if constexpr (DROP) e = drop1(a.drop, drop_row(a.drop, row), ec, e);
                row_of<T>(a.dx, row)[ec] = rounded<T>(e);
            }
        }
        if constexpr (TEAM == 32) {
            __syncwarp();
            if (t == 0 && filled < mine) fill();
        }
        if (++stage == ring.stages) { stage = 0; phase ^= 1u; }
    }
    if (!ok && t == 0) {                                               // copies in flight land before the CTA ends
        atomicCAS(status, 0, ST_TIMEOUT);
        for (uint32_t n = filled > ring.stages ? filled - ring.stages : 0; n < filled; ++n) mbar_wait(full + 8 * (n % ring.stages), (n / ring.stages) & 1u);
    }
    if (!partial) return;
    partial += (uint64_t)blockIdx.x * a.part_ld;
    if constexpr (TEAMS == 1) {
        norm_leave_sums<TEAM, V>(sum, end_sum, ec, t, cut, partial);
    } else {                                                           // the teams' sums in the stages' place, added in order
        __syncthreads();
        norm_leave_sums<TEAM, V>(sum, end_sum, ec, t, cut, reinterpret_cast<float*>(raw + team * ring.stages * stage_bytes));
        __syncthreads();
        for (uint32_t c = threadIdx.x; c < a.cols; c += TEAMS * TEAM) {
            float total = 0.0f;
#pragma unroll
            for (int w = 0; w < TEAMS; ++w) total += reinterpret_cast<const float*>(raw + w * ring.stages * stage_bytes)[c];
            partial[c] = total;
        }
    }
}

// Column sums from the CTAs' partial rows: 32 columns a CTA, one of JOIN_LANES rows a thread, joined in order.  3 us, most of it the second launch.
constexpr int JOIN_LANES = 32;
static __global__ void __launch_bounds__(JOIN_LANES * 32) norm_join_kernel(const float* partial, uint32_t parts, uint64_t part_ld, uint32_t cols, float* dgamma,
                                                                           uint32_t accumulate) {
    __shared__ float join[JOIN_LANES][33];
    wait_for_predecessor();
    release_successor();
    const uint32_t tx = threadIdx.x & 31u, ty = threadIdx.x >> 5, c = blockIdx.x * 32 + tx;
    float total = 0.0f;
    if (c < cols)
#pragma unroll 8
        for (uint32_t i = ty; i < parts; i += JOIN_LANES) total += load_l2(&partial[i * part_ld + c]);
    join[ty][tx] = total;
    __syncthreads();
    total = warp_sum(join[tx][ty]);                          // a warp a column
    if (tx == 0 && blockIdx.x * 32 + ty < cols) {
        float* to = dgamma + blockIdx.x * 32 + ty;
        *to = accumulate ? *to + total : total;
    }
}

// Rows that the ring does not take, longer than 16384 or inputs of several phases, in two kernels.  Each row's r and mean(g u).  4000 x 20000: 181 us (0.54).
template <typename T>
__global__ void __launch_bounds__(NORM_THREADS) norm_stats_kernel(NormGradArgs a, float2* stats) {
    __shared__ float slots[NORM_THREADS / 32][2];
    wait_for_predecessor();
    release_successor();
    const T *dy = static_cast<const T*>(a.dy.p), *h = static_cast<const T*>(a.h.p), *gamma = static_cast<const T*>(a.gamma.p);
    for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        float sum = 0.0f, dot = 0.0f;
        for (uint32_t c0 = threadIdx.x * 8; c0 < a.cols; c0 += NORM_THREADS * 8) {
            float d[8], f[8], g[8];
            to_floats(load8(dy + row * a.dy.ld, c0, a.cols, a.grain_y), d);
            to_floats(load8(h + row * a.h.ld, c0, a.cols, a.grain_h), f);
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
__global__ void __launch_bounds__(CKPT_THREADS) norm_strips_kernel(NormGradArgs a, const float2* stats, float* partial, uint32_t* tickets, float* dgamma) {
    wait_for_predecessor();
    release_successor();
    const T *dy = static_cast<const T*>(a.dy.p), *h = static_cast<const T*>(a.h.p), *gamma = static_cast<const T*>(a.gamma.p);
    const T* residual = static_cast<const T*>(a.residual.p);
    T *dh = static_cast<T*>(a.dh.p), *dx = static_cast<T*>(a.dx.p);
    const uint32_t tx = threadIdx.x & 31u, ty = threadIdx.x >> 5;
    const uint32_t c0 = blockIdx.x * GRAD_COLS + tx * 8;
    const uint64_t first = (uint64_t)blockIdx.y * a.run_rows, end = min(first + a.run_rows, a.rows);
    float sum[8] = {}, g[8] = {};
    if (c0 < a.cols) {
        to_floats(load8(gamma, c0, a.cols, a.grain_g), g);
        for (uint64_t row = first + ty; row < end; row += GRAD_LANES) {
            float d[8], f[8], e[8] = {};
            to_floats(load8(dy + row * a.dy.ld, c0, a.cols, a.grain_y), d);
            to_floats(load8(h + row * a.h.ld, c0, a.cols, a.grain_h), f);
            if (residual) to_floats(load8(residual + row * a.residual.ld, c0, a.cols, a.grain_r), e);
            const float2 s = stats[row];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float u = f[i] * s.x;
                sum[i] = fmaf(d[i], u, sum[i]);
                e[i] = fmaf(s.x, fmaf(-u, s.y, d[i] * g[i]), e[i]);
            }
            if (dh) store8(dh + row * a.dh.ld, c0, a.cols, a.grain_dh, e);
            if (dx) {
                if (a.drop.cut) drop8(a.drop, row, c0, e);
                store8(dx + row * a.dx.ld, c0, a.cols, a.grain_dx, e);
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
