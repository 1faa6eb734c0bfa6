// 8-bit activation checkpoints: pack, unpack, and the activation's backward pass that reads them.
//
// A row is cut into groups of 32 features.  With m the largest finite magnitude of a group, e is the least exponent
// with m <= 127 2^e and every element is kept as q = rint(x 2^-e), one byte, with e + 127 in one more byte per group.
// The scale is a power of two so that q 2^e is exactly a bf16 or fp16 value: what reads the checkpoint (a matrix
// product, an activation's slope) works on the stored numbers themselves and nothing is rounded a second time.
#pragma once
#include "sc_layer_common.cuh"

namespace sc {

constexpr int CKPT_THREADS = 256;
constexpr int CKPT_UNROLL = 4;                // items (8 elements) a thread has in flight

// Items are chunks of 8 elements, four to a group, numbered along the rows; a thread walks them with a fixed stride.
struct ItemWalk {
    uint64_t rows, total;                     // total = rows * chunks
    uint32_t cols, chunks;                    // chunks per row (a multiple of 4)
    uint32_t vec;                             // 16-byte accesses are aligned and no chunk straddles a row's end
};

struct Item { uint64_t row; uint32_t chunk; };

__device__ __forceinline__ Item item_at(const ItemWalk& w, uint64_t i) {
    Item it;
    if (w.total <= 0xFFFFFFFFull) { const uint32_t r = (uint32_t)i / w.chunks; it.row = r; it.chunk = (uint32_t)i - r * w.chunks; }
    else { it.row = i / w.chunks; it.chunk = (uint32_t)(i - it.row * w.chunks); }
    return it;
}

template <typename T> struct Raw8 { uint4 v; };
template <> struct Raw8<float> { uint4 v, w; };

template <typename T>
__device__ __forceinline__ Raw8<T> load8(const T* row, uint32_t c0, uint32_t cols, uint32_t vec) {
    Raw8<T> r{};
    if (vec) {
        if (c0 < cols) {
            r.v = __ldcs(reinterpret_cast<const uint4*>(row + c0));
            if constexpr (sizeof(T) == 4) r.w = __ldcs(reinterpret_cast<const uint4*>(row + c0) + 1);
        }
    } else {
        T* e = reinterpret_cast<T*>(&r);
#pragma unroll
        for (int i = 0; i < 8; ++i) if (c0 + i < cols) e[i] = row[c0 + i];
    }
    return r;
}

template <typename T>
__device__ __forceinline__ void to_floats(const Raw8<T>& r, float f[8]) {
    if constexpr (sizeof(T) == 2) {
        const uint32_t w[4] = {r.v.x, r.v.y, r.v.z, r.v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { const float2 p = Elem<T>::unpack(w[i]); f[2 * i] = p.x; f[2 * i + 1] = p.y; }
    } else {
        const uint32_t w[8] = {r.v.x, r.v.y, r.v.z, r.v.w, r.w.x, r.w.y, r.w.z, r.w.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(w[i]);
    }
}

// Bits of the largest magnitude of 8 elements as a float; infinities and NaN order above every finite value.
template <typename T>
__device__ __forceinline__ uint32_t abs_max8(const Raw8<T>& r) {
    if constexpr (sizeof(T) == 2) {
        const uint32_t m = __vmaxu2(__vmaxu2(r.v.x & Elem<T>::ABS, r.v.y & Elem<T>::ABS), __vmaxu2(r.v.z & Elem<T>::ABS, r.v.w & Elem<T>::ABS));
        const uint32_t h = max(m & 0xFFFFu, m >> 16);
        if constexpr (Elem<T>::INF16 == 0x7F80u) return h << 16;
        return __float_as_uint(Elem<T>::unpack(h).x) & 0x7FFFFFFFu;
    } else {
        const uint32_t w[8] = {r.v.x, r.v.y, r.v.z, r.v.w, r.w.x, r.w.y, r.w.z, r.w.w};
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, w[i] & 0x7FFFFFFFu);
        return m;
    }
}

// One pass: 2 (4) bytes read and 1 + 1/32 written per element; four lanes hold a group and share its maximum.
template <typename T>
__global__ void __launch_bounds__(CKPT_THREADS) checkpoint_pack_kernel(const T* __restrict__ x, uint64_t ldx, ItemWalk w,
                                                                       uint8_t* __restrict__ q, uint8_t* __restrict__ scales) {
    const uint64_t stride = (uint64_t)gridDim.x * CKPT_THREADS;
    const uint32_t lane = threadIdx.x & 31u;
    const uint64_t groups = w.chunks >> 2;
    // total is a multiple of 4 and a warp's items are consecutive, so a group's four lanes stay together
    for (uint64_t base = (uint64_t)blockIdx.x * CKPT_THREADS + threadIdx.x; base - lane < w.total; base += stride * CKPT_UNROLL) {
        Raw8<T> raw[CKPT_UNROLL];
        Item it[CKPT_UNROLL];
#pragma unroll
        for (int u = 0; u < CKPT_UNROLL; ++u) {
            const uint64_t i = base + u * stride;
            it[u] = item_at(w, i < w.total ? i : 0);
            raw[u] = Raw8<T>{};
            if (i < w.total) raw[u] = load8(x + it[u].row * ldx, it[u].chunk * 8, w.cols, w.vec);
        }
#pragma unroll
        for (int u = 0; u < CKPT_UNROLL; ++u) {
            uint32_t m = abs_max8(raw[u]);
            m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
            m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 2));
            float f[8];
            to_floats(raw[u], f);
            uint32_t b[8];
            const int e = ckpt_encode8<T>(f, m, b);
            if (base + u * stride >= w.total) continue;
            const uint32_t c0 = it[u].chunk * 8;
            uint8_t* dst = q + it[u].row * w.cols + c0;
            if (w.vec) {
                if (c0 < w.cols) {
                    __stcs(reinterpret_cast<uint2*>(dst), ckpt_join8(b));
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) if (c0 + i < w.cols) dst[i] = (uint8_t)b[i];
            }
            if ((it[u].chunk & 3u) == 0u) scales[it[u].row * groups + (it[u].chunk >> 2)] = (uint8_t)(e + 127);
        }
    }
}

template <typename T>
__device__ __forceinline__ void store8(T* row, uint32_t c0, uint32_t cols, uint32_t vec, const float f[8]) {
    if (vec) {
        if (c0 >= cols) return;
        if constexpr (sizeof(T) == 2) {
            const uint4 o = make_uint4(Elem<T>::pack(f[0], f[1]), Elem<T>::pack(f[2], f[3]), Elem<T>::pack(f[4], f[5]), Elem<T>::pack(f[6], f[7]));
            *reinterpret_cast<uint4*>(row + c0) = o;
        } else {
            *reinterpret_cast<float4*>(row + c0) = make_float4(f[0], f[1], f[2], f[3]);
            *(reinterpret_cast<float4*>(row + c0) + 1) = make_float4(f[4], f[5], f[6], f[7]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) if (c0 + i < cols) row[c0 + i] = Elem<T>::from_float(f[i]);
    }
}

__device__ __forceinline__ uint2 load_q8(const uint8_t* row, uint32_t c0, uint32_t cols, uint32_t vec) {
    uint2 r = make_uint2(0u, 0u);
    if (vec) {
        if (c0 < cols) r = __ldcs(reinterpret_cast<const uint2*>(row + c0));
    } else {
        uint8_t* b = reinterpret_cast<uint8_t*>(&r);
#pragma unroll
        for (int i = 0; i < 8; ++i) if (c0 + i < cols) b[i] = row[c0 + i];
    }
    return r;
}

template <typename T>
__global__ void __launch_bounds__(CKPT_THREADS) checkpoint_unpack_kernel(const uint8_t* __restrict__ q, const uint8_t* __restrict__ scales, ItemWalk w,
                                                                         T* __restrict__ out, uint64_t ldo) {
    const uint64_t stride = (uint64_t)gridDim.x * CKPT_THREADS;
    const uint64_t groups = w.chunks >> 2;
    for (uint64_t base = (uint64_t)blockIdx.x * CKPT_THREADS + threadIdx.x; base < w.total; base += stride * CKPT_UNROLL) {
        uint2 raw[CKPT_UNROLL];
        uint32_t sb[CKPT_UNROLL];
        Item it[CKPT_UNROLL];
#pragma unroll
        for (int u = 0; u < CKPT_UNROLL; ++u) {
            const uint64_t i = base + u * stride;
            it[u] = item_at(w, i < w.total ? i : 0);
            if (i >= w.total) continue;
            raw[u] = load_q8(q + it[u].row * w.cols, it[u].chunk * 8, w.cols, w.vec);
            sb[u] = scales[it[u].row * groups + (it[u].chunk >> 2)];
        }
#pragma unroll
        for (int u = 0; u < CKPT_UNROLL; ++u) {
            if (base + u * stride >= w.total) continue;
            float f[8];
            ckpt_values4(raw[u].x, ckpt_scale(sb[u]), f);
            ckpt_values4(raw[u].y, ckpt_scale(sb[u]), f + 4);
            store8(out + it[u].row * ldo, it[u].chunk * 8, w.cols, w.vec, f);
        }
    }
}

// ---------------------------------------------------------------------------
// dz = dy * act'(z^) and db = column sums of dz
// ---------------------------------------------------------------------------
// A CTA owns a strip of 256 columns and a run of rows: 32 threads side by side with 8 columns each, 8 rows at a time.
// Column sums are kept in registers in 32 bits, joined over the CTA's 8 row lanes in shared memory and written as one
// partial row per run; the last CTA of a strip to finish adds the runs' partial rows in order, so the result does not
// depend on the order in which the CTAs ran.
constexpr int GRAD_COLS = 256, GRAD_LANES = 8;

struct GradArgs {
    uint64_t rows, lddy, lddz;
    uint32_t cols, groups, runs, run_rows, vec, accumulate;
};

template <typename T, int ACT>
__global__ void __launch_bounds__(CKPT_THREADS) activation_grad_kernel(const T* dy, const uint8_t* __restrict__ q, const uint8_t* __restrict__ scales,
                                                                       GradArgs a, T* dz, float* __restrict__ partial,
                                                                       uint32_t* __restrict__ tickets, float* __restrict__ db) {
    const uint32_t tx = threadIdx.x & 31u, ty = threadIdx.x >> 5;
    const uint32_t c0 = blockIdx.x * GRAD_COLS + tx * 8;
    const uint64_t r0 = (uint64_t)blockIdx.y * a.run_rows;
    const uint64_t r1 = min(r0 + a.run_rows, a.rows);
    float sum[8] = {};
    if (c0 < a.cols) {
#pragma unroll 2
        for (uint64_t r = r0 + ty; r < r1; r += GRAD_LANES) {
            const Raw8<T> g = load8(dy + r * a.lddy, c0, a.cols, a.vec);
            float f[8];
            to_floats(g, f);
            if constexpr (ACT != SC_ACT_NONE) {
                const uint2 k = load_q8(q + r * a.cols, c0, a.cols, a.vec);
                const float s = ckpt_scale(scales[r * a.groups + (c0 >> 5)]);
                float z[8];
                ckpt_values4(k.x, s, z);
                ckpt_values4(k.y, s, z + 4);
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] *= activation_slope<ACT>(z[i]);
            }
            if (dz) store8(dz + r * a.lddz, c0, a.cols, a.vec, f);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] += f[i];
        }
    }
    if (!db) return;
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
            for (uint32_t j = 0; j < a.runs; ++j) total += __ldcg(&partial[(uint64_t)j * a.cols + c]);
        if (threadIdx.x == 0) tickets[blockIdx.x] = 0u;               // zero again for the next call
    }
    if (c < a.cols) db[c] = a.accumulate ? db[c] + total : total;
}

}  // namespace sc
