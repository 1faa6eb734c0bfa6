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
constexpr int CKPT_UNROLL = 4;                // items a thread has in flight

// Items are halves of a group, 16 elements, numbered along the rows.  A thread's items are a fixed stride apart, which is
// kept as rows and items within a row: one division at the start, an addition and a comparison from then on.
struct ItemWalk {
    uint64_t total, stride_rows;              // total = rows * items
    uint32_t cols, items, stride_items;       // items per row (even)
    uint32_t grain_x, grain_q;                // elements that one access of a row, or of q, may take
};

struct ItemAt {
    uint64_t row;
    uint32_t item;
    __device__ ItemAt(const ItemWalk& w, uint64_t i) : row(i / w.items) { item = (uint32_t)(i - row * w.items); }
    __device__ void next(const ItemWalk& w) {
        row += w.stride_rows;
        item += w.stride_items;
        if (item >= w.items) { item -= w.items; ++row; }
    }
};

template <typename T> struct Raw8 { uint4 v; };
template <> struct Raw8<float> { uint4 v, w; };

// A grain is the widest run of elements, a power of two, at whose multiples every row of a matrix is aligned to the run's size:
// 16-bit rows of grain 8 take 16-byte accesses, and so on down to single elements.  What is narrower than 16 bytes, and a
// row's ragged end, goes through these functions, which are kept out of line.
static __device__ __noinline__ uint4 load_narrow(const uint16_t* p, uint32_t n, uint32_t grain) {
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (n >= 8 && grain >= 4) {
        const uint2 a = *reinterpret_cast<const uint2*>(p), b = *(reinterpret_cast<const uint2*>(p) + 1);
        v = make_uint4(a.x, a.y, b.x, b.y);
    } else if (n >= 8 && grain == 2) {
        const uint32_t* w = reinterpret_cast<const uint32_t*>(p);
        v = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
        uint16_t e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = i < (int)n ? p[i] : (uint16_t)0;
        v = make_uint4(e[0] | (uint32_t)e[1] << 16, e[2] | (uint32_t)e[3] << 16, e[4] | (uint32_t)e[5] << 16, e[6] | (uint32_t)e[7] << 16);
    }
    return v;
}
static __device__ __noinline__ void store_narrow(uint16_t* p, uint4 v, uint32_t n, uint32_t grain) {
    if (n >= 8 && grain >= 4) {
        *reinterpret_cast<uint2*>(p) = make_uint2(v.x, v.y);
        *(reinterpret_cast<uint2*>(p) + 1) = make_uint2(v.z, v.w);
    } else if (n >= 8 && grain == 2) {
        uint32_t* w = reinterpret_cast<uint32_t*>(p);
        w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
    } else {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) if (i < (int)n) p[i] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
    }
}
static __device__ __noinline__ uint2 load_q_narrow(const uint8_t* p, uint32_t n, uint32_t grain) {
    if (n >= 8 && grain >= 4) return make_uint2(*reinterpret_cast<const uint32_t*>(p), *(reinterpret_cast<const uint32_t*>(p) + 1));
    uint32_t v[2] = {0u, 0u};
    if (n >= 8 && grain == 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i >> 1] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[i] << (16 * (i & 1));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) if (i < (int)n) v[i >> 2] |= (uint32_t)p[i] << (8 * (i & 3));
    }
    return make_uint2(v[0], v[1]);
}
static __device__ __noinline__ void store_q_narrow(uint8_t* p, uint2 v, uint32_t n, uint32_t grain) {
    const uint32_t w[2] = {v.x, v.y};
    if (n >= 8 && grain >= 4) {
        reinterpret_cast<uint32_t*>(p)[0] = v.x;
        reinterpret_cast<uint32_t*>(p)[1] = v.y;
    } else if (n >= 8 && grain == 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) reinterpret_cast<uint16_t*>(p)[i] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) if (i < (int)n) p[i] = (uint8_t)(w[i >> 2] >> (8 * (i & 3)));
    }
}

// Eight elements from column c0; zero past the row's end.
template <typename T>
__device__ __forceinline__ Raw8<T> load8(const T* row, uint32_t c0, uint32_t cols, uint32_t grain) {
    Raw8<T> r{};
    if constexpr (sizeof(T) == 2) {
        if (grain >= 8 && c0 + 8 <= cols) r.v = load_stream16(row + c0);
        else if (c0 < cols) r.v = load_narrow(reinterpret_cast<const uint16_t*>(row + c0), cols - c0, grain);
    } else {
        if (grain >= 4 && c0 + 8 <= cols) {
            r.v = load_stream16(row + c0);
            r.w = load_stream16(reinterpret_cast<const uint4*>(row + c0) + 1);
        } else {
            uint32_t e[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) e[i] = c0 + i < cols ? __float_as_uint(row[c0 + i]) : 0u;
            r.v = make_uint4(e[0], e[1], e[2], e[3]);
            r.w = make_uint4(e[4], e[5], e[6], e[7]);
        }
    }
    return r;
}

// 32 bytes in one access: whole sectors per thread.
__device__ __forceinline__ void load32(const void* p, uint4& a, uint4& b) {
    asm volatile("ld.global.cs.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(a.x), "=r"(a.y), "=r"(a.z), "=r"(a.w), "=r"(b.x), "=r"(b.y), "=r"(b.z), "=r"(b.w) : "l"(p));
}
__device__ __forceinline__ void store32(void* p, uint4 a, uint4 b) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"l"(p), "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b.x), "r"(b.y), "r"(b.z), "r"(b.w) : "memory");
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

// `dst`: where column c0 is kept.
__device__ __forceinline__ void store_q8(uint8_t* dst, uint32_t c0, uint32_t cols, uint32_t grain, uint2 v) {
    if (grain >= 8 && c0 + 8 <= cols) __stcs(reinterpret_cast<uint2*>(dst), v);
    else if (c0 < cols) store_q_narrow(dst, v, cols - c0, grain);
}

// One pass: 2 (4) bytes read and 1 + 1/32 written per element; two lanes hold a group and share its maximum.  Bound by HBM:
// 16384 x 8192 bf16 in 67-71 us, 5.8-6.1 TB/s (0.89-0.95 of the measured copy rate); items of half a group and 32-byte accesses
// brought it there from 0.65 (8 elements a thread: twice the address arithmetic, 16-byte halves of sectors).  From fp32 108 us (0.97).
template <typename T>
__global__ void __launch_bounds__(CKPT_THREADS, sizeof(T) == 2 ? 4 : 3) checkpoint_pack_kernel(const T* x, uint64_t ldx, ItemWalk w,
                                                                       uint8_t* q, uint8_t* scales) {
    constexpr int UNROLL = sizeof(T) == 2 ? CKPT_UNROLL : 2;
    wait_for_predecessor();
    release_successor();
    const uint64_t stride = (uint64_t)gridDim.x * CKPT_THREADS, groups = w.items >> 1;
    uint64_t base = (uint64_t)blockIdx.x * CKPT_THREADS + threadIdx.x;
    const uint32_t lane = threadIdx.x & 31u;
    ItemAt at(w, base);
    // total is even and a warp's items are consecutive, so a group's two lanes stay together
    for (; base - lane < w.total; base += stride * UNROLL) {
        Raw8<T> raw[UNROLL][2];
        ItemAt from = at;
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            raw[u][0] = raw[u][1] = Raw8<T>{};
            if (base + u * stride < w.total) {
                const T* row = x + at.row * ldx;
                const uint32_t c0 = at.item * 16;
                if (sizeof(T) == 2 && w.grain_x >= 16 && c0 + 16 <= w.cols) {
                    load32(row + c0, raw[u][0].v, raw[u][1].v);
                } else {
                    raw[u][0] = load8(row, c0, w.cols, w.grain_x);
                    raw[u][1] = load8(row, c0 + 8, w.cols, w.grain_x);
                }
            }
            at.next(w);
        }
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            uint32_t m = max(abs_max8(raw[u][0]), abs_max8(raw[u][1]));
            m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
            int e = ckpt_exponent<T>(m);
            const bool odd = m >= 0x7F800000u || e == Elem<T>::EMAX;   // the two lanes agree
            if (odd) {
                m = 0;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float f[8];
                    to_floats(raw[u][h], f);
                    m = max(m, finite_max8(f));
                }
                m = max(m, __shfl_xor_sync(3u << (lane & 30u), m, 1));
                e = ckpt_exponent<T>(m);
            }
            uint2 b[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float f[8];
                to_floats(raw[u][h], f);
                b[h] = odd ? ckpt_bytes8_any<T>(f, e) : ckpt_bytes8(f, e);
            }
            if (base + u * stride < w.total) {
                const uint32_t c0 = from.item * 16;
                uint8_t* dst = q + from.row * w.cols + c0;
                if (w.grain_q >= 16 && c0 + 16 <= w.cols) {
                    __stcs(reinterpret_cast<uint4*>(dst), make_uint4(b[0].x, b[0].y, b[1].x, b[1].y));
                } else {
                    store_q8(dst, c0, w.cols, w.grain_q, b[0]);
                    store_q8(dst + 8, c0 + 8, w.cols, w.grain_q, b[1]);
                }
                if ((from.item & 1u) == 0u) scales[from.row * groups + (from.item >> 1)] = (uint8_t)(e + 127);
            }
            from.next(w);
        }
    }
}

template <typename T>
__device__ __forceinline__ void store8(T* row, uint32_t c0, uint32_t cols, uint32_t grain, const float f[8]) {
    if constexpr (sizeof(T) == 2) {
        const uint4 o = make_uint4(Elem<T>::pack(f[0], f[1]), Elem<T>::pack(f[2], f[3]), Elem<T>::pack(f[4], f[5]), Elem<T>::pack(f[6], f[7]));
        if (grain >= 8 && c0 + 8 <= cols) *reinterpret_cast<uint4*>(row + c0) = o;
        else if (c0 < cols) store_narrow(reinterpret_cast<uint16_t*>(row + c0), o, cols - c0, grain);
    } else if (grain >= 4 && c0 + 8 <= cols) {
        *reinterpret_cast<float4*>(row + c0) = make_float4(f[0], f[1], f[2], f[3]);
        *(reinterpret_cast<float4*>(row + c0) + 1) = make_float4(f[4], f[5], f[6], f[7]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) if (c0 + i < cols) row[c0 + i] = f[i];
    }
}

template <typename T>
__device__ __forceinline__ uint4 packed8(const Pair v[4]) {
    uint32_t o[4] = {};
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) { const float2 f = both(v[i]); o[i] = Elem<T>::pack(f.x, f.y); }
    }
    return make_uint4(o[0], o[1], o[2], o[3]);
}
template <typename T>
__device__ __forceinline__ void store8(T* row, uint32_t c0, uint32_t cols, uint32_t grain, const Pair v[4]) {
    float f[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) { const float2 p = both(v[i]); f[2 * i] = p.x; f[2 * i + 1] = p.y; }
    store8(row, c0, cols, grain, f);
}

__device__ __forceinline__ uint2 load_q8(const uint8_t* row, uint32_t c0, uint32_t cols, uint32_t grain) {
    if (grain >= 8 && c0 + 8 <= cols) return load_stream8(row + c0);
    return c0 < cols ? load_q_narrow(row + c0, cols - c0, grain) : make_uint2(0u, 0u);
}

// The reverse, bound by HBM in the same way: 16384 x 8192 bf16 in 71 us, 5.75 TB/s (0.89).  To fp32 165 us (0.63), in 16-byte stores
// that lie 64 bytes apart across a warp.
template <typename T>
__global__ void __launch_bounds__(CKPT_THREADS, sizeof(T) == 2 ? 4 : 3) checkpoint_unpack_kernel(const uint8_t* q, const uint8_t* scales, ItemWalk w,
                                                                         T* out, uint64_t ldo) {
    wait_for_predecessor();
    release_successor();
    const uint64_t stride = (uint64_t)gridDim.x * CKPT_THREADS, groups = w.items >> 1;
    uint64_t base = (uint64_t)blockIdx.x * CKPT_THREADS + threadIdx.x;
    ItemAt at(w, base);
    for (; base < w.total; base += stride * CKPT_UNROLL) {
        uint2 raw[CKPT_UNROLL][2];
        uint32_t sb[CKPT_UNROLL];
        ItemAt from = at;
#pragma unroll
        for (int u = 0; u < CKPT_UNROLL; ++u) {
            if (base + u * stride < w.total) {
                const uint8_t* row = q + at.row * w.cols;
                const uint32_t c0 = at.item * 16;
                if (w.grain_q >= 16 && c0 + 16 <= w.cols) {
                    const uint4 v = load_stream16(row + c0);
                    raw[u][0] = make_uint2(v.x, v.y);
                    raw[u][1] = make_uint2(v.z, v.w);
                } else {
                    raw[u][0] = load_q8(row, c0, w.cols, w.grain_q);
                    raw[u][1] = load_q8(row, c0 + 8, w.cols, w.grain_q);
                }
                sb[u] = scales[at.row * groups + (at.item >> 1)];
            }
            at.next(w);
        }
#pragma unroll
        for (int u = 0; u < CKPT_UNROLL; ++u) {
            if (base + u * stride < w.total) {
                const Scale k = ckpt_scale(sb[u]);
                const uint32_t c0 = from.item * 16;
                T* row = out + from.row * ldo;
                Pair f[2][4];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (sb[u] <= LARGE_SCALE) ckpt_values8<false>(raw[u][h], k, f[h]);
                    else ckpt_values8<true>(raw[u][h], k, f[h]);
                }
                if (sizeof(T) == 2 && w.grain_x >= 16 && c0 + 16 <= w.cols) {
                    store32(row + c0, packed8<T>(f[0]), packed8<T>(f[1]));
                } else {
                    store8(row, c0, w.cols, w.grain_x, f[0]);
                    store8(row, c0 + 8, w.cols, w.grain_x, f[1]);
                }
            }
            from.next(w);
        }
    }
}

// The same for rows, or a q, that take narrow accesses only: a lane works on two neighbouring elements, so that a warp's
// accesses stay contiguous; sixteen lanes hold a group.  Three times the instructions of the wide form, a quarter of its
// transactions on such rows.
constexpr int NARROW_UNROLL = 4;              // runs of 64 elements a warp has in flight

struct NarrowWalk {
    uint64_t total, stride_rows;              // total = rows * runs; a warp's runs are a fixed stride apart, in rows and runs
    uint32_t cols, runs, stride_runs;         // runs of 64 elements a row
    uint32_t two_x, two_q;                    // whether two elements of a row, or of q, go in one access
};
struct RunAt {
    uint64_t row;
    uint32_t run;
    __device__ RunAt(const NarrowWalk& w, uint64_t i) : row(i / w.runs) { run = (uint32_t)(i - row * w.runs); }
    __device__ void next(const NarrowWalk& w) {
        row += w.stride_rows;
        run += w.stride_runs;
        if (run >= w.runs) { run -= w.runs; ++row; }
    }
};

template <typename T>
__global__ void __launch_bounds__(CKPT_THREADS) checkpoint_pack_narrow_kernel(const T* x, uint64_t ldx, NarrowWalk w,
                                                                              uint8_t* q, uint8_t* scales) {
    wait_for_predecessor();
    release_successor();
    const uint32_t lane = threadIdx.x & 31u, groups = (w.cols + CKPT_GROUP - 1) / CKPT_GROUP;
    const uint64_t first = ((uint64_t)blockIdx.x * CKPT_THREADS + threadIdx.x) >> 5, stride = (uint64_t)gridDim.x * (CKPT_THREADS / 32);
    RunAt at(w, first);
    for (uint64_t base = first; base < w.total; base += stride * NARROW_UNROLL) {
        float f[NARROW_UNROLL][2];
        uint64_t row[NARROW_UNROLL];
        uint32_t c[NARROW_UNROLL];
#pragma unroll
        for (int u = 0; u < NARROW_UNROLL; ++u) {
            row[u] = at.row;
            c[u] = base + u * stride < w.total ? at.run * 64 + lane * 2 : w.cols;
            at.next(w);
            const T* p = x + row[u] * ldx + c[u];
            f[u][0] = f[u][1] = 0.0f;
            if (sizeof(T) == 2 && w.two_x && c[u] + 1 < w.cols) {
                uint32_t v = *reinterpret_cast<const uint32_t*>(p);
                const T* e = reinterpret_cast<const T*>(&v);
                f[u][0] = Elem<T>::to_float(e[0]);
                f[u][1] = Elem<T>::to_float(e[1]);
            } else {
                if (c[u] < w.cols) f[u][0] = Elem<T>::to_float(p[0]);
                if (c[u] + 1 < w.cols) f[u][1] = Elem<T>::to_float(p[1]);
            }
        }
#pragma unroll
        for (int u = 0; u < NARROW_UNROLL; ++u) {
            const uint32_t a = __float_as_uint(f[u][0]) & 0x7FFFFFFFu, b = __float_as_uint(f[u][1]) & 0x7FFFFFFFu;
            uint32_t m = max(a < 0x7F800000u ? a : 0u, b < 0x7F800000u ? b : 0u);
#pragma unroll
            for (int d = 1; d < 16; d <<= 1) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, d));
            const int e = ckpt_exponent<T>(m);
            const float inv = pow2(-e), most = e == Elem<T>::EMAX ? 63.0f : 127.0f;
            const uint32_t b0 = ckpt_byte_any(f[u][0], inv, most), b1 = ckpt_byte_any(f[u][1], inv, most);
            uint8_t* dst = q + row[u] * w.cols + c[u];
            if (w.two_q && c[u] + 1 < w.cols) {
                *reinterpret_cast<uint16_t*>(dst) = (uint16_t)(b0 | b1 << 8);
            } else {
                if (c[u] < w.cols) dst[0] = (uint8_t)b0;
                if (c[u] + 1 < w.cols) dst[1] = (uint8_t)b1;
            }
            if ((lane & 15u) == 0u && c[u] < w.cols) scales[row[u] * groups + (c[u] >> 5)] = (uint8_t)(e + 127);
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(CKPT_THREADS) checkpoint_unpack_narrow_kernel(const uint8_t* q, const uint8_t* scales, NarrowWalk w,
                                                                                T* out, uint64_t ldo) {
    wait_for_predecessor();
    release_successor();
    const uint32_t lane = threadIdx.x & 31u, groups = (w.cols + CKPT_GROUP - 1) / CKPT_GROUP;
    const uint64_t first = ((uint64_t)blockIdx.x * CKPT_THREADS + threadIdx.x) >> 5, stride = (uint64_t)gridDim.x * (CKPT_THREADS / 32);
    RunAt at(w, first);
    for (uint64_t base = first; base < w.total; base += stride * NARROW_UNROLL) {
        uint32_t b[NARROW_UNROLL], sb[NARROW_UNROLL], c[NARROW_UNROLL];
        uint64_t row[NARROW_UNROLL];
#pragma unroll
        for (int u = 0; u < NARROW_UNROLL; ++u) {
            row[u] = at.row;
            c[u] = base + u * stride < w.total ? at.run * 64 + lane * 2 : w.cols;
            at.next(w);
            const uint8_t* p = q + row[u] * w.cols + c[u];
            b[u] = sb[u] = 0u;
            if (w.two_q && c[u] + 1 < w.cols) {
                b[u] = *reinterpret_cast<const uint16_t*>(p);
            } else {
                if (c[u] < w.cols) b[u] = p[0];
                if (c[u] + 1 < w.cols) b[u] |= (uint32_t)p[1] << 8;
            }
            if (c[u] < w.cols) sb[u] = scales[row[u] * groups + (c[u] >> 5)];
        }
#pragma unroll
        for (int u = 0; u < NARROW_UNROLL; ++u) {
            const float s = __uint_as_float(sb[u] << 23), nan = __uint_as_float(0x7FFFFFFFu);
            const uint32_t lo = b[u] & 0xFFu, hi = b[u] >> 8;
            const T v[2] = {Elem<T>::from_float(lo == 0x80u ? nan : (float)(int8_t)lo * s), Elem<T>::from_float(hi == 0x80u ? nan : (float)(int8_t)hi * s)};
            T* dst = out + row[u] * ldo + c[u];
            if (sizeof(T) == 2 && w.two_x && c[u] + 1 < w.cols) {
                *reinterpret_cast<uint32_t*>(dst) = *reinterpret_cast<const uint16_t*>(&v[0]) | (uint32_t)*reinterpret_cast<const uint16_t*>(&v[1]) << 16;
            } else {
                if (c[u] < w.cols) dst[0] = v[0];
                if (c[u] + 1 < w.cols) dst[1] = v[1];
            }
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
//
// 2 + 1 + 1/32 bytes read and 2 written per element.  8192 x 16384 bf16: the bias gradient alone (2 bytes read) 49 us (0.84 of the
// measured copy rate), relu 114-116 us (0.90-0.92), silu 120-133 us (0.79-0.87), tanh gelu 130-145 us (0.72-0.80), gelu 149 us (0.70).
// The first two are bound by HBM.  In the others no unit is full: tanh gelu and gelu use 60 and 64 % of the issue slots,
// the multiply-add pipe 48 and 55 % of the cycles, the special-function unit 48 and 41 %; 35 and 27 % of a warp's
// time goes by waiting for its loads (silu 48 %), of which a thread has one row of dy and q, 24 bytes, in flight.  Paired fp32 arithmetic
// and one exponential shared by gelu's tail and density took them from 0.37 and 0.50.  Four CTAs per SM with one row ahead
// beat three with two, or two with three.
constexpr int GRAD_COLS = 256, GRAD_LANES = 8;

struct GradArgs {
    uint64_t rows, lddy, lddz;
    uint32_t cols, groups, runs, run_rows, accumulate, grain_y, grain_z, grain_q;
};

// WIDE: a multiple of 8 columns, rows that take 16-byte accesses and a q that takes 8-byte ones.
template <typename T, int ACT, bool WIDE>
__global__ void __launch_bounds__(CKPT_THREADS, 4) activation_grad_kernel(const T* dy, const uint8_t* q, const uint8_t* scales,
                                                                          GradArgs a, T* dz, float* partial,
                                                                          uint32_t* tickets, float* db) {
    wait_for_predecessor();
    release_successor();
    const uint32_t tx = threadIdx.x & 31u, ty = threadIdx.x >> 5;
    const uint32_t c0 = blockIdx.x * GRAD_COLS + tx * 8;
    const uint64_t r0 = (uint64_t)blockIdx.y * a.run_rows + ty;
    Pair sum[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) sum[i] = pair(0.0f);
    if (c0 < a.cols) {
        const uint32_t left = (uint32_t)(min((uint64_t)(blockIdx.y + 1) * a.run_rows, a.rows) - (uint64_t)blockIdx.y * a.run_rows);
        const T* from = dy + r0 * a.lddy;
        T* to = dz + r0 * a.lddz;
        const uint8_t *qr = q + r0 * a.cols, *sr = scales + r0 * a.groups + (c0 >> 5);
        const uint64_t step_y = GRAD_LANES * a.lddy, step_z = GRAD_LANES * a.lddz, step_q = (uint64_t)GRAD_LANES * a.cols, step_s = (uint64_t)GRAD_LANES * a.groups;
        // a thread works on one row while its next one is on the way
        struct Row { Raw8<T> g; uint2 k; uint32_t sb; };
        const auto fetch = [&](Row& row, uint32_t r) {
            if (r < left) {
                if constexpr (WIDE) row.g.v = load_stream16(from + c0);
                else row.g = load8(from, c0, a.cols, a.grain_y);
                if constexpr (ACT != SC_ACT_NONE) {
                    if constexpr (WIDE) row.k = load_stream8(qr + c0);
                    else row.k = load_q8(qr, c0, a.cols, a.grain_q);
                    row.sb = *sr;
                }
            }
            from += step_y; qr += step_q; sr += step_s;
        };
        const auto work = [&](const Row& row, uint32_t r) {
            if (r < left) {
                float f[8];
                to_floats(row.g, f);
                Pair v[4], z[4];
                if constexpr (ACT != SC_ACT_NONE) ckpt_values8<false>(row.k, slope_scale(row.sb), z);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    v[i] = pair(f[2 * i], f[2 * i + 1]);
                    if constexpr (ACT != SC_ACT_NONE) v[i] = v[i] * activation_slope<ACT>(z[i]);
                    sum[i] = sum[i] + v[i];
                }
                if (dz) {
                    if constexpr (WIDE) *reinterpret_cast<uint4*>(to + c0) = packed8<T>(v);
                    else store8(to, c0, a.cols, a.grain_z, v);
                }
            }
            to += step_z;
        };
        Row x, y;
        fetch(x, ty);
        for (uint32_t r = ty; r < left; r += 2 * GRAD_LANES) {
            fetch(y, r + GRAD_LANES);
            work(x, r);
            fetch(x, r + 2 * GRAD_LANES);
            work(y, r + GRAD_LANES);
        }
    }
    if (!db) return;
    __shared__ float join[GRAD_LANES][GRAD_COLS];
    __shared__ uint32_t last;
#pragma unroll
    for (int i = 0; i < 4; ++i) { const float2 f = both(sum[i]); join[ty][tx * 8 + 2 * i] = f.x; join[ty][tx * 8 + 2 * i + 1] = f.y; }
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
    if (c < a.cols) db[c] = a.accumulate ? db[c] + total : total;
}

}  // namespace sc
