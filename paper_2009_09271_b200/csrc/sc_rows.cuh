// Rows of any alignment, eight elements a thread.
//
// A row is cut where its 16-bit elements cross 16-byte boundaries: a chunk's first column is a multiple of 8 less the row's shift,
// the number of elements between its first one and the boundary before it.  Matrices of one odd width have the same shift in
// the same row, so all of them move in whole accesses, with single elements at a row's ends only.  WIDE is the case without: every
// row starts on a boundary and is a multiple of 8 long.
#pragma once
#include "sc_checkpoint.cuh"

namespace sc {

// A matrix to read: `span` elements from its first to its last.  `vec`: its rows have the shifts of the phase (and are 16-byte accesses).
struct InRows {
    const void* p;
    uint64_t ld, span;
    uint32_t vec;
};
struct OutRows {
    void* p;
    uint64_t ld;
    uint32_t vec;
};
// Row r is (first + r ld) mod 8 elements past a boundary.
struct Phase { uint32_t first, ld; };
template <bool WIDE>
__device__ __forceinline__ int row_shift(const Phase& p, uint64_t row) { return WIDE ? 0 : (int)((p.first + (uint32_t)row * p.ld) & 7u); }

static __device__ __noinline__ uint4 load_some(const uint16_t* row, int c0, int cols) {
    uint16_t e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = (uint32_t)c0 + i < (uint32_t)cols ? row[c0 + i] : (uint16_t)0;
    return make_uint4(e[0] | (uint32_t)e[1] << 16, e[2] | (uint32_t)e[3] << 16, e[4] | (uint32_t)e[5] << 16, e[6] | (uint32_t)e[7] << 16);
}
// The first n of eight elements that start on a 16-byte boundary, the rest 0.
__device__ __forceinline__ uint4 load_begin(const uint16_t* p, int n) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = 2 * i + 1 < n ? reinterpret_cast<const uint32_t*>(p)[i] : 2 * i < n ? (uint32_t)p[2 * i] : 0u;
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// What of a chunk lies in the row, one element at a time.
static __device__ __noinline__ void store_each(uint16_t* row, int c0, int cols, uint4 v) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) if ((uint32_t)c0 + i < (uint32_t)cols) row[c0 + i] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
}
static __device__ __noinline__ void store_each_byte(uint8_t* row, int c0, int cols, uint2 v) {
#pragma unroll
    for (int i = 0; i < 8; ++i) if ((uint32_t)c0 + i < (uint32_t)cols) row[c0 + i] = (uint8_t)((i < 4 ? v.x : v.y) >> (8 * (i & 3)));
}
// A chunk on a boundary that is cut at one end: accesses of four, two and one elements.
__device__ __forceinline__ void store_some(uint16_t* row, int c0, int cols, uint4 v, uint32_t vec) {
    uint16_t* p = row + c0;
    if (!vec || (c0 < 0 && c0 > cols - 8)) {
        store_each(row, c0, cols, v);
    } else if (c0 >= 0) {                                              // the row's last n elements
        const int n = cols - c0;
        if (n & 4) { *reinterpret_cast<uint2*>(p) = make_uint2(v.x, v.y); v.x = v.z; v.y = v.w; p += 4; }
        if (n & 2) { *reinterpret_cast<uint32_t*>(p) = v.x; v.x = v.y; p += 2; }
        if (n & 1) *p = (uint16_t)v.x;
    } else {                                                           // its first n, at the chunk's end
        const int n = 8 + c0;
        if (n & 4) { *reinterpret_cast<uint2*>(p + 4) = make_uint2(v.z, v.w); v.z = v.x; v.w = v.y; p -= 4; }
        if (n & 2) { *reinterpret_cast<uint32_t*>(p + 6) = v.w; v.w = v.z; p -= 2; }
        if (n & 1) p[7] = (uint16_t)(v.w >> 16);
    }
}
__device__ __forceinline__ void store_some_bytes(uint8_t* row, int c0, int cols, uint2 v, uint32_t vec) {
    uint8_t* p = row + c0;
    if (!vec || (c0 < 0 && c0 > cols - 8)) {
        store_each_byte(row, c0, cols, v);
    } else if (c0 >= 0) {
        const int n = cols - c0;
        if (n & 4) { *reinterpret_cast<uint32_t*>(p) = v.x; v.x = v.y; p += 4; }
        if (n & 2) { *reinterpret_cast<uint16_t*>(p) = (uint16_t)v.x; v.x >>= 16; p += 2; }
        if (n & 1) *p = (uint8_t)v.x;
    } else {
        const int n = 8 + c0;
        if (n & 4) { *reinterpret_cast<uint32_t*>(p + 4) = v.y; v.y = v.x; p -= 4; }
        if (n & 2) { *reinterpret_cast<uint16_t*>(p + 6) = (uint16_t)(v.y >> 16); v.y <<= 16; p -= 2; }
        if (n & 1) p[7] = (uint8_t)(v.y >> 24);
    }
}
// Of eight elements from column c0 those outside the row become 0.
__device__ __forceinline__ void keep_row(uint4& v, int c0, int cols) {
    uint32_t* w = reinterpret_cast<uint32_t*>(&v);
#pragma unroll
    for (int i = 0; i < 4; ++i)
        w[i] &= ((uint32_t)c0 + 2 * i < (uint32_t)cols ? 0xFFFFu : 0u) | ((uint32_t)c0 + 2 * i + 1 < (uint32_t)cols ? 0xFFFF0000u : 0u);
}

// The first column of a row's chunk; `cols` where the chunk has none of the row's.  Rows may end next to 2^31.
__device__ __forceinline__ int chunk_col(uint32_t chunk, int shift, uint32_t cols) {
    return chunk * 8 < cols + (uint32_t)shift ? (int)(chunk * 8 - (uint32_t)shift) : (int)cols;
}

// One row to read.  A chunk at its end is read whole where that stays within the matrix: `head`, `tail`.
template <typename T>
struct RowIn {
    const T* p;
    bool vec, head, tail;
};
template <typename T, bool WIDE>
__device__ __forceinline__ RowIn<T> row_in(const InRows& m, uint64_t row, int cols) {
    const uint64_t at = row * m.ld;
    return {static_cast<const T*>(m.p) + at, WIDE || m.vec, WIDE || at >= 7, WIDE || at + (uint32_t)cols + 7 <= m.span};
}
// Elements c0 to c0 + 7 of a row.  What lies outside it is 0, or comes out as anything where row_keep8 does not follow: that waits for the
// load, so it stands where the values are used.
template <typename T, bool WIDE>
__device__ __forceinline__ Raw8<T> row_load8(const RowIn<T>& r, int c0, int cols) {
    Raw8<T> v{};
    if (c0 >= cols) return v;
    if (WIDE || (r.vec && (c0 >= 0 || (r.head && sizeof(T) == 2)) && (c0 <= cols - 8 || (r.tail && sizeof(T) == 2)))) {
        v.v = load_stream16(r.p + c0);
        if constexpr (sizeof(T) == 4) v.w = load_stream16(reinterpret_cast<const uint4*>(r.p + c0) + 1);
    } else if constexpr (sizeof(T) == 4) {
        uint32_t e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = (uint32_t)c0 + i < (uint32_t)cols ? __float_as_uint(r.p[c0 + i]) : 0u;
        v.v = make_uint4(e[0], e[1], e[2], e[3]);
        v.w = make_uint4(e[4], e[5], e[6], e[7]);
    } else {
        v.v = load_some(reinterpret_cast<const uint16_t*>(r.p), c0, cols);
    }
    return v;
}
template <typename T, bool WIDE>
__device__ __forceinline__ void row_keep8(Raw8<T>& v, int c0, int cols) {
    if constexpr (!WIDE && sizeof(T) == 2)
        if (c0 < 0 || c0 > cols - 8) keep_row(v.v, c0, cols);
}
// Elements c0 to c0 + 7 of a row that starts on a boundary while the chunk does not: they lie across two aligned eights.  The first one is
// loaded ahead, the second where they are used; it is some other thread's first one.  Zero outside the row.
template <typename T, bool WIDE>
__device__ __forceinline__ Raw8<T> across_load8(const InRows& m, int c0, int cols) {
    if constexpr (WIDE) {
        return row_load8<T, true>(RowIn<T>{static_cast<const T*>(m.p), true, true, true}, c0, cols);
    } else {
        Raw8<T> r{};
        const int c = c0 & ~7;
        const uint16_t* p = static_cast<const uint16_t*>(m.p);
        if (m.vec && c >= 0 && c < cols) r.v = c <= cols - 8 ? load_stream16(p + c) : load_begin(p + c, cols - c);
        return r;
    }
}
template <typename T, bool WIDE>
__device__ __forceinline__ Raw8<T> across_join8(const InRows& m, const Raw8<T>& first, int c0, int cols) {
    if constexpr (WIDE) {
        return first;
    } else {
        const int by = c0 & 7;
        if (m.vec && by == 0) return first;
        Raw8<T> r{};
        if (!m.vec) {
            if (c0 < cols) r.v = load_some(static_cast<const uint16_t*>(m.p), c0, cols);
            return r;
        }
        const uint4 a = first.v, b = across_load8<T, false>(m, c0 + 8, cols).v;
        uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
        if (by & 4)
#pragma unroll
            for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
        if (by & 2)
#pragma unroll
            for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
        if (by & 1)
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 16);
        r.v = make_uint4(w[0], w[1], w[2], w[3]);
        return r;
    }
}
template <typename T>
__device__ __forceinline__ void to_pairs(const Raw8<T>& r, Pair v[4]) {
    float f[8];
    to_floats(r, f);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = pair(f[2 * i], f[2 * i + 1]);
}
template <typename T, bool WIDE>
__device__ __forceinline__ void row_store8(const OutRows& m, uint64_t row, int c0, int cols, const Pair v[4]) {
    if (c0 >= cols) return;
    T* to = static_cast<T*>(m.p) + row * m.ld;
    const uint4 o = packed8<T>(v);
    if (WIDE || (m.vec && c0 >= 0 && c0 <= cols - 8)) *reinterpret_cast<uint4*>(to + c0) = o;
    else store_some(reinterpret_cast<uint16_t*>(to), c0, cols, o, m.vec);
}
template <bool WIDE>
__device__ __forceinline__ void row_store_bytes8(const OutRows& m, uint64_t row, int c0, int cols, uint2 b) {
    if (c0 >= cols) return;
    uint8_t* to = static_cast<uint8_t*>(m.p) + row * m.ld;
    if (WIDE || (m.vec && c0 >= 0 && c0 <= cols - 8)) *reinterpret_cast<uint2*>(to + c0) = b;
    else store_some_bytes(to, c0, cols, b, m.vec);
}
template <bool WIDE>
__device__ __forceinline__ uint2 row_load_bytes8(const InRows& m, uint64_t row, int c0, int cols) {
    if (c0 >= cols) return make_uint2(0u, 0u);
    const uint8_t* from = static_cast<const uint8_t*>(m.p) + row * m.ld;
    if (WIDE || (m.vec && c0 >= 0 && c0 <= cols - 8)) return load_stream8(from + c0);
    uint32_t b[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) b[i] = (uint32_t)c0 + i < (uint32_t)cols ? from[c0 + i] : 0u;
    return ckpt_join8(b);
}

}  // namespace sc
