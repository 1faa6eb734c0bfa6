// Rows of any alignment, eight elements a thread.
//
// A row is cut where its 16-bit elements cross 16-byte boundaries: into whole chunks of eight elements between two boundaries, and its
// ends, up to seven elements before the first boundary and up to seven after the last, which one warp handles one element a lane.
// Matrices of one odd width have the same cut in the same row, so all of them move in whole accesses; one whose rows are cut elsewhere
// has its chunks moved in single elements.  WIDE is the case without ends: every row starts on a boundary and is a multiple of 8 long.
// With checks for the ends at each chunk instead, rows of 4097 took 1.5 to 2.6 times as long as rows of 4096; now it is 1.1 to 1.3.
#pragma once
#include "sc_checkpoint.cuh"

namespace sc {

// A matrix to read.  `vec`: its rows are cut as the phase says (and chunks are 16-byte accesses).
struct InRows {
    const void* p;
    uint64_t ld;
    uint32_t vec;
};
struct OutRows {
    void* p;
    uint64_t ld;
    uint32_t vec;
};
// Row r starts (first + r ld) mod 8 elements past a boundary.
struct Phase { uint32_t first, ld; };

// Whether thread t of a team is in its last warp, which has the rows' ends.
template <int TEAM>
__device__ __forceinline__ bool last_warp(uint32_t t) {
    if constexpr (TEAM == 32) return true;
    else return t >= TEAM - 32;
}
// A row's cut: `lead` elements, `whole` chunks from there, and the rest.
struct RowCut { int lead; uint32_t whole; };
template <bool WIDE>
__device__ __forceinline__ RowCut row_cut(const Phase& p, uint64_t row, uint32_t cols) {
    if constexpr (WIDE) return {0, cols / 8};
    const uint32_t lead = min((8u - (p.first + (uint32_t)row * p.ld)) & 7u, cols);
    return {(int)lead, (cols - lead) / 8};
}
// The column of the ends' element that a lane has, -1: none.  Lanes 0 to 6 have the elements before the chunks, 8 to 14 those behind.
__device__ __forceinline__ int end_col(const RowCut& cut, uint32_t cols, uint32_t lane) {
    const uint32_t rest = (uint32_t)cut.lead + cut.whole * 8, l = lane - 8;
    return lane < 8 ? (lane < (uint32_t)cut.lead ? (int)lane : -1) : l < 8 && rest + l < cols ? (int)(rest + l) : -1;
}

// Eight elements of any alignment.
static __device__ __noinline__ uint4 load_each(const uint16_t* p) {
    uint32_t e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = p[i];
    return make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
}
static __device__ __noinline__ void store_each(uint16_t* p, uint4 v) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
}
static __device__ __noinline__ uint2 load_each_byte(const uint8_t* p) {
    uint32_t b[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) b[i] = p[i];
    return ckpt_join8(b);
}
static __device__ __noinline__ void store_each_byte(uint8_t* p, uint2 v) {
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = (uint8_t)((i < 4 ? v.x : v.y) >> (8 * (i & 3)));
}
// The first n of eight elements that start on a 16-byte boundary, the rest 0.
__device__ __forceinline__ uint4 load_begin(const uint16_t* p, int n) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = 2 * i + 1 < n ? reinterpret_cast<const uint32_t*>(p)[i] : 2 * i < n ? (uint32_t)p[2 * i] : 0u;
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// The whole chunk from column c of a row that begins at `row`.
template <typename T, bool WIDE>
__device__ __forceinline__ Raw8<T> chunk_load8(const InRows& m, const T* row, int c) {
    Raw8<T> v{};
    if (WIDE || m.vec) {
        v.v = load_stream16(row + c);
        if constexpr (sizeof(T) == 4) v.w = load_stream16(reinterpret_cast<const uint4*>(row + c) + 1);
    } else if constexpr (sizeof(T) == 2) {
        v.v = load_each(reinterpret_cast<const uint16_t*>(row) + c);
    }
    return v;
}
template <typename T>
__device__ __forceinline__ const T* row_of(const InRows& m, uint64_t row) { return static_cast<const T*>(m.p) + row * m.ld; }
template <typename T>
__device__ __forceinline__ T* row_of(const OutRows& m, uint64_t row) { return static_cast<T*>(m.p) + row * m.ld; }

// Elements c0 to c0 + 7 of one row that starts on a boundary while the chunk does not: they lie across two aligned eights.  The first one is
// loaded ahead, the second where they are used; it is some other thread's first one.
template <typename T, bool WIDE>
__device__ __forceinline__ Raw8<T> across_load8(const InRows& m, int c0, int cols) {
    Raw8<T> r{};
    const int c = c0 & ~7;
    if (WIDE || (m.vec && c <= cols - 8)) r.v = load_stream16(static_cast<const T*>(m.p) + c);
    else if (m.vec && c < cols) r.v = load_begin(static_cast<const uint16_t*>(m.p) + c, cols - c);
    return r;
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
            r.v = load_each(static_cast<const uint16_t*>(m.p) + c0);
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
__device__ __forceinline__ void chunk_store8(const OutRows& m, T* row, int c, const Pair v[4]) {
    const uint4 o = packed8<T>(v);
    if (WIDE || m.vec) *reinterpret_cast<uint4*>(row + c) = o;
    else store_each(reinterpret_cast<uint16_t*>(row) + c, o);
}
template <bool WIDE>
__device__ __forceinline__ void chunk_store_bytes8(const OutRows& m, uint8_t* row, int c, uint2 b) {
    if (WIDE || m.vec) *reinterpret_cast<uint2*>(row + c) = b;
    else store_each_byte(row + c, b);
}
__device__ __forceinline__ uint2 chunk_load_bytes8(const InRows& m, const uint8_t* row, int c) {
    return m.vec ? load_stream8(row + c) : load_each_byte(row + c);
}
// One element, and a number rounded to one.
template <typename T> __device__ __forceinline__ float element(T v) { return (float)v; }
template <typename T> __device__ __forceinline__ T rounded(float v);
template <> __device__ __forceinline__ __nv_bfloat16 rounded<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half rounded<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ float rounded<float>(float v) { return v; }

}  // namespace sc
