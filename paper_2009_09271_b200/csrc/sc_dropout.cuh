// Dropout whose mask is made, not stored: sixteen bits an element from the counter-based generator.
//
// Four neighbouring elements of a row share one 64-bit word, mix64(key, row * ceil(cols / 4) + column / 4), the first of them its
// low 16 bits.  An element is kept where its bits, as an integer, are at least `cut`; what is kept is scaled by 65536 / (65536 - cut),
// the reciprocal of the probability that the bits really give, so that the mean stays the input's.  The gradient is the same
// call on the gradient.
#pragma once
#include "sc_common.cuh"
#include "sc_rows.cuh"

namespace sc {

constexpr uint64_t SALT_DROPOUT = 0x64726F70ull;

// mix64(a, b) mixes a + (b + 1) GENERATOR_STEP: neighbouring words are a step apart before they are mixed.
constexpr uint64_t GENERATOR_STEP = 0x9E3779B97F4A7C15ull;

struct Drop {
    uint64_t key;
    uint32_t cut;              // 0: everything is kept as it is; 65536: nothing is kept
    uint32_t groups;           // words a row
    float scale;
};

// A row's words, and the ones around them: word j is mix64(key, row * groups + j).
__device__ __forceinline__ uint64_t drop_row(const Drop& d, uint64_t row) { return d.key + row * d.groups * GENERATOR_STEP; }

// Four elements and their word.  What is dropped is 0 whatever it was.
__device__ __forceinline__ void drop4(const Drop& d, uint64_t word, Pair v[2]) {
    const uint32_t lo = (uint32_t)word, hi = (uint32_t)(word >> 32);
    const float2 a = both(v[0]), b = both(v[1]);
    v[0] = pair((lo & 0xFFFFu) >= d.cut ? a.x * d.scale : 0.0f, (lo >> 16) >= d.cut ? a.y * d.scale : 0.0f);
    v[1] = pair((hi & 0xFFFFu) >= d.cut ? b.x * d.scale : 0.0f, (hi >> 16) >= d.cut ? b.y * d.scale : 0.0f);
}
// Eight elements from column c0 of the row whose words begin at `base`.  Where c0 is no multiple of 4 they lie across three words.
template <bool WIDE>
__device__ __forceinline__ void drop_pairs(const Drop& d, uint64_t base, int c0, Pair v[4]) {
    const uint64_t z = base + (uint64_t)(int64_t)(c0 >> 2) * GENERATOR_STEP;
    uint64_t w[2] = {mix64(z, 0), mix64(z + GENERATOR_STEP, 0)};
    if (!WIDE && (c0 & 3)) {
        const uint32_t by = 16 * (c0 & 3);
        const uint64_t next = mix64(z + 2 * GENERATOR_STEP, 0);
        w[0] = w[0] >> by | w[1] << (64 - by);
        w[1] = w[1] >> by | next << (64 - by);
    }
    drop4(d, w[0], v);
    drop4(d, w[1], v + 2);
}
// The element of column c alone.
__device__ __forceinline__ float drop1(const Drop& d, uint64_t base, int c, float v) {
    const uint64_t word = mix64(base + (uint64_t)(c >> 2) * GENERATOR_STEP, 0);
    return ((uint32_t)(word >> (16 * (c & 3))) & 0xFFFFu) >= d.cut ? v * d.scale : 0.0f;
}
__device__ __forceinline__ void drop8(const Drop& d, uint64_t row, uint32_t c0, float f[8]) {
    Pair v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = pair(f[2 * i], f[2 * i + 1]);
    drop_pairs<true>(d, drop_row(d, row), (int)c0, v);
#pragma unroll
    for (int i = 0; i < 4; ++i) { const float2 p = both(v[i]); f[2 * i] = p.x; f[2 * i + 1] = p.y; }
}

// y = residual + dropout(x).  A team of threads has a row, or with blockIdx.y a part of one, V times eight elements a thread at a time, so that a
// row's words have one base: found anew for every eight elements it was half the generator's cost.  16384 x 8192 bf16: onto a residual 124 us
// (6.5 TB/s, 0.99 of the measured copy rate; 135 with the base found anew), without one 93 (0.88), where the generator's 64-bit products,
// at half the multiply-add rate, are what is left beside HBM.
struct DropArgs {
    uint64_t rows;
    InRows x, residual;
    OutRows y;
    uint32_t cols;
    Phase phase;
    Drop drop;
};
template <typename T, int TEAM, int V, bool RESIDUAL, bool WIDE>
__global__ void __launch_bounds__(TEAM == 32 ? 256 : TEAM) dropout_kernel(DropArgs a) {
    constexpr int TEAMS = TEAM == 32 ? 8 : 1;
    wait_for_predecessor();
    release_successor();
    const uint32_t t = TEAM == 32 ? threadIdx.x & 31u : threadIdx.x;
    const uint64_t row = (uint64_t)blockIdx.x * TEAMS + (TEAM == 32 ? threadIdx.x >> 5 : 0u);
    if (row >= a.rows) return;
    const RowCut cut = row_cut<WIDE>(a.phase, row, a.cols);
    const T *x = row_of<T>(a.x, row), *res = row_of<T>(a.residual, row);
    T* y = row_of<T>(a.y, row);
    const uint64_t base = drop_row(a.drop, row);
    if (!WIDE && blockIdx.y == 0 && last_warp<TEAM>(t)) {                  // the ends
        const int c = end_col(cut, a.cols, t & 31u);
        if (c >= 0) {
            float f = element(x[c]);
            if (a.drop.cut) f = drop1(a.drop, base, c, f);
            if (RESIDUAL) f += element(res[c]);
            y[c] = rounded<T>(f);
        }
    }
    for (uint32_t first = blockIdx.y * (TEAM * V) + t; first < cut.whole; first += gridDim.y * (TEAM * V)) {
        Raw8<T> in[V], add[V];
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (first + j * TEAM < cut.whole) {
                const int c = cut.lead + (int)(first + j * TEAM) * 8;
                in[j] = chunk_load8<T, WIDE>(a.x, x, c);
                if (RESIDUAL) add[j] = chunk_load8<T, WIDE>(a.residual, res, c);
            }
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (first + j * TEAM < cut.whole) {
                const int c = cut.lead + (int)(first + j * TEAM) * 8;
                Pair v[4];
                to_pairs(in[j], v);
                if (a.drop.cut) drop_pairs<WIDE>(a.drop, base, c, v);
                if constexpr (RESIDUAL) {
                    Pair r[4];
                    to_pairs(add[j], r);
#pragma unroll
                    for (int k = 0; k < 4; ++k) v[k] = v[k] + r[k];
                }
                chunk_store8<T, WIDE>(a.y, y, c, v);
            }
    }
}

}  // namespace sc
