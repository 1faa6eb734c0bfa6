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
// Eight elements from column c0 of the row whose words begin at `base`.  Where c0 is no multiple of 4 they lie across three words; the elements
// of other rows may come out as anything.
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
__device__ __forceinline__ void drop8(const Drop& d, uint64_t row, uint32_t c0, float f[8]) {
    Pair v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = pair(f[2 * i], f[2 * i + 1]);
    drop_pairs<true>(d, drop_row(d, row), (int)c0, v);
#pragma unroll
    for (int i = 0; i < 4; ++i) { const float2 p = both(v[i]); f[2 * i] = p.x; f[2 * i + 1] = p.y; }
}

// y = residual + dropout(x), eight elements a thread and item, several items in flight.
struct DropArgs {
    InRows x, residual;
    OutRows y;
    Phase phase;
    Drop drop;
};
constexpr int DROP_UNROLL = 4;
template <typename T, bool RESIDUAL, bool WIDE>
__global__ void __launch_bounds__(CKPT_THREADS) dropout_kernel(ItemWalk w, DropArgs a) {
    wait_for_predecessor();
    release_successor();
    const uint64_t first = (uint64_t)blockIdx.x * CKPT_THREADS + threadIdx.x, stride = (uint64_t)gridDim.x * CKPT_THREADS;
    const int cols = (int)w.cols;
    ItemAt at(w, first);
    for (uint64_t base = first; base < w.total; base += stride * DROP_UNROLL) {
        Raw8<T> in[DROP_UNROLL], res[DROP_UNROLL];
        ItemAt from = at;
#pragma unroll
        for (int u = 0; u < DROP_UNROLL; ++u) {
            if (base + u * stride < w.total) {
                const int c0 = chunk_col(at.item, row_shift<WIDE>(a.phase, at.row), w.cols);
                in[u] = row_load8<T, WIDE>(row_in<T, WIDE>(a.x, at.row, cols), c0, cols);
                if (RESIDUAL) res[u] = row_load8<T, WIDE>(row_in<T, WIDE>(a.residual, at.row, cols), c0, cols);
            }
            at.next(w);
        }
#pragma unroll
        for (int u = 0; u < DROP_UNROLL; ++u) {
            if (base + u * stride < w.total) {
                const int c0 = chunk_col(from.item, row_shift<WIDE>(a.phase, from.row), w.cols);
                Pair v[4];
                to_pairs(in[u], v);
                if (a.drop.cut) drop_pairs<WIDE>(a.drop, drop_row(a.drop, from.row), c0, v);
                if constexpr (RESIDUAL) {
                    Pair r[4];
                    to_pairs(res[u], r);
#pragma unroll
                    for (int k = 0; k < 4; ++k) v[k] = v[k] + r[k];
                }
                row_store8<T, WIDE>(a.y, from.row, c0, cols, v);
            }
            from.next(w);
        }
    }
}

}  // namespace sc
