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

struct Drop {
    uint64_t key;
    uint32_t cut;              // 0: everything is kept as it is; 65536: nothing is kept
    uint32_t groups;           // words a row
    float scale;
};

// Eight elements from column c0, a multiple of 8.  What is dropped is 0 whatever it was.
__device__ __forceinline__ void drop8(const Drop& d, uint64_t row, uint32_t c0, float f[8]) {
    const uint64_t at = row * d.groups + (c0 >> 2);
    const uint64_t w[2] = {mix64(d.key, at), mix64(d.key, at + 1)};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t bits = (uint32_t)(w[i >> 2] >> (16 * (i & 3))) & 0xFFFFu;
        f[i] = bits >= d.cut ? f[i] * d.scale : 0.0f;
    }
}

// The same from any column, before the row's first as well: the elements of other rows may come out as anything.
__device__ __forceinline__ void drop8_any(const Drop& d, uint64_t row, int c0, float f[8]) {
    const uint64_t at = row * d.groups + (uint64_t)(int64_t)(c0 >> 2);
    const uint32_t by = 16 * (c0 & 3);
    uint64_t w[2] = {mix64(d.key, at), mix64(d.key, at + 1)};
    if (by) {
        const uint64_t next = mix64(d.key, at + 2);
        w[0] = w[0] >> by | w[1] << (64 - by);
        w[1] = w[1] >> by | next << (64 - by);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t bits = (uint32_t)(w[i >> 2] >> (16 * (i & 3))) & 0xFFFFu;
        f[i] = bits >= d.cut ? f[i] * d.scale : 0.0f;
    }
}
template <bool WIDE>
__device__ __forceinline__ void drop_pairs(const Drop& d, uint64_t row, int c0, Pair v[4]) {
    float f[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) { const float2 p = both(v[i]); f[2 * i] = p.x; f[2 * i + 1] = p.y; }
    if constexpr (WIDE) drop8(d, row, (uint32_t)c0, f);
    else drop8_any(d, row, c0, f);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = pair(f[2 * i], f[2 * i + 1]);
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
                if (a.drop.cut) drop_pairs<WIDE>(a.drop, from.row, c0, v);
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
