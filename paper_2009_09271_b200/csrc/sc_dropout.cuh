// Dropout whose mask is made, not stored: sixteen bits an element from the counter-based generator.
//
// Four neighbouring elements of a row share one 64-bit word, mix64(key, row * ceil(cols / 4) + column / 4), the first of them its
// low 16 bits.  An element is kept where its bits, as an integer, are at least `cut`; what is kept is scaled by 65536 / (65536 - cut),
// the reciprocal of the probability that the bits really give, so that the mean stays the input's.  The gradient is the same
// call on the gradient.
#pragma once
#include "sc_checkpoint.cuh"
#include "sc_common.cuh"

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

struct DropArgs {
    uint64_t ldx, ldr, ldy;
    uint32_t grain_x, grain_r, grain_y;
    Drop drop;
};

// y = residual + dropout(x): one pass, eight elements a thread and item.
template <typename T>
__global__ void __launch_bounds__(CKPT_THREADS) dropout_kernel(const T* x, const T* residual, T* y, ItemWalk w, DropArgs a) {
    wait_for_predecessor();
    release_successor();
    const uint64_t first = (uint64_t)blockIdx.x * CKPT_THREADS + threadIdx.x, stride = (uint64_t)gridDim.x * CKPT_THREADS;
    ItemAt at(w, first);
    for (uint64_t i = first; i < w.total; i += stride, at.next(w)) {
        const uint32_t c0 = at.item * 8;
        float f[8], r[8];
        to_floats(load8(x + at.row * a.ldx, c0, w.cols, a.grain_x), f);
        if (residual) to_floats(load8(residual + at.row * a.ldr, c0, w.cols, a.grain_r), r);
        if (a.drop.cut) drop8(a.drop, at.row, c0, f);
        if (residual)
#pragma unroll
            for (int k = 0; k < 8; ++k) f[k] += r[k];
        store8(y + at.row * a.ldy, c0, w.cols, a.grain_y, f);
    }
}

}  // namespace sc
