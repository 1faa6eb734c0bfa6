// The layer's three matrix products, out[i, j] = sum_r A[i, r] B[j, r], and what follows each in its epilogue:
//   forward       y  = act(x W^T + b) + residual          A = x [M, K],   B = W [N, K],    r over K
//   input grad    dx = (dz W + residual) * act'(z^)       A = dz [M, N],  B = W^T [K, N],  r over N
//   weight grad   dW (+)= dz^T x^                         A = dz^T [N, M], B = x^T [K, M], r over M
#pragma once
#include "sc_checkpoint.cuh"
#include "sc_layer_common.cuh"
#include "sc_tcgen05.cuh"

namespace sc {

enum { PRODUCT_FORWARD = 0, PRODUCT_INPUT = 1, PRODUCT_WEIGHT = 2 };

struct Epilogue {
    const void* bias;          // forward: [cols] or null
    const void* residual;      // forward, input grad: rows of ldr, or null
    void* out;                 // 16-bit rows of ldo; weight grad: fp32 rows of ldo
    uint8_t* q;                // forward: checkpoint of z to write, or null; input grad: checkpoint to read, or null
    uint8_t* scales;
    uint64_t ldr, ldo, rows;
    uint32_t cols, groups;
    int act;
    uint32_t accumulate;
    uint32_t grain_out, grain_res, grain_q, grain_bias;      // elements that one access of a row may take
    uint32_t scales_by4;       // block_rows: four neighbouring scales of a row go out in one access
};

// What follows the product for 8 columns from c0 of one row.  All 32 lanes of a warp call it; four neighbouring lanes hold
// 32 consecutive columns of one row, from a multiple of 32, so they share a checkpoint group.  `bias`: of these columns.
// `slot`: 0, or the row's 128 bytes of shared memory, where the 16-bit result and the checkpoint's bytes (from byte 64) are
// left for rows_out instead of being written to rows that take narrow accesses only.
template <typename T, int MODE, int ACT>
__device__ __forceinline__ void epilogue8(const Epilogue& ep, uint64_t row, uint32_t c0, const float bias[8], float v[8], uint32_t slot = 0) {
    const bool in = row < ep.rows && c0 < ep.cols;
    if constexpr (MODE == PRODUCT_WEIGHT) {
        if (!in) return;
        float* out = static_cast<float*>(ep.out) + row * ep.ldo + c0;
        if (ep.accumulate) {
#pragma unroll
            for (int i = 0; i < 8; ++i) if (c0 + i < ep.cols) out[i] += v[i];
        } else {
            store8(out - c0, c0, ep.cols, ep.grain_out, v);
        }
    } else {
        float res[8] = {};
        if (in && ep.residual) to_floats(load8(static_cast<const T*>(ep.residual) + row * ep.ldr, c0, ep.cols, ep.grain_res), res);
        if constexpr (MODE == PRODUCT_FORWARD) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += bias[i];
            if (ep.q) {
                uint32_t m = 0;                         // columns past the end hold zeros: no product, no bias
#pragma unroll
                for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7FFFFFFFu);
                m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
                m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 2));
                int e;
                const uint2 b = ckpt_encode8<T>(v, m, e);
                if (slot) asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(slot + 64 + (c0 & 31u)), "r"(b.x), "r"(b.y) : "memory");
                if (in) {
                    if (!slot) store_q8(ep.q + row * ep.cols + c0, c0, ep.cols, ep.grain_q, b);
                    if ((c0 & 31u) == 0u) ep.scales[row * ep.groups + (c0 >> 5)] = (uint8_t)(e + 127);
                }
            }
            if (!in) return;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 f = both(activation<ACT>(pair(v[2 * i], v[2 * i + 1])) + pair(res[2 * i], res[2 * i + 1]));
                v[2 * i] = f.x; v[2 * i + 1] = f.y;
            }
        } else {
            if (!in) return;
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += res[i];
            if constexpr (ACT != SC_ACT_NONE) {
                const uint2 k = load_q8(ep.q + row * ep.cols, c0, ep.cols, ep.grain_q);
                const Scale s = slope_scale(ep.scales[row * ep.groups + (c0 >> 5)]);
                Pair z[4];
                ckpt_values8<false>(k, s, z);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 f = both(pair(v[2 * i], v[2 * i + 1]) * activation_slope<ACT>(z[i]));
                    v[2 * i] = f.x; v[2 * i + 1] = f.y;
                }
            }
        }
        if (slot) {
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(slot + (c0 & 31u) * 2), "r"(Elem<T>::pack(v[0], v[1])), "r"(Elem<T>::pack(v[2], v[3])),
                         "r"(Elem<T>::pack(v[4], v[5])), "r"(Elem<T>::pack(v[6], v[7])) : "memory");
        } else {
            store8(static_cast<T*>(ep.out) + row * ep.ldo, c0, ep.cols, ep.grain_out, v);
        }
    }
}

// The 32 x 32 block that epilogue8 left in shared memory, to rows of any alignment: neighbouring lanes write neighbouring
// elements, two at a time where the rows allow.
static __device__ __noinline__ void rows_out(const Epilogue& ep, uint32_t stage_addr, uint64_t row0, uint32_t col0, bool kept) {
    const uint32_t lane = threadIdx.x & 31u;
    const uint32_t rows = row0 < ep.rows ? (uint32_t)min((uint64_t)32, ep.rows - row0) : 0u, cols = col0 < ep.cols ? min(32u, ep.cols - col0) : 0u;
    uint16_t* y = static_cast<uint16_t*>(ep.out) + row0 * ep.ldo + col0;
    if (ep.grain_out >= 2) {
        const uint32_t c = (lane & 15u) * 2;
#pragma unroll 4
        for (uint32_t r = lane >> 4; r < rows; r += 2) {
            uint32_t v;
            asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(stage_addr + r * 128 + c * 2) : "memory");
            if (c + 1 < cols) *reinterpret_cast<uint32_t*>(y + r * ep.ldo + c) = v;
            else if (c < cols) y[r * ep.ldo + c] = (uint16_t)v;
        }
    } else {
#pragma unroll 4
        for (uint32_t r = 0; r < rows; ++r) {
            uint16_t v;
            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(stage_addr + r * 128 + lane * 2) : "memory");
            if (lane < cols) y[r * ep.ldo + lane] = v;
        }
    }
    if (!kept) return;
    uint8_t* q = ep.q + row0 * ep.cols + col0;
    if (ep.grain_q >= 2) {
        const uint32_t c = (lane & 15u) * 2;
#pragma unroll 4
        for (uint32_t r = lane >> 4; r < rows; r += 2) {
            uint16_t v;
            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(stage_addr + r * 128 + 64 + c) : "memory");
            if (c + 1 < cols) *reinterpret_cast<uint16_t*>(q + (uint64_t)r * ep.cols + c) = v;
            else if (c < cols) q[(uint64_t)r * ep.cols + c] = (uint8_t)v;
        }
    } else {
#pragma unroll 4
        for (uint32_t r = 0; r < rows; ++r) {
            uint32_t v;
            asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(stage_addr + r * 128 + 64 + lane) : "memory");
            if (lane < cols) q[(uint64_t)r * ep.cols + lane] = (uint8_t)v;
        }
    }
}

// The bias of 8 columns; zero past the end.
template <typename T, int MODE>
__device__ __forceinline__ void load_bias(const Epilogue& ep, uint32_t c0, float b[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) b[i] = 0.0f;
    if constexpr (MODE == PRODUCT_FORWARD)
        if (ep.bias && c0 < ep.cols) to_floats(load8(static_cast<const T*>(ep.bias), c0, ep.cols, ep.grain_bias), b);
}

// ---------------------------------------------------------------------------
// The product on the 5th-generation tensor cores
// ---------------------------------------------------------------------------
// CTAs (CG = 1) or pairs of CTAs that share one matrix instruction (CG = 2) walk output tiles of 128 CG x BN; each CTA of
// a pair holds 128 rows of A, half of B's rows, and the accumulator of its own 128 output rows.  A producer warp streams
// 64-deep slices of both operands into a ring of shared-memory stages by TMA (128-byte swizzle; edges are filled with
// zeros), one thread issues the matrix instructions into one of two accumulators in TMEM, and eight warps empty the
// other one.  A 16-bit result leaves by block_rows, rows that do not take 16-byte accesses by block_out, which moves
// 32 x 32 blocks through shared memory so that neighbouring lanes work along rows.
//
// Bound by the tensor pipe and, where calls follow each other, by the power cap (1000 W; SM clock 1.2-1.5 GHz).
// 8192 x 16384 x 4096 bf16: forward 775-840 us (1.31-1.42 PFLOP/s; the library's product alone 772-800 us beside it), with tanh
// gelu and checkpoint 832-900 us, input gradient 790-890 us, weight gradient 850-935 us.  At 4096 x 8192 x 4096 the tensor
// pipe is active for 78 to 82 % of the elapsed cycles.  What it took: pairs of CTAs (B read once a pair), the issuing warp kept
// converged with one elected lane (a branch on the lane number cost 10 %), an accumulator hand-over without a release at
// cluster scope, and the epilogue's loops rolled (fetched cold, they were most of a small call).
//
// The tensor cores add to an fp32 accumulator by cutting, not rounding: measured, a sum of n steps of 16 products comes
// out about n 2^-24 of its size too small (2e-7 after 256 products, 9e-6 after 8192, 4e-5 after 32768 of random sign).  A
// bf16 result does not see that; of an fp16 one 16384 products of one sign take up to a quarter of a half step.  The weight gradient is fp32, so its accumulators are emptied every 6 blocks
// (384 products) and added up in registers, with rounding: 3.6e-7 after 8192, at the price of 3 to 5 % of the time.
constexpr int TC_ROWS = 128, TC_STEP = 64, TC_THREADS = 384, TC_EPI_WARPS = 8, TC_CHUNK = 6;
constexpr int TC_LEAST_REGS = 160;             // 160 x 384 >= 56 x 128 + 208 x 256, for builds that shift registers
constexpr uint32_t TC_SMEM_LIMIT = 232448;

template <int BN, int CG>
struct TcShape {
    static constexpr int B_ROWS = BN / CG;
    static constexpr uint32_t A_BYTES = TC_ROWS * TC_STEP * 2, B_BYTES = B_ROWS * TC_STEP * 2, STAGE = A_BYTES + B_BYTES;
    static constexpr uint32_t STAGING = TC_EPI_WARPS * 32 * 32 * 4;
    static constexpr int STAGES = (TC_SMEM_LIMIT - 1024 - 256 - STAGING) / STAGE > 8 ? 8 : (TC_SMEM_LIMIT - 1024 - 256 - STAGING) / STAGE;
    static constexpr uint32_t SMEM = STAGES * STAGE + STAGING + 1024 + 256;
    static constexpr uint32_t TMEM_COLS = 2 * BN;
};

struct TcArgs {
    uint32_t tiles_i, tiles_j, tiles;      // output tiles
    uint32_t splits;                       // parts of the reduction; more than one: fp32 partial sums go to `partial`
    uint32_t blocks;                       // reduction blocks of 64
    uint32_t idesc, a_box_rows;
    uint64_t part_stride;                  // elements between two parts
    uint32_t part_ld;
    uint32_t tma_out;                      // fp32 goes out by TMA: partial sums always, the weight gradient where its rows allow
    uint32_t rows_form;                    // 16-bit result and all that goes with it: rows take 16-byte accesses (q: 8-byte)
    float* partial;
    int* status;
};

// Tiles in groups of 8 rows of tiles, down the rows first, so that the tiles in flight share operands in L2.
__device__ __forceinline__ void tile_at(const TcArgs& a, uint32_t t, uint32_t& ti, uint32_t& tj) {
    const uint32_t per = 8 * a.tiles_j, g = t / per, first = g * 8, high = min(8u, a.tiles_i - first), in = t - g * per;
    ti = first + in % high;
    tj = in / high;
}

// One 32 x 32 block, thread t holding row t, to its place.  The 16-byte units of a row are permuted by its number, which
// makes both directions free of bank conflicts.
template <typename T, int MODE>
__device__ __forceinline__ void block_out(const CUtensorMap* map_out, const TcArgs& a, const Epilogue& ep, uint32_t stage_addr, const uint32_t (&v)[32], uint64_t row0, uint32_t col0,
                                          uint32_t split) {
    const uint32_t lane = threadIdx.x & 31u;
    if (a.tma_out) {                       // the last block's copy has left the buffer
        if (lane == 0) tma_store_wait_read();
        __syncwarp();
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) {
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(stage_addr + lane * 128 + ((u ^ (lane & 7)) * 16)),
                     "r"(v[4 * u]), "r"(v[4 * u + 1]), "r"(v[4 * u + 2]), "r"(v[4 * u + 3]) : "memory");
    }
    __syncwarp();
    const uint32_t c0 = col0 + (lane & 3u) * 8;
    const auto fetch = [&](int i, float f[8]) {
        const uint32_t r = (lane >> 2) + 8 * i, u = (lane & 3u) * 2;
        asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(f[0]), "=f"(f[1]), "=f"(f[2]), "=f"(f[3])
                     : "r"(stage_addr + r * 128 + ((u ^ (r & 7)) * 16)) : "memory");
        asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(f[4]), "=f"(f[5]), "=f"(f[6]), "=f"(f[7])
                     : "r"(stage_addr + r * 128 + (((u + 1) ^ (r & 7)) * 16)) : "memory");
        return row0 + r;
    };
    if (a.tma_out) {                       // the permutation above is the 128-byte swizzle
        smem_to_async_fence();
        __syncwarp();
        if (lane == 0 && row0 < ep.rows && col0 < ep.cols) {
            // the addition happens in L2, without waiting for what is there: one per element, so in no order that could change
            if (MODE == PRODUCT_WEIGHT && ep.accumulate && a.splits == 1) tma_add_3d(map_out, stage_addr, (int32_t)col0, (int32_t)row0, 0);
            else tma_store_3d(map_out, stage_addr, (int32_t)col0, (int32_t)row0, (int32_t)split);
            tma_store_commit();
        }
        return;
    }
    if constexpr (MODE == PRODUCT_WEIGHT) {
        // Rows at any 4-byte offset: one row of 32 a store, eight rows at a time.
        const uint32_t c = col0 + lane;
        float* out = static_cast<float*>(ep.out) + row0 * ep.ldo + c;
        const uint32_t rows = c < ep.cols && row0 < ep.rows ? (uint32_t)min((uint64_t)32, ep.rows - row0) : 0u;
#pragma unroll 1
        for (uint32_t r0 = 0; r0 < 32; r0 += 8) {
            float f[8];
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i)
                asm volatile("ld.shared.f32 %0, [%1];" : "=f"(f[i]) : "r"(stage_addr + (r0 + i) * 128 + (((lane >> 2) ^ i) * 16) + (lane & 3u) * 4) : "memory");
            if (ep.accumulate) {
#pragma unroll
                for (uint32_t i = 0; i < 8; ++i, out += ep.ldo)
                    if (r0 + i < rows) asm volatile("red.relaxed.gpu.global.add.f32 [%0], %1;" ::"l"(out), "f"(f[i]) : "memory");
            } else {
#pragma unroll
                for (uint32_t i = 0; i < 8; ++i, out += ep.ldo)
                    if (r0 + i < rows) *out = f[i];
            }
        }
    } else {
        float bias[8];
        load_bias<T, MODE>(ep, c0, bias);
        const bool narrow = ep.grain_out == 1 || (MODE == PRODUCT_FORWARD && ep.q && ep.grain_q == 1);
        with_activation(ep.act, [&](auto act) {
#pragma unroll 1                                              // little code: it is fetched cold in a small call
            for (int i = 0; i < 4; ++i) {
                float f[8];
                const uint64_t row = fetch(i, f);
                if (narrow) __syncwarp();                     // the row's four lanes have read it
                epilogue8<T, MODE, decltype(act)::value>(ep, row, c0, bias, f, narrow ? stage_addr + (uint32_t)(row - row0) * 128 : 0u);
            }
        });
        if (narrow) {
            __syncwarp();
            rows_out(ep, stage_addr, row0, col0, MODE == PRODUCT_FORWARD && ep.q);
        }
    }
    __syncwarp();
}

// One 32 x 32 block of a 16-bit result, thread t holding row t from TMEM to the end: a checkpoint group is one thread's own, its
// bytes go out as one sector, and the result leaves by TMA from a 2 KB buffer of 64-byte rows (64-byte swizzle), two of
// which take turns.  About a third of the instructions of block_out, which serves rows of other alignments.
template <typename T, int MODE, int ACT>
__device__ __forceinline__ void block_rows(const CUtensorMap* map_out, const Epilogue& ep, uint32_t buffer, const uint32_t (&v)[32], uint64_t row0,
                                           uint32_t col0, uint32_t& scale4) {
    const uint32_t lane = threadIdx.x & 31u;
    const uint64_t row = row0 + lane;
    const bool in = row < ep.rows && col0 < ep.cols, whole = col0 + 32 <= ep.cols;
    Pair z[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = pair(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1]));
    if constexpr (MODE == PRODUCT_FORWARD) {
        if (ep.bias) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float b[8];
                load_bias<T, MODE>(ep, col0 + 8 * j, b);
#pragma unroll
                for (int i = 0; i < 4; ++i) z[4 * j + i] = z[4 * j + i] + pair(b[2 * i], b[2 * i + 1]);
            }
        }
        if (ep.q) {
            uint32_t m = 0;                                 // columns past the end hold no product and no bias
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float2 f = both(z[i]);
                m = max(max(m, __float_as_uint(f.x) & 0x7FFFFFFFu), __float_as_uint(f.y) & 0x7FFFFFFFu);
            }
            int e = ckpt_exponent<T>(m);
            const bool odd = m >= 0x7F800000u || e == Elem<T>::EMAX;
            if (odd) {
                m = 0;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float2 f = both(z[i]);
                    const uint32_t a = __float_as_uint(f.x) & 0x7FFFFFFFu, b = __float_as_uint(f.y) & 0x7FFFFFFFu;
                    m = max(max(m, a < 0x7F800000u ? a : 0u), b < 0x7F800000u ? b : 0u);
                }
                e = ckpt_exponent<T>(m);
            }
            uint2 b[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float f[8];
#pragma unroll
                for (int i = 0; i < 4; ++i) { const float2 p = both(z[4 * j + i]); f[2 * i] = p.x; f[2 * i + 1] = p.y; }
                b[j] = ckpt_bytes8(f, e);
            }
            if (odd) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float f[8];
#pragma unroll
                    for (int i = 0; i < 4; ++i) { const float2 p = both(z[4 * j + i]); f[2 * i] = p.x; f[2 * i + 1] = p.y; }
                    b[j] = ckpt_bytes8_any<T>(f, e);
                }
            }
            if (in) {
                uint8_t* q = ep.q + row * ep.cols + col0;
                const uint4 b01 = make_uint4(b[0].x, b[0].y, b[1].x, b[1].y), b23 = make_uint4(b[2].x, b[2].y, b[3].x, b[3].y);
                if (whole && ep.grain_q >= 32) {
                    store32(q, b01, b23);
                } else if (whole && ep.grain_q >= 16) {
                    reinterpret_cast<uint4*>(q)[0] = b01;
                    reinterpret_cast<uint4*>(q)[1] = b23;
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) store_q8(q + 8 * j, col0 + 8 * j, ep.cols, ep.grain_q, b[j]);
                }
                // the scales of four blocks in a row go out together where they are aligned; a warp's first block is one of four
                scale4 = scale4 >> 8 | (uint32_t)(e + 127) << 24;
                uint8_t* s = ep.scales + row * ep.groups + (col0 >> 5);
                if (!ep.scales_by4) *s = (uint8_t)(e + 127);
                else if ((col0 & 96u) == 96u) *reinterpret_cast<uint32_t*>(s - 3) = scale4;
            }
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) z[i] = activation<ACT>(z[i]);
    }
    if (ep.residual && in) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float r[8];
            to_floats(load8(static_cast<const T*>(ep.residual) + row * ep.ldr, col0 + 8 * j, ep.cols, 8u), r);
#pragma unroll
            for (int i = 0; i < 4; ++i) z[4 * j + i] = z[4 * j + i] + pair(r[2 * i], r[2 * i + 1]);
        }
    }
    if constexpr (MODE == PRODUCT_INPUT && ACT != SC_ACT_NONE) {
        if (in) {
            const uint8_t* q = ep.q + row * ep.cols;
            const Scale s = slope_scale(ep.scales[row * ep.groups + (col0 >> 5)]);
            uint2 k[4];
            if (whole && ep.grain_q >= 16) {
                const uint4 a = load_stream16(q + col0), b = load_stream16(reinterpret_cast<const uint4*>(q + col0) + 1);
                k[0] = make_uint2(a.x, a.y); k[1] = make_uint2(a.z, a.w); k[2] = make_uint2(b.x, b.y); k[3] = make_uint2(b.z, b.w);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) k[j] = load_q8(q, col0 + 8 * j, ep.cols, ep.grain_q);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                Pair h[4];
                ckpt_values8<false>(k[j], s, h);
#pragma unroll
                for (int i = 0; i < 4; ++i) z[4 * j + i] = z[4 * j + i] * activation_slope<ACT>(h[i]);
            }
        }
    }
    if (lane == 0) tma_store_wait_read_but_one();           // the copy before last has left this buffer
    __syncwarp();
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const uint4 o = packed8<T>(z + 4 * u);
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(buffer + lane * 64 + ((u ^ ((lane >> 1) & 3)) * 16)), "r"(o.x), "r"(o.y), "r"(o.z),
                     "r"(o.w) : "memory");
    }
    smem_to_async_fence();
    __syncwarp();
    if (lane == 0) {
        if (row0 < ep.rows && col0 < ep.cols) tma_store_2d(map_out, buffer, (int32_t)col0, (int32_t)row0);
        tma_store_commit();
    }
}

template <typename T, int MODE, int BN, int CG>
__global__ void __launch_bounds__(TC_THREADS, 1) product_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                                                                const __grid_constant__ CUtensorMap map_out, TcArgs a, Epilogue ep) {
    using S = TcShape<BN, CG>;
    constexpr bool A_MN = MODE == PRODUCT_WEIGHT, B_MN = MODE != PRODUCT_FORWARD;
    constexpr bool SUM = MODE == PRODUCT_WEIGHT;
    extern __shared__ uint8_t raw[];
    const uint32_t base = (smem_addr(raw) + 1023u) & ~1023u;
    const uint32_t staging = base + S::STAGES * S::STAGE;
    const uint32_t bars = staging + S::STAGING;
    const uint32_t full = bars, empty = bars + 8 * S::STAGES, tfull = empty + 8 * S::STAGES, tempty = tfull + 16, slot = tempty + 16;
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;
    const uint32_t rank = CG == 2 ? cluster_rank() : 0u;
    const uint32_t first = blockIdx.x / CG, step = gridDim.x / CG;

    if (threadIdx.x == 0) {
        for (int s = 0; s < S::STAGES; ++s) { mbar_init(full + 8 * s, 1); mbar_init(empty + 8 * s, 1); }
        for (int s = 0; s < 2; ++s) { mbar_init(tfull + 8 * s, 1); mbar_init(tempty + 8 * s, TC_EPI_WARPS * CG); }
        mbar_init_fence();
        tma_prefetch_map(&map_a);
        tma_prefetch_map(&map_b);
        if (a.tma_out || a.rows_form) tma_prefetch_map(&map_out);
    }
    if (warp == 2) tmem_alloc<CG>(slot, S::TMEM_COLS);
    tcgen05_fence_before();
    __syncthreads();
    if constexpr (CG == 2) cluster_sync();
    tcgen05_fence_after();
    uint32_t tmem;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(tmem) : "r"(slot));
    wait_for_predecessor();
    release_successor();

    const uint32_t work = a.tiles * a.splits;
    // The register sums of a 256-wide tile need more than an even share: of the registers that the CTA is
    // launched with, four warps keep 56 a thread and eight get 208 (the host checks that the sum fits).
    constexpr bool REGS = SUM && BN == 256;
    if (warp < 4) {
        if constexpr (REGS) asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        bool ok = true;
        if (warp == 0) {
            // in a pair the first CTA's barriers count the bytes of both
            const uint32_t bytes = CG * ((A_MN ? S::A_BYTES : a.a_box_rows * TC_STEP * 2) + S::B_BYTES);
            uint32_t stage = 0, phase = 0, issued = 0;
            for (uint32_t w = first; w < work && ok; w += step) {
                const uint32_t split = w / a.tiles;
                uint32_t ti, tj;
                tile_at(a, w - split * a.tiles, ti, tj);
                const uint32_t k0 = (uint64_t)a.blocks * split / a.splits, k1 = (uint64_t)a.blocks * (split + 1) / a.splits;
                const int32_t i0 = (int32_t)((ti * CG + rank) * TC_ROWS), j0 = (int32_t)(tj * BN + rank * S::B_ROWS);
                for (uint32_t k = k0; k < k1; ++k) {
                    if (!(ok = warp_wait(empty + 8 * stage, phase ^ 1u))) break;
                    const uint32_t sa = base + stage * S::STAGE, sb = sa + S::A_BYTES;
                    if (elect_one()) {
                        if (rank == 0) mbar_expect_tx(full + 8 * stage, bytes);
                        const uint32_t bar = CG == 2 ? map_to_rank(full + 8 * stage, 0) : full + 8 * stage;
                        const int32_t r = (int32_t)(k * TC_STEP);
                        if constexpr (A_MN) {
#pragma unroll
                            for (int c = 0; c < TC_ROWS; c += 64) tma_load_2d<CG>(sa + c * TC_STEP * 2, &map_a, bar, i0 + c, r);
                        } else {
                            tma_load_2d<CG>(sa, &map_a, bar, r, i0);
                        }
                        if constexpr (B_MN) {
#pragma unroll
                            for (int c = 0; c < S::B_ROWS; c += 64) tma_load_2d<CG>(sb + c * TC_STEP * 2, &map_b, bar, j0 + c, r);
                        } else {
                            tma_load_2d<CG>(sb, &map_b, bar, r, j0);
                        }
                    }
                    __syncwarp();
                    ++issued;
                    if (++stage == S::STAGES) { stage = 0; phase ^= 1u; }
                }
            }
            if (!ok) {                     // the copies in flight land before the CTA ends (two seconds have passed since the last)
                if (lane == 0) atomicCAS(a.status, 0, ST_TIMEOUT);
                if (rank == 0)
                    for (uint32_t n = issued > (uint32_t)S::STAGES ? issued - S::STAGES : 0; n < issued; ++n)
                        mbar_wait(full + 8 * (n % S::STAGES), (n / S::STAGES) & 1u);
            }
        } else if (warp == 1 && rank == 0) {
            uint32_t stage = 0, phase = 0, acc = 0, acc_phase = 0;
            const uint64_t da0 = A_MN ? smem_desc(base, TC_STEP * 128, 1024) : smem_desc(base, 16, 1024);
            const uint64_t db0 = B_MN ? smem_desc(base + S::A_BYTES, TC_STEP * 128, 1024) : smem_desc(base + S::A_BYTES, 16, 1024);
            for (uint32_t w = first; w < work && ok; w += step) {
                const uint32_t split = w / a.tiles;
                const uint32_t k0 = (uint64_t)a.blocks * split / a.splits, k1 = (uint64_t)a.blocks * (split + 1) / a.splits;
                for (uint32_t c0 = k0; c0 < k1 && ok;) {
                    const uint32_t c1 = SUM ? min(c0 + TC_CHUNK, k1) : k1;
                    if (!(ok = warp_wait(tempty + 8 * acc, acc_phase ^ 1u))) break;
                    tcgen05_fence_after();
                    for (uint32_t k = c0; k < c1; ++k) {
                        if (!(ok = warp_wait(full + 8 * stage, phase))) break;
                        tcgen05_fence_after();
                        const uint32_t next = stage + 1 == S::STAGES ? 0 : stage + 1, next_phase = next ? phase : phase ^ 1u;
                        const uint64_t da = da0 + stage * (S::STAGE >> 4), db = db0 + stage * (S::STAGE >> 4);
                        const uint32_t d = tmem + acc * BN;
                        if (elect_one()) {
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                mma_f16<CG>(d, da + (A_MN ? 128 : 2) * i, db + (B_MN ? 128 : 2) * i, a.idesc, k > c0 || i > 0);
                            mma_commit<CG>(empty + 8 * stage);
                            if (k + 1 == c1) mma_commit<CG>(tfull + 8 * acc);
                        }
                        __syncwarp();
                        stage = next; phase = next_phase;
                    }
                    if ((acc ^= 1u) == 0) acc_phase ^= 1u;
                    c0 = c1;
                }
            }
            if (!ok && lane == 0) atomicCAS(a.status, 0, ST_TIMEOUT);
        }
        __syncwarp();
    } else {
        if constexpr (REGS) asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
        const uint32_t e = warp - 4, quarter = warp & 3u, half = e >> 2;
        const uint32_t stage_addr = staging + e * 4096;
        const uint32_t from = tmem + ((quarter * 32) << 16) + half * (BN / 2);
        uint32_t acc = 0, acc_phase = 0, turn = 0;
        bool ok = true;
        for (uint32_t w = first; w < work && ok; w += step) {
            const uint32_t split = w / a.tiles;
            uint32_t ti, tj;
            tile_at(a, w - split * a.tiles, ti, tj);
            const uint64_t row0 = (uint64_t)(ti * CG + rank) * TC_ROWS + quarter * 32;
            const uint32_t col0 = tj * BN + half * (BN / 2);
            if constexpr (SUM) {
                const uint32_t k0 = (uint64_t)a.blocks * split / a.splits, k1 = (uint64_t)a.blocks * (split + 1) / a.splits;
                uint32_t sum[BN / 64][32];               // fp32, by their bits
#pragma unroll
                for (int c = 0; c < BN / 64; ++c)
#pragma unroll
                    for (int i = 0; i < 32; ++i) sum[c][i] = 0u;
                for (uint32_t c0 = k0; c0 < k1; c0 += TC_CHUNK) {
                    if (!(ok = warp_wait(tfull + 8 * acc, acc_phase))) break;
                    __syncwarp();
                    tcgen05_fence_after();
#pragma unroll
                    for (int c = 0; c < BN / 64; ++c) {
                        uint32_t v[32];
                        tmem_load32(from + acc * BN + c * 32, v);
                        tmem_load_wait(v);
#pragma unroll
                        for (int i = 0; i < 32; ++i) sum[c][i] = __float_as_uint(__uint_as_float(sum[c][i]) + __uint_as_float(v[i]));
                    }
                    tcgen05_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_cluster(CG == 2 ? map_to_rank(tempty + 8 * acc, 0) : tempty + 8 * acc);
                    if ((acc ^= 1u) == 0) acc_phase ^= 1u;
                }
                if (!ok) break;
#pragma unroll
                for (int c = 0; c < BN / 64; ++c) block_out<T, MODE>(&map_out, a, ep, stage_addr, sum[c], row0, col0 + c * 32, split);
            } else {
                if (!(ok = warp_wait(tfull + 8 * acc, acc_phase))) break;
                __syncwarp();
                tcgen05_fence_after();
                uint32_t scale4 = 0;
#pragma unroll 1
                for (int c = 0; c < BN / 2; c += 32) {
                    uint32_t v[32];
                    tmem_load32(from + acc * BN + c, v);
                    tmem_load_wait(v);
                    if (c + 32 >= BN / 2) {             // this warp has taken all it needs from the accumulator
                        tcgen05_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive_cluster(CG == 2 ? map_to_rank(tempty + 8 * acc, 0) : tempty + 8 * acc);
                    }
                    if (a.rows_form) {
                        with_activation(ep.act, [&](auto act) {
                            block_rows<T, MODE, decltype(act)::value>(&map_out, ep, stage_addr + turn, v, row0, col0 + c, scale4);
                        });
                        turn ^= 2048u;                      // the two buffers take turns from block to block, whatever the tile
                    } else
                        block_out<T, MODE>(&map_out, a, ep, stage_addr, v, row0, col0 + c, split);
                }
                if ((acc ^= 1u) == 0) acc_phase ^= 1u;
            }
        }
        if ((a.tma_out || a.rows_form) && lane == 0) tma_store_wait();
        if (!ok && lane == 0) atomicCAS(a.status, 0, ST_TIMEOUT);
        __syncwarp();
    }
    tcgen05_fence_before();
    __syncthreads();
    if constexpr (CG == 2) cluster_sync();
    tcgen05_fence_after();
    if (warp == 2) tmem_free<CG>(tmem, S::TMEM_COLS);
}

// ---------------------------------------------------------------------------
// Forward product of a few tokens
// ---------------------------------------------------------------------------
// With one to four tokens the weights' bytes are everything, and four multiply-adds a weight still fit beside their loads.
// A warp owns four rows of W and walks its share of the reduction, 16 bytes a lane and row; WK warps split a row, WN warps
// sit side by side, and the last step joins them in shared memory.  WN = 8 puts 32 outputs, a checkpoint group, in one CTA.
// 1 x 4096 x 4096 bf16 takes 7.8 us with W from HBM (33.6 MB, 4.3 TB/s), 1 x 16384 x 4096 24.7 us (5.4 TB/s), 1 x 1024 x 1024 2.0 us:
// bound by the weights' bytes, from three tokens on by the registers that limit the loads in flight.
template <typename T, int TOKENS, int WN, int WK, bool WIDE>
__global__ void __launch_bounds__(WN * WK * 32) product_tokens_kernel(const T* x, uint64_t ldx, const T* w, uint64_t ldw,
                                                                      uint32_t K, uint32_t grain_x, uint32_t grain_w, Epilogue ep) {
    constexpr int ROWS = 4, COLS = ROWS * WN;
    wait_for_predecessor();
    release_successor();
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u, wn = warp / WK, wk = warp % WK;
    const uint32_t n0 = blockIdx.x * COLS + wn * ROWS, tokens = (uint32_t)ep.rows;
    float acc[ROWS][TOKENS] = {};
    constexpr uint32_t STEP = 8 * 32 * WK;
#pragma unroll 2
    for (uint32_t k = (wk * 32 + lane) * 8; k < K; k += STEP) {
        Raw8<T> rw[ROWS], rx[TOKENS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            rw[r] = Raw8<T>{};
            if (n0 + r < ep.cols) rw[r] = load8(w + (uint64_t)(n0 + r) * ldw, k, K, WIDE ? 8u : grain_w);
        }
#pragma unroll
        for (int m = 0; m < TOKENS; ++m) {
            rx[m] = Raw8<T>{};
            if (m < tokens) {
                if (WIDE && k + 8 <= K) rx[m].v = *reinterpret_cast<const uint4*>(x + m * ldx + k);
                else rx[m] = load8(x + m * ldx, k, K, WIDE ? 8u : grain_x);
            }
        }
        float fx[TOKENS][8];
#pragma unroll
        for (int m = 0; m < TOKENS; ++m) to_floats(rx[m], fx[m]);
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            float fw[8];
            to_floats(rw[r], fw);
#pragma unroll
            for (int m = 0; m < TOKENS; ++m)
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[r][m] = fmaf(fw[i], fx[m][i], acc[r][m]);
        }
    }
    __shared__ float part[WK][TOKENS][COLS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int m = 0; m < TOKENS; ++m) {
            float v = acc[r][m];
#pragma unroll
            for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
            if (lane == 0) part[wk][m][wn * ROWS + r] = v;
        }
    __syncthreads();
    if (warp) return;
    // lane 4 m + j: token m, eight of the CTA's outputs
    const uint32_t m = lane >> 2, j = (lane & 3u) * 8;
    const bool own = m < TOKENS && j < COLS;
    const uint32_t c0 = own ? blockIdx.x * COLS + j : ep.cols;
    float f[8] = {}, bias[8];
    if (own)
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int s = 0; s < WK; ++s) f[i] += part[s][m][j + i];
    load_bias<T, PRODUCT_FORWARD>(ep, c0, bias);
    with_activation(ep.act, [&](auto act) { epilogue8<T, PRODUCT_FORWARD, decltype(act)::value>(ep, m, c0, bias, f); });
}

// ---------------------------------------------------------------------------
// Weight gradient of a few tokens
// ---------------------------------------------------------------------------
// Up to 8 tokens: the fp32 result's own bytes are everything (8 multiply-adds a value, two at a time, fit beside them), so each
// value is made where it is stored.  A CTA owns 128 columns and `run` rows; every warp holds the columns' inputs in
// registers, read from the checkpoint or from x, and walks its rows with the rows' dz in shared memory (each twice, as the
// paired arithmetic wants it), one 128-byte store at a time, whatever the alignment.  4096 x 4096: 14.4 us at 4 tokens and
// 16.3 at 8, against 18.2 on the tiles (with the checkpoint's copy); a fill of the output takes 12.3.  With 16 tokens it took 31.
template <typename T, int TOKENS, bool KEPT>
__global__ void __launch_bounds__(256) weight_tokens_kernel(const T* dz, uint64_t lddz, const T* x, uint64_t ldx,
                                                            const uint8_t* q, const uint8_t* scales, uint32_t tokens, uint32_t run,
                                                            Epilogue ep) {
    extern __shared__ __align__(16) float2 rows_dz[];              // [run][TOKENS]
    wait_for_predecessor();
    release_successor();
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    const uint32_t c0 = blockIdx.x * 128 + lane, K = ep.cols;
    const uint64_t n0 = (uint64_t)blockIdx.y * run;
    const uint32_t rows = (uint32_t)min((uint64_t)run, ep.rows - n0);
    for (uint32_t i = threadIdx.x; i < rows * TOKENS; i += 256) {
        const uint32_t m = i / rows, r = i - m * rows;
        const float d = m < tokens ? Elem<T>::to_float(dz[m * lddz + n0 + r]) : 0.0f;
        rows_dz[r * TOKENS + m] = make_float2(d, d);
    }
    // all loads first, from clamped places; columns past the end are not stored
    float v[TOKENS][4];
    if constexpr (KEPT) {
        uint32_t k[TOKENS][4];
#pragma unroll
        for (int m = 0; m < TOKENS; ++m)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint64_t row = min((uint32_t)m, tokens - 1);
                const uint32_t c = min(c0 + 32 * j, K - 1);
                k[m][j] = q[row * K + c];
                v[m][j] = __uint_as_float((uint32_t)scales[row * ep.groups + (c >> 5)] << 23);
            }
#pragma unroll
        for (int m = 0; m < TOKENS; ++m)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[m][j] *= (float)(int8_t)k[m][j];
                // a bf16 value whatever the checkpoint was made from; an fp16 value unless that was a type of wider range: rounded then, as by unpacking
                if constexpr (std::is_same<T, __half>::value) v[m][j] = __half2float(__float2half_rn(v[m][j]));
                if (k[m][j] == 0x80u) v[m][j] = __uint_as_float(0x7FFFFFFFu);
                if (m >= (int)tokens) v[m][j] = 0.0f;
            }
    } else {
#pragma unroll
        for (int m = 0; m < TOKENS; ++m)
#pragma unroll
            for (int j = 0; j < 4; ++j) v[m][j] = Elem<T>::to_float(x[min((uint32_t)m, tokens - 1) * ldx + min(c0 + 32 * j, K - 1)]);
#pragma unroll
        for (int m = 0; m < TOKENS; ++m)
#pragma unroll
            for (int j = 0; j < 4; ++j) if (m >= (int)tokens) v[m][j] = 0.0f;
    }
    __syncthreads();
    float* out = static_cast<float*>(ep.out) + n0 * ep.ldo + c0;
#pragma unroll 2
    for (uint32_t r = warp; r < rows; r += 8) {
        Pair lo[2] = {pair(0.0f), pair(0.0f)}, hi[2] = {pair(0.0f), pair(0.0f)};     // two chains each
#pragma unroll
        for (int m = 0; m < TOKENS; m += 2) {
            const float4 d = *reinterpret_cast<const float4*>(&rows_dz[r * TOKENS + m]);
            lo[0] = fma2(pair(d.x, d.y), pair(v[m][0], v[m][1]), lo[0]);
            hi[0] = fma2(pair(d.x, d.y), pair(v[m][2], v[m][3]), hi[0]);
            lo[1] = fma2(pair(d.z, d.w), pair(v[m + 1][0], v[m + 1][1]), lo[1]);
            hi[1] = fma2(pair(d.z, d.w), pair(v[m + 1][2], v[m + 1][3]), hi[1]);
        }
        const float2 a01 = both(lo[0] + lo[1]), a23 = both(hi[0] + hi[1]);
        const float acc[4] = {a01.x, a01.y, a23.x, a23.y};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float* o = out + r * ep.ldo + 32 * j;
            if (c0 + 32 * j >= K) continue;
            if (ep.accumulate) asm volatile("red.relaxed.gpu.global.add.f32 [%0], %1;" ::"l"(o), "f"(acc[j]) : "memory");
            else *o = acc[j];
        }
    }
}

// Joins the parts of a split product in order and applies the epilogue; no parts at all is an empty sum.  2 to 6 us: parts are
// few enough to be read from L2.
template <typename T, int MODE>
__global__ void __launch_bounds__(256) product_join_kernel(const float* partial, uint32_t splits, uint64_t part_stride, uint32_t part_ld,
                                                           Epilogue ep) {
    wait_for_predecessor();
    release_successor();
    const uint32_t chunks = 4 * ((ep.cols + 31) / 32);
    const uint64_t total = ep.rows * chunks, stride = (uint64_t)gridDim.x * 256;
    const uint32_t lane = threadIdx.x & 31u;
    for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i - lane < total; i += stride) {
        const uint64_t row = i < total ? i / chunks : ep.rows;
        const uint32_t c0 = (uint32_t)(i - row * chunks) * 8;
        float f[8] = {};
        if (i < total && c0 < ep.cols) {
            const float4* p = reinterpret_cast<const float4*>(partial + row * part_ld + c0);
            for (uint32_t s = 0; s < splits; ++s, p += part_stride / 4) {
                const float4 x = load_l2(p), y = load_l2(p + 1);
                f[0] += x.x; f[1] += x.y; f[2] += x.z; f[3] += x.w;
                f[4] += y.x; f[5] += y.y; f[6] += y.z; f[7] += y.w;
            }
        }
        if constexpr (MODE == PRODUCT_WEIGHT) {
            epilogue8<T, MODE, SC_ACT_NONE>(ep, row, c0, nullptr, f);
        } else {
            float bias[8];
            load_bias<T, MODE>(ep, c0, bias);
            with_activation(ep.act, [&](auto act) { epilogue8<T, MODE, decltype(act)::value>(ep, row, c0, bias, f); });
        }
    }
}

// Rows copied to a 16-byte aligned place with rows a multiple of 8 elements apart, where the tensor cores' loads can reach them.
// Rows of single-element alignment are read 32 elements a warp and access, the others a chunk of 8 a thread.
struct LayoutArgs {
    const uint16_t* src;
    uint16_t* dst;
    uint64_t ld, rows;
    uint32_t cols, ldd, grain;
};
__device__ __forceinline__ void layout_rows(const LayoutArgs& a, uint32_t block, uint32_t blocks) {
    const uint64_t first = (uint64_t)block * 256 + threadIdx.x, stride = (uint64_t)blocks * 256;
    if (a.grain == 1) {
        const uint32_t lane = threadIdx.x & 31u, runs = (a.ldd + 255) / 256;
        for (uint64_t i = first >> 5; i < a.rows * runs; i += stride >> 5) {
            const uint64_t row = i / runs;
            const uint32_t c0 = (uint32_t)(i - row * runs) * 256 + lane;
            uint16_t v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = c0 + 32 * k < a.cols ? a.src[row * a.ld + c0 + 32 * k] : (uint16_t)0;
#pragma unroll
            for (int k = 0; k < 8; ++k) if (c0 + 32 * k < a.ldd) a.dst[row * a.ldd + c0 + 32 * k] = v[k];
        }
    } else {
        const uint32_t chunks = a.ldd / 8;
        for (uint64_t i = first; i < a.rows * chunks; i += stride) {
            const uint64_t row = i / chunks;
            const uint32_t c0 = (uint32_t)(i - row * chunks) * 8;
            *reinterpret_cast<uint4*>(a.dst + row * a.ldd + c0) = load_narrow(a.src + row * a.ld + c0, a.cols - c0, a.grain);
        }
    }
}
// One or both operands of a product: blockIdx.y chooses.
static __global__ void __launch_bounds__(256) layout_kernel(LayoutArgs a, LayoutArgs b) {
    wait_for_predecessor();
    release_successor();
    layout_rows(blockIdx.y ? b : a, blockIdx.x, gridDim.x);
}

}  // namespace sc
