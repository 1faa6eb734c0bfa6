// The layer's three matrix products, out[i, j] = sum_r A[i, r] B[j, r], and what follows each in its epilogue:
//   forward       y  = act(x W^T + b) + residual          A = x [M, K],   B = W [N, K],    r over K
//   input grad    dx = (dz W + residual) * act'(z^)       A = dz [M, N],  B = W^T [K, N],  r over N
//   weight grad   dW (+)= dz^T x^                         A = dz^T [N, M], B = x^T [K, M], r over M
#pragma once
#include "sc_layer_common.cuh"

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
};

// Operand with any strides, element (i, r) at i * si + r * sr.
struct Operand {
    const void* p;
    uint64_t si, sr;
};

template <typename T, int MODE>
__global__ void __launch_bounds__(256) product_plain_kernel(Operand A, Operand B, uint64_t red, Epilogue ep) {
    constexpr int TILE_I = 64, TILE_J = 64, STEP = 16;
    __shared__ float sa[STEP][TILE_I + 4], sb[STEP][TILE_J + 4];
    const uint64_t i0 = (uint64_t)blockIdx.y * TILE_I;
    const uint32_t j0 = blockIdx.x * TILE_J;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const T* a = static_cast<const T*>(A.p);
    const T* b = static_cast<const T*>(B.p);
    float acc[4][4] = {}, sum[4][4] = {};                // a long sum is kept as a sum of sums of 256 products
    for (uint64_t r0 = 0; r0 < red; r0 += STEP) {
        for (int t = threadIdx.x; t < TILE_I * STEP; t += 256) {
            // the index that is contiguous in memory runs fastest over the threads
            const int i = A.sr == 1 ? t / STEP : t % TILE_I, r = A.sr == 1 ? t % STEP : t / TILE_I;
            const int j = B.sr == 1 ? t / STEP : t % TILE_J, s = B.sr == 1 ? t % STEP : t / TILE_J;
            sa[r][i] = i0 + i < ep.rows && r0 + r < red ? Elem<T>::to_float(a[(i0 + i) * A.si + (r0 + r) * A.sr]) : 0.0f;
            sb[s][j] = j0 + j < ep.cols && r0 + s < red ? Elem<T>::to_float(b[(uint64_t)(j0 + j) * B.si + (r0 + s) * B.sr]) : 0.0f;
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < STEP; ++r) {
            float va[4], vb[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) { va[u] = sa[r][ty * 4 + u]; vb[u] = sb[r][tx * 4 + u]; }
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int v = 0; v < 4; ++v) acc[u][v] = fmaf(va[u], vb[v], acc[u][v]);
        }
        __syncthreads();
        if ((r0 + STEP) % 256 == 0 || r0 + STEP >= red) {
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int v = 0; v < 4; ++v) { sum[u][v] += acc[u][v]; acc[u][v] = 0.0f; }
        }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const uint64_t i = i0 + ty * 4 + u;
        const uint32_t j = j0 + tx * 4;
        float z[4];
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            z[v] = sum[u][v];
            if (i >= ep.rows || j + v >= ep.cols) continue;
            if constexpr (MODE == PRODUCT_WEIGHT) {
                float* dw = static_cast<float*>(ep.out) + i * ep.ldo + j + v;
                *dw = ep.accumulate ? *dw + z[v] : z[v];
            } else {
                const T* res = ep.residual ? static_cast<const T*>(ep.residual) + i * ep.ldr + j + v : nullptr;
                T* out = static_cast<T*>(ep.out) + i * ep.ldo + j + v;
                if constexpr (MODE == PRODUCT_FORWARD) {
                    if (ep.bias) z[v] += Elem<T>::to_float(static_cast<const T*>(ep.bias)[j + v]);
                    float y = activation(ep.act, z[v]);
                    if (res) y += Elem<T>::to_float(*res);
                    *out = Elem<T>::from_float(y);
                } else {
                    if (res) z[v] += Elem<T>::to_float(*res);
                    if (ep.q) {
                        const uint32_t b = ep.q[i * ep.cols + j + v];
                        float k[4];
                        ckpt_values4(b, ckpt_scale(ep.scales[i * ep.groups + ((j + v) >> 5)]), k);
                        z[v] *= activation_slope(ep.act, k[0]);
                    }
                    *out = Elem<T>::from_float(z[v]);
                }
            }
        }
        if constexpr (MODE == PRODUCT_FORWARD) {
            if (!ep.q) continue;
            uint32_t m = 0;                                   // eight lanes hold a group
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const uint32_t k = __float_as_uint(z[v]) & 0x7FFFFFFFu;
                if (j + v < ep.cols && k < 0x7F800000u) m = max(m, k);
            }
#pragma unroll
            for (int d = 1; d < 8; d <<= 1) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, d));
            const int e = ckpt_exponent<T>(m);
            const float inv = pow2(-e), most = e == Elem<T>::EMAX ? 63.0f : 127.0f;
            if (i >= ep.rows) continue;
#pragma unroll
            for (int v = 0; v < 4; ++v)
                if (j + v < ep.cols) ep.q[i * ep.cols + j + v] = (uint8_t)ckpt_byte_any(z[v], inv, most);
            if ((tx & 7) == 0 && j < ep.cols) ep.scales[i * ep.groups + (j >> 5)] = (uint8_t)(e + 127);
        }
    }
}

}  // namespace sc
