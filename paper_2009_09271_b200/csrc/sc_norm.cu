// Host side of 8-bit rows, the root-mean-square norm and dropout, declared in include/sparsecomm.h.
#include <cmath>

#include "sc_layer_host.cuh"
#include "sc_norm.cuh"

namespace {

// Items of eight elements, and the distances that a grid of `item_grid` CTAs walks in.
uint32_t item_grid(const sc_ctx* c, uint64_t total) {
    return (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>(ceil_div(total, CKPT_THREADS), (uint64_t)c->sm_count * 8));
}
ItemWalk item_walk(const sc_ctx* c, size_t rows, size_t cols) {
    ItemWalk w{};
    w.cols = (uint32_t)cols;
    w.items = (uint32_t)ceil_div(cols, 8);
    w.total = (uint64_t)rows * w.items;
    const uint64_t stride = (uint64_t)item_grid(c, w.total) * CKPT_THREADS;
    w.stride_rows = stride / w.items;
    w.stride_items = (uint32_t)(stride % w.items);
    return w;
}
uint32_t row_grid(const sc_ctx* c, size_t rows) { return (uint32_t)std::min<uint64_t>(rows, (uint64_t)c->sm_count * 8); }

inline uint32_t grain16(const void* p, size_t rows, size_t ld) { return grain_of(p, rows > 1 ? ld : 0, 2, 8); }

// The cut that p stands for; false where p is no probability.
bool drop_of(double p, uint64_t seed, size_t cols, Drop& d) {
    if (!(p >= 0.0 && p <= 1.0)) return false;
    d.cut = (uint32_t)std::lrint(p * 65536.0);
    d.key = mix64(seed, SALT_DROPOUT);
    d.groups = (uint32_t)ceil_div(cols, 4);
    d.scale = d.cut < 65536 ? 65536.0f / (float)(65536 - d.cut) : 0.0f;
    return true;
}
inline bool eps_ok(float eps) { return eps >= 0.0f && eps <= 3.402823466e38f; }

// Column sums of the norm's gradient: runs of rows as for the activation's gradient.
struct StripPlan { uint32_t strips, runs, run_rows; size_t partial, stats; };
StripPlan strip_plan(const sc_ctx* c, size_t rows, size_t cols) {
    StripPlan p{};
    p.strips = (uint32_t)ceil_div(cols, GRAD_COLS);
    const uint64_t runs = std::max<uint64_t>(1, std::min<uint64_t>((uint64_t)c->sm_count * 8 / p.strips, ceil_div(rows, 32)));
    p.run_rows = (uint32_t)(ceil_div(ceil_div(rows, runs), GRAD_LANES) * GRAD_LANES);
    p.runs = (uint32_t)ceil_div(rows, p.run_rows);
    p.partial = p.runs > 1 ? ((size_t)p.runs * cols * sizeof(float) + 255) & ~(size_t)255 : 0;
    p.stats = rows * sizeof(float2);
    return p;
}

}  // namespace

extern "C" {

int sc_quantize(sc_ctx* ctx, int type, const void* x, size_t ldx, size_t rows, size_t cols, int8_t* q, size_t ldq, float* scales, void* stream) {
    if (!ctx) return SC_ERR_INVALID;
    if (type != SC_F32 && !known_type(type)) return SC_ERR_UNSUPPORTED;
    if (const int rc = check_matrix(x, ldx, rows, cols, type_bytes(type))) return rc;
    if (const int rc = check_matrix(q, ldq, rows, cols, 1)) return rc;
    if (rows == 0 || cols == 0) return SC_OK;
    if (!scales || !aligned(scales, 4)) return SC_ERR_INVALID;
    DeviceGuard guard(ctx->device);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    QuantizeArgs a{};
    a.rows = rows; a.ldx = ldx; a.ldq = ldq; a.cols = (uint32_t)cols;
    a.grain_x = grain_of(x, rows > 1 ? ldx : 0, type_bytes(type), 8);
    a.grain_q = grain_of(q, rows > 1 ? ldq : 0, 1, 8);
    uint8_t* qb = reinterpret_cast<uint8_t*>(q);
    Launch l(ctx, KIND_QUANTIZE, st);
#define SC_QUANTIZE(T) launch(quantize_kernel<T>, row_grid(ctx, rows), NORM_THREADS, 0, 1, st, static_cast<const T*>(x), a, qb, scales)
    if (type == SC_BF16) SC_QUANTIZE(__nv_bfloat16);
    else if (type == SC_F16) SC_QUANTIZE(__half);
    else SC_QUANTIZE(float);
#undef SC_QUANTIZE
    SC_CUDA(cudaGetLastError());
    return SC_OK;
}

int sc_dequantize(sc_ctx* ctx, int type, const int8_t* q, size_t ldq, const float* scales, size_t rows, size_t cols, void* out, size_t ldo,
                  void* stream) {
    if (!ctx) return SC_ERR_INVALID;
    if (type != SC_F32 && !known_type(type)) return SC_ERR_UNSUPPORTED;
    if (const int rc = check_matrix(q, ldq, rows, cols, 1)) return rc;
    if (const int rc = check_matrix(out, ldo, rows, cols, type_bytes(type))) return rc;
    if (rows == 0 || cols == 0) return SC_OK;
    if (!scales || !aligned(scales, 4)) return SC_ERR_INVALID;
    DeviceGuard guard(ctx->device);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    ItemWalk w = item_walk(ctx, rows, cols);
    w.grain_x = grain_of(out, rows > 1 ? ldo : 0, type_bytes(type), 8);
    w.grain_q = grain_of(q, rows > 1 ? ldq : 0, 1, 8);
    const uint8_t* qb = reinterpret_cast<const uint8_t*>(q);
    Launch l(ctx, KIND_DEQUANTIZE, st);
#define SC_DEQUANTIZE(T) launch(dequantize_kernel<T>, item_grid(ctx, w.total), CKPT_THREADS, 0, 1, st, qb, ldq, scales, w, static_cast<T*>(out), ldo)
    if (type == SC_BF16) SC_DEQUANTIZE(__nv_bfloat16);
    else if (type == SC_F16) SC_DEQUANTIZE(__half);
    else SC_DEQUANTIZE(float);
#undef SC_DEQUANTIZE
    SC_CUDA(cudaGetLastError());
    return SC_OK;
}

int sc_dropout(sc_ctx* ctx, int type, const void* x, size_t ldx, const void* residual, size_t ldr, double p, uint64_t seed, size_t rows, size_t cols,
               void* y, size_t ldy, void* stream) {
    if (!ctx) return SC_ERR_INVALID;
    if (!known_type(type)) return SC_ERR_UNSUPPORTED;
    if (const int rc = check_matrix(x, ldx, rows, cols, 2)) return rc;
    if (residual) if (const int rc = check_matrix(residual, ldr, rows, cols, 2)) return rc;
    if (const int rc = check_matrix(y, ldy, rows, cols, 2)) return rc;
    DropArgs a{};
    if (!drop_of(p, seed, cols, a.drop)) return SC_ERR_INVALID;
    if (rows == 0 || cols == 0) return SC_OK;
    DeviceGuard guard(ctx->device);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const ItemWalk w = item_walk(ctx, rows, cols);
    a.ldx = ldx; a.ldr = ldr; a.ldy = ldy;
    a.grain_x = grain16(x, rows, ldx); a.grain_r = grain16(residual, rows, ldr); a.grain_y = grain16(y, rows, ldy);
    Launch l(ctx, KIND_DROPOUT, st);
#define SC_DROPOUT(T) launch(dropout_kernel<T>, item_grid(ctx, w.total), CKPT_THREADS, 0, 1, st, static_cast<const T*>(x), static_cast<const T*>(residual), \
                             static_cast<T*>(y), w, a)
    if (type == SC_BF16) SC_DROPOUT(__nv_bfloat16);
    else SC_DROPOUT(__half);
#undef SC_DROPOUT
    SC_CUDA(cudaGetLastError());
    return SC_OK;
}

int sc_rms_norm(sc_ctx* ctx, int type, const void* x, size_t ldx, const void* residual, size_t ldr, const void* gamma, float eps, double p, uint64_t seed,
                size_t rows, size_t cols, void* h, size_t ldh, void* y, size_t ldy, int8_t* q, size_t ldq, float* scales, void* stream) {
    if (!ctx) return SC_ERR_INVALID;
    if (!known_type(type)) return SC_ERR_UNSUPPORTED;
    if (!eps_ok(eps)) return SC_ERR_INVALID;
    if (const int rc = check_matrix(x, ldx, rows, cols, 2)) return rc;
    if (residual) if (const int rc = check_matrix(residual, ldr, rows, cols, 2)) return rc;
    if (h) if (const int rc = check_matrix(h, ldh, rows, cols, 2)) return rc;
    if (y) if (const int rc = check_matrix(y, ldy, rows, cols, 2)) return rc;
    if (q) if (const int rc = check_matrix(q, ldq, rows, cols, 1)) return rc;
    NormArgs a{};
    if (!drop_of(p, seed, cols, a.drop)) return SC_ERR_INVALID;
    if (rows == 0 || cols == 0) return SC_OK;
    if (!gamma || !aligned(gamma, 2) || !aligned(scales, 4) || (q == nullptr) != (scales == nullptr) || (!y && !q)) return SC_ERR_INVALID;
    DeviceGuard guard(ctx->device);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    a.rows = rows; a.ldx = ldx; a.ldr = ldr; a.ldh = ldh; a.ldy = ldy; a.ldq = ldq; a.cols = (uint32_t)cols;
    a.grain_x = grain16(x, rows, ldx); a.grain_r = grain16(residual, rows, ldr); a.grain_g = grain_of(gamma, 0, 2, 8);
    a.grain_h = grain16(h, rows, ldh); a.grain_y = grain16(y, rows, ldy); a.grain_q = grain_of(q, rows > 1 ? ldq : 0, 1, 8);
    a.eps = eps; a.mean = 1.0f / (float)cols;
    uint8_t* qb = reinterpret_cast<uint8_t*>(q);
    Launch l(ctx, KIND_RMS_NORM, st);
#define SC_NORM(T) launch(rms_norm_kernel<T>, row_grid(ctx, rows), NORM_THREADS, 0, 1, st, static_cast<const T*>(x), static_cast<const T*>(residual), \
                          static_cast<const T*>(gamma), a, static_cast<T*>(h), static_cast<T*>(y), qb, scales)
    if (type == SC_BF16) SC_NORM(__nv_bfloat16);
    else SC_NORM(__half);
#undef SC_NORM
    SC_CUDA(cudaGetLastError());
    return SC_OK;
}

int sc_rms_norm_grad(sc_ctx* ctx, int type, const void* dy, size_t lddy, const void* h, size_t ldh, const void* gamma, float eps, const void* residual,
                     size_t ldr, double p, uint64_t seed, size_t rows, size_t cols, void* dh, size_t lddh, void* dx, size_t lddx, float* dgamma,
                     int accumulate, void* stream) {
    if (!ctx) return SC_ERR_INVALID;
    if (!known_type(type)) return SC_ERR_UNSUPPORTED;
    if (!eps_ok(eps) || !aligned(dgamma, 4)) return SC_ERR_INVALID;
    if (const int rc = check_matrix(dy, lddy, rows, cols, 2)) return rc;
    if (const int rc = check_matrix(h, ldh, rows, cols, 2)) return rc;
    if (residual) if (const int rc = check_matrix(residual, ldr, rows, cols, 2)) return rc;
    if (dh) if (const int rc = check_matrix(dh, lddh, rows, cols, 2)) return rc;
    if (dx) if (const int rc = check_matrix(dx, lddx, rows, cols, 2)) return rc;
    NormGradArgs a{};
    if (!drop_of(p, seed, cols, a.drop)) return SC_ERR_INVALID;
    if (cols == 0) return SC_OK;
    DeviceGuard guard(ctx->device);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (rows == 0) {
        if (dgamma && !accumulate) SC_CUDA(cudaMemsetAsync(dgamma, 0, cols * sizeof(float), st));
        return SC_OK;
    }
    if (!gamma || !aligned(gamma, 2) || (!dh && !dx && !dgamma)) return SC_ERR_INVALID;
    const StripPlan plan = strip_plan(ctx, rows, cols);
    if (const int rc = layer_scratch(ctx, plan.partial + plan.stats, st)) return rc;
    a.rows = rows; a.lddy = lddy; a.ldh = ldh; a.ldr = ldr; a.lddh = lddh; a.lddx = lddx; a.cols = (uint32_t)cols;
    a.grain_y = grain16(dy, rows, lddy); a.grain_h = grain16(h, rows, ldh); a.grain_g = grain_of(gamma, 0, 2, 8);
    a.grain_r = grain16(residual, rows, ldr); a.grain_dh = grain16(dh, rows, lddh); a.grain_dx = grain16(dx, rows, lddx);
    a.runs = plan.runs; a.run_rows = plan.run_rows; a.accumulate = accumulate ? 1u : 0u;
    a.eps = eps; a.mean = 1.0f / (float)cols;
    float* partial = reinterpret_cast<float*>(ctx->d_layer + TICKET_BYTES);
    float2* stats = reinterpret_cast<float2*>(ctx->d_layer + TICKET_BYTES + plan.partial);
    uint32_t* tickets = reinterpret_cast<uint32_t*>(ctx->d_layer);
    const dim3 grid(plan.strips, plan.runs);
#define SC_NORM_GRAD(T)                                                                                                                        \
    do {                                                                                                                                       \
        const T *dyp = static_cast<const T*>(dy), *hp = static_cast<const T*>(h), *gp = static_cast<const T*>(gamma);                          \
        {                                                                                                                                      \
            Launch l(ctx, KIND_RMS_NORM_GRAD, st);                                                                                             \
            launch(norm_stats_kernel<T>, row_grid(ctx, rows), NORM_THREADS, 0, 1, st, dyp, hp, gp, a, stats);                                  \
        }                                                                                                                                      \
        Launch l(ctx, KIND_RMS_NORM_GRAD, st);                                                                                                 \
        launch(norm_strips_kernel<T>, grid, CKPT_THREADS, 0, 1, st, dyp, hp, gp, static_cast<const T*>(residual), a, stats, static_cast<T*>(dh), \
               static_cast<T*>(dx), partial, tickets, dgamma);                                                                                 \
    } while (0)
    if (type == SC_BF16) SC_NORM_GRAD(__nv_bfloat16);
    else SC_NORM_GRAD(__half);
#undef SC_NORM_GRAD
    SC_CUDA(cudaGetLastError());
    return SC_OK;
}

}  // extern "C"
