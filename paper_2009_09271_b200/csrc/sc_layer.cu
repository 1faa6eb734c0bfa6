// Host side of the layer operators declared in include/sparsecomm.h: argument checks, scratch, launches.
#include <algorithm>

#include "sc_checkpoint.cuh"
#include "sc_context.cuh"
#include "sc_product.cuh"

namespace {

constexpr uint64_t MAX_DIM = 1ull << 31;      // rows and columns; offsets are 64-bit throughout

inline bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
inline uint64_t ceil_div(uint64_t a, uint64_t b) { return (a + b - 1) / b; }

inline bool known_type(int type) { return type == SC_BF16 || type == SC_F16; }
inline bool known_act(int act) { return act >= SC_ACT_NONE && act <= SC_ACT_SILU; }
inline size_t type_bytes(int type) { return type == SC_F32 ? 4 : 2; }

// A matrix argument: rows of `cols` elements, `ld` apart.
int check_matrix(const void* p, size_t ld, size_t rows, size_t cols, size_t elem) {
    if (rows >= MAX_DIM || cols >= MAX_DIM) return SC_ERR_RANGE;
    if (ld < cols && rows > 1) return SC_ERR_INVALID;
    if (rows == 0 || cols == 0) return SC_OK;
    return p && aligned(p, elem) ? SC_OK : SC_ERR_INVALID;
}

// The layer operators' scratch: 64 KB of tickets, zero between calls, then `bytes` of workspace.
constexpr size_t TICKET_BYTES = 65536;
constexpr uint32_t MAX_TICKETS = TICKET_BYTES / sizeof(uint32_t);

int layer_scratch(sc_ctx* c, size_t bytes, cudaStream_t st) {
    if (c->d_layer && c->layer_bytes >= bytes) return SC_OK;
    cudaStreamCaptureStatus cap = cudaStreamCaptureStatusNone;
    SC_CUDA(cudaStreamIsCapturing(st, &cap));
    if (cap != cudaStreamCaptureStatusNone) return SC_ERR_WORKSPACE;      // reserve before the capture
    if (c->d_layer) {
        SC_CUDA(cudaStreamSynchronize(st));
        cudaFree(c->d_layer);
        c->scratch_bytes -= TICKET_BYTES + c->layer_bytes;
        c->d_layer = nullptr; c->layer_bytes = 0;
    }
    bytes = (bytes + 255) & ~(size_t)255;
    void* p = nullptr;
    if (cudaMalloc(&p, TICKET_BYTES + bytes) != cudaSuccess) { cudaGetLastError(); return SC_ERR_WORKSPACE; }
    if (cudaMemsetAsync(p, 0, TICKET_BYTES, st) != cudaSuccess) { cudaFree(p); return SC_ERR_CUDA; }
    c->d_layer = static_cast<unsigned char*>(p);
    c->layer_bytes = bytes;
    c->scratch_bytes += TICKET_BYTES + bytes;
    return SC_OK;
}

ItemWalk item_walk(size_t rows, size_t cols, bool vec) {
    ItemWalk w{};
    w.rows = rows; w.cols = (uint32_t)cols;
    w.chunks = (uint32_t)(4 * ckpt_groups(cols));
    w.total = (uint64_t)rows * w.chunks;
    w.vec = vec ? 1u : 0u;
    return w;
}

uint32_t item_grid(const sc_ctx* c, uint64_t total) {
    return (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>(ceil_div(total, CKPT_THREADS * CKPT_UNROLL), (uint64_t)c->sm_count * 8));
}

template <typename T>
void launch_pack(sc_ctx* c, const void* x, size_t ldx, size_t rows, size_t cols, uint8_t* q, uint8_t* scales, cudaStream_t st) {
    const bool vec = aligned(x, 16) && (ldx * sizeof(T)) % 16 == 0 && cols % 8 == 0 && aligned(q, 8);
    const ItemWalk w = item_walk(rows, cols, vec);
    Launch l(c, KIND_CKPT_PACK, st);
    checkpoint_pack_kernel<T><<<item_grid(c, w.total), CKPT_THREADS, 0, st>>>(static_cast<const T*>(x), ldx, w, q, scales);
}

template <typename T>
void launch_unpack(sc_ctx* c, const uint8_t* q, const uint8_t* scales, size_t rows, size_t cols, void* out, size_t ldo, cudaStream_t st) {
    const bool vec = aligned(out, 16) && (ldo * sizeof(T)) % 16 == 0 && cols % 8 == 0 && aligned(q, 8);
    const ItemWalk w = item_walk(rows, cols, vec);
    Launch l(c, KIND_CKPT_UNPACK, st);
    checkpoint_unpack_kernel<T><<<item_grid(c, w.total), CKPT_THREADS, 0, st>>>(q, scales, w, static_cast<T*>(out), ldo);
}

struct GradPlan { uint32_t strips, runs, run_rows; size_t bytes; };

// Runs of rows: enough CTAs to fill the GPU (about eight per SM), none of fewer than 32 rows.
GradPlan grad_plan(const sc_ctx* c, size_t rows, size_t cols) {
    GradPlan p{};
    p.strips = (uint32_t)ceil_div(cols, GRAD_COLS);
    uint64_t runs = std::max<uint64_t>(1, std::min<uint64_t>((uint64_t)c->sm_count * 8 / p.strips, ceil_div(rows, 32)));
    p.run_rows = (uint32_t)(ceil_div(ceil_div(rows, runs), GRAD_LANES) * GRAD_LANES);
    p.runs = (uint32_t)ceil_div(rows, p.run_rows);
    p.bytes = p.runs > 1 ? (size_t)p.runs * cols * sizeof(float) : 0;
    return p;
}

template <typename T>
void launch_product(int mode, const Operand& A, const Operand& B, size_t red, const Epilogue& ep, cudaStream_t st) {
    const dim3 grid((uint32_t)ceil_div(ep.cols, 64), (uint32_t)ceil_div(ep.rows, 64));
    if (mode == PRODUCT_FORWARD) product_plain_kernel<T, PRODUCT_FORWARD><<<grid, 256, 0, st>>>(A, B, red, ep);
    else if (mode == PRODUCT_INPUT) product_plain_kernel<T, PRODUCT_INPUT><<<grid, 256, 0, st>>>(A, B, red, ep);
    else product_plain_kernel<T, PRODUCT_WEIGHT><<<grid, 256, 0, st>>>(A, B, red, ep);
}

void launch_product(int type, int mode, const Operand& A, const Operand& B, size_t red, const Epilogue& ep, cudaStream_t st) {
    if (type == SC_BF16) launch_product<__nv_bfloat16>(mode, A, B, red, ep, st);
    else launch_product<__half>(mode, A, B, red, ep, st);
}

}  // namespace

extern "C" {

int sc_layer_reserve(sc_ctx* ctx, size_t M, size_t N, size_t K) {
    if (!ctx) return SC_ERR_INVALID;
    if (M >= MAX_DIM || N >= MAX_DIM || K >= MAX_DIM) return SC_ERR_RANGE;
    DeviceGuard guard(ctx->device);
    const size_t bytes = 2 * M * K + std::max(grad_plan(ctx, std::max<size_t>(M, 1), std::max<size_t>(N, 1)).bytes, grad_plan(ctx, std::max<size_t>(M, 1), std::max<size_t>(K, 1)).bytes);
    return layer_scratch(ctx, bytes, nullptr);
}

int sc_checkpoint_pack(sc_ctx* ctx, int type, const void* x, size_t ldx, size_t rows, size_t cols, int8_t* q, uint8_t* scales, void* stream) {
    if (!ctx) return SC_ERR_INVALID;
    if (type != SC_F32 && !known_type(type)) return SC_ERR_UNSUPPORTED;
    if (const int rc = check_matrix(x, ldx, rows, cols, type_bytes(type))) return rc;
    if (rows == 0 || cols == 0) return SC_OK;
    if (!q || !scales) return SC_ERR_INVALID;
    DeviceGuard guard(ctx->device);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    uint8_t* qb = reinterpret_cast<uint8_t*>(q);
    if (type == SC_BF16) launch_pack<__nv_bfloat16>(ctx, x, ldx, rows, cols, qb, scales, st);
    else if (type == SC_F16) launch_pack<__half>(ctx, x, ldx, rows, cols, qb, scales, st);
    else launch_pack<float>(ctx, x, ldx, rows, cols, qb, scales, st);
    SC_CUDA(cudaGetLastError());
    return SC_OK;
}

int sc_checkpoint_unpack(sc_ctx* ctx, int type, const int8_t* q, const uint8_t* scales, size_t rows, size_t cols, void* out, size_t ldo, void* stream) {
    if (!ctx) return SC_ERR_INVALID;
    if (type != SC_F32 && !known_type(type)) return SC_ERR_UNSUPPORTED;
    if (const int rc = check_matrix(out, ldo, rows, cols, type_bytes(type))) return rc;
    if (rows == 0 || cols == 0) return SC_OK;
    if (!q || !scales) return SC_ERR_INVALID;
    DeviceGuard guard(ctx->device);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const uint8_t* qb = reinterpret_cast<const uint8_t*>(q);
    if (type == SC_BF16) launch_unpack<__nv_bfloat16>(ctx, qb, scales, rows, cols, out, ldo, st);
    else if (type == SC_F16) launch_unpack<__half>(ctx, qb, scales, rows, cols, out, ldo, st);
    else launch_unpack<float>(ctx, qb, scales, rows, cols, out, ldo, st);
    SC_CUDA(cudaGetLastError());
    return SC_OK;
}

int sc_activation_grad(sc_ctx* ctx, int type, int act, const void* dy, size_t lddy, const int8_t* q, const uint8_t* scales,
                       size_t rows, size_t cols, void* dz, size_t lddz, float* db, int accumulate, void* stream) {
    if (!ctx) return SC_ERR_INVALID;
    if (!known_type(type)) return SC_ERR_UNSUPPORTED;
    if (!known_act(act)) return SC_ERR_INVALID;
    if (const int rc = check_matrix(dy, lddy, rows, cols, 2)) return rc;
    if (dz) if (const int rc = check_matrix(dz, lddz, rows, cols, 2)) return rc;
    if (!dz && !db) return SC_ERR_INVALID;
    if (!aligned(db, 4)) return SC_ERR_INVALID;
    if (cols == 0) return SC_OK;
    const bool kept = act != SC_ACT_NONE;
    if (kept && rows && (!q || !scales)) return SC_ERR_INVALID;
    if (ceil_div(cols, GRAD_COLS) > MAX_TICKETS) return SC_ERR_RANGE;
    DeviceGuard guard(ctx->device);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (rows == 0) {
        if (db && !accumulate) SC_CUDA(cudaMemsetAsync(db, 0, cols * sizeof(float), st));
        return SC_OK;
    }
    const GradPlan p = grad_plan(ctx, rows, cols);
    if (db) if (const int rc = layer_scratch(ctx, p.bytes, st)) return rc;
    GradArgs a{};
    a.rows = rows; a.lddy = lddy; a.lddz = lddz; a.cols = (uint32_t)cols; a.groups = (uint32_t)ckpt_groups(cols);
    a.runs = p.runs; a.run_rows = p.run_rows; a.accumulate = accumulate ? 1u : 0u; a.act = act;
    a.vec = cols % 8 == 0 && aligned(dy, 16) && lddy % 8 == 0 && (!dz || (aligned(dz, 16) && lddz % 8 == 0)) && (!kept || aligned(q, 8)) ? 1u : 0u;
    float* partial = reinterpret_cast<float*>(ctx->d_layer ? ctx->d_layer + TICKET_BYTES : nullptr);
    uint32_t* tickets = reinterpret_cast<uint32_t*>(ctx->d_layer);
    const dim3 grid(p.strips, p.runs);
    const uint8_t* qb = reinterpret_cast<const uint8_t*>(q);
    {
        Launch l(ctx, KIND_ACT_GRAD, st);
#define SC_GRAD(T, KEPT) activation_grad_kernel<T, KEPT><<<grid, CKPT_THREADS, 0, st>>>( \
            static_cast<const T*>(dy), qb, scales, a, static_cast<T*>(dz), partial, tickets, db)
        if (type == SC_BF16) { if (kept) SC_GRAD(__nv_bfloat16, true); else SC_GRAD(__nv_bfloat16, false); }
        else { if (kept) SC_GRAD(__half, true); else SC_GRAD(__half, false); }
#undef SC_GRAD
    }
    SC_CUDA(cudaGetLastError());
    return SC_OK;
}

int sc_linear(sc_ctx* ctx, int type, int act, const void* x, size_t ldx, const void* w, size_t ldw, const void* bias,
              const void* residual, size_t ldr, size_t M, size_t N, size_t K, void* y, size_t ldy, int8_t* q, uint8_t* scales, void* stream) {
    if (!ctx) return SC_ERR_INVALID;
    if (!known_type(type)) return SC_ERR_UNSUPPORTED;
    if (!known_act(act) || (q == nullptr) != (scales == nullptr) || !aligned(bias, 2)) return SC_ERR_INVALID;
    if (const int rc = check_matrix(x, ldx, M, K, 2)) return rc;
    if (const int rc = check_matrix(w, ldw, N, K, 2)) return rc;
    if (const int rc = check_matrix(y, ldy, M, N, 2)) return rc;
    if (residual) if (const int rc = check_matrix(residual, ldr, M, N, 2)) return rc;
    if (M == 0 || N == 0) return SC_OK;
    DeviceGuard guard(ctx->device);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    Epilogue ep{};
    ep.bias = bias; ep.residual = residual; ep.ldr = ldr; ep.out = y; ep.ldo = ldy; ep.rows = M; ep.cols = (uint32_t)N;
    ep.q = reinterpret_cast<uint8_t*>(q); ep.scales = scales; ep.groups = (uint32_t)ckpt_groups(N); ep.act = act;
    { Launch l(ctx, KIND_LINEAR, st);
      launch_product(type, PRODUCT_FORWARD, Operand{x, ldx, 1}, Operand{w, ldw, 1}, K, ep, st); }
    SC_CUDA(cudaGetLastError());
    return SC_OK;
}

int sc_linear_grad_input(sc_ctx* ctx, int type, int act, const void* dz, size_t lddz, const void* w, size_t ldw, const void* residual,
                         size_t ldr, const int8_t* q, const uint8_t* scales, size_t M, size_t N, size_t K, void* dx, size_t lddx, void* stream) {
    if (!ctx) return SC_ERR_INVALID;
    if (!known_type(type)) return SC_ERR_UNSUPPORTED;
    if (!known_act(act)) return SC_ERR_INVALID;
    if (const int rc = check_matrix(dz, lddz, M, N, 2)) return rc;
    if (const int rc = check_matrix(w, ldw, N, K, 2)) return rc;
    if (const int rc = check_matrix(dx, lddx, M, K, 2)) return rc;
    if (residual) if (const int rc = check_matrix(residual, ldr, M, K, 2)) return rc;
    if (M == 0 || K == 0) return SC_OK;
    if (act != SC_ACT_NONE && (!q || !scales)) return SC_ERR_INVALID;
    DeviceGuard guard(ctx->device);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    Epilogue ep{};
    ep.residual = residual; ep.ldr = ldr; ep.out = dx; ep.ldo = lddx; ep.rows = M; ep.cols = (uint32_t)K; ep.act = act;
    if (act != SC_ACT_NONE) {
        ep.q = const_cast<uint8_t*>(reinterpret_cast<const uint8_t*>(q));
        ep.scales = const_cast<uint8_t*>(scales);
        ep.groups = (uint32_t)ckpt_groups(K);
    }
    { Launch l(ctx, KIND_LINEAR_DX, st);
      launch_product(type, PRODUCT_INPUT, Operand{dz, lddz, 1}, Operand{w, 1, ldw}, N, ep, st); }
    SC_CUDA(cudaGetLastError());
    return SC_OK;
}

int sc_linear_grad_weight(sc_ctx* ctx, int type, const void* dz, size_t lddz, const void* x, size_t ldx, const int8_t* q,
                          const uint8_t* scales, size_t M, size_t N, size_t K, float* dw, size_t lddw, int accumulate, void* stream) {
    if (!ctx) return SC_ERR_INVALID;
    if (!known_type(type)) return SC_ERR_UNSUPPORTED;
    if ((x != nullptr) == (q != nullptr) && M && K) return SC_ERR_INVALID;
    if (const int rc = check_matrix(dz, lddz, M, N, 2)) return rc;
    if (const int rc = check_matrix(dw, lddw, N, K, 4)) return rc;
    if (x) if (const int rc = check_matrix(x, ldx, M, K, 2)) return rc;
    if (N == 0 || K == 0) return SC_OK;
    if (q && !scales) return SC_ERR_INVALID;
    DeviceGuard guard(ctx->device);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (q && M) {
        if (const int rc = layer_scratch(ctx, 2 * M * K, st)) return rc;
        void* wide = ctx->d_layer + TICKET_BYTES;
        const uint8_t* qb = reinterpret_cast<const uint8_t*>(q);
        if (type == SC_BF16) launch_unpack<__nv_bfloat16>(ctx, qb, scales, M, K, wide, K, st);
        else launch_unpack<__half>(ctx, qb, scales, M, K, wide, K, st);
        x = wide; ldx = K;
    }
    Epilogue ep{};
    ep.out = dw; ep.ldo = lddw; ep.rows = N; ep.cols = (uint32_t)K; ep.accumulate = accumulate ? 1u : 0u;
    { Launch l(ctx, KIND_LINEAR_DW, st);
      launch_product(type, PRODUCT_WEIGHT, Operand{dz, 1, lddz}, Operand{x, 1, ldx}, M, ep, st); }
    SC_CUDA(cudaGetLastError());
    return SC_OK;
}

}  // extern "C"
