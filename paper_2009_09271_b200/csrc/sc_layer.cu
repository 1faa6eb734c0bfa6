// Host side of the layer operators declared in include/sparsecomm.h: arguments, kernels, launches.
#include "sc_checkpoint.cuh"
#include "sc_product_host.cuh"

namespace {

uint32_t item_grid(const sc_ctx* c, uint64_t total) {
    return (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>(ceil_div(total, CKPT_THREADS), (uint64_t)c->sm_count * 8));
}

ItemWalk item_walk(const sc_ctx* c, size_t rows, size_t cols, const uint8_t* q, const void* x, size_t ldx, size_t elem) {
    ItemWalk w{};
    w.cols = (uint32_t)cols;
    w.items = (uint32_t)(2 * ckpt_groups(cols));
    w.total = (uint64_t)rows * w.items;
    const uint64_t stride = (uint64_t)item_grid(c, w.total) * CKPT_THREADS;
    w.stride_rows = stride / w.items;
    w.stride_items = (uint32_t)(stride % w.items);
    w.grain_x = grain_of(x, rows > 1 ? ldx : 0, elem, 16);
    w.grain_q = grain_of(q, rows > 1 ? cols : 0, 1, 16);
    return w;
}

// Rows that are aligned to single elements only, or such a q, take the narrow form: unpacking 5181 x 265 takes 7.8 us in it and
// 13.3 in the wide form.  With rows of two elements and more the wide form is ahead (3853 x 10730: 66 us against 105).
bool narrow_walk(const sc_ctx* c, const ItemWalk& wide, size_t rows, size_t cols, NarrowWalk& w, uint32_t& grid) {
    if (wide.grain_q > 1 && wide.grain_x > 1) return false;
    w.cols = (uint32_t)cols;
    w.runs = (uint32_t)ceil_div(cols, 64);
    w.total = (uint64_t)rows * w.runs;
    grid = (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>(ceil_div(w.total, CKPT_THREADS / 32), (uint64_t)c->sm_count * 8));
    const uint64_t stride = (uint64_t)grid * (CKPT_THREADS / 32);
    w.stride_rows = stride / w.runs;
    w.stride_runs = (uint32_t)(stride % w.runs);
    w.two_x = wide.grain_x >= 2; w.two_q = wide.grain_q >= 2;
    return true;
}

template <typename T>
void launch_pack(sc_ctx* c, const void* x, size_t ldx, size_t rows, size_t cols, uint8_t* q, uint8_t* scales, cudaStream_t st) {
    const ItemWalk w = item_walk(c, rows, cols, q, x, ldx, sizeof(T));
    NarrowWalk n{};
    uint32_t grid = 0;
    Launch l(c, KIND_CKPT_PACK, st);
    if (narrow_walk(c, w, rows, cols, n, grid))
        launch(checkpoint_pack_narrow_kernel<T>, grid, CKPT_THREADS, 0, 1, st, static_cast<const T*>(x), ldx, n, q, scales);
    else
        launch(checkpoint_pack_kernel<T>, item_grid(c, w.total), CKPT_THREADS, 0, 1, st, static_cast<const T*>(x), ldx, w, q, scales);
}

template <typename T>
void launch_unpack(sc_ctx* c, const uint8_t* q, const uint8_t* scales, size_t rows, size_t cols, void* out, size_t ldo, cudaStream_t st) {
    const ItemWalk w = item_walk(c, rows, cols, q, out, ldo, sizeof(T));
    NarrowWalk n{};
    uint32_t grid = 0;
    Launch l(c, KIND_CKPT_UNPACK, st);
    if (narrow_walk(c, w, rows, cols, n, grid))
        launch(checkpoint_unpack_narrow_kernel<T>, grid, CKPT_THREADS, 0, 1, st, q, scales, n, static_cast<T*>(out), ldo);
    else
        launch(checkpoint_unpack_kernel<T>, item_grid(c, w.total), CKPT_THREADS, 0, 1, st, q, scales, w, static_cast<T*>(out), ldo);
}

struct GradPlan { uint32_t strips, runs, run_rows; size_t bytes; };

// Runs of rows: enough CTAs to fill the GPU (about eight per SM), none of fewer than 32 rows.  A strip has a ticket where it has more
// than one run, which takes at most four strips per SM: far fewer than there are tickets.
GradPlan grad_plan(const sc_ctx* c, size_t rows, size_t cols) {
    GradPlan p{};
    p.strips = (uint32_t)ceil_div(cols, GRAD_COLS);
    uint64_t runs = std::max<uint64_t>(1, std::min<uint64_t>((uint64_t)c->sm_count * 8 / p.strips, ceil_div(rows, 32)));
    p.run_rows = (uint32_t)(ceil_div(ceil_div(rows, runs), GRAD_LANES) * GRAD_LANES);
    p.runs = (uint32_t)ceil_div(rows, p.run_rows);
    p.bytes = p.runs > 1 ? (size_t)p.runs * cols * sizeof(float) : 0;
    return p;
}

template <typename T, int TOKENS>
void run_tokens(const Stored& x, const Stored& w, const Epilogue& ep, cudaStream_t st) {
    const uint32_t gx = grain_of(x.p, x.rows > 1 ? x.ld : 0, 2, 8), gw = grain_of(w.p, w.rows > 1 ? w.ld : 0, 2, 8);
    const bool wide = gx == 8 && gw == 8;
    const T *xp = static_cast<const T*>(x.p), *wp = static_cast<const T*>(w.p);
    const uint32_t K = (uint32_t)x.cols;
#define SC_TOKENS(WN, WK, WIDE) launch(product_tokens_kernel<T, TOKENS, WN, WK, WIDE>, (uint32_t)ceil_div(ep.cols, 4 * WN), WN * WK * 32, 0, 1, st, xp, x.ld, wp, w.ld, K, gx, gw, ep)
    if (ep.q) { if (wide) SC_TOKENS(8, 4, true); else SC_TOKENS(8, 4, false); }
    else if (wide) SC_TOKENS(2, 4, true);
    else SC_TOKENS(2, 4, false);
#undef SC_TOKENS
}

template <typename T>
void run_tokens(const Stored& x, const Stored& w, const Epilogue& ep, cudaStream_t st) {
    if (ep.rows == 1) run_tokens<T, 1>(x, w, ep, st);
    else if (ep.rows == 2) run_tokens<T, 2>(x, w, ep, st);
    else run_tokens<T, 4>(x, w, ep, st);
}

// One and two tokens are ahead of the tiles at every size measured (1 x 4096 x 4096: 7.8 against 11.6 us, 2 x 16384 x 4096: 26
// against 31); three and four while the call is short (1024 x 1024: 2.9 against 7.8 us; 4096 x 4096: 13.1 against 12.1).
bool few_tokens(uint64_t M, uint64_t N, uint64_t K) { return K && (M <= 2 || (M <= 4 && N * K <= (8u << 20))); }

template <int MODE>
int run_product(sc_ctx* c, int kind, int type, const Stored& A, const Stored& B, uint64_t red, const Epilogue& ep, size_t used, cudaStream_t st) {
    // the weight gradient is fp32 whatever the operands are: one build serves both types
    if constexpr (MODE != PRODUCT_WEIGHT)
        if (type == SC_F16) return run_product<__half, MODE>(c, kind, type, A, B, red, ep, used, st);
    return run_product<__nv_bfloat16, MODE>(c, kind, type, A, B, red, ep, used, st);
}

constexpr uint64_t FEW_WEIGHT_TOKENS = 8;

template <typename T, int TOKENS, bool KEPT>
void launch_weight_tokens(sc_ctx* c, const void* dz, size_t lddz, const void* x, size_t ldx, const uint8_t* q, const uint8_t* scales, size_t M,
                          const Epilogue& ep, cudaStream_t st) {
    // rows per CTA: one round of the CTAs that fit on the SMs, where that leaves 8 to 512 rows each
    const uint64_t columns = ceil_div(ep.cols, 128), strips = std::max<uint64_t>(1, (uint64_t)c->sm_count * (TOKENS == 4 ? 5 : 3) / columns);
    const uint32_t run = (uint32_t)std::min<uint64_t>(512, std::max<uint64_t>(8, ceil_div(ep.rows, strips)));
    launch(weight_tokens_kernel<T, TOKENS, KEPT>, dim3((uint32_t)columns, (uint32_t)ceil_div(ep.rows, run)), 256, run * TOKENS * sizeof(float2), 1, st,
           static_cast<const T*>(dz), lddz, static_cast<const T*>(x), ldx, q, scales, (uint32_t)M, run, ep);
}

template <typename T>
void run_weight_tokens(sc_ctx* c, const void* dz, size_t lddz, const void* x, size_t ldx, const uint8_t* q, const uint8_t* scales, size_t M, const Epilogue& ep,
                       cudaStream_t st) {
    if (q) { if (M <= 4) launch_weight_tokens<T, 4, true>(c, dz, lddz, x, ldx, q, scales, M, ep, st);
             else launch_weight_tokens<T, 8, true>(c, dz, lddz, x, ldx, q, scales, M, ep, st); }
    else if (M <= 4) launch_weight_tokens<T, 4, false>(c, dz, lddz, x, ldx, q, scales, M, ep, st);
    else launch_weight_tokens<T, 8, false>(c, dz, lddz, x, ldx, q, scales, M, ep, st);
}

// A wait of the layer products where nothing arrives.
__global__ void layer_wait_probe_kernel(long long limit, int* status) {
    __shared__ __align__(8) unsigned long long word;
    const uint32_t bar = smem_addr(&word);
    if (threadIdx.x == 0) { mbar_init(bar, 1); mbar_init_fence(); }
    __syncwarp();
    if (!warp_wait(bar, 0, limit) && threadIdx.x == 0) atomicCAS(status, 0, ST_TIMEOUT);
}

}  // namespace

int layer_wait_probe(sc_ctx* c, long long limit_cycles, cudaStream_t st) {
    layer_wait_probe_kernel<<<1, 32, 0, st>>>(std::min(limit_cycles, MBAR_LIMIT_CYCLES), c->d_status);
    return cudaGetLastError() == cudaSuccess ? SC_OK : SC_ERR_CUDA;
}

extern "C" {

int sc_layer_reserve(sc_ctx* ctx, size_t M, size_t N, size_t K) {
    if (!ctx) return SC_ERR_INVALID;
    if (M >= MAX_DIM || N >= MAX_DIM || K >= MAX_DIM) return SC_ERR_RANGE;
    DeviceGuard guard(ctx->device);
    // the operands' copies (x^ always, the others where rows are not 16-byte aligned) and partial sums; the bias gradient's
    // partial rows are far below the latter
    const size_t copies[3] = {layout_bytes(M, K), layout_bytes(N, K), layout_bytes(M, N)};
    size_t bytes = PARTIAL_CAP;
    for (const size_t n : copies) {
        if (n > SIZE_MAX / 4) return SC_ERR_WORKSPACE;                    // a sum of three would wrap
        bytes += n;
    }
    return layer_scratch(ctx, bytes, nullptr);
}

int sc_debug_layer_tiles(sc_ctx* ctx, int rows, int cols, int parts) {
    if (!ctx) return SC_ERR_INVALID;
    const bool none = rows == 0 && cols == 0 && parts == 0;
    const bool pair = rows == 256 && cols == 256, single = rows == 128 && (cols == 64 || cols == 128 || cols == 256);
    if (!none && ((!pair && !single) || parts < 1 || parts > 64)) return SC_ERR_INVALID;
    ctx->layer_force_bn = cols; ctx->layer_force_cg = pair ? 2 : 1; ctx->layer_force_parts = (uint32_t)parts;
    for (ProductPlan& p : ctx->layer_plans) p = ProductPlan{};
    return SC_OK;
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
    DeviceGuard guard(ctx->device);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (rows == 0) {
        if (db && !accumulate) SC_CUDA(cudaMemsetAsync(db, 0, cols * sizeof(float), st));
        return SC_OK;
    }
    const GradPlan p = grad_plan(ctx, rows, cols);
    if (db && p.runs > 1) if (const int rc = layer_scratch(ctx, p.bytes, st)) return rc;
    GradArgs a{};
    a.rows = rows; a.lddy = lddy; a.lddz = lddz; a.cols = (uint32_t)cols; a.groups = (uint32_t)ckpt_groups(cols);
    a.runs = p.runs; a.run_rows = p.run_rows; a.accumulate = accumulate ? 1u : 0u;
    a.grain_y = grain_of(dy, rows > 1 ? lddy : 0, 2, 8);
    a.grain_z = grain_of(dz, rows > 1 ? lddz : 0, 2, 8);
    a.grain_q = grain_of(q, rows > 1 ? cols : 0, 1, 8);
    const bool wide = cols % 8 == 0 && a.grain_y == 8 && a.grain_z == 8 && (!kept || a.grain_q == 8);
    float* partial = reinterpret_cast<float*>(ctx->d_layer ? ctx->d_layer + TICKET_BYTES : nullptr);
    uint32_t* tickets = reinterpret_cast<uint32_t*>(ctx->d_layer);
    const dim3 grid(p.strips, p.runs);
    const uint8_t* qb = reinterpret_cast<const uint8_t*>(q);
    {
        Launch l(ctx, KIND_ACT_GRAD, st);
#define SC_GRAD(T, ACT, WIDE) launch(activation_grad_kernel<T, ACT, WIDE>, grid, CKPT_THREADS, 0, 1, st, \
            static_cast<const T*>(dy), qb, scales, a, static_cast<T*>(dz), partial, tickets, db)
#define SC_GRAD_ACT(ACT)                                                                                     \
        case ACT:                                                                                            \
            if (type == SC_BF16) { if (wide) SC_GRAD(__nv_bfloat16, ACT, true); else SC_GRAD(__nv_bfloat16, ACT, false); } \
            else { if (wide) SC_GRAD(__half, ACT, true); else SC_GRAD(__half, ACT, false); }                  \
            break;
        switch (act) { SC_GRAD_ACT(SC_ACT_NONE) SC_GRAD_ACT(SC_ACT_RELU) SC_GRAD_ACT(SC_ACT_GELU) SC_GRAD_ACT(SC_ACT_GELU_TANH) SC_GRAD_ACT(SC_ACT_SILU) }
#undef SC_GRAD_ACT
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
    ep.grain_out = grain_of(y, M > 1 ? ldy : 0, 2, 8); ep.grain_res = grain_of(residual, M > 1 ? ldr : 0, 2, 8);
    ep.grain_q = grain_of(q, M > 1 ? N : 0, 1, 32); ep.grain_bias = grain_of(bias, 0, 2, 8);
    if (few_tokens(M, N, K)) {
        Launch l(ctx, KIND_LINEAR, st);
        const Stored xs{x, M, K, ldx}, ws{w, N, K, ldw};
        if (type == SC_BF16) run_tokens<__nv_bfloat16>(xs, ws, ep, st);
        else run_tokens<__half>(xs, ws, ep, st);
        SC_CUDA(cudaGetLastError());
        return SC_OK;
    }
    if (const int rc = run_product<PRODUCT_FORWARD>(ctx, KIND_LINEAR, type, Stored{x, M, K, ldx}, Stored{w, N, K, ldw}, K, ep, 0, st)) return rc;
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
    ep.grain_out = grain_of(dx, M > 1 ? lddx : 0, 2, 8); ep.grain_res = grain_of(residual, M > 1 ? ldr : 0, 2, 8);
    ep.grain_q = grain_of(q, M > 1 ? K : 0, 1, 16);
    if (const int rc = run_product<PRODUCT_INPUT>(ctx, KIND_LINEAR_DX, type, Stored{dz, M, N, lddz}, Stored{w, N, K, ldw}, N, ep, 0, st)) return rc;
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
    Epilogue ep{};
    ep.out = dw; ep.ldo = lddw; ep.rows = N; ep.cols = (uint32_t)K; ep.accumulate = accumulate ? 1u : 0u;
    if (N == 1) ep.ldo = lddw = (K + 3) & ~(size_t)3;                // the distance between rows says nothing
    ep.grain_out = grain_of(dw, lddw, 4, 4);
    ep.groups = (uint32_t)ckpt_groups(K);
    if (M && M <= FEW_WEIGHT_TOKENS && N <= 65535ull * 8) {
        const uint8_t* qb = reinterpret_cast<const uint8_t*>(q);
        Launch l(ctx, KIND_LINEAR_DW, st);
        if (type == SC_BF16) run_weight_tokens<__nv_bfloat16>(ctx, dz, lddz, x, ldx, qb, scales, M, ep, st);
        else run_weight_tokens<__half>(ctx, dz, lddz, x, ldx, qb, scales, M, ep, st);
        SC_CUDA(cudaGetLastError());
        return SC_OK;
    }
    size_t used = 0;
    if (q && M) {                                  // the checkpoint's values, rows 16-byte aligned
        used = layout_bytes(M, K);
        const Stored dzs{dz, M, N, lddz};
        if (const int rc = layer_scratch(ctx, used + product_plan(ctx, PRODUCT_WEIGHT, N, K, M).bytes + (tma_ready(dzs) ? 0 : layout_bytes(M, N)), st)) return rc;
        void* wide = ctx->d_layer + TICKET_BYTES;
        const uint8_t* qb = reinterpret_cast<const uint8_t*>(q);
        if (type == SC_BF16) launch_unpack<__nv_bfloat16>(ctx, qb, scales, M, K, wide, round8(K), st);
        else launch_unpack<__half>(ctx, qb, scales, M, K, wide, round8(K), st);
        x = wide; ldx = round8(K);
    }
    if (const int rc = run_product<PRODUCT_WEIGHT>(ctx, KIND_LINEAR_DW, type, Stored{dz, M, N, lddz}, Stored{x, M, K, ldx}, M, ep, used, st)) return rc;
    SC_CUDA(cudaGetLastError());
    return SC_OK;
}

}  // extern "C"
