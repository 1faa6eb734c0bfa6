// Host side of the linear layer on 8-bit integers, declared in include/sparsecomm.h.
#include "sc_product_host.cuh"

namespace {

constexpr uint64_t MAX_TERMS = 131071;        // products of up to 2^14 that a 32-bit integer sum holds: 131071 2^14 < 2^31

template <typename T, int TOKENS>
void run_tokens(const Stored& x, const Stored& w, const Epilogue& ep, cudaStream_t st) {
    const uint8_t *xp = static_cast<const uint8_t*>(x.p), *wp = static_cast<const uint8_t*>(w.p);
    const uint32_t K = (uint32_t)x.cols;
    if (ep.q) launch(quantized_tokens_kernel<T, TOKENS, 8>, (uint32_t)ceil_div(ep.cols, 32), 8 * 4 * 32, 0, 1, st, xp, x.ld, wp, w.ld, K, ep);
    else launch(quantized_tokens_kernel<T, TOKENS, 2>, (uint32_t)ceil_div(ep.cols, 8), 2 * 4 * 32, 0, 1, st, xp, x.ld, wp, w.ld, K, ep);
}
template <typename T, int EIGHTS>
void run_eights(const Stored& x, const Stored& w, const Epilogue& ep, cudaStream_t st) {
    const uint8_t *xp = static_cast<const uint8_t*>(x.p), *wp = static_cast<const uint8_t*>(w.p);
    const uint32_t K = (uint32_t)x.cols;
    if (ep.q) launch(quantized_eights_kernel<T, EIGHTS, 2>, (uint32_t)ceil_div(ep.cols, 32), 2 * TOKENS_WK * 32, 0, 1, st, xp, x.ld, wp, w.ld, K, ep);
    else launch(quantized_eights_kernel<T, EIGHTS, 1>, (uint32_t)ceil_div(ep.cols, 16), TOKENS_WK * 32, 0, 1, st, xp, x.ld, wp, w.ld, K, ep);
}

// What the kernels without tiles take: rows that are 16-byte aligned and a multiple of 16 long.  Up to 8 tokens they are ahead of the tiles
// (8 x 4096 x 4096: 7.3 against 10.5 us, 8 x 16384 x 4096 19 against 20), but for long sums, where they are up to a tenth behind (8 x 4096 x 16384 19.5 against
// 17.8), and up to 32 while the weights are few (32 x 4096 x 4096 10.7 against 11.5; 16 x 16384 x 4096 26 against 17).
bool few_tokens(const Stored& x, const Stored& w) {
    return tma_ready(x) && tma_ready(w) && x.cols % 16 == 0 && (x.rows <= 8 || (x.rows <= 32 && w.rows * w.cols <= (32u << 20)));
}

template <typename T>
int run(sc_ctx* c, int type, const Stored& x, const Stored& w, const Epilogue& ep, cudaStream_t st) {
    // an empty sum has nothing to scale: the forward product's epilogue alone
    if (x.cols == 0) return run_product<T, PRODUCT_FORWARD>(c, KIND_LINEAR_QUANTIZED, type, x, w, 0, ep, 0, st);
    if (!c->layer_force_bn && few_tokens(x, w)) {
        Launch l(c, KIND_LINEAR_QUANTIZED, st);
        if (ep.rows == 1) run_tokens<T, 1>(x, w, ep, st);
        else if (ep.rows == 2) run_tokens<T, 2>(x, w, ep, st);
        else if (ep.rows <= 8) run_eights<T, 1>(x, w, ep, st);
        else if (ep.rows <= 16) run_eights<T, 2>(x, w, ep, st);
        else run_eights<T, 4>(x, w, ep, st);
        return SC_OK;
    }
    return run_product<T, PRODUCT_QUANTIZED>(c, KIND_LINEAR_QUANTIZED, type, x, w, x.cols, ep, 0, st);
}

}  // namespace

extern "C" {

int sc_linear_quantized(sc_ctx* ctx, int type, int act, const int8_t* x, size_t ldx, const float* x_scales, const int8_t* w, size_t ldw,
                        const float* w_scales, const void* bias, const void* residual, size_t ldr, size_t M, size_t N, size_t K, void* y, size_t ldy,
                        int8_t* q, uint8_t* scales, void* stream) {
    if (!ctx) return SC_ERR_INVALID;
    if (!known_type(type)) return SC_ERR_UNSUPPORTED;
    if (!known_act(act) || (q == nullptr) != (scales == nullptr) || !aligned(bias, 2) || !aligned(x_scales, 4) || !aligned(w_scales, 4)) return SC_ERR_INVALID;
    if (const int rc = check_matrix(x, ldx, M, K, 1)) return rc;
    if (const int rc = check_matrix(w, ldw, N, K, 1)) return rc;
    if (const int rc = check_matrix(y, ldy, M, N, 2)) return rc;
    if (residual) if (const int rc = check_matrix(residual, ldr, M, N, 2)) return rc;
    if (K > MAX_TERMS) return SC_ERR_RANGE;
    if (M == 0 || N == 0) return SC_OK;
    if (K && (!x_scales || !w_scales)) return SC_ERR_INVALID;
    DeviceGuard guard(ctx->device);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    Epilogue ep{};
    ep.bias = bias; ep.residual = residual; ep.ldr = ldr; ep.out = y; ep.ldo = ldy; ep.rows = M; ep.cols = (uint32_t)N;
    ep.q = reinterpret_cast<uint8_t*>(q); ep.scales = scales; ep.groups = (uint32_t)ckpt_groups(N); ep.act = act;
    ep.row_scale = x_scales; ep.col_scale = w_scales; ep.scales_by16 = aligned(w_scales, 16);
    ep.grain_out = grain_of(y, M > 1 ? ldy : 0, 2, 8); ep.grain_res = grain_of(residual, M > 1 ? ldr : 0, 2, 8);
    ep.grain_q = grain_of(q, M > 1 ? N : 0, 1, 32); ep.grain_bias = grain_of(bias, 0, 2, 8);
    const Stored xs{x, M, K, ldx, 1}, ws{w, N, K, ldw, 1};
    const int rc = type == SC_BF16 ? run<__nv_bfloat16>(ctx, type, xs, ws, ep, st) : run<__half>(ctx, type, xs, ws, ep, st);
    if (rc) return rc;
    SC_CUDA(cudaGetLastError());
    return SC_OK;
}

}  // extern "C"
