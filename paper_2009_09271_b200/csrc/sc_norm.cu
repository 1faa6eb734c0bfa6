// Host side of 8-bit rows, the root-mean-square norm and dropout, declared in include/sparsecomm.h.
#include <atomic>
#include <cmath>

#include "sc_layer_host.cuh"
#include "sc_norm.cuh"

namespace {

// The walk of a grid over `items` items a row, and the grid: eight CTAs an SM, or as many as give each thread one round of so many items.
ItemWalk item_walk(const sc_ctx* c, size_t rows, size_t cols, uint64_t items, uint32_t& grid, int round) {
    ItemWalk w{};
    w.cols = (uint32_t)cols;
    w.items = (uint32_t)items;
    w.total = (uint64_t)rows * w.items;
    const uint64_t few = std::min<uint64_t>(ceil_div(w.total, CKPT_THREADS), (uint64_t)c->sm_count * 8), one = ceil_div(w.total, (uint64_t)CKPT_THREADS * round);
    grid = (uint32_t)std::min<uint64_t>(std::max(few, one), 1u << 30);
    const uint64_t stride = (uint64_t)grid * CKPT_THREADS;
    w.stride_rows = stride / w.items;
    w.stride_items = (uint32_t)(stride % w.items);
    return w;
}
uint32_t row_grid(const sc_ctx* c, size_t rows) { return (uint32_t)std::min<uint64_t>(rows, (uint64_t)c->sm_count * 8); }

inline uint32_t grain16(const void* p, size_t rows, size_t ld) { return grain_of(p, rows > 1 ? ld : 0, 2, 8); }

// How a matrix's rows are cut, and whether another's are cut the same (one that is not there is).
Phase phase_of(const void* p, size_t rows, size_t ld, size_t elem) {
    return Phase{(uint32_t)(reinterpret_cast<uintptr_t>(p) / elem) & 7u, rows > 1 ? (uint32_t)ld & 7u : 0u};
}
bool in_phase(const Phase& phase, const void* p, size_t rows, size_t ld, size_t elem) {
    const Phase own = phase_of(p, rows, ld, elem);
    return !p || (own.first == phase.first && own.ld == phase.ld);
}
InRows in_rows(const Phase& phase, const void* p, size_t rows, size_t ld, size_t elem = 2) { return InRows{p, ld, in_phase(phase, p, rows, ld, elem)}; }
OutRows out_rows(const Phase& phase, void* p, size_t rows, size_t ld, size_t elem = 2) { return OutRows{p, ld, in_phase(phase, p, rows, ld, elem)}; }
inline bool unshifted(const Phase& phase, size_t cols) { return phase.first == 0 && phase.ld == 0 && cols % 8 == 0; }

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

// Runs f(team, elements / 8 a thread) for the threads that hold a row's chunks of eight; false where it is too long for them.  How a row
// is shared out, and with it the order of its sums, depends on its length and on how the first operand's rows are cut, not on where the results
// or the other operands lie.
template <typename F>
bool with_team(uint64_t chunks, F&& f) {
    using std::integral_constant;
#define SC_TEAM(TEAM, V) if (chunks <= (uint64_t)TEAM * V) { f(integral_constant<int, TEAM>(), integral_constant<int, V>()); return true; }
    SC_TEAM(32, 1) SC_TEAM(32, 2) SC_TEAM(32, 4) SC_TEAM(128, 2) SC_TEAM(256, 2) SC_TEAM(256, 4) SC_TEAM(512, 4) SC_TEAM(1024, 4)
#undef SC_TEAM
    return false;
}
inline uint32_t team_grid(int team, size_t rows) { return (uint32_t)(team == 32 ? ceil_div(rows, 8) : rows); }
inline int team_threads(int team) { return team == 32 ? 256 : team; }

template <typename T>
void run_quantize(sc_ctx* c, const QuantizeArgs& a, float* scales, cudaStream_t st) {
    const bool wide = unshifted(a.phase, a.cols) && a.q.vec;
    const bool held = with_team(a.cols / 8, [&](auto team, auto v) {
        constexpr int TEAM = decltype(team)::value, V = decltype(v)::value;
        if (wide) launch(quantize_rows_kernel<T, TEAM, V, true>, team_grid(TEAM, a.rows), team_threads(TEAM), 0, 1, st, a, scales);
        else launch(quantize_rows_kernel<T, TEAM, V, false>, team_grid(TEAM, a.rows), team_threads(TEAM), 0, 1, st, a, scales);
    });
    if (!held) launch(quantize_kernel<T>, row_grid(c, a.rows), NORM_THREADS, 0, 1, st, a, scales);
}

template <typename T>
void run_dequantize(sc_ctx* c, const void* q, size_t ldq, const float* scales, size_t rows, size_t cols, void* out, size_t ldo, cudaStream_t st) {
    uint32_t grid = 0;
    const uint32_t grain_x = grain_of(out, rows > 1 ? ldo : 0, sizeof(T), 16), grain_q = grain_of(q, rows > 1 ? ldq : 0, 1, 16);
    if (cols % 16 == 0 && grain_q >= 16 && grain_x * sizeof(T) >= 32) {
        // 16384 x 8192 to bf16: 62 us in one round, 69 with eight CTAs an SM
        const ItemWalk w = item_walk(c, rows, cols, cols / 16, grid, DEQUANTIZE_UNROLL);
        launch(dequantize_kernel<T>, grid, CKPT_THREADS, 0, 1, st, static_cast<const uint8_t*>(q), ldq, scales, w, static_cast<T*>(out), ldo);
    } else {
        DequantizeArgs a{};
        a.rows = rows; a.cols = (uint32_t)cols; a.scales = scales;
        a.phase = phase_of(out, rows, ldo, sizeof(T));
        a.q = in_rows(a.phase, q, rows, ldq, 1); a.out = out_rows(a.phase, out, rows, ldo, sizeof(T));
        const uint64_t chunks = std::max(a.cols / 8, 1u);
        const auto start = [&](auto team, auto v) {
            constexpr int TEAM = decltype(team)::value, V = decltype(v)::value;
            launch(dequantize_rows_kernel<T, TEAM, V>, dim3(team_grid(TEAM, rows), (uint32_t)std::min<uint64_t>(ceil_div(chunks, TEAM * V), 65535)), team_threads(TEAM), 0, 1, st, a);
        };
        using std::integral_constant;
        if (chunks <= 32) start(integral_constant<int, 32>(), integral_constant<int, 1>());
        else if (chunks <= 64) start(integral_constant<int, 32>(), integral_constant<int, 2>());
        // a warp a row once there are rows for every warp (16384 x 1001: 10.2 against 17.9 us), a chunk a thread for fewer (300 x 1001: 1.7 against 1.8)
        else if (chunks <= 128 && rows > 16ull * c->sm_count) start(integral_constant<int, 32>(), integral_constant<int, 4>());
        else if (chunks <= 128) start(integral_constant<int, 128>(), integral_constant<int, 1>());
        else if (chunks <= 256) start(integral_constant<int, 128>(), integral_constant<int, 2>());
        else start(integral_constant<int, 256>(), integral_constant<int, 2>());
    }
}

template <typename T>
void run_dropout(const sc_ctx* c, const DropArgs& a, cudaStream_t st) {
    const bool wide = unshifted(a.phase, a.cols) && a.residual.vec && a.y.vec;
    const uint64_t chunks = std::max(a.cols / 8, 1u);
    const auto start = [&](auto team, auto v) {
        constexpr int TEAM = decltype(team)::value, V = decltype(v)::value;
        const dim3 grid(team_grid(TEAM, a.rows), (uint32_t)std::min<uint64_t>(ceil_div(chunks, TEAM * V), 65535));
        if (a.residual.p) {
            if (wide) launch(dropout_kernel<T, TEAM, V, true, true>, grid, team_threads(TEAM), 0, 1, st, a);
            else launch(dropout_kernel<T, TEAM, V, true, false>, grid, team_threads(TEAM), 0, 1, st, a);
        } else if (wide) launch(dropout_kernel<T, TEAM, V, false, true>, grid, team_threads(TEAM), 0, 1, st, a);
        else launch(dropout_kernel<T, TEAM, V, false, false>, grid, team_threads(TEAM), 0, 1, st, a);
    };
    using std::integral_constant;
    if (chunks <= 32) start(integral_constant<int, 32>(), integral_constant<int, 1>());
    else if (chunks <= 64) start(integral_constant<int, 32>(), integral_constant<int, 2>());
    // a warp a row once there are rows for every warp (65536 x 1024 without a residual 46 against 69 us), a chunk a thread for fewer (509 x 1024:
    // 1.7 against 2.2) and for cut rows (8000 x 1001: 11.8 against 14.1)
    else if (chunks <= 128 && unshifted(a.phase, a.cols) && a.rows > 16ull * c->sm_count) start(integral_constant<int, 32>(), integral_constant<int, 4>());
    else if (chunks <= 128) start(integral_constant<int, 128>(), integral_constant<int, 1>());
    else if (chunks <= 256) start(integral_constant<int, 128>(), integral_constant<int, 2>());
    else if (chunks <= 512 || a.residual.p) start(integral_constant<int, 256>(), integral_constant<int, 2>());
    else start(integral_constant<int, 256>(), integral_constant<int, 4>());
}

template <typename T, bool DROP>
void run_norm(sc_ctx* c, const NormArgs& a, float* scales, cudaStream_t st) {
    const bool wide = unshifted(a.phase, a.cols) && a.residual.vec && a.gamma.vec && a.h.vec && a.y.vec && a.q.vec;
    const uint64_t chunks = a.cols / 8;
    // cut rows carry more code a chunk: 16384 x 1001 takes 25.7 us with one chunk a thread, 29.6 with four; 64 x 1001 2.1 and 3.9
    if (!unshifted(a.phase, a.cols) && chunks > 64 && chunks <= 128) {
        launch(rms_norm_rows_kernel<T, 128, 1, DROP, false>, team_grid(128, a.rows), team_threads(128), 0, 1, st, a, scales);
        return;
    }
    const bool held = with_team(chunks, [&](auto team, auto v) {
        constexpr int TEAM = decltype(team)::value, V = decltype(v)::value;
        if (wide) launch(rms_norm_rows_kernel<T, TEAM, V, DROP, true>, team_grid(TEAM, a.rows), team_threads(TEAM), 0, 1, st, a, scales);
        else launch(rms_norm_rows_kernel<T, TEAM, V, DROP, false>, team_grid(TEAM, a.rows), team_threads(TEAM), 0, 1, st, a, scales);
    });
    if (!held) launch(rms_norm_kernel<T>, row_grid(c, a.rows), NORM_THREADS, 0, 1, st, a, scales);
}

constexpr uint32_t RING_BYTES = 208 * 1024;          // shared memory for the stages of the norm gradient's rings on an SM

// Column sums of the gradient of rows too long for a ring: runs of rows as for the activation's gradient.
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


// Shared memory of the ring kernels: all of a CTA's, once per build and device.
template <typename T, int TEAM, int V, bool DROP, bool WIDE>
int ring_ready(const sc_ctx* c) {
    static std::atomic<uint64_t> ready{0};
    const uint64_t bit = c->device < 64 ? 1ull << c->device : 0;
    if (!(ready.load(std::memory_order_relaxed) & bit)) {
        SC_CUDA(cudaFuncSetAttribute(norm_grad_ring_kernel<T, TEAM, V, DROP, WIDE>, cudaFuncAttributeMaxDynamicSharedMemorySize, RING_BYTES));
        ready.fetch_or(bit, std::memory_order_relaxed);
    }
    return SC_OK;
}

template <typename T, int TEAM, int V, bool DROP, bool WIDE>
int launch_norm_grad(sc_ctx* c, NormGradArgs a, float* dgamma, cudaStream_t st) {
    constexpr uint32_t TEAMS = ring_teams(TEAM, V), FIT = ring_ctas(TEAM, V);
    // as many stages as leave room for every CTA that fits otherwise, two at least
    NormRing ring{};
    ring.row_bytes = 16 * (a.cols / 8 + !WIDE); ring.operands = a.residual.p ? 3 : 2;
    const uint32_t stage = TEAMS * ring.row_bytes * ring.operands;
    ring.stages = std::min(RING_MOST_STAGES, std::max(2u, RING_BYTES / FIT / stage));
    const uint32_t per_sm = std::max(1u, std::min(FIT, RING_BYTES / (ring.stages * stage)));
    uint32_t grid = (uint32_t)std::min<uint64_t>(ceil_div(a.rows, TEAMS), (uint64_t)c->sm_count * per_sm);
    if (grid < ceil_div(a.rows, TEAMS) && grid >= 8) grid &= ~7u;                          // a team's rows are a multiple of 8 apart
    a.part_ld = ((uint64_t)a.cols + 7) & ~7ull;
    float* partial = nullptr;
    if (dgamma) {
        if (const int rc = layer_scratch(c, grid * a.part_ld * sizeof(float), st)) return rc;
        partial = reinterpret_cast<float*>(c->d_layer + TICKET_BYTES);
    }
    if (const int rc = ring_ready<T, TEAM, V, DROP, WIDE>(c)) return rc;
    {
        Launch l(c, KIND_RMS_NORM_GRAD, st);
        launch(norm_grad_ring_kernel<T, TEAM, V, DROP, WIDE>, grid, TEAMS * TEAM, ring.stages * stage, 1, st, a, ring, partial, c->d_status);
    }
    if (dgamma) {
        Launch l(c, KIND_RMS_NORM_GRAD, st);
        launch(norm_join_kernel, (uint32_t)ceil_div(a.cols, 32), JOIN_LANES * 32, 0, 1, st, partial, grid, a.part_ld, a.cols, dgamma, a.accumulate);
    }
    return SC_OK;
}

template <typename T>
int run_norm_grad(sc_ctx* c, NormGradArgs a, float* dgamma, cudaStream_t st) {
    const bool wide = unshifted(a.phase, a.cols) && a.h.vec && a.gamma.vec && a.residual.vec && a.dh.vec && a.dx.vec, drop = a.drop.cut && a.dx.p;
    const bool ringed = a.h.vec && a.residual.vec;                 // results of another cut leave in single elements
    const uint32_t chunks = a.cols / 8;
#define SC_TEAM(TEAM, V) \
    if (ringed && chunks <= TEAM * V) { \
        if (wide) return drop ? launch_norm_grad<T, TEAM, V, true, true>(c, a, dgamma, st) : launch_norm_grad<T, TEAM, V, false, true>(c, a, dgamma, st); \
        return drop ? launch_norm_grad<T, TEAM, V, true, false>(c, a, dgamma, st) : launch_norm_grad<T, TEAM, V, false, false>(c, a, dgamma, st); \
    }
    SC_TEAM(32, 1) SC_TEAM(32, 2)
    // Up to some thousand cut rows are over sooner with a chunk a thread, whose code is fetched cold (509 x 1001: 6.1 against 7.9 us, 2000 x 1001
    // 11.0 against 12.9); more are not (4000 x 1001: 16.4 against 16.3, 16384 x 1001 42 against 31), nor are rows without ends (2048 x 1024:
    // 9.5 against 8.2).  The order of a row's sums goes with the choice.
    if (ringed && !unshifted(a.phase, a.cols) && chunks <= 128 && a.rows <= 16ull * c->sm_count)
        return drop ? launch_norm_grad<T, 128, 1, true, false>(c, a, dgamma, st) : launch_norm_grad<T, 128, 1, false, false>(c, a, dgamma, st);
    SC_TEAM(32, 4) SC_TEAM(128, 2) SC_TEAM(256, 2) SC_TEAM(256, 4) SC_TEAM(512, 4)
#undef SC_TEAM
    // rows too long for a ring's stages, or inputs of several phases
    const StripPlan plan = strip_plan(c, a.rows, a.cols);
    if (const int rc = layer_scratch(c, plan.partial + plan.stats, st)) return rc;
    a.runs = plan.runs; a.run_rows = plan.run_rows;
    float* partial = reinterpret_cast<float*>(c->d_layer + TICKET_BYTES);
    float2* stats = reinterpret_cast<float2*>(c->d_layer + TICKET_BYTES + plan.partial);
    {
        Launch l(c, KIND_RMS_NORM_GRAD, st);
        launch(norm_stats_kernel<T>, row_grid(c, a.rows), NORM_THREADS, 0, 1, st, a, stats);
    }
    Launch l(c, KIND_RMS_NORM_GRAD, st);
    launch(norm_strips_kernel<T>, dim3(plan.strips, plan.runs), CKPT_THREADS, 0, 1, st, a, stats, partial, reinterpret_cast<uint32_t*>(c->d_layer), dgamma);
    return SC_OK;
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
    a.rows = rows; a.cols = (uint32_t)cols;
    a.grain_x = grain_of(x, rows > 1 ? ldx : 0, type_bytes(type), 8);
    a.grain_q = grain_of(q, rows > 1 ? ldq : 0, 1, 8);
    a.phase = phase_of(x, rows, ldx, type_bytes(type));
    a.x = in_rows(a.phase, x, rows, ldx, type_bytes(type));
    a.q = out_rows(a.phase, q, rows, ldq, 1);
    Launch l(ctx, KIND_QUANTIZE, st);
    if (type == SC_BF16) run_quantize<__nv_bfloat16>(ctx, a, scales, st);
    else if (type == SC_F16) run_quantize<__half>(ctx, a, scales, st);
    else run_quantize<float>(ctx, a, scales, st);
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
    Launch l(ctx, KIND_DEQUANTIZE, st);
    if (type == SC_BF16) run_dequantize<__nv_bfloat16>(ctx, q, ldq, scales, rows, cols, out, ldo, st);
    else if (type == SC_F16) run_dequantize<__half>(ctx, q, ldq, scales, rows, cols, out, ldo, st);
    else run_dequantize<float>(ctx, q, ldq, scales, rows, cols, out, ldo, st);
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
    a.rows = rows; a.cols = (uint32_t)cols;
    a.phase = phase_of(x, rows, ldx, 2);
    a.x = in_rows(a.phase, x, rows, ldx); a.residual = in_rows(a.phase, residual, rows, ldr); a.y = out_rows(a.phase, y, rows, ldy);
    Launch l(ctx, KIND_DROPOUT, st);
    if (type == SC_BF16) run_dropout<__nv_bfloat16>(ctx, a, st);
    else run_dropout<__half>(ctx, a, st);
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
    a.rows = rows; a.cols = (uint32_t)cols;
    a.grain_x = grain16(x, rows, ldx); a.grain_r = grain16(residual, rows, ldr); a.grain_g = grain_of(gamma, 0, 2, 8);
    a.grain_h = grain16(h, rows, ldh); a.grain_y = grain16(y, rows, ldy); a.grain_q = grain_of(q, rows > 1 ? ldq : 0, 1, 8);
    a.eps = eps; a.mean = 1.0f / (float)cols;
    a.phase = phase_of(x, rows, ldx, 2);
    a.x = in_rows(a.phase, x, rows, ldx); a.residual = in_rows(a.phase, residual, rows, ldr);
    a.gamma = InRows{gamma, 0, aligned(gamma, 16)};
    a.h = out_rows(a.phase, h, rows, ldh); a.y = out_rows(a.phase, y, rows, ldy); a.q = out_rows(a.phase, q, rows, ldq, 1);
    Launch l(ctx, KIND_RMS_NORM, st);
    if (type == SC_BF16) { if (a.drop.cut) run_norm<__nv_bfloat16, true>(ctx, a, scales, st); else run_norm<__nv_bfloat16, false>(ctx, a, scales, st); }
    else if (a.drop.cut) run_norm<__half, true>(ctx, a, scales, st);
    else run_norm<__half, false>(ctx, a, scales, st);
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
    a.rows = rows; a.cols = (uint32_t)cols;
    a.grain_y = grain16(dy, rows, lddy); a.grain_h = grain16(h, rows, ldh); a.grain_g = grain_of(gamma, 0, 2, 8);
    a.grain_r = grain16(residual, rows, ldr); a.grain_dh = grain16(dh, rows, lddh); a.grain_dx = grain16(dx, rows, lddx);
    a.accumulate = accumulate ? 1u : 0u; a.eps = eps; a.mean = 1.0f / (float)cols;
    a.phase = phase_of(dy, rows, lddy, 2);
    a.dy = in_rows(a.phase, dy, rows, lddy); a.h = in_rows(a.phase, h, rows, ldh); a.residual = in_rows(a.phase, residual, rows, ldr);
    a.gamma = InRows{gamma, 0, aligned(gamma, 16)};
    a.dh = out_rows(a.phase, dh, rows, lddh); a.dx = out_rows(a.phase, dx, rows, lddx);
    const int rc = type == SC_BF16 ? run_norm_grad<__nv_bfloat16>(ctx, a, dgamma, st) : run_norm_grad<__half>(ctx, a, dgamma, st);
    if (rc) return rc;
    SC_CUDA(cudaGetLastError());
    return SC_OK;
}

}  // extern "C"
