// Host side of the layer operators declared in include/sparsecomm.h: argument checks, scratch, launches.
#include <algorithm>
#include <atomic>

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

// The widest run of elements, up to `most`, at whose multiples rows `ld` apart are aligned to the run's size.
uint32_t grain_of(const void* p, size_t ld, size_t elem, uint32_t most) {
    while (most > 1 && (!aligned(p, most * elem) || ld % most)) most /= 2;
    return most;
}

// A matrix argument: rows of `cols` elements, `ld` apart.
int check_matrix(const void* p, size_t ld, size_t rows, size_t cols, size_t elem) {
    if (rows >= MAX_DIM || cols >= MAX_DIM) return SC_ERR_RANGE;
    if (ld < cols && rows > 1) return SC_ERR_INVALID;
    if (rows == 0 || cols == 0) return SC_OK;
    return p && aligned(p, elem) ? SC_OK : SC_ERR_INVALID;
}

// The layer operators' scratch: 64 KB of tickets, zero between calls, then `bytes` of workspace.  Only calls that use it ask for it.
constexpr size_t TICKET_BYTES = 65536;

int layer_scratch(sc_ctx* c, size_t bytes, cudaStream_t st) {
    cudaStreamCaptureStatus cap = cudaStreamCaptureStatusNone;
    SC_CUDA(cudaStreamIsCapturing(st, &cap));
    const bool capturing = cap != cudaStreamCaptureStatusNone;
    if (c->d_layer && c->layer_bytes >= bytes) {
        c->layer_captured |= capturing;
        return SC_OK;
    }
    if (capturing) return SC_ERR_WORKSPACE;                               // reserve before the capture
    bytes = (bytes + 255) & ~(size_t)255;
    void* p = nullptr;
    if (c->d_layer) {
        SC_CUDA(cudaStreamSynchronize(st));
        if (c->layer_captured) {                                          // a graph may still use it: kept until sc_destroy
            if (c->layer_retired_count == sc_ctx::MAX_RETIRED) return SC_ERR_WORKSPACE;
            c->layer_retired[c->layer_retired_count++] = c->d_layer;
        } else {
            cudaFree(c->d_layer);
            c->scratch_bytes -= TICKET_BYTES + c->layer_bytes;
        }
        c->d_layer = nullptr; c->layer_bytes = 0; c->layer_captured = false;
    }
    if (cudaMalloc(&p, TICKET_BYTES + bytes) != cudaSuccess) { cudaGetLastError(); return SC_ERR_WORKSPACE; }
    // finished before any stream can use it
    if (cudaMemsetAsync(p, 0, TICKET_BYTES, st) != cudaSuccess || cudaStreamSynchronize(st) != cudaSuccess) { cudaFree(p); return SC_ERR_CUDA; }
    c->d_layer = static_cast<unsigned char*>(p);
    c->layer_bytes = bytes;
    c->scratch_bytes += TICKET_BYTES + bytes;
    return SC_OK;
}

uint32_t item_grid(const sc_ctx* c, uint64_t total) {
    return (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>(ceil_div(total, CKPT_THREADS), (uint64_t)c->sm_count * 8));
}

// Launches a layer kernel (optionally in clusters) that may begin while its predecessor on the stream ends.
template <typename... P, typename... A>
cudaError_t launch(void (*kernel)(P...), dim3 grid, int threads, size_t smem, int cluster, cudaStream_t st, A... args) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2]{};
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim = {(unsigned)cluster, 1, 1};
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
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

// ---------------------------------------------------------------------------
// matrix products
// ---------------------------------------------------------------------------
// A stored 16-bit matrix: `rows` rows of `cols` elements, `ld` apart.
struct Stored {
    const void* p;
    uint64_t rows, cols, ld;
    Stored(const void* p_, uint64_t rows_, uint64_t cols_, uint64_t ld_) : p(p_), rows(rows_), cols(cols_), ld(rows_ > 1 ? ld_ : (cols_ + 7) & ~7ull) {}
};

inline uint64_t round8(uint64_t n) { return (n + 7) & ~7ull; }
inline bool tma_ready(const Stored& m) { return aligned(m.p, 16) && m.ld % 8 == 0; }
inline size_t layout_bytes(uint64_t rows, uint64_t cols) { return (rows * round8(cols) * 2 + 255) & ~(size_t)255; }

decltype(&cuTensorMapEncodeTiled) encode_fn() {
    static decltype(&cuTensorMapEncodeTiled) fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult found = cudaDriverEntryPointSymbolNotFound;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) p = nullptr;
        return reinterpret_cast<decltype(&cuTensorMapEncodeTiled)>(p);
    }();
    return fn;
}

// Boxes of 64 elements (one 128-byte swizzled row) by `box_rows` rows; what lies outside the matrix reads as zero.
bool tile_map(CUtensorMap* map, int type, const Stored& m, uint32_t box_rows) {
    const auto fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[2] = {m.cols, m.rows}, strides[1] = {m.ld * 2};
    const cuuint32_t box[2] = {64, box_rows}, steps[2] = {1, 1};
    return fn(map, type == SC_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, const_cast<void*>(m.p), dims, strides, box,
              steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The fp32 result, or `parts` of them, stored in blocks of 32 x 32.
bool out_map(CUtensorMap* map, float* p, uint64_t rows, uint64_t cols, uint64_t ld, uint32_t parts, uint64_t part_stride) {
    const auto fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[3] = {cols, rows, parts}, strides[2] = {ld * 4, part_stride * 4};
    const cuuint32_t box[3] = {32, 32, 1}, steps[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 3, p, dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The 16-bit result, stored in blocks of 32 x 32.
bool rows_map(CUtensorMap* map, int type, void* p, uint64_t rows, uint64_t cols, uint64_t ld) {
    const auto fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[2] = {cols, rows}, strides[1] = {ld * 2};
    const cuuint32_t box[2] = {32, 32}, steps[2] = {1, 1};
    return fn(map, type == SC_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, p, dims, strides, box, steps,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

constexpr size_t PARTIAL_CAP = 64u << 20;      // bytes of partial sums a split product may use

using ProductPlan = sc_ctx::LayerPlan;

// Tile shape and number of parts by an estimate in SM cycles: waves of tiles, each as long as its reduction or as the
// emptying of the accumulator before it, and the partial sums' way to memory and back.  A block of 64 reduction steps costs
// the tensor pipe 512 cycles for 256 columns (pairs; a little more for one CTA, which loads twice B), or what its bytes
// take from L2 (50 to 60 a cycle and SM).  Against the best of all shapes and splits, swept over 23 sizes and the three products
// (9 to 32001 tokens, widths 512 to 9000), the choice is within 12 % in 66 of 69 cases, at the median 0.1 % off.  The others: 9 x 1024 x 1024
// forward 7.3 us against 6.0, the input gradients of 300 x 4096 x 1024 (13.7 against 11.6) and 100 x 9000 x 512 (16.6 against 10.0): short calls
// whose split is too coarse.
ProductPlan product_plan(sc_ctx* c, int mode, uint64_t rows, uint64_t cols, uint64_t red) {
    for (const ProductPlan& p : c->layer_plans)                // a step's few sizes come again and again
        if (p.rows == rows && p.cols == cols && p.red == red && p.mode == mode) return p;
    ProductPlan best{rows, cols, red, mode, 256, 1, 1, (cols + 31) & ~31ull, 0};
    const uint64_t blocks = ceil_div(red, TC_STEP);
    if (c->layer_force_bn && !(c->layer_force_cg == 2 && rows <= TC_ROWS)) {
        const uint64_t parts = std::min<uint64_t>(c->layer_force_parts, blocks), bytes = parts > 1 ? parts * rows * best.part_ld * sizeof(float) : 0;
        best.bn = c->layer_force_bn; best.cg = c->layer_force_cg;
        if (bytes <= PARTIAL_CAP) { best.splits = (uint32_t)parts; best.bytes = bytes; }
        return best;
    }
    double best_cost = 0;
    const double box = (double)std::min<uint64_t>(rows, TC_ROWS);
    for (int shape = 0; shape < 4; ++shape) {                 // 256 x 256 by pairs, then 128 x 256, 128, 64
        const int cg = shape == 0 ? 2 : 1, bn = shape == 0 ? 256 : 512 >> shape;
        if (cg == 2 && rows <= TC_ROWS) continue;
        const uint64_t tiles = ceil_div(rows, TC_ROWS * cg) * ceil_div(cols, bn), units = c->sm_count / cg;
        const double block_cost = cg == 2 ? 540.0 : bn == 256 ? 620.0 : std::max(350.0, (box + bn) * 128 / (bn == 64 ? 50.0 : 60.0));
        for (uint32_t s = 1; s <= blocks && s <= 64; ++s) {
            const size_t bytes = s > 1 ? s * rows * best.part_ld * sizeof(float) : 0;
            if (bytes > PARTIAL_CAP || (s > 1 && tiles * s > units * 2)) break;
            const double main = (double)ceil_div(blocks, s) * block_cost, out = 800.0 + bn * (mode == PRODUCT_WEIGHT || s > 1 ? 25.0 : 16.0);
            const double cost = 4000.0 + (double)ceil_div(tiles * s, units) * std::max(main, out) + out + (s > 1 ? 3000.0 + 2.0 * bytes / 2500.0 : 0.0);
            if (best_cost == 0 || cost < best_cost) { best_cost = cost; best.bn = bn; best.cg = cg; best.splits = s; best.bytes = bytes; }
        }
    }
    c->layer_plans[c->layer_plan_next] = best;
    c->layer_plan_next = (c->layer_plan_next + 1) % sc_ctx::LAYER_PLANS;
    return best;
}

template <typename T, int MODE, int BN, int CG>
int launch_tiles(sc_ctx* c, const CUtensorMap& ma, const CUtensorMap& mb, const CUtensorMap& mo, const TcArgs& a, const Epilogue& ep, cudaStream_t st) {
    static std::atomic<uint64_t> ready{0};         // devices on which this build may use its shared memory
    const uint64_t bit = c->device < 64 ? 1ull << c->device : 0;
    if (!(ready.load(std::memory_order_relaxed) & bit)) {
        cudaFuncAttributes f{};
        SC_CUDA(cudaFuncSetAttribute(product_kernel<T, MODE, BN, CG>, cudaFuncAttributeMaxDynamicSharedMemorySize, TcShape<BN, CG>::SMEM));
        SC_CUDA(cudaFuncGetAttributes(&f, product_kernel<T, MODE, BN, CG>));
        // a register split beyond the launch's total would wait for ever
        if (MODE == PRODUCT_WEIGHT && BN == 256 && f.numRegs < TC_LEAST_REGS) return SC_ERR_UNSUPPORTED;
        ready.fetch_or(bit, std::memory_order_relaxed);
    }
    const uint32_t grid = CG * (uint32_t)std::min<uint64_t>((uint64_t)a.tiles * a.splits, c->sm_count / CG);
    return launch(product_kernel<T, MODE, BN, CG>, grid, TC_THREADS, TcShape<BN, CG>::SMEM, CG, st, ma, mb, mo, a, ep) == cudaSuccess ? SC_OK : SC_ERR_CUDA;
}

template <typename T, int MODE>
int run_product(sc_ctx* c, int kind, int type, Stored A, Stored B, uint64_t red, Epilogue ep, size_t used, cudaStream_t st) {
    constexpr bool A_MN = MODE == PRODUCT_WEIGHT, B_MN = MODE != PRODUCT_FORWARD;
    const uint64_t chunks = 4 * ckpt_groups(ep.cols);
    const uint32_t join_grid = (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>(ceil_div(ep.rows * chunks, 256), (uint64_t)c->sm_count * 8));
    if (red == 0) {
        Launch l(c, KIND_LAYER_JOIN, st);
        launch(product_join_kernel<T, MODE>, join_grid, 256, 0, 1, st, nullptr, 0, 0, 0, ep);
        return SC_OK;
    }
    const ProductPlan p = product_plan(c, MODE, ep.rows, ep.cols, red);
    const uint64_t tiles = ceil_div(ep.rows, TC_ROWS * p.cg) * ceil_div(ep.cols, p.bn);
    if (tiles * p.splits > 0x7FFFFFFFull) return SC_ERR_RANGE;
    const size_t copy_a = tma_ready(A) ? 0 : layout_bytes(A.rows, A.cols), copy_b = tma_ready(B) ? 0 : layout_bytes(B.rows, B.cols);
    const size_t need = used + p.bytes + copy_a + copy_b;
    if (need) if (const int rc = layer_scratch(c, need, st)) return rc;
    unsigned char* at = need ? c->d_layer + TICKET_BYTES + used : nullptr;
    float* partial = reinterpret_cast<float*>(at);
    at += p.bytes;
    LayoutArgs copies[2];
    int ncopies = 0;
    uint64_t work = 0;
    for (Stored* m : {&A, &B}) {
        if (tma_ready(*m)) continue;
        const uint32_t ldd = (uint32_t)round8(m->cols);
        copies[ncopies++] = LayoutArgs{static_cast<const uint16_t*>(m->p), reinterpret_cast<uint16_t*>(at), m->ld, m->rows, (uint32_t)m->cols, ldd,
                                       std::min(4u, grain_of(m->p, m->rows > 1 ? m->ld : 0, 2, 8))};
        work = std::max(work, m->rows * (ldd / 8));
        m->p = at; m->ld = ldd;
        at += layout_bytes(m->rows, m->cols);
    }
    if (ncopies) {
        Launch l(c, KIND_LAYER_LAYOUT, st);
        launch(layout_kernel, dim3((uint32_t)std::min<uint64_t>(ceil_div(work, 256), (uint64_t)c->sm_count * 8), ncopies), 256, 0, 1, st, copies[0],
               copies[ncopies - 1]);
    }
    TcArgs a{};
    a.tiles_i = (uint32_t)ceil_div(ep.rows, TC_ROWS * p.cg); a.tiles_j = (uint32_t)ceil_div(ep.cols, p.bn); a.tiles = (uint32_t)tiles;
    a.splits = p.splits; a.blocks = (uint32_t)ceil_div(red, TC_STEP);
    a.idesc = mma_idesc(TC_ROWS * p.cg, p.bn, type == SC_BF16, A_MN, B_MN);
    a.a_box_rows = A_MN ? 64u : (uint32_t)std::min<uint64_t>(TC_ROWS, round8(ep.rows));
    a.part_ld = (uint32_t)p.part_ld; a.part_stride = ep.rows * p.part_ld; a.partial = partial; a.status = c->d_status;
    // partial sums are whole to the next multiple of 32 columns: a checkpoint group's maximum is taken over all of its columns
    // A tile store ends on a 16-byte boundary: measured, it writes a row's last, partly covered 16 bytes whole.  Results whose
    // rows are not a multiple of 16 bytes long leave by the kernels' own stores.
    a.tma_out = p.splits > 1 || (MODE == PRODUCT_WEIGHT && ep.grain_out >= 4 && ep.cols % 4 == 0);
    if constexpr (MODE != PRODUCT_WEIGHT)
        // a warp's 128 columns of a 256-wide tile are four whole groups of the row
        ep.scales_by4 = MODE == PRODUCT_FORWARD && p.bn == 256 && ep.cols % 128 == 0 && aligned(ep.scales, 4);
    if constexpr (MODE != PRODUCT_WEIGHT)
        a.rows_form = p.splits == 1 && ep.cols % 8 == 0 && ep.grain_out >= 8 && (!ep.residual || ep.grain_res >= 8) && (!ep.q || ep.grain_q >= 8);
    CUtensorMap ma, mb, mo{};
    if (a.rows_form && !rows_map(&mo, type, ep.out, ep.rows, ep.cols, ep.rows > 1 ? ep.ldo : round8(ep.cols))) return SC_ERR_CUDA;
    if (a.tma_out && !(p.splits > 1 ? out_map(&mo, partial, ep.rows, p.part_ld, p.part_ld, p.splits, a.part_stride)
                                    : out_map(&mo, static_cast<float*>(ep.out), ep.rows, ep.cols, ep.ldo, 1, ep.rows * ep.ldo)))
        return SC_ERR_CUDA;
    if (!tile_map(&ma, type, A, a.a_box_rows) || !tile_map(&mb, type, B, B_MN ? 64u : (uint32_t)(p.bn / p.cg))) return SC_ERR_CUDA;
    {
        Launch l(c, kind, st);
        int rc;
        if (p.cg == 2) rc = launch_tiles<T, MODE, 256, 2>(c, ma, mb, mo, a, ep, st);
        else if (p.bn == 256) rc = launch_tiles<T, MODE, 256, 1>(c, ma, mb, mo, a, ep, st);
        else if (p.bn == 128) rc = launch_tiles<T, MODE, 128, 1>(c, ma, mb, mo, a, ep, st);
        else rc = launch_tiles<T, MODE, 64, 1>(c, ma, mb, mo, a, ep, st);
        if (rc) return rc;
    }
    if (p.splits > 1) {
        Launch l(c, KIND_LAYER_JOIN, st);
        launch(product_join_kernel<T, MODE>, join_grid, 256, 0, 1, st, partial, p.splits, a.part_stride, a.part_ld, ep);
    }
    return SC_OK;
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
