// Host side of the products on the tensor cores: operand layouts, tensor maps, tile choice, launches.
#pragma once
#include <atomic>

#include "sc_layer_host.cuh"
#include "sc_product.cuh"

namespace {

// A stored matrix of 16-bit (or 8-bit) elements: `rows` rows of `cols` elements, `ld` apart.
struct Stored {
    const void* p;
    uint64_t rows, cols, ld;
    uint32_t elem;
    Stored(const void* p_, uint64_t rows_, uint64_t cols_, uint64_t ld_, uint32_t elem_ = 2)
        : p(p_), rows(rows_), cols(cols_), ld(rows_ > 1 ? ld_ : (cols_ + 15) & ~15ull), elem(elem_) {}
};

inline uint64_t round8(uint64_t n) { return (n + 7) & ~7ull; }
inline bool tma_ready(const Stored& m) { return aligned(m.p, 16) && m.ld * m.elem % 16 == 0; }
// A copy's rows are 16-byte aligned: elements between them, and its bytes.  Long rows of bytes start on whole cache lines: with tiles' rows
// across two of them 8192 x 16384 x 4097 took 443 us instead of 340.
inline uint64_t layout_ld(const Stored& m) {
    const uint64_t to = m.cols >= 128 ? 128 : 16;
    return m.elem == 1 ? (m.cols + to - 1) & ~(to - 1) : round8(m.cols);
}
inline size_t layout_bytes(const Stored& m) { return (m.rows * layout_ld(m) * m.elem + 255) & ~(size_t)255; }
inline size_t layout_bytes(uint64_t rows, uint64_t cols) { return (rows * round8(cols) * 2 + 255) & ~(size_t)255; }

inline decltype(&cuTensorMapEncodeTiled) encode_fn() {
    static decltype(&cuTensorMapEncodeTiled) fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult found = cudaDriverEntryPointSymbolNotFound;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) p = nullptr;
        return reinterpret_cast<decltype(&cuTensorMapEncodeTiled)>(p);
    }();
    return fn;
}

// Boxes of 64 16-bit (128 8-bit) elements, one 128-byte swizzled row, by `box_rows` rows; what lies outside the matrix reads as zero.
inline bool tile_map(CUtensorMap* map, int type, const Stored& m, uint32_t box_rows) {
    const auto fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[2] = {m.cols, m.rows}, strides[1] = {m.ld * m.elem};
    const cuuint32_t box[2] = {128 / m.elem, box_rows}, steps[2] = {1, 1};
    const CUtensorMapDataType kind = m.elem == 1 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : type == SC_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    return fn(map, kind, 2, const_cast<void*>(m.p), dims, strides, box,
              steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The fp32 result, or `parts` of them, stored in blocks of 32 x 32.
inline bool out_map(CUtensorMap* map, float* p, uint64_t rows, uint64_t cols, uint64_t ld, uint32_t parts, uint64_t part_stride) {
    const auto fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[3] = {cols, rows, parts}, strides[2] = {ld * 4, part_stride * 4};
    const cuuint32_t box[3] = {32, 32, 1}, steps[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 3, p, dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The 16-bit result, stored in blocks of 32 x 32.
inline bool rows_map(CUtensorMap* map, int type, void* p, uint64_t rows, uint64_t cols, uint64_t ld) {
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
inline ProductPlan product_plan(sc_ctx* c, int mode, uint64_t rows, uint64_t cols, uint64_t red) {
    for (const ProductPlan& p : c->layer_plans)                // a step's few sizes come again and again
        if (p.rows == rows && p.cols == cols && p.red == red && p.mode == mode) return p;
    ProductPlan best{rows, cols, red, mode, 256, 1, 1, (cols + 31) & ~31ull, 0};
    const uint64_t blocks = ceil_div(red, product_step(mode));
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
    constexpr bool A_MN = MODE == PRODUCT_WEIGHT, B_MN = epilogue_of(MODE) != PRODUCT_FORWARD;
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
    const size_t copy_a = tma_ready(A) ? 0 : layout_bytes(A), copy_b = tma_ready(B) ? 0 : layout_bytes(B);
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
        const uint32_t ldd = (uint32_t)layout_ld(*m);
        copies[ncopies++] = LayoutArgs{static_cast<const uint16_t*>(m->p), reinterpret_cast<uint16_t*>(at), m->ld, m->rows, (uint32_t)m->cols, ldd,
                                       std::min(4u, grain_of(m->p, m->rows > 1 ? m->ld : 0, m->elem, 8))};
        work = std::max(work, m->elem == 1 ? m->rows * ceil_div(m->cols, 16 * LAYOUT_RUNS) * 32 : m->rows * (ldd / 8));
        m->p = at; m->ld = ldd;
        at += layout_bytes(*m);
    }
    if (ncopies) {
        Launch l(c, KIND_LAYER_LAYOUT, st);
        launch(MODE == PRODUCT_QUANTIZED ? layout_bytes_kernel : layout_kernel, dim3((uint32_t)std::min<uint64_t>(ceil_div(work, 256), (uint64_t)c->sm_count * 8), ncopies), 256, 0, 1, st, copies[0],
               copies[ncopies - 1]);
    }
    TcArgs a{};
    a.tiles_i = (uint32_t)ceil_div(ep.rows, TC_ROWS * p.cg); a.tiles_j = (uint32_t)ceil_div(ep.cols, p.bn); a.tiles = (uint32_t)tiles;
    a.splits = p.splits; a.blocks = (uint32_t)ceil_div(red, product_step(MODE));
    a.idesc = MODE == PRODUCT_QUANTIZED ? mma_idesc_i8(TC_ROWS * p.cg, p.bn) : mma_idesc(TC_ROWS * p.cg, p.bn, type == SC_BF16, A_MN, B_MN);
    a.a_box_rows = A_MN ? 64u : (uint32_t)std::min<uint64_t>(TC_ROWS, round8(ep.rows));
    a.part_ld = (uint32_t)p.part_ld; a.part_stride = ep.rows * p.part_ld; a.partial = partial; a.status = c->d_status;
    // partial sums are whole to the next multiple of 32 columns: a checkpoint group's maximum is taken over all of its columns
    // A tile store ends on a 16-byte boundary: measured, it writes a row's last, partly covered 16 bytes whole.  Results whose
    // rows are not a multiple of 16 bytes long leave by the kernels' own stores.
    a.tma_out = p.splits > 1 || (MODE == PRODUCT_WEIGHT && ep.grain_out >= 4 && ep.cols % 4 == 0);
    if constexpr (MODE != PRODUCT_WEIGHT)
        // a warp's 128 columns of a 256-wide tile are four whole groups of the row
        ep.scales_by4 = epilogue_of(MODE) == PRODUCT_FORWARD && p.bn == 256 && ep.cols % 128 == 0 && aligned(ep.scales, 4);
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

}  // namespace
