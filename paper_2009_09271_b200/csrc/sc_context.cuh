// Host-side state shared by the C ABI's translation units: the context, its scratch and launch bookkeeping.
#pragma once
#include <algorithm>
#include <cstdint>
#include <vector>

#include "../../include/sparsecomm.h"
#include "sc_common.cuh"

using namespace sc;

struct sc_ctx {
    int device = 0;
    int sm_count = 0;
    size_t max_n = 0;
    int max_W = 0, max_seg = 0;
    size_t max_tiles_per_worker = 0;
    size_t max_mask_words = 0;      // per seed group
    size_t max_atiles = 0;
    size_t scratch_bytes = 0;

    SegEntry* d_segs = nullptr;
    uint32_t* d_fast_list = nullptr;
    uint32_t* d_tiny_list = nullptr;      // [max_segments]: short segments, the <= TINY_SMALL_MAX ones first
    uint32_t tiny_small = 0, tiny_large = 0, tiny_large_max_n = 0;
    int occ_tiny_small = 1;
    uint32_t* d_lists = nullptr;     // tiles of the large segments | their pack groups (each max_tiles long)
    uint32_t n_fast_tiles = 0, n_fast_groups = 0;
    uint32_t* d_hist = nullptr;      // radix histograms of the fall-back (cleared by the fall-back kernel itself)
    TopkState* d_state = nullptr;
    unsigned long long* d_desc = nullptr;
    unsigned long long* d_ticket = nullptr;
    uint32_t* d_mask = nullptr;
    uint32_t* d_bounds = nullptr;
    uint32_t* d_offsets = nullptr;   // per seed group / worker: exclusive kept-count prefix over tiles
    // sampled-bracket top-k path.  Everything that must start at zero in a top-k call lies in one block
    // (one memset): counters and the barrier word, then the per-problem states, then the candidate histograms.
    unsigned char* d_zero = nullptr;
    size_t zero_bytes = 0;
    FastState* d_fstate = nullptr;   // inside d_zero
    uint32_t* d_sample = nullptr;
    uint2* d_cand = nullptr;
    uint2* d_list2 = nullptr;
    uint32_t* d_tile_sure = nullptr;
    uint32_t* d_tile_csum = nullptr;
    uint32_t* d_tile_cbase = nullptr;
    uint32_t* d_tile_ccnt = nullptr;
    uint32_t* d_tile_fbase = nullptr;
    uint32_t* d_tile_fcnt = nullptr;
    uint32_t* d_tile_tie = nullptr;
    size_t max_main_grid = 0;            // CTAs of the top-k pass in the build chosen for the current table
    size_t main_grid_v[2] = {0, 0};      // [0]: three CTAs per SM, [1]: the two-CTA build
    int main_wide = 0;                   // 1: the current table uses the two-CTA build
    uint2* d_flagged = nullptr;      // grown on demand: its size depends on k
    size_t flagged_slots = 0;
    size_t max_fast_per_worker = 0, max_cand_per_worker = 0;
    uint32_t last_topk_problems = 0; // (worker, segment) pairs of the most recent top-k call
    uint32_t max_sample_m = 0, fast_big = 0, fast_huge = 0;   // of the fast list: the first fast_huge are long segments, the first fast_big have large samples
    float gamma = 1.0f;                  // step size of the accumulate line (sc_set_gamma)
    int occ_main = 1, occ_main_wide = 1, occ_emit_v[4] = {1, 1, 1, 1}, occ_fallback = 1, occ_filter = 1;
    uint32_t lookback_poll_limit = 0, barrier_poll_limit = 0;   // set by sc_create
    uint64_t* d_seeds = nullptr;
    int* d_status = nullptr;

    std::vector<sc_segment> cached_segs;
    size_t cached_n = 0;
    bool layout_valid = false;
    Layout layout{};

    uint32_t epoch = 0;
    uint64_t launches = 0;

    int occ_pack_mask = 1, occ_block = 1, occ_agg = 1, occ_agg_big = 1, occ_agg_warp = 1;
    int occ_agg_fine[5] = {1, 1, 1, 1, 1};

    // optional per-kernel timing (sc_profile)
    bool prof_on = false;
    struct ProfRec { int kind; cudaEvent_t a, b; };
    std::vector<ProfRec> prof_recs;
    std::vector<cudaEvent_t> prof_free;

    // host-buffer entry point
    float* d_stage_grads = nullptr;
    float* d_stage_vals = nullptr;
    uint32_t* d_stage_idx = nullptr;
    float* d_stage_out = nullptr;
    size_t stage_grads_elems = 0, stage_msg_elems = 0, stage_out_elems = 0;
    cudaStream_t copy_stream = nullptr;
    cudaStream_t aux_stream = nullptr;   // short top-k segments run here, beside the large ones
    cudaEvent_t ev_fork = nullptr, ev_join = nullptr;
    cudaEvent_t ev_start = nullptr;
    std::vector<cudaEvent_t> ev_worker;

    // layer operators (sc_layer.cu): one block, grown on demand, and tickets that are zero between calls
    unsigned char* d_layer = nullptr;
    size_t layer_bytes = 0;
    struct LayerPlan { uint64_t rows, cols, red; int mode, bn, cg; uint32_t splits; uint64_t part_ld; size_t bytes; };
    static constexpr int LAYER_PLANS = 16;
    LayerPlan layer_plans[LAYER_PLANS] = {};     // tile shapes of the sizes seen last
    int layer_plan_next = 0;
    int layer_force_bn = 0, layer_force_cg = 1;  // sc_debug_layer_tiles: 0, or the width and the CTAs of every tile
    uint32_t layer_force_parts = 1;
    bool layer_captured = false;                 // a captured call used the block: growing must not free it
    static constexpr int MAX_RETIRED = 64;
    unsigned char* layer_retired[MAX_RETIRED] = {};
    int layer_retired_count = 0;
};

namespace {

#define SC_CUDA(call)                                   \
    do {                                                \
        cudaError_t err__ = (call);                     \
        if (err__ != cudaSuccess) return SC_ERR_CUDA;   \
    } while (0)

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

template <typename T>
int dev_alloc(sc_ctx* c, T** p, size_t count) {
    size_t bytes = std::max<size_t>(count, 1) * sizeof(T);
    if (cudaMalloc(reinterpret_cast<void**>(p), bytes) != cudaSuccess) { *p = nullptr; return SC_ERR_WORKSPACE; }
    c->scratch_bytes += bytes;
    return SC_OK;
}

class DeviceGuard {
  public:
    explicit DeviceGuard(int dev) { cudaGetDevice(&prev_); if (prev_ != dev) { cudaSetDevice(dev); set_ = true; } }
    ~DeviceGuard() { if (set_) cudaSetDevice(prev_); }
  private:
    int prev_ = 0;
    bool set_ = false;
};

enum { KIND_SCATTER = 0, KIND_MASK_COUNT, KIND_ROW_SCAN, KIND_RANDK_PACK, KIND_RANDBLOCK, KIND_AGG_BOUNDS, KIND_AGG_TILES,
       KIND_AGG_WARP, KIND_AGG_FINE, KIND_AGG_APPLY, KIND_TINY, KIND_BRACKET, KIND_MAIN, KIND_FILTER, KIND_FINISH, KIND_RESOLVE_SMALL, KIND_EMIT,
       KIND_FALLBACK, KIND_CKPT_PACK, KIND_CKPT_UNPACK, KIND_ACT_GRAD, KIND_LINEAR, KIND_LINEAR_DX, KIND_LINEAR_DW, KIND_LAYER_JOIN,
       KIND_LAYER_LAYOUT, KIND_COUNT };
const char* const kKindNames[KIND_COUNT] = {"randk_scatter", "mask_count", "row_scan", "randk_pack", "randblock", "agg_bounds",
                                            "agg_tiles", "agg_warp", "agg_fine", "agg_apply", "topk_tiny", "topk_bracket",
                                            "topk_main", "topk_filter", "topk_finish", "topk_resolve_small", "topk_emit", "topk_fallback",
                                            "checkpoint_pack", "checkpoint_unpack", "activation_grad", "linear", "linear_grad_input",
                                            "linear_grad_weight", "layer_join", "layer_layout"};

// Counts a kernel launch and, when profiling is on, brackets it with two events.
class Launch {
  public:
    Launch(sc_ctx* c, int kind, cudaStream_t st) : c_(c), st_(st) {
        ++c->launches;
        if (!c->prof_on) return;
        rec_.kind = kind;
        rec_.a = take(); rec_.b = take();
        if (rec_.a && rec_.b) { cudaEventRecord(rec_.a, st_); on_ = true; }
    }
    ~Launch() {
        if (!on_) return;
        cudaEventRecord(rec_.b, st_);
        c_->prof_recs.push_back(rec_);
    }
  private:
    cudaEvent_t take() {
        if (!c_->prof_free.empty()) { cudaEvent_t e = c_->prof_free.back(); c_->prof_free.pop_back(); return e; }
        cudaEvent_t e = nullptr;
        if (cudaEventCreate(&e) != cudaSuccess) return nullptr;
        return e;
    }
    sc_ctx* c_;
    cudaStream_t st_;
    sc_ctx::ProfRec rec_{};
    bool on_ = false;
};

}  // namespace

// sc_layer.cu: a kernel that waits as the layer products do, for something that never arrives.
int layer_wait_probe(sc_ctx* c, long long limit_cycles, cudaStream_t st);
