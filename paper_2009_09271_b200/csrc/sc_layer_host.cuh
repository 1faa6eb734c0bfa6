// Host side that the layer operators' translation units share: argument checks, scratch, launches.
#pragma once
#include <algorithm>

#include "sc_context.cuh"
#include "sc_layer_common.cuh"

namespace {

constexpr uint64_t MAX_DIM = 1ull << 31;      // rows and columns; offsets are 64-bit throughout

inline bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
inline uint64_t ceil_div(uint64_t a, uint64_t b) { return (a + b - 1) / b; }

inline bool known_type(int type) { return type == SC_BF16 || type == SC_F16; }
inline bool known_act(int act) { return act >= SC_ACT_NONE && act <= SC_ACT_SILU; }
inline size_t type_bytes(int type) { return type == SC_F32 ? 4 : 2; }

// The widest run of elements, up to `most`, at whose multiples rows `ld` apart are aligned to the run's size.
inline uint32_t grain_of(const void* p, size_t ld, size_t elem, uint32_t most) {
    while (most > 1 && (!aligned(p, most * elem) || ld % most)) most /= 2;
    return most;
}

// A matrix argument: rows of `cols` elements, `ld` apart.
inline int check_matrix(const void* p, size_t ld, size_t rows, size_t cols, size_t elem) {
    if (rows >= MAX_DIM || cols >= MAX_DIM) return SC_ERR_RANGE;
    if (ld < cols && rows > 1) return SC_ERR_INVALID;
    if (rows == 0 || cols == 0) return SC_OK;
    return p && aligned(p, elem) ? SC_OK : SC_ERR_INVALID;
}

// The layer operators' scratch: 64 KB of tickets, zero between calls, then `bytes` of workspace.  Only calls that use it ask for it.
constexpr size_t TICKET_BYTES = 65536;

inline int layer_scratch(sc_ctx* c, size_t bytes, cudaStream_t st) {
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

}  // namespace
