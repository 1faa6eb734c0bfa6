/*
 * sparsecomm.h -- C ABI of the sparsified-SGD gradient compressor for NVIDIA B200 (sm_100a).
 *
 * The library implements the per-step hot path of "Sparsified SGD with
 * error-feedback" (Algorithm 1 of "Sparse Communication for Training Deep
 * Networks"): for every worker w
 *     p   = g + e            accumulate the residual   (Algorithm 1, accumulate line; gamma folded into g)
 *     q^w = C(p)             keep k coordinates        (Methodology: Top-k, Random-k, Block-random-k)
 *     e'  = p - q^w          kept coordinates become 0 (Methodology prose on error feedback)
 * and, after the exchange,
 *     q   = (sum_w q^w) / W  dense average             (Algorithm 1, aggregate line; abstract: "average")
 *
 * Conventions
 *  - All data pointers are DEVICE pointers owned by the caller unless a name
 *    starts with h_ (then it is a HOST pointer).  The library never frees them.
 *  - fp32 IEEE-754 round-to-nearest, denormals kept; coordinates are uint32.
 *  - Every call is asynchronous on `stream` (a cudaStream_t passed as void*; NULL
 *    is the legacy default stream) and returns a status code, never throws.
 *    Argument errors are detected on the host before any launch and leave every
 *    buffer untouched.  Problems seen on the device (a bounded wait that ran out,
 *    a coordinate outside its range) set a sticky status word read by
 *    sc_sync_status().
 *  - A context owns scratch memory and is bound to the device that was current
 *    in sc_create().  Use one context per stream; calls on one context must not
 *    overlap on the GPU.
 *  - grad/residual/out must not alias; base pointers must be 16-byte aligned.
 *  - Messages: coordinates ascending and distinct, vals[j] = p[idx[j]].  With a
 *    segment table (layer-wise scope, Methodology "scope of sparsification")
 *    segment s owns message slots [K_s, K_s + k_s), K_s = sum of earlier k, and
 *    its coordinates are global (segment offset added).  Segment s of a call
 *    draws its coordinates from the seed mix64(seed, s).
 */
#ifndef SPARSECOMM_H
#define SPARSECOMM_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct sc_ctx sc_ctx;

/* Compressor C(.) -- Methodology, "compressor or sparsification scheme". */
enum { SC_TOPK = 0,       /* k largest |p|, ties to the lowest coordinate            */
       SC_RANDK = 1,      /* k distinct coordinates from a seeded bijection of [0,n)  */
       SC_RANDBLOCK = 2,  /* one seeded start a in [0,n-k], coordinates a..a+k-1      */
       SC_RANDBLOCK_WRAP = 3 /* start a in [0,n), coordinates (a+j) mod n: a variant of the
                               block scheme (Methodology, Block-random-k) in which every
                               coordinate is kept with the same probability k/n; the
                               message is still ascending (wrapped head first)          */ };

enum { SC_OK = 0,
       SC_ERR_INVALID = -1,      /* null pointer, misaligned base pointer, unknown scheme, bad table */
       SC_ERR_RANGE = -2,        /* k > n, n >= 2^32, W < 1, sizes beyond what the context was made for */
       SC_ERR_WORKSPACE = -3,    /* scratch allocation failed */
       SC_ERR_CUDA = -4,         /* a CUDA runtime call failed */
       SC_ERR_TIMEOUT = -5,      /* a bounded device-side wait gave up (reported by sc_sync_status) */
       SC_ERR_UNSUPPORTED = -6,
       SC_ERR_DEVICE_CHECK = -7  /* a device-side range check failed (e.g. unsorted message) */ };

/* One tensor of the gradient: elements [offset, offset+n) keep k coordinates. */
typedef struct { uint64_t offset, n, k; } sc_segment;

/* Allocates the context and all scratch for problems up to max_n elements per
 * worker, max_W workers and max_segments segments (cudaMalloc; synchronous). */
int sc_create(sc_ctx** out, size_t max_n, int max_W, int max_segments);
void sc_destroy(sc_ctx* ctx);
const char* sc_strerror(int code);

/* Step size of the accumulate line of Algorithm 1, p = gamma * g + e.  The default, 1, is the plain
 * fp32 add (the caller has folded gamma into g).  Any other value makes every later compress call of
 * this context evaluate the line as ONE fused multiply-add per element (a single rounding), so the
 * caller can pass the raw gradient.  Host-side state, no device work; always returns SC_OK for a
 * valid context. */
int sc_set_gamma(sc_ctx* ctx, float gamma);

/* Synchronises `stream`, then returns (and clears) the sticky device status. */
int sc_sync_status(sc_ctx* ctx, void* stream);

/* Bytes of device scratch the context holds; kernels launched so far. */
size_t sc_scratch_bytes(const sc_ctx* ctx);
uint64_t sc_launch_count(const sc_ctx* ctx);

/* Instrumentation (no counterpart in the paper).  sc_profile(ctx, 1) makes every
 * later kernel launch of this context be bracketed by two CUDA events on the
 * launching stream and forgets earlier records; sc_profile(ctx, 0) stops it.
 * sc_profile_read waits for the recorded launches and fills, for each of
 * sc_profile_kinds() kernel kinds (named by sc_profile_name), the summed device
 * time in milliseconds and the number of launches (HOST arrays of that length). */
int sc_profile(sc_ctx* ctx, int enable);
int sc_profile_kinds(void);
const char* sc_profile_name(int kind);
int sc_profile_read(sc_ctx* ctx, double* h_ms, uint64_t* h_launches);

/* Instrumentation (no counterpart in the paper).  Top-k of a segment of 65,536 or
 * more elements first tries a one-pass path whose work depends on a sampled
 * bracket of the threshold; if the exact counts show the bracket missed, it redoes
 * the selection with a multi-pass radix select.  Both give the same bits.  After
 * synchronising `stream` this fills h_counts[3] for the most recent top-k call:
 * (worker, segment) pairs served by [0] the radix select in shared memory because the
 * segment is short, [1] the one-pass path, [2] the radix select after a missed bracket. */
int sc_topk_path_counts(sc_ctx* ctx, void* stream, uint32_t* h_counts);

/* Instrumentation (no counterpart in the paper).  More about the most recent top-k call, after
 * synchronising `stream`: h_counts[8] (HOST) = (worker, segment) pairs [0] served in shared memory
 * (short segments), [1] served by the one-pass path, [2] redone by the radix select; of the large
 * segments: [3] those for which the sample showed one massive key value (a "tie key": exact zeros of a
 * sparse tensor, a constant tensor) whose elements are counted instead of listed, [4] those whose
 * threshold turned out to BE that key (tie-key elements admitted by coordinate order); reasons for
 * [2]: [5] a list overflowed, [6] the exact counts disproved the bracket, [7] too many candidates share
 * the threshold's histogram bin. */
int sc_topk_path_detail(sc_ctx* ctx, void* stream, uint32_t* h_counts);

/* Instrumentation for tests of the bounded device-side waits (no counterpart in the paper).  The
 * fall-back radix select is one kernel whose CTAs meet at grid-wide barriers and whose pack phase looks
 * back at its predecessors' counts; both waits give up after a number of polls, record
 * SC_ERR_TIMEOUT in the status word and let the kernel return.  sc_debug_set_poll_limits changes the
 * two limits for later calls of this context (0 restores the default).  sc_debug_wait_probe launches a
 * small kernel that runs one of the waits where what it waits for never arrives: which = 0, a barrier
 * that expects one CTA more than the launch has; which = 1, a look-back at a count nobody publishes;
 * which = 2, a wait of the layer products (about two seconds by default, here 100 cycles per barrier poll if that is less).
 * The kernel returns when the limit is reached (set a small one first); sc_sync_status then reports
 * SC_ERR_TIMEOUT. */
int sc_debug_set_poll_limits(sc_ctx* ctx, uint32_t lookback_polls, uint32_t barrier_polls);
int sc_debug_wait_probe(sc_ctx* ctx, int which, void* stream);

/* Algorithm 1, accumulate + compress + residual lines, one worker, global scope.
 * grad[n] read-only; residual[n] in/out (reads e, writes e'); out_vals[k],
 * out_idx[k] written.  k == 0 is allowed (residual <- gamma g + e, see sc_set_gamma). */
int sc_compress(sc_ctx* ctx, int scheme, const float* grad, float* residual, size_t n, size_t k,
                uint64_t seed, float* out_vals, uint32_t* out_idx, void* stream);

/* Same for W workers and a segment table in one call.  grads and residuals are
 * W rows of n elements (row w at +w*n); segs is a HOST array of nseg segments,
 * ascending and non-overlapping inside [0,n); elements outside every segment
 * are left alone.  h_seeds is a HOST array of W seeds; equal seeds give equal
 * coordinates (workers sharing their seed state, Methodology).  Messages: row w of out_vals /
 * out_idx has K = sum k_s entries (row w at +w*K). */
int sc_compress_batch(sc_ctx* ctx, int scheme, int W, const float* grads, float* residuals, size_t n,
                      const sc_segment* segs, int nseg, const uint64_t* h_seeds,
                      float* out_vals, uint32_t* out_idx, void* stream);

/* Algorithm 1, aggregate line, read as an average: out[i] = (sum over w = 0..W-1,
 * in that order, starting from +0.0, of q^w[i]) / (float)W; untouched i give
 * +0.0.  vals and idx are W rows of k entries, each row ascending and distinct,
 * all coordinates < n.  out[n] is fully overwritten. */
int sc_aggregate(sc_ctx* ctx, int W, const float* vals, const uint32_t* idx, size_t k, size_t n,
                 float* out, void* stream);

/* The same when all workers kept the same coordinates (the paper's allReduce
 * case): vals is W rows of k, idx is ONE row of k. */
int sc_aggregate_shared(sc_ctx* ctx, int W, const float* vals, const uint32_t* idx, size_t k, size_t n,
                        float* out, void* stream);

/* Algorithm 1, aggregate line fused with the model-update line (x <- x - q, q read as the
 * average as above): x[i] <- x[i] - (sum over w = 0..W-1, in order, from +0.0, of q^w[i]) / W
 * for every coordinate some worker sent; all other x[i] are left untouched.  The result is
 * bit-identical to computing the dense average with sc_aggregate and subtracting it, but the
 * dense vector is never written or read.  Same message conventions as sc_aggregate; x[n] is
 * updated in place.  The _shared form takes ONE row of coordinates for all workers. */
int sc_aggregate_apply(sc_ctx* ctx, int W, const float* vals, const uint32_t* idx, size_t k, size_t n,
                       float* x, void* stream);
int sc_aggregate_apply_shared(sc_ctx* ctx, int W, const float* vals, const uint32_t* idx, size_t k, size_t n,
                              float* x, void* stream);

/* The paper has no counterpart for this entry point: it is sc_aggregate for callers that
 * are not allowed to allocate device memory.  Every other entry point needs an sc_ctx, and
 * sc_create calls cudaMalloc.  That rules the library out for code that runs after a
 * framework has handed all free device memory to its own pool (a later cudaMalloc fails),
 * and for code inside a latency-critical section, since cudaMalloc may synchronise the
 * whole device.  sc_aggregate_static needs no context and calls no cudaMalloc, cudaFree or
 * any other allocating routine: its scratch (the per-tile message bounds, about 1 MB) is a
 * fixed __device__ array inside the library, present on every GPU that loads the library
 * until the process exits.
 *   - Same arguments and result as sc_aggregate, same bits, for W <= 64 and
 *     n <= 16,777,216.  Anything larger returns SC_ERR_RANGE before touching a buffer.
 *   - The first call on a device looks up the array's address on that device (the device
 *     must be current) and remembers it; make that first call before any stream capture.
 *   - All calls on one GPU share the one array, which keeps the previous call's contents
 *     (what has to start at zero is cleared on `stream` by the call itself).  Two calls
 *     whose kernels can overlap on the GPU (different streams, no ordering) race on it.
 *   - A message that breaks the ascending-coordinate rule is skipped silently here: there
 *     is no context whose status word could report it. */
int sc_aggregate_static(int W, const float* vals, const uint32_t* idx, size_t k, size_t n,
                        float* out, void* stream);

/* One whole step: sc_compress_batch followed by the aggregate over the W
 * messages it produced (the shared-coordinate form when all seeds are equal and
 * the scheme is not top-k).  out[n] receives the dense average. */
int sc_step(sc_ctx* ctx, int scheme, int W, const float* grads, float* residuals, size_t n,
            const sc_segment* segs, int nseg, const uint64_t* h_seeds,
            float* out_vals, uint32_t* out_idx, float* out, void* stream);

/* One whole step of Algorithm 1 without the dense average: sc_compress_batch followed by the
 * model-update line applied at the sent coordinates only, x[i] <- x[i] - (sum over w, in order, from
 * +0.0, of q^w[i]) / W (the same bits as sc_step followed by x - out, see sc_aggregate_apply).  x[n] is
 * updated in place; no dense vector of n elements is written or read besides g, e and the touched x. */
int sc_step_apply(sc_ctx* ctx, int scheme, int W, const float* grads, float* residuals, size_t n,
                  const sc_segment* segs, int nseg, const uint64_t* h_seeds,
                  float* out_vals, uint32_t* out_idx, float* x, void* stream);

/* One whole step with the step's inputs and result in HOST memory: h_grads
 * (W rows of n, ideally pinned) is copied to device staging owned by the
 * context, worker by worker, overlapped with the compression of the previous
 * worker; the dense average is copied back to h_out[n].  residuals stay on the
 * device (they are the only state carried between steps).  The first call
 * allocates the staging (cudaMalloc).  Returns after the result is in h_out. */
int sc_step_host(sc_ctx* ctx, int scheme, int W, const float* h_grads, float* residuals, size_t n,
                 const sc_segment* segs, int nseg, const uint64_t* h_seeds, float* h_out, void* stream);

/* ---------------------------------------------------------------------------------------------------------
 * Layer operators: a linear layer whose activations are kept in 8 bits between its forward and its backward
 * pass.  They produce the gradient rows that the calls above compress: the weight and bias gradients are fp32
 * and are written (or added) straight into a worker's row, at any element offset.
 *
 *     forward        z = x W^T + b,  y = act(z) + residual        x [M, K], W [N, K], z and y [M, N]
 *     checkpoints    8 bits an element of x and z, instead of 16
 *     backward       dz = dy * act'(z^),  db = column sums of dz
 *                    dx = dz W,           dW = dz^T x^            ^: the value that the checkpoint holds
 *
 * Matrices are rows of the stated length, `ld` elements apart (ld >= the row's length; any value, any base
 * aligned to its element; 16-byte aligned rows are the fast case).  Everything is computed in fp32 from the 16-bit
 * inputs and rounded once, to the type of the output.  The tensor cores add 16 products at a time to their fp32 sums and cut
 * instead of rounding, so that a sum of n products may be up to n 2^-27 of its largest running value short (16384 of one
 * sign: at most 1.2e-4 of the result); dW, an fp32 result, is added up with rounding every 384 products.  Empty sizes are allowed: no rows or
 * columns, nothing is written; an empty sum is 0.  Sizes are below 2^31.  Unless a call says otherwise outputs alias no input.
 *
 * Checkpoint of a matrix [rows, cols]: q, rows * cols int8, and scales, rows * ceil(cols / 32) bytes, both dense.
 * Each run of 32 elements of a row has one scale 2^e, stored as e + 127: e is the least exponent with
 * m <= 127 * 2^e for the largest finite magnitude m of the run, within [-126, 122] (SC_F16: [-24, 10]);
 * q = x 2^-e rounded to the nearest integer, ties to even, and within +-127 (+-63 where e is the largest of its range).
 * An element that is not finite is kept as q = -128, which reads as NaN.  Elements within half a step of 0 read as 0, where
 * relu's slope is 0.  The value q * 2^e is exactly a value of
 * the type, so what reads a checkpoint adds no rounding of its own.
 * --------------------------------------------------------------------------------------------------------- */
enum { SC_BF16 = 0, SC_F16 = 1, SC_F32 = 2 /* checkpoints only */ };
enum { SC_ACT_NONE = 0, SC_ACT_RELU = 1, SC_ACT_GELU = 2 /* z Phi(z) */,
       SC_ACT_GELU_TANH = 3 /* z (1 + tanh(sqrt(2/pi) (z + 0.044715 z^3))) / 2 */, SC_ACT_SILU = 4 /* z / (1 + e^-z) */ };

/* The layer operators keep their workspace in the context.  A call that needs more than it has allocates
 * (synchronous), or returns SC_ERR_WORKSPACE while its stream is being captured.  sc_layer_reserve allocates
 * ahead what any layer call of at most these sizes needs.  A block that captured calls used is kept until sc_destroy. */
int sc_layer_reserve(sc_ctx* ctx, size_t M, size_t N, size_t K);

/* Instrumentation for tests: later products of this context run in tiles of rows x cols outputs (256 x 256, 128 x 256, 128 x 128 or
 * 128 x 64), their sums cut into `parts` (1 to 64), instead of what the library chooses for the size; 0, 0, 0 restores its choice.  Products
 * of up to 128 rows take no 256-row tiles, sums no more parts than blocks of 64 terms or 64 MB of partial sums allow, and the few
 * tokens that are served without tiles still are.  Host-side state, no device work. */
int sc_debug_layer_tiles(sc_ctx* ctx, int rows, int cols, int parts);

/* Checkpoint of x, and the values of a checkpoint (rounded to `type` where the checkpoint was made from another). */
int sc_checkpoint_pack(sc_ctx* ctx, int type, const void* x, size_t ldx, size_t rows, size_t cols,
                       int8_t* q, uint8_t* scales, void* stream);
int sc_checkpoint_unpack(sc_ctx* ctx, int type, const int8_t* q, const uint8_t* scales, size_t rows, size_t cols,
                         void* out, size_t ldo, void* stream);

/* dz = dy * act'(z^) with z^ the checkpoint (q, scales) of the pre-activation, and db[cols] = column sums of dz
 * before its rounding (accumulate: added to db).  dz or db may be NULL; dz may be dy (same ld).  With SC_ACT_NONE the
 * checkpoint is not read: the call gives the bias gradient of dy. */
int sc_activation_grad(sc_ctx* ctx, int type, int act, const void* dy, size_t lddy, const int8_t* q, const uint8_t* scales,
                       size_t rows, size_t cols, void* dz, size_t lddz, float* db, int accumulate, void* stream);

/* y = act(x W^T + bias) + residual.  bias[N] and residual [M, N] are of the type and may be NULL; y may be residual
 * (same ld).  With q and scales the checkpoint of z = x W^T + bias, taken from its fp32 values, is written too. */
int sc_linear(sc_ctx* ctx, int type, int act, const void* x, size_t ldx, const void* w, size_t ldw, const void* bias,
              const void* residual, size_t ldr, size_t M, size_t N, size_t K, void* y, size_t ldy,
              int8_t* q, uint8_t* scales, void* stream);

/* dx = (dz W + residual) * act'(z^): the gradient of the layer's input, plus a residual branch's gradient [M, K]
 * (NULL: none), through the activation that made that input (SC_ACT_NONE, or z^ [M, K] as q and scales).  dx may be
 * residual (same ld). */
int sc_linear_grad_input(sc_ctx* ctx, int type, int act, const void* dz, size_t lddz, const void* w, size_t ldw,
                         const void* residual, size_t ldr, const int8_t* q, const uint8_t* scales,
                         size_t M, size_t N, size_t K, void* dx, size_t lddx, void* stream);

/* dW = dz^T x in fp32, rows of lddw (accumulate: added to dW, where values below 2^-126 may count as 0).  The layer's input is given once: as x, or as its
 * checkpoint (q, scales) with x NULL, whose values are those of sc_checkpoint_unpack to `type`. */
int sc_linear_grad_weight(sc_ctx* ctx, int type, const void* dz, size_t lddz, const void* x, size_t ldx,
                          const int8_t* q, const uint8_t* scales, size_t M, size_t N, size_t K,
                          float* dw, size_t lddw, int accumulate, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* SPARSECOMM_H */
