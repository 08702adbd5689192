/*
 * darb.h -- C ABI of libdarb: density-adaptive regular-block (DARB) pruned
 * matrices on one GB300 GPU (sm_103a).
 *
 * DARB (Ren et al., "DARB: A Density-Adaptive Regular-Block Pruning for Deep
 * Neural Networks", arXiv 1911.08020) splits every row of a weight matrix into
 * equal blocks whose size depends on the row (Sec. 3.2), keeps the one weight of
 * largest magnitude in each block (block-max weight masking, BMWM, Sec. 3.1),
 * and stores per block only that value and its position inside the block
 * (log2 m bits, Sec. 4.2).  Multiplying by such a matrix needs, per block, one
 * small selection among m activations (Sec. 3.2, Fig. 6(b)).
 *
 * This library encodes dense matrices into that format on the GPU and
 * multiplies with them, alone or fused into LSTM / GRU cell steps.
 *
 * Conventions shared by every call:
 *  - Every call returns a darb_status_t and never aborts the process.
 *  - Matrices are row-major with an explicit leading dimension in elements.
 *    Activations X are cols x batch with the batch contiguous (row k of X
 *    starts at X + k * ldx); outputs Y are rows x batch (row r at Y + r * ldy).
 *  - Pointers documented as "device" must be CUDA device (or managed) memory
 *    of the current device; "host" pointers are ordinary host memory.
 *  - The caller owns every buffer it passes; a handle owns the encoded matrix
 *    and any scratch it allocates, and releases both in darb_destroy.
 *  - Work is enqueued on the caller's stream.  Only darb_encode, darb_import,
 *    darb_export, darb_sync_status, darb_rnn_reserve, darb_adamw_create,
 *    darb_muon_create, the two _sync_status of their plans and the destroy calls
 *    synchronise; the others are asynchronous.
 *    darb_spmm allocates nothing; the step calls on large matrices or batches
 *    use scratch owned by the handle (darb_rnn_reserve sizes it up front).
 *  - Only these calls take scratch from the device's stream-ordered memory
 *    pool: darb_spmm_ex with DARB_PATH_TENSOR_CORES, the sequence calls, and
 *    darb_layer_norm_grad and darb_policy_loss where they are given none.  They
 *    return it to the pool on the same stream.  The first such call on a device raises the release threshold of the device's current
 *    pool to 1 GiB if it is lower, so that freed scratch stays mapped across
 *    synchronisations; darb_spmm never touches the pool.
 *  - There is no CPU fallback: without a usable CUDA device the GPU calls
 *    return DARB_ERR_CUDA.
 */
#ifndef DARB_H
#define DARB_H

#include <stdint.h>
#include <cuda_runtime_api.h>

#if defined(__GNUC__)
#define DARB_API __attribute__((visibility("default")))
#else
#define DARB_API
#endif

#ifdef __cplusplus
extern "C" {
#endif

typedef struct darb_handle_s *darb_handle_t;

typedef enum {
    DARB_OK = 0,
    DARB_ERR_INVALID_ARG = 1,   /* null pointer, size <= 0, ld < width, m out of [1,256],
                                   shape mismatch, unknown or destroyed handle          */
    DARB_ERR_NONFINITE = 2,     /* a NaN weight was found while encoding                 */
    DARB_ERR_OOM = 3,           /* a device or host allocation failed                    */
    DARB_ERR_CUDA = 4,          /* a CUDA runtime call or kernel launch failed           */
    DARB_ERR_TIMEOUT = 5,       /* a bounded device-side wait gave up (darb_sync_status)  */
    DARB_ERR_UNSUPPORTED = 6    /* arguments valid but not supported by these kernels    */
} darb_status_t;

typedef enum { DARB_F32 = 0, DARB_BF16 = 1 } darb_dtype_t;

/* How the activations of a call lie in memory.  DARB_TOKEN_ROWS: token t is a row
 * of contiguous features at t * ld.  DARB_TOKEN_COLUMNS: features x tokens, feature
 * f of token t at f * ld + t -- the layout that darb_spmm and the steps read and write.
 * In the calls that take a layout, matrices of one leading dimension that lie side by side
 * in a wider buffer do not overlap, nor does a vector that lies between a matrix's lines;
 * of different leading dimensions everything from the first to the last element counts. */
typedef enum { DARB_TOKEN_ROWS = 0, DARB_TOKEN_COLUMNS = 1 } darb_layout_t;

/* Largest block size the format stores (offsets take at most 8 bits). */
#define DARB_MAX_BLOCK 256

/* Most alternatives that darb_token_logprobs lists for a token. */
#define DARB_MAX_TOP 32

/*
 * Density-adaptive block-size rule (Sec. 3.2, the worked example with matrix
 * density 21.88%).  Host only; no CUDA call.
 *   row_nnz  host int64[rows]: retained weights per row after irregular pruning,
 *            0 <= row_nnz[r] <= cols.
 *   m_out    host int32[rows]: block size per row.
 * A row denser than the whole matrix has its density rounded UP to the next
 * power-of-two density 1/m, a sparser row DOWN; m = 1 / rounded density.
 * Readings where the paper is silent: a row exactly at the matrix density is
 * rounded up; an empty row gets m_max; the result is clamped to [m_min, m_max].
 * Errors: DARB_ERR_INVALID_ARG for null pointers, rows/cols <= 0, row_nnz out of
 * range, or not 1 <= m_min <= m_max <= DARB_MAX_BLOCK.
 */
DARB_API darb_status_t darb_assign_block_sizes(const int64_t *row_nnz, int64_t rows, int64_t cols,
                                      int32_t m_min, int32_t m_max, int32_t *m_out);

/*
 * Block sizes from the weights themselves (Sec. 3.2): the K = `keep` weights
 * of largest magnitude form the mask of irregular pruning (Sec. 2, "Irregular Pruning"), used
 * only to measure each row's density; darb_assign_block_sizes then turns the
 * row counts into block sizes.  Weights tied with the K-th largest magnitude
 * all count (the paper does not break such ties), so the counts may add up to
 * slightly more than K.  Magnitudes are compared on the stored values (bf16
 * or fp32); +0 and -0 tie; an infinity is the largest.
 *   W        device, rows x cols row-major, leading dimension ldw (elements),
 *            aligned to its element size
 *   keep     1 <= keep <= rows * cols (and rows * cols < 2^32)
 *   row_nnz_out  host int64[rows] receiving the counts, or NULL
 *   m_out    host int32[rows] receiving the block sizes
 * Runs on `stream` and synchronises it.  Device scratch (8 bytes per row) is
 * kept by the library between calls, one buffer per device; concurrent calls
 * take turns on it.
 * Errors: DARB_ERR_INVALID_ARG; DARB_ERR_NONFINITE if W holds a NaN;
 * DARB_ERR_UNSUPPORTED if rows * cols >= 2^32; DARB_ERR_OOM; DARB_ERR_CUDA.
 */
DARB_API darb_status_t darb_assign_from_weights(const void *W, darb_dtype_t wtype, int64_t rows, int64_t cols,
                                                int64_t ldw, int64_t keep, int32_t m_min, int32_t m_max,
                                                int64_t *row_nnz_out, int32_t *m_out, cudaStream_t stream);

/*
 * BMWM encode (Sec. 3.1 steps (1)-(3), with the per-row block size of Sec. 3.2).
 *   W      device, rows x cols, row-major, leading dimension ldw >= cols
 *          (elements); fp32 or bf16 as wtype says.  Any alignment.
 *   m      host int32[rows], 1 <= m[r] <= DARB_MAX_BLOCK (any value, not only
 *          powers of two).
 *   out    receives a new handle.
 * Row r is split into ceil(cols / m[r]) blocks, block j covering columns
 * [j*m[r], min((j+1)*m[r], cols)) (a shorter last block still keeps one
 * weight).  In each block the weight of largest magnitude is kept; among
 * equal magnitudes (including +0 / -0) the lowest column wins.  +-Inf are the
 * largest magnitudes.  The kept value is stored bit for bit in wtype.
 * Allocates the handle's device memory, runs on `stream` and synchronises it
 * before returning; W may be freed afterwards.
 * Errors: DARB_ERR_INVALID_ARG; DARB_ERR_NONFINITE if W holds a NaN (no handle
 * is returned); DARB_ERR_OOM; DARB_ERR_CUDA.
 */
DARB_API darb_status_t darb_encode(const void *W, darb_dtype_t wtype, int64_t rows, int64_t cols,
                          int64_t ldw, const int32_t *m, darb_handle_t *out, cudaStream_t stream);

/*
 * Re-run BMWM on a new W of the handle's shape and dtype, keeping its block
 * sizes, into the handle's existing memory (e.g. after a retraining step of
 * Sec. 4's prune-retrain loop).  Asynchronous on `stream`, allocates nothing.
 * A NaN in W is recorded on the device and reported by darb_sync_status.
 * The handle must not be in use by work on another stream meanwhile.
 */
DARB_API darb_status_t darb_reencode(darb_handle_t h, const void *W, int64_t ldw, cudaStream_t stream);

/*
 * darb_reencode from weights in HOST memory (Sec. 3.1's BMWM on a W that
 * lives on the host, as a serving or training loop hands it over).
 *   W      host, rows x ldw elements of the handle's dtype, row-major,
 *          ldw >= cols; only the first cols of each row are read.
 *   W_dev  device, rows x ldw elements (aligned to the element size), owned
 *          by the caller: W is copied there (rows of cols elements at pitch
 *          ldw), then re-encoded from it; it keeps the copy afterwards.
 * The copy and the encode are ordered on `stream`.  With pinned host memory
 * the call is asynchronous; with pageable memory the copy completes before
 * the call returns.  Allocates nothing.
 * Errors: as darb_reencode, and DARB_ERR_INVALID_ARG for a null W_dev;
 * DARB_ERR_CUDA if the copy cannot be issued.
 */
DARB_API darb_status_t darb_reencode_host(darb_handle_t h, const void *W, int64_t ldw, void *W_dev,
                                          cudaStream_t stream);

/* Synchronise `stream` and report what the handle's kernels recorded on the
 * device since the last call, then clear it: DARB_ERR_TIMEOUT if a bounded
 * device wait (for a bulk copy, or of a sequence call for another CTA) gave up
 * -- results of that call are not valid, the device stays usable -- else
 * DARB_ERR_NONFINITE if a (re)encode met a NaN, else DARB_OK.                */
DARB_API darb_status_t darb_sync_status(darb_handle_t h, cudaStream_t stream);

/*
 * Y = W_darb X: for row r and batch column b,
 *   Y[r, b] = sum_j val[r, j] * X[j*m_r + off[r, j], b]
 * (block j of the row selects one activation row, Sec. 3.2 / Fig. 6(b)).
 *   X  device fp32, cols x batch, ldx >= batch, 4-byte aligned.
 *   Y  device fp32, rows x batch, ldy >= batch; overwritten.  Must not
 *      overlap X.
 * Every kept weight is multiplied only by the activation its block selects
 * (a NaN or infinity in an activation row that no kept weight selects does
 * not reach Y), in fp32, on the CUDA cores, for every dtype and batch.
 * Asynchronous on `stream`; allocates nothing; the handle is only read, so
 * calls on several streams may share it.  A bounded device wait that gave up
 * is reported by darb_sync_status.
 * Errors: DARB_ERR_INVALID_ARG (null, batch <= 0, ld < batch, X or Y not
 * 4-byte aligned, Y overlapping X); DARB_ERR_UNSUPPORTED (batch above 2^19);
 * DARB_ERR_CUDA.
 */
DARB_API darb_status_t darb_spmm(darb_handle_t h, const float *X, int64_t ldx, int64_t batch, float *Y,
                        int64_t ldy, cudaStream_t stream);

/*
 * darb_spmm with X and Y in HOST memory (Sec. 3.2's product as a caller
 * outside the GPU sees it: activations in, outputs back).
 *   X      host fp32, cols x batch, ldx >= batch.
 *   Y      host fp32, rows x batch, ldy >= batch; receives the product.
 *   X_dev  device fp32, cols x batch (rows of batch floats), owned by the
 *          caller: X is copied there first.
 *   Y_dev  device fp32, rows x batch (rows of batch floats), owned by the
 *          caller: the product is written there, then copied into Y.  Must
 *          not overlap X_dev.
 * Copy in, product (darb_spmm on X_dev, Y_dev) and copy out are ordered on
 * `stream`; with pinned host memory the call is asynchronous and Y holds the
 * product once `stream` has been synchronised.  Allocates nothing.
 * Errors: as darb_spmm (X_dev and Y_dev checked as its X and Y, X and Y for
 * null); DARB_ERR_CUDA if a copy cannot be issued.
 */
DARB_API darb_status_t darb_spmm_host(darb_handle_t h, const float *X, int64_t ldx, int64_t batch, float *Y,
                                      int64_t ldy, float *X_dev, float *Y_dev, cudaStream_t stream);

/* Which kernels compute a product (the paper has no counterpart: these are two
 * ways of evaluating the same sum on the GPU).                               */
typedef enum {
    DARB_PATH_AUTO = 0,          /* what darb_spmm does: the CUDA-core gather        */
    DARB_PATH_CUDA_CORES = 1,    /* gather-multiply-add on the CUDA cores (any weights) */
    DARB_PATH_TENSOR_CORES = 2   /* densified tiles on the tensor cores (bf16 weights) */
} darb_path_t;

/*
 * darb_spmm with the kernel family chosen by the caller.  DARB_PATH_AUTO and
 * DARB_PATH_CUDA_CORES are darb_spmm.  DARB_PATH_TENSOR_CORES is an opt-in
 * alternative that is not the paper's per-block selection: it multiplies every activation
 * of a stage by the densified tile, zeros included, with X split into two
 * bf16 parts (x = hi + lo): |Y - exact| <= 2^-16 * sum |val * x| plus fp32
 * rounding, a NaN or infinity in X may make rows NaN that do not select it,
 * and |x| must stay below the largest bf16.  It needs bf16 weights, and it
 * takes the split of X (4 bytes per element of X, batch rounded up to 8) from
 * the device's stream-ordered memory pool on `stream` for the duration of the
 * call (DARB_ERR_OOM if the pool cannot supply it); the CUDA-core path
 * allocates nothing.
 * Errors: as darb_spmm; DARB_ERR_INVALID_ARG for an unknown path;
 * DARB_ERR_UNSUPPORTED if DARB_PATH_TENSOR_CORES cannot take the call.
 */
DARB_API darb_status_t darb_spmm_ex(darb_handle_t h, const float *X, int64_t ldx, int64_t batch, float *Y,
                                    int64_t ldy, darb_path_t path, cudaStream_t stream);

/* The kernel family darb_spmm takes for this handle and batch (*path: always
 * DARB_PATH_CUDA_CORES), and how many kernels it launches per call (*kernels:
 * 1).  Host only.
 * Errors: DARB_ERR_INVALID_ARG (unknown handle, batch <= 0, null outputs). */
DARB_API darb_status_t darb_spmm_path(darb_handle_t h, int64_t batch, darb_path_t *path, int32_t *kernels);

/*
 * One LSTM cell step whose gate matrix is the handle (rows = 4H, cols = I + H),
 * multiplied with the stacked input [x_t; h_{t-1}].  Gate rows [0,H) = i,
 * [H,2H) = f, [2H,3H) = g, [3H,4H) = o (the paper names LSTMs, Sec. 4.1, but
 * writes no cell equations; this is the standard cell):
 *   c_t = sigmoid(f) * c_{t-1} + sigmoid(i) * tanh(g),  h_t = sigmoid(o) * tanh(c_t)
 *   x      device fp32, I x B (batch contiguous); may be NULL when I == 0
 *   h_prev, c_prev   device fp32, H x B
 *   bias   device fp32 [4H] added to the gate pre-activations, or NULL
 *   h_out, c_out     device fp32, H x B; must not overlap any input
 * Most steps keep their gate sums on chip and need no scratch.  A step whose
 * stacked input is too tall for that (from some 14000 rows), whose batch is
 * above 1024, or that is faster on the kernels that exchange gate sums through
 * memory (large matrices; decided by the sizes, the dtype and the alignment)
 * uses scratch owned by the handle (4H x B floats of gate sums and at most
 * H x ceil(B / t) counters, t = 1, 2, 4 or 8 by batch), allocated by the first such call that
 * needs more than the handle holds (that call synchronises); call
 * darb_rnn_reserve first to size it up front.  Step calls on one handle must
 * be ordered on one stream.
 * Errors: DARB_ERR_INVALID_ARG (null, shape mismatch, B <= 0); DARB_ERR_OOM;
 * DARB_ERR_CUDA.
 */
DARB_API darb_status_t darb_lstm_step(darb_handle_t h, int64_t I, int64_t H, int64_t B, const float *x,
                             const float *h_prev, const float *c_prev, const float *bias,
                             float *h_out, float *c_out, cudaStream_t stream);

/*
 * One GRU cell step whose gate matrix is the handle (rows = 3H, cols = I + H).
 * Gate rows [0,H) = r, [H,2H) = z, [2H,3H) = n; columns [0,I) multiply x_t and
 * [I,I+H) multiply h_{t-1}, and the two parts are kept apart (the paper names
 * GRUs, Sec. 4.1, without equations; this is the standard cell):
 *   a = W[:, :I] x + b_ih,  bh = W[:, I:] h + b_hh
 *   r = sigmoid(a_r + bh_r), z = sigmoid(a_z + bh_z), n = tanh(a_n + r * bh_n)
 *   h_t = (1 - z) * n + z * h_{t-1}
 *   x device fp32 I x B (NULL allowed when I == 0); h_prev device fp32 H x B;
 *   b_ih, b_hh device fp32 [3H] or NULL; h_out device fp32 H x B, not
 *   overlapping any input.
 * Scratch, ordering and errors as for darb_lstm_step (scratch 2 x 3H x B floats).
 */
DARB_API darb_status_t darb_gru_step(darb_handle_t h, int64_t I, int64_t H, int64_t B, const float *x,
                            const float *h_prev, const float *b_ih, const float *b_hh,
                            float *h_out, cudaStream_t stream);

/*
 * T consecutive LSTM steps (the cell of darb_lstm_step) in one persistent
 * launch: the recurrence of an RNN layer over a whole input sequence (the
 * LSTM models of Sec. 4.1 run one step per token).  The batch columns are cut
 * into groups, each run by its own CTAs; a CTA keeps its share of the gate
 * matrix decoded in shared memory for all T steps, so W is read from memory
 * once per call instead of once per step.  The steps of a group are separated
 * by a barrier over its CTAs, or, where a column tile of h is at most 32 KB, by
 * the values of h themselves, which carry the number of their step.
 *   x_seq  device fp32, T x I x B (step t at x_seq + t*I*B); NULL allowed when I == 0
 *   h0, c0 device fp32, H x B: the state before the first step
 *   bias   device fp32 [4H] or NULL
 *   h_seq  device fp32, T x H x B: h_t of every step
 *   c_seq  device fp32, T x H x B: c_t of every step, or NULL
 *   c_last device fp32, H x B: c_T, or NULL
 * No output may overlap an input or another output.  T == 0 launches nothing
 * and copies c0 to c_last.  The results equal T calls of darb_lstm_step up to
 * the order of the fp32 additions inside each gate sum.
 * When x_t is at least a third of the stacked input (2I >= H), the sequence
 * has 64 to 2^19 columns (T * B) and the workspace below stays under 1 GiB,
 * the x parts of all T steps are computed first as one product
 * W [x_0 .. x_{T-1}; 0] of T * B columns (darb_spmm's kernels and numerics,
 * the CUDA-core gather); the recurrence then stages and
 * multiplies only h_{t-1}.
 * Resources: a preparing launch and one cooperative launch of at most one CTA
 * per SM, and a stream-ordered workspace of
 *   - 128 bytes for every column group (at most one a CTA), and 128 more;
 *   - H x B floats when c_last is NULL and the cell state does not fit on chip;
 *   - two buffers of h, H rounded up to 4 rows x B rounded up to whole column
 *     tiles (of 1 to 32 columns): 4 bytes an element, 8 where a tile of h is at
 *     most 32 KB;
 *   - when the x parts are precomputed, (I + H + 4H) x T*B floats (T*B rounded
 *     up to 4); else, unless I is 0 or x_seq is laid out so already (I a multiple
 *     of 4, B one whole tile, a 16-byte aligned base), a copy of x_seq with I
 *     rounded up to 4 rows and B to whole tiles, if that is at most 1 GiB and
 *     the memory pool can supply it; x_seq is read in place if not.
 * DARB_ERR_OOM if the pool cannot supply the rest.  A wait of more than 1 s for
 * another CTA ends the launch and is reported by darb_sync_status as
 * DARB_ERR_TIMEOUT.  For testing that path, the environment variable
 * DARB_TEST_BARRIER_TIMEOUT=1 (read at every launch) shortens the limit to 1 ms
 * and makes CTA 0 withhold its first arrival or its first values of h, so the
 * launch times out on purpose; DARB_TEST_POOL_LIMIT=n makes the pool refuse
 * workspaces of more than n bytes.
 * Errors: DARB_ERR_INVALID_ARG (shape mismatch, null, overlap, T < 0);
 * DARB_ERR_UNSUPPORTED when a CTA's share of the decoded matrix plus one
 * column tile of [x_t; h_{t-1}] does not fit in shared memory, or cols > 65535;
 * DARB_ERR_OOM; DARB_ERR_CUDA.
 */
DARB_API darb_status_t darb_lstm_sequence(darb_handle_t h, int64_t T, int64_t I, int64_t H, int64_t B,
                                          const float *x_seq, const float *h0, const float *c0,
                                          const float *bias, float *h_seq, float *c_seq, float *c_last,
                                          cudaStream_t stream);

/*
 * T consecutive GRU steps (the cell of darb_gru_step) in one persistent
 * launch, as darb_lstm_sequence.
 *   x_seq device fp32, T x I x B (NULL allowed when I == 0); h0 device fp32
 *   H x B; b_ih, b_hh device fp32 [3H] or NULL; h_seq device fp32, T x H x B,
 *   not overlapping any input.
 * Precomputed x parts, resources and errors as darb_lstm_sequence (workspace
 * with 3H rows of x parts).
 */
DARB_API darb_status_t darb_gru_sequence(darb_handle_t h, int64_t T, int64_t I, int64_t H, int64_t B,
                                         const float *x_seq, const float *h0, const float *b_ih,
                                         const float *b_hh, float *h_seq, cudaStream_t stream);

/*
 * darb_lstm_step without any allocation: the same step, same arguments and
 * same results, with the scratch of the steps that need some (gate sums and
 * arrival counters) in one fixed array of 4 MiB inside this library instead of
 * memory owned by the handle.  It is for callers that cannot let a library call cudaMalloc at step
 * time -- a serving loop with a fixed memory budget, code that must not
 * synchronise the device mid-stream, or allocations that must all go through
 * the caller's own pool.  The paper has no counterpart; it is a property of
 * this library's interface only.
 *   - Limit: 4H*B floats (rounded up to 256 bytes) plus H*ceil(B/t) counters
 *     (t = 1, 2, 4 or 8 by batch) must fit in 4 MiB, whether or not the step
 *     uses them; larger calls return DARB_ERR_UNSUPPORTED and do nothing.
 *   - Every GPU that loads the library holds the 4 MiB until the process exits.
 *   - The first call on each device looks up the array's device address (one
 *     cudaGetSymbolAddress); make that first call before any stream capture.
 *   - All calls on a device share the one array, which keeps the last call's
 *     contents; a call that uses it clears its counters on `stream`.  Calls that
 *     overlap on the GPU (other streams, or unordered launches) race on it.
 * Errors as darb_lstm_step, plus DARB_ERR_UNSUPPORTED for the size limit.
 */
DARB_API darb_status_t darb_lstm_step_noalloc(darb_handle_t h, int64_t I, int64_t H, int64_t B,
                                              const float *x, const float *h_prev, const float *c_prev,
                                              const float *bias, float *h_out, float *c_out,
                                              cudaStream_t stream);

/* Size the handle's RNN step scratch for batches up to max_batch now, so that
 * later step calls allocate nothing (e.g. before capturing them in a CUDA
 * graph).  Synchronises the device.  Errors: INVALID_ARG, OOM, CUDA.          */
DARB_API darb_status_t darb_rnn_reserve(darb_handle_t h, int64_t max_batch);

/*
 * What a model answers with, scored: for each token the log probability of the
 * entry that was given, the entropy of the distribution and its k most probable
 * entries, from the logits in one pass (the perplexity that Sec. 4.1 reports
 * is exp of the mean negative log probability).  With x the token's logits,
 *   lse = log sum_v exp(x_v),  log p_v = x_v - lse,  entropy = -sum_v p_v log p_v.
 *   logits   device, tokens x vocab in `layout`, fp32 or bf16 (dtype), leading
 *            dimension ld (>= vocab for token rows, >= tokens for token columns)
 *   targets  device int64[tokens]: the entry whose log probability is wanted;
 *            negative: none (log probability 0); vocab or more: NaN.  NULL if
 *            logprob is NULL, and only then
 *   k        0 <= k <= min(DARB_MAX_TOP, vocab)
 *   logprob, entropy, lse   device fp32[tokens]; each may be NULL
 *   top_logprob, top_index  device fp32 / int32 [tokens x k], most probable
 *            first, equal logits by index (NaN counts as the largest); NULL
 *            allowed when k == 0
 * A logit of -inf is a masked entry (p = 0).  A token whose entries are all -inf
 * has lse and log probabilities of -inf and an entropy of 0.  A token with a NaN or
 * +inf among its logits has NaN results (its top_index stands).  No other log
 * probability is above 0 and no other entropy below it.  All sums are fp32 and in
 * a fixed order.  tokens == 0 does nothing.
 * No output may overlap another buffer of the call.  Asynchronous on `stream`;
 * allocates nothing; one launch.
 * Errors: DARB_ERR_INVALID_ARG; DARB_ERR_UNSUPPORTED (more than 2^27 tokens,
 * 2^30 entries, or 2^48 elements from the first to the last logit); DARB_ERR_CUDA.
 */
DARB_API darb_status_t darb_token_logprobs(const void *logits, darb_dtype_t dtype, darb_layout_t layout,
                                           int64_t tokens, int64_t vocab, int64_t ld, const int64_t *targets,
                                           int32_t k, float *logprob, float *entropy, float *lse,
                                           float *top_logprob, int32_t *top_index, cudaStream_t stream);

/*
 * The gradient of darb_token_logprobs with respect to the logits: with a and b
 * the incoming gradients of log probability and entropy,
 *   d_logits_v = a ([v = target] - p_v) - b p_v (log p_v + entropy).
 * (The gradient of the mean loss over n tokens has a = -1/n.)
 *   logits, targets   as in the forward call; lse, entropy its results
 *   d_logprob, d_entropy   device fp32[tokens]; NULL: no such gradient (targets
 *            may then be NULL, and without d_entropy entropy may be NULL)
 *   d_logits device, tokens x vocab in `layout`, of the logits' dtype, leading
 *            dimension ld_grad; may be the logits themselves (same pointer and
 *            leading dimension), otherwise it may not overlap another buffer
 * A token without a target gets no gradient of its log probability, a token
 * whose entries are all -inf none at all; a target of vocab or more gives NaN.
 * One fp32 number for lse leaves p with a relative error of up to 2^-16 while lse is
 * within +-512.  The sums of a token past that are taken again from its logits,
 * which takes longer.
 * Asynchronous on `stream`; allocates nothing; one launch.
 * Errors: as darb_token_logprobs.
 */
DARB_API darb_status_t darb_token_logprobs_grad(const void *logits, darb_dtype_t dtype, darb_layout_t layout,
                                                int64_t tokens, int64_t vocab, int64_t ld, const int64_t *targets,
                                                const float *lse, const float *entropy, const float *d_logprob,
                                                const float *d_entropy, void *d_logits, int64_t ld_grad,
                                                cudaStream_t stream);

/*
 * Layer norm over the features of each token (the normalisation between the
 * layers that the library multiplies):
 *   mean = sum_f x_f / F,  rstd = 1 / sqrt(sum_f (x_f - mean)^2 / F + eps),
 *   y_f = (x_f - mean) * rstd * gamma_f + beta_f.
 *   x, y     device, fp32 or bf16 (dtype), leading dimensions ld_x, ld_y.  Token
 *            rows: tokens x features, steps = 1.  Token columns: `steps` matrices
 *            of features x tokens one after the other (matrix s at
 *            s * features * ld), as the sequence calls write them
 *   gamma, beta   device fp32[features]; NULL: 1 and 0
 *   mean, rstd    device fp32[steps x tokens]: the statistics the backward pass
 *            needs; each may be NULL
 * The mean and the centred squares are summed in fp32, the squares after the mean
 * is known.  y may be x itself (same pointer and leading dimension); no other
 * overlap of an output is allowed.  No tokens: nothing is done.
 * A bounded device wait that gave up (DARB_ERR_TIMEOUT elsewhere; it has no handle
 * to be reported through) leaves NaN in the tokens it was for.
 * Asynchronous on `stream`; allocates nothing; one launch.
 * Errors: DARB_ERR_INVALID_ARG (also a negative or NaN eps); DARB_ERR_UNSUPPORTED
 * (sizes as darb_token_logprobs, features up to 2^24); DARB_ERR_CUDA.
 */
DARB_API darb_status_t darb_layer_norm(const void *x, darb_dtype_t dtype, darb_layout_t layout, int64_t steps,
                                       int64_t tokens, int64_t features, int64_t ld_x, const float *gamma,
                                       const float *beta, float eps, void *y, int64_t ld_y, float *mean, float *rstd,
                                       cudaStream_t stream);

/*
 * The backward pass of darb_layer_norm.  With xh = (x - mean) * rstd and
 * g = dy * gamma, per token
 *   dx_f = rstd * (g_f - sum g / F - xh_f * sum(g xh) / F),
 * and over all tokens dgamma_f = sum dy_f xh_f, dbeta_f = sum dy_f.
 *   dy, x, dx   device, of one dtype and layout, with leading dimensions of
 *            their own; dx may be dy itself (same pointer and leading dimension)
 *   gamma    device fp32[features] or NULL (1)
 *   mean, rstd  what the forward pass wrote
 *   dgamma, dbeta  device fp32[features], overwritten (with zeros when there
 *            are no tokens); both NULL: not wanted
 *   work     device scratch of darb_layer_norm_grad_work bytes, 16-byte aligned, the
 *            caller's; NULL: taken from the device's stream-ordered memory pool for
 *            the duration of the call.  Not used when dgamma and dbeta are NULL
 * The sums over the tokens are fp32, in an order fixed by the sizes and alignments.
 * Asynchronous on `stream`; allocates nothing else.  Errors: as darb_layer_norm,
 * and DARB_ERR_OOM if the pool cannot supply the scratch.
 */
DARB_API darb_status_t darb_layer_norm_grad(const void *dy, int64_t ld_dy, const void *x, int64_t ld_x,
                                            darb_dtype_t dtype, darb_layout_t layout, int64_t steps, int64_t tokens,
                                            int64_t features, const float *gamma, const float *mean,
                                            const float *rstd, void *dx, int64_t ld_dx, float *dgamma, float *dbeta,
                                            void *work, cudaStream_t stream);

/* Bytes of scratch that darb_layer_norm_grad needs on the current device.
 * Errors: DARB_ERR_INVALID_ARG (sizes, null output); DARB_ERR_UNSUPPORTED (sizes
 * that darb_layer_norm_grad does not take).                                   */
DARB_API darb_status_t darb_layer_norm_grad_work(darb_layout_t layout, int64_t steps, int64_t tokens, int64_t features,
                                                 int64_t *bytes);

/* What a gate of darb_gated_scan holds: the logit of the share of the old state that
 * is kept, or that share itself. */
typedef enum { DARB_GATES_LOGITS = 0, DARB_GATES_VALUES = 1 } darb_gates_t;

/*
 * A gated linear recurrence over whole sequences: the recurrent layer whose gates do
 * not need the step before, so that those of all steps are one darb_spmm.  Per channel
 *   a_t = sigmoid(gate_t) (DARB_GATES_VALUES: gate_t),
 *   h_t = a_t h_(t-1) + (1 - a_t) x_t   (coupled == 0: a_t h_(t-1) + x_t).
 *   gate, x, h   device, fp32 or bf16 (dtype).  Element (o, t, i) -- outer, step, inner
 *            -- is at o * ld + t * step + i, with leading dimensions and steps of their
 *            own.  What the sequence calls write (steps x features x batch) has inner =
 *            features * batch; a product of all steps (features x (steps * batch)) has
 *            outer = features, inner = batch; token rows (batch x steps x features) have
 *            outer = batch, inner = features.  No two elements of a tensor may share a place
 *   h0       device fp32[outer x inner], the state before step 0; NULL: 0
 *   h_last   device fp32[outer x inner], the state after the last step; NULL: not wanted.
 *            May be h0 itself (a state that is carried from call to call)
 * The state is fp32 from step to step; h is rounded to its type as it is written.  h may
 * be x itself (same pointer and strides); no other overlap is allowed.  A logit of -inf
 * starts anew (a = 0), one of +inf keeps the state (a = 1; steps are put together in a fixed
 * order of their own, so that its last place may change); a NaN makes its channel NaN from
 * there on, and so may an infinite state, as soon as the product of the gates since is 0 in
 * 32 bits.  Gates above 1 in magnitude are allowed
 * as long as their products over any 8192 steps stay finite.
 * No channels: nothing is done; steps == 0: h_last is h0.
 * Asynchronous on `stream`; allocates nothing; one launch (steps == 0: a copy).
 * Errors: DARB_ERR_INVALID_ARG; DARB_ERR_UNSUPPORTED (more than 2^30 steps or channels,
 * or 2^48 elements from the first to the last of a tensor); DARB_ERR_CUDA.
 */
DARB_API darb_status_t darb_gated_scan(const void *gate, int64_t ld_gate, int64_t step_gate, const void *x,
                                       int64_t ld_x, int64_t step_x, darb_dtype_t dtype, darb_gates_t gates,
                                       int coupled, int64_t outer, int64_t steps, int64_t inner, const float *h0,
                                       void *h, int64_t ld_h, int64_t step_h, float *h_last, cudaStream_t stream);

/*
 * The backward pass of darb_gated_scan.  From the last step to the first, with c what
 * flows to a step from the one after it (d_last at the end),
 *   g = dh_t + c,  d_x_t = g (1 - a_t)  (coupled == 0: g),
 *   d_gate_t = g (h_(t-1) - x_t) a_t (1 - a_t)   (coupled == 0: without x_t;
 *            DARB_GATES_VALUES: without a_t (1 - a_t)),
 *   c = a_t g,  and at the end d_h0 = c.
 *   gate, x, h0, gates, coupled   as in the forward call; h its result
 *   dh       device, the gradient that comes in at every step, of the same dtype
 *   d_last   device fp32[outer x inner], the gradient of h_last; NULL: 0
 *   d_gate, d_x   device, of the same dtype; d_gate may be the gate itself and d_x may be x
 *            (same pointer and strides)
 *   d_h0     device fp32[outer x inner]; NULL: not wanted.  May be d_last itself
 * No other overlap of an output is allowed.  steps == 0: d_h0 is d_last.
 * Asynchronous on `stream`; allocates nothing; one launch.  Errors: as darb_gated_scan.
 */
DARB_API darb_status_t darb_gated_scan_grad(const void *dh, int64_t ld_dh, int64_t step_dh, const void *gate,
                                            int64_t ld_gate, int64_t step_gate, const void *x, int64_t ld_x,
                                            int64_t step_x, const void *h, int64_t ld_h, int64_t step_h,
                                            darb_dtype_t dtype, darb_gates_t gates, int coupled, int64_t outer,
                                            int64_t steps, int64_t inner, const float *h0, const float *d_last,
                                            void *d_gate, int64_t ld_dgate, int64_t step_dgate, void *d_x,
                                            int64_t ld_dx, int64_t step_dx, float *d_h0, cudaStream_t stream);

/* Whether darb_policy_loss takes a ratio for every token or one for every sequence
 * (the exponential of the mean difference of its tokens), and whether every token or
 * every sequence counts the same in the means. */
typedef enum { DARB_PER_TOKEN = 0, DARB_PER_SEQUENCE = 1 } darb_per_t;

/*
 * The clipped policy loss of sequences that a model drew itself, with a KL term and
 * an entropy bonus, and its gradients in the same call.  It takes what
 * darb_token_logprobs gives and leaves what darb_token_logprobs_grad takes.  Of the
 * tokens that count, with r = e^(logprob - old) (or the sequence's), A the sequence's
 * advantage, x = ref - logprob and w = 1 / (tokens) or 1 / (sequences with a token * tokens
 * of the sequence):
 *   policy = -sum w min(r A, clip(r, 1 - clip_low, 1 + clip_high) A)
 *   kl = sum w (e^x - 1 - x),  entropy = sum w H
 *   loss = policy + kl_coef kl - entropy_coef entropy
 *   logprob, old_logprob   device fp32[tokens]
 *   ref_logprob, entropy   device fp32[tokens]; NULL allowed where kl_coef (entropy_coef
 *            and d_entropy) do without
 *   mask     device, a byte a token: 0 does not count; NULL: all count.  What the other
 *            buffers hold at tokens that do not count is not looked at
 *   advantage  device fp32[sequences]
 *   offsets  device int64[sequences + 1]: sequence s has the tokens from offsets[s] up
 *            to offsets[s + 1]; they must not fall, nor be below 0 or above `tokens`
 *            (else results are not defined, but nothing outside the buffers is touched).
 *            Tokens before the first and behind the last sequence do not count
 *   clip_low   0 .. 1 (1: r is not clipped from below); clip_high >= 0 (+inf: not from above)
 *   kl_coef, entropy_coef   finite as 32 bits hold them
 *   stats    device fp32[5]: loss, policy, kl, entropy, and the share of the weight whose
 *            ratio is clipped; terms without their buffers are 0
 *   d_logprob, d_entropy   device fp32[tokens]: the gradients of the loss; d_entropy NULL: not
 *            wanted.  0 at masked tokens; of tokens outside of all sequences left as it was
 *   work     device scratch of darb_policy_loss_work bytes (16-byte aligned), not to be shared
 *            by calls that may run at the same time; NULL: from the device's memory pool
 * Where nothing counts the stats and gradients are 0.  A border is decided as the exact
 * difference decides it; sums are in a fixed order, over more than 256 tokens in 64 bits.
 * No output may overlap another buffer.  Asynchronous on `stream`; allocates nothing but work;
 * one launch up to 4096 tokens, else three (past 1.6 million, four).
 * Errors: DARB_ERR_INVALID_ARG; DARB_ERR_UNSUPPORTED (more than 2^27 tokens or sequences);
 * DARB_ERR_OOM; DARB_ERR_CUDA.
 */
DARB_API darb_status_t darb_policy_loss(int64_t tokens, int64_t sequences, const float *logprob,
                                        const float *old_logprob, const float *ref_logprob, const float *entropy,
                                        const uint8_t *mask, const float *advantage, const int64_t *offsets,
                                        double clip_low, double clip_high, double kl_coef, double entropy_coef,
                                        darb_per_t ratio, darb_per_t mean, float *stats, float *d_logprob,
                                        float *d_entropy, void *work, cudaStream_t stream);

/* Bytes of scratch that darb_policy_loss needs for so many tokens (0 up to 4096). */
DARB_API darb_status_t darb_policy_loss_work(int64_t tokens, int64_t *bytes);

/* Elements that share a scale where darb_adamw_step holds states in 8 bits. */
#define DARB_ADAMW_BLOCK 256

typedef struct darb_adamw_s *darb_adamw_t;

/*
 * A plan for AdamW steps over n tensors at once (the update of the dense weights
 * between two re-encodes of Sec. 4's prune-retrain loop).  All tensors are dense
 * and the caller's; they have to stay where they are while the plan lives.
 *   numel    host int64[n], 0 allowed
 *   params   host array of n device pointers, fp32, updated by every step
 *   m, v     host arrays of n device pointers, the moments.  m_scale and v_scale
 *            NULL: fp32, m and v.  Otherwise e4m3 codes (one byte an element) of m
 *            and of sqrt(v), with
 *   m_scale, v_scale  host arrays of n device pointers, fp32, one value for every
 *            DARB_ADAMW_BLOCK elements of the tensor (the last block may be
 *            short); an element is code * scale.  Zero codes and scales are zero
 *            moments
 *   copies   host array of n device pointers (NULL entries allowed), bf16: the
 *            updated parameter rounded, e.g. for darb_reencode; NULL: none
 *   gtype    type of the gradients
 * No two of the buffers may overlap.  Allocates the plan's tables on the current
 * device, runs on `stream` and synchronises it.
 * Errors: DARB_ERR_INVALID_ARG; DARB_ERR_UNSUPPORTED (2^31 chunks of 2048
 * elements or more); DARB_ERR_OOM; DARB_ERR_CUDA.
 */
DARB_API darb_status_t darb_adamw_create(int32_t n, const int64_t *numel, float *const *params, void *const *m,
                                         void *const *v, float *const *m_scale, float *const *v_scale,
                                         void *const *copies, darb_dtype_t gtype, darb_adamw_t *out,
                                         cudaStream_t stream);

/*
 * One step: with g' = g * *grad_scale and t = step,
 *   m = beta1 m + (1 - beta1) g',  v = beta2 v + (1 - beta2) g'^2,
 *   p = p (1 - lr weight_decay)
 *       - lr / (1 - beta1^t) * m / (sqrt(v) / sqrt(1 - beta2^t) + eps).
 *   grads    host array of n device pointers of the plan's gradient type; a NULL
 *            entry leaves its tensor and states as they are
 *   grad_scale  device fp32 scalar (what clipping by the norm gives), or NULL: 1
 *   step     t >= 1
 *   seed     of the states' rounding in 8 bits; another one for every step (the
 *            step itself, for instance).  The same inputs and seed give the same
 *            results.  Not used with fp32 states
 * Each operation above is one IEEE fp32 operation; in 8 bits the update uses m
 * and v before they are rounded, and a block's scale is its largest magnitude /
 * 448, the codes rounded up or down at random so that the mean is kept (a root
 * that is not zero keeps a code that is not zero).  A NaN or infinity reaches its
 * own element, and in 8 bits the states of its block.
 * Asynchronous on `stream`; allocates nothing; one launch for every 448 tensors.
 * Steps of one plan must be ordered on one stream.
 * Errors: DARB_ERR_INVALID_ARG (an unknown plan, a step below 1, lr, eps or
 * weight_decay negative or not finite, a beta outside [0, 1), a gradient or
 * grad_scale that overlaps a buffer of any of the plan's tensors); DARB_ERR_CUDA.
 */
DARB_API darb_status_t darb_adamw_step(darb_adamw_t plan, const void *const *grads, const float *grad_scale,
                                       int64_t step, uint64_t seed, double lr, double beta1, double beta2, double eps,
                                       double weight_decay, cudaStream_t stream);

/* Synchronise `stream` and report what the plan's steps recorded since the last
 * call, then clear it: DARB_ERR_TIMEOUT if a bounded device wait for a bulk copy
 * gave up (the tensors are then not all updated), else DARB_OK.                */
DARB_API darb_status_t darb_adamw_sync_status(darb_adamw_t plan, cudaStream_t stream);

/* Release a plan (not its tensors); NULL is a no-op.  Waits for the device.    */
DARB_API darb_status_t darb_adamw_destroy(darb_adamw_t plan);

typedef struct darb_muon_s *darb_muon_t;

/*
 * A plan for updates of n weight matrices whose momentum is orthogonalised by
 * Newton-Schulz products, next to darb_adamw_create (which is left the vectors).  The
 * matrices are dense, row after row, and the caller's; they have to stay where they are
 * while the plan lives.
 *   rows, cols   host int64[n], 0 allowed, 32768 at most
 *   params   host array of n device pointers, fp32[rows x cols], updated by every step
 *   m        host array of n device pointers, fp32, the momentum
 *   copies   host array of n device pointers (NULL entries allowed), bf16: the updated
 *            parameters rounded, e.g. for darb_reencode; NULL: none
 *   gtype    type of the gradients
 * No two of the buffers may overlap.  Allocates tables and scratch on the current device (8
 * bytes an element and 8 bytes for every pair of the shorter side's), runs on `stream` and
 * synchronises it.
 * Errors: DARB_ERR_INVALID_ARG; DARB_ERR_UNSUPPORTED (a longer side); DARB_ERR_OOM;
 * DARB_ERR_CUDA.
 */
DARB_API darb_status_t darb_muon_create(int32_t n, const int64_t *rows, const int64_t *cols, float *const *params,
                                        float *const *m, void *const *copies, darb_dtype_t gtype, darb_muon_t *out,
                                        cudaStream_t stream);

/*
 * One step: with g' = g * *grad_scale and |u| the root of the sum of all squares,
 *   m = beta m + (1 - beta) g',  u = (1 - beta) g' + beta m (nesterov == 0: m),
 *   X = u / (|u| + eps), transposed where there are more rows than columns,
 *   five times  A = X X^T,  X = 3.4445 X + (-4.7750 A + 2.0315 A A) X,
 *   p = p (1 - lr weight_decay) - lr 0.2 sqrt(max(rows, cols)) X.
 *   grads    host array of n device pointers of the plan's gradient type, as dense as the
 *            parameters; a NULL entry leaves its matrix and momentum as they are
 *   grad_scale  device fp32 scalar (what clipping by the norm gives), or NULL: 1
 * The products' operands are fp16 with all sums in fp32, and the diagonals of A and its
 * polynomial are kept in fp32.  With bf16 gradients X is off by about 1e-3 of itself
 * (its norm), with fp32 gradients, whose operands are two fp16 numbers each, by about
 * 1e-5.  A NaN or infinity in a gradient makes its whole matrix NaN; zero gradients
 * and momentum give X = 0.
 * Asynchronous on `stream`; allocates nothing; 17 launches (two more for every further
 * 448 matrices).  Results do not depend on the order of anything.  Steps of one plan must
 * be ordered on one stream.
 * Errors: DARB_ERR_INVALID_ARG (an unknown plan; lr or weight_decay negative; lr, eps or 1 - lr weight_decay
 * not finite in 32 bits; beta outside [0, 1); an eps that is not above 0 in 32 bits; a gradient or grad_scale that overlaps a
 * buffer of any of the plan's matrices); DARB_ERR_CUDA.
 */
DARB_API darb_status_t darb_muon_step(darb_muon_t plan, const void *const *grads, const float *grad_scale, double lr,
                                      double beta, double weight_decay, double eps, int nesterov, cudaStream_t stream);

/* As darb_adamw_sync_status: DARB_ERR_TIMEOUT if a bounded device wait gave up. */
DARB_API darb_status_t darb_muon_sync_status(darb_muon_t plan, cudaStream_t stream);

/* Release a plan (not its matrices); NULL is a no-op.  Waits for the device.   */
DARB_API darb_status_t darb_muon_destroy(darb_muon_t plan);

typedef struct {
    int64_t rows, cols;
    int64_t nnzb;            /* kept weights = blocks = sum_r ceil(cols / m_r)           */
    darb_dtype_t wtype;
    int32_t nbins;           /* distinct block sizes                                     */
    int32_t ngroups;         /* 32-row groups the kernels work on                        */
    int64_t value_bytes;     /* nnzb * sizeof(value): the values the paper stores       */
    int64_t offset_bytes;    /* stored offsets: 4 bits per block if m <= 16, else 8     */
    int64_t meta_bytes;      /* per-row block size and pointer (int32 + uint16)         */
    int64_t index_bits_min;  /* sum over blocks of ceil(log2 m): the paper's index bits */
    int64_t device_bytes;    /* device memory the handle holds (incl. padding, scratch) */
} darb_info_t;

/* Shape and storage accounting of a handle (Sec. 4.2 index-storage analysis). */
DARB_API darb_status_t darb_info(darb_handle_t h, darb_info_t *info);

/*
 * Copy the encoding out in canonical order: blocks in (row, j) order.
 *   val      host, nnzb values of the handle's dtype (fp32 or bf16 bits)
 *   off      host uint8[nnzb], position of the kept weight inside its block
 *   blk_ptr  host int64[rows + 1], first block of each row; blk_ptr[rows] = nnzb
 *   m        host int32[rows], block size of each row
 * Any of the four may be NULL to skip it.  Synchronises the device.
 */
DARB_API darb_status_t darb_export(darb_handle_t h, void *val, uint8_t *off, int64_t *blk_ptr, int32_t *m);

/* Build a handle from canonical host arrays (the inverse of darb_export).
 * off[p] must be < m[r] and j*m[r] + off[p] < cols.  Synchronises `stream`.  */
DARB_API darb_status_t darb_import(const void *val, const uint8_t *off, const int32_t *m,
                          darb_dtype_t wtype, int64_t rows, int64_t cols, darb_handle_t *out,
                          cudaStream_t stream);

/* Whether the library's kernels are launched with programmatic dependent
 * launch (PDL: a kernel may start its prologue, and read the handle's
 * immutable data, while the previous kernel on the stream drains; its reads
 * of X and writes of Y still wait for that kernel).  Process wide, on by
 * default; applies to launches made after the call (a CUDA graph keeps what
 * it captured).  For measuring the overlap; results are the same either way.
 * The paper has no counterpart.  Always DARB_OK.                             */
DARB_API darb_status_t darb_set_pdl(int enabled);

/* Release a handle and all device memory it owns; NULL is a no-op.  Waits for
 * the device to finish using it.                                              */
DARB_API darb_status_t darb_destroy(darb_handle_t h);

/* Static, human-readable name of a status code. */
DARB_API const char *darb_status_string(darb_status_t s);

#ifdef __cplusplus
}
#endif

#endif /* DARB_H */
