/*
 * hc.h -- C ABI of libhc, the GB300 (sm_103a) sparse contact operators of
 * "ECO: Efficient Human-Contact Representation for Human-Scene Interaction".
 *
 * A sparse contact mask over body-mesh vertices selects the rows of a dense
 * human-scene tensor (Eq. 1); the selected rows are decomposed into a
 * coordinate list C' and compact features S' (Eq. 2); sparse layers then run
 * on the compact rows only (Sec. 3.2): convolution over each vertex's spiral
 * neighbourhood (Eqs. 4-5), linear (Eq. 6) and activation (Eq. 10).
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 *  - Every pointer argument is a DEVICE pointer on the current CUDA device,
 *    except where a comment says otherwise. The caller owns every buffer;
 *    nothing is retained after the call returns.
 *  - Work is enqueued on `stream` (NULL = the legacy default stream) and is
 *    asynchronous: the return status reports argument checks and launch
 *    errors only. Problems found on the device (an out-of-range index, a
 *    count above capacity, a bounded wait that ran out) set a sticky device
 *    status word, read and cleared by hc_get_device_status().
 *  - The active-row count N' stays on the device (`count`, one int32), so a
 *    chain of calls needs no host synchronisation and can be captured into a
 *    CUDA graph once the library has set itself up on the device (see
 *    hc_mask_compact).
 *  - Layouts are row-major. dtype HC_F32 means IEEE binary32; HC_BF16 means
 *    bfloat16 storage with fp32 accumulation (tensor cores) and a
 *    round-to-nearest-even store. Bias is always fp32. The input, weight and
 *    output of one call share one dtype.
 *  - Neighbours outside the active set contribute nothing (Eq. 4 keeps only
 *    kernel taps whose coordinate is present in C), which equals the dense
 *    layer on the masked input (Eq. 1) restricted to active rows.
 *  - Sizes are int; B*V and every row count must stay below 2^31.
 */
#ifndef HC_H
#define HC_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct CUstream_st* hc_stream_t; /* same type as cudaStream_t */

typedef enum {
    HC_OK = 0,
    HC_ERR_INVALID_ARG = 1,   /* null pointer, bad size, bad enum, misaligned pointer */
    HC_ERR_UNSUPPORTED = 2,   /* valid but not supported (e.g. L > HC_MAX_SPIRAL) */
    HC_ERR_CAPACITY = 3,      /* device: count exceeded the stated capacity */
    HC_ERR_INVALID_INDEX = 4, /* device: spiral/row_of/coords entry out of range */
    HC_ERR_TIMEOUT = 5,       /* device: a bounded wait inside a kernel ran out */
    HC_ERR_CUDA = 6           /* CUDA runtime error; see hc_last_error_string() */
} hc_status;

typedef enum { HC_F32 = 0, HC_BF16 = 1 } hc_dtype;
typedef enum { HC_ACT_NONE = 0, HC_ACT_ELU = 1, HC_ACT_RELU = 2 } hc_act;
typedef enum {
    HC_LAYOUT_DENSE = 0,  /* [B, V, C]: row (b, v) at (b*V + v)*C */
    HC_LAYOUT_COMPACT = 1 /* [N', C]: row n is the n-th entry of coords */
} hc_layout;

#define HC_MAX_SPIRAL 32 /* largest spiral length L */

/*
 * hc_mask_compact -- decomposition of a masked tensor into coordinates (Eq. 2)
 * and the inverse index map idx() used by the sparse convolution (Eq. 4).
 *
 *   mask     [B, V] uint8. Row (b, v) is active iff mask[b*V + v] != 0
 *            (the paper's mask holds 0/1, Eq. 1; any nonzero byte counts).
 *   coords   [B*V, 2] int32 capacity. Receives the active rows as (b, v)
 *            pairs in ascending (b, v) order: the coordinate matrix C'.
 *   row_of   [B, V] int32, or NULL. Receives the position of (b, v) in
 *            coords, or -1 if inactive.
 *   batch_offsets [B+1] int32, or NULL. Receives the number of active rows
 *            in frames before b; batch_offsets[B] = N'. Rows of frame b are
 *            [batch_offsets[b], batch_offsets[b+1]).
 *   count    one int32: receives N'.
 * B >= 0, V >= 0; B*V == 0 gives N' = 0. Results are bit-exact and unique.
 *
 * Scratch: a small per-(device, stream) workspace (one int32 per 4096 mask
 * bytes) is allocated by the library on the first call that needs it and
 * kept until process exit. Make the first call on each device and stream
 * outside stream capture; later calls allocate nothing unless a larger mask
 * is seen. Calls on one stream are ordered; calls on different streams use
 * different workspaces. All operators share a stream's workspace: a call that
 * needs a larger one synchronises the stream and replaces it. A workspace that
 * was in use during a capture then stays allocated beside the new one, so a
 * graph may be replayed after larger calls on its stream. A graph uses the
 * workspace of the stream it was captured on, wherever it is replayed: replays
 * of such graphs and calls on that stream must not overlap.
 * A call holds its stream's workspace until its last launch: calls of several
 * threads on one stream follow each other whole.
 */
hc_status hc_mask_compact(const uint8_t* mask, int B, int V, int32_t* coords,
                          int32_t* row_of, int32_t* batch_offsets, int32_t* count,
                          hc_stream_t stream);

/*
 * hc_mask_compact_static -- hc_mask_compact that allocates nothing. The paper
 * has no counterpart; this entry point exists for callers of this library
 * that cannot allocate device memory at the moment they compact a mask:
 * processes that hand all device memory to their own pool up front and must
 * not allocate behind its back, and code on a path where a cudaMalloc or
 * cudaFree (which can synchronise the whole device) is not allowed.
 *
 * Same arguments, results and errors as hc_mask_compact (bit-identical
 * outputs). Differences:
 *  - Scratch: a fixed array of HC_STATIC_MAX_MASK_BYTES / 4096 int32 (16 KiB)
 *    inside the library's device image, present on every GPU that loads the
 *    library until the process exits. No cudaMalloc, cudaFree or allocating
 *    library routine is called.
 *  - Limit: B*V may not exceed HC_STATIC_MAX_MASK_BYTES; larger masks are
 *    rejected with HC_ERR_UNSUPPORTED before anything is launched.
 *  - Set-up: the first call on each device looks up the array's device
 *    address (with that device current); make that first call before any
 *    stream capture.
 *  - Sharing: every call on a device uses the same array, which keeps the
 *    previous call's contents (each call rewrites what it reads, so no
 *    clearing is needed). Calls whose kernels overlap on the GPU (e.g. on
 *    two streams without ordering between them) race on it.
 */
#define HC_STATIC_MAX_MASK_BYTES (4096 * 4096)
hc_status hc_mask_compact_static(const uint8_t* mask, int B, int V, int32_t* coords,
                                 int32_t* row_of, int32_t* batch_offsets, int32_t* count,
                                 hc_stream_t stream);

/*
 * hc_sparse_spiral_conv_fwd -- sparse convolution on the spiral
 * neighbourhood (Eqs. 4-5) with fused bias (Eq. 6) and activation (Eq. 10).
 *
 * For each active row n < N' with coordinate (b, v) = coords[n]:
 *   y[n, o] = act( bias[o] + sum_{l<L} sum_{c<C_in}
 *                  S(b, spiral[v*L + l])[c] * W[(l*C_in + c)*C_out + o] )
 * where S(b, u) is the input row of (b, u) when u >= 0 and row_of[b*V+u] >= 0,
 * and the term is absent otherwise. Slot 0 of the spiral is the vertex
 * itself (the centre tap); -1 entries mean "no neighbour".
 *
 *   x        x_layout DENSE: [B, V, C_in]; COMPACT: [N', C_in] in coords order
 *   coords, row_of, count   as written by hc_mask_compact (row_of required)
 *   spiral   [V, L] int32, entries in [-1, V)
 *   W        [L*C_in, C_out] of dtype dt, row index l*C_in + c
 *   bias     [C_out] fp32, or NULL for zero
 *   y        [B*V, C_out] capacity of dtype dt; rows 0..N'-1 are written,
 *            in coords order (the conv outputs the centre coordinates, Eq. 5).
 * 1 <= L <= HC_MAX_SPIRAL, C_in >= 1, C_out >= 1.
 * Out-of-range spiral/row_of/coords entries contribute nothing and set
 * HC_ERR_INVALID_INDEX; a count above B*V is clamped and sets HC_ERR_CAPACITY.
 * bf16 with C_out % 8 == 0 and 16-byte aligned W, y runs on the tensor cores
 * (tcgen05); other shapes run on CUDA cores. With C_in % 8 != 0 (x then
 * needs only 2-byte alignment) x and W are first copied, with zero channels
 * appended up to C_pad = the next multiple of 8, into the per-stream
 * workspace (x_rows * C_pad * 2 + L * C_pad * C_out * 2 bytes; compact inputs
 * copy their first N' rows only); the sums are unchanged. With C_out = 128
 * and B*V of at least 256 rows per SM, the kernel reads N' on the device and
 * multiplies 256-row items (two 128-row halves sharing each weight stage) when
 * every SM gets one, 128-row items otherwise; the results are the same bits
 * either way.
 */
hc_status hc_sparse_spiral_conv_fwd(const void* x, hc_layout x_layout, hc_dtype dt,
                                    const int32_t* coords, const int32_t* row_of,
                                    const int32_t* count, const int32_t* spiral, int B, int V,
                                    int L, int C_in, int C_out, const void* W, const float* bias,
                                    hc_act act, void* y, hc_stream_t stream);

/*
 * hc_conv_rulebook -- the indexing matrix of the sparse convolution (Eq. 4),
 * materialised: for every active row n < N' and spiral slot l < L,
 *   rulebook[l*(B*V) + n] = the input row feeding that tap, or -1 when the
 *   tap is absent (spiral[v*L+l] == -1, or the neighbour (b, u) is inactive).
 * The input row is b*V + u for x_layout DENSE and row_of[b*V + u] for
 * COMPACT. The coordinates do not change from layer to layer (Eq. 5), so one
 * rulebook serves every conv layer run on the same mask.
 *   coords, row_of, count   as written by hc_mask_compact
 *   spiral    [V, L] int32, entries in [-1, V)
 *   rulebook  [L, B*V] int32, slot-major, caller-owned; columns n >= N'
 *             are not written.
 * Out-of-range entries are reported (HC_ERR_INVALID_INDEX) and stored as -1.
 */
hc_status hc_conv_rulebook(const int32_t* coords, const int32_t* row_of, const int32_t* count,
                           const int32_t* spiral, int B, int V, int L, hc_layout x_layout,
                           int32_t* rulebook, hc_stream_t stream);

/*
 * hc_mask_compact_rulebook -- hc_mask_compact followed by hc_conv_rulebook on
 * its output (Eq. 2 and the Eq. 4 indexing matrix), in two kernels when
 * V <= 65535: a count pass, then one pass per (frame, block of 1024
 * vertices) that ranks the frame's mask bytes in shared memory and writes
 * coords, row_of, batch_offsets, count and the rulebook columns of its
 * active vertices, every tap lookup answered from shared memory. Larger
 * frames run the two operations' own kernels. The results are identical to
 * the two calls (bit-exact).
 *   mask, B, V, coords, row_of, batch_offsets, count   as hc_mask_compact
 *                                                      (row_of required)
 *   spiral, L, x_layout, rulebook                      as hc_conv_rulebook
 * Out-of-range spiral entries are reported (HC_ERR_INVALID_INDEX) and their
 * taps stored as -1. Uses the library's per-stream workspace (one int32 per
 * 4096 mask bytes).
 */
hc_status hc_mask_compact_rulebook(const uint8_t* mask, int B, int V, const int32_t* spiral, int L,
                                   hc_layout x_layout, int32_t* coords, int32_t* row_of,
                                   int32_t* batch_offsets, int32_t* count, int32_t* rulebook,
                                   hc_stream_t stream);

/*
 * hc_sparse_conv_rulebook_fwd -- the sparse convolution (Eq. 5) with fused
 * bias (Eq. 6) and activation (Eq. 10), through a precomputed rulebook:
 *   y[n, o] = act( bias[o] + sum_{l<L, r = rulebook[l*capacity+n] >= 0}
 *                  sum_{c<C_in} x[r, c] * W[(l*C_in + c)*C_out + o] ),  n < N'
 *   x         [x_rows, C_in] of dtype dt; rulebook entries must lie in
 *             [-1, x_rows) (others are reported and skipped)
 *   rulebook  [L, capacity] int32 as written by hc_conv_rulebook
 *             (capacity = B*V there)
 *   count     N' on the device, at most capacity (clamped, HC_ERR_CAPACITY)
 *   W, bias, act as for hc_sparse_spiral_conv_fwd.
 *   y         [capacity, C_out] compact output of dtype dt, or NULL.
 *   out       [B, V, C_out] dense output of dtype dt, or NULL: when given, row
 *             n is also written at coords[n] = (b, v), the scatter of
 *             hc_scatter_dense fused into the epilogue (inactive rows of out
 *             are not touched). Needs coords (as written by hc_mask_compact),
 *             B >= 1 and V >= 1. At least one of y and out must be given.
 * Results equal hc_sparse_spiral_conv_fwd (and hc_scatter_dense without
 * zero fill) on the same inputs.
 */
hc_status hc_sparse_conv_rulebook_fwd(const void* x, hc_dtype dt, int x_rows,
                                      const int32_t* rulebook, const int32_t* count, int capacity,
                                      int L, int C_in, int C_out, const void* W, const float* bias,
                                      hc_act act, void* y, const int32_t* coords, int B, int V,
                                      void* out, hc_stream_t stream);

/*
 * hc_sparse_conv_rulebook_fwd_hint -- hc_sparse_conv_rulebook_fwd with the
 * caller's host-side estimate of N' (rows_hint >= 0; 0 = unknown), which
 * the call uses only to choose how the tensor cores tile the rows. The
 * tiling that is fastest for many rows (two 128-row halves per item sharing
 * every weight stage, multiplied as one M = 128 channels x N = 256 rows
 * product) is slower when there are too few items to fill the GPU; it
 * applies to bf16, C_out = 128, and neither out nor group-norm statistics.
 * With rows_hint giving at least one such item per SM (about 39k rows on
 * 152 SMs) the launch uses it directly; with a smaller nonzero estimate it
 * uses one-half items; with none (0, and in hc_sparse_conv_rulebook_fwd)
 * a call whose capacity could fill the SMs with such items launches a
 * kernel that reads N' on the device and chooses (a little slower than a
 * direct launch at small N': ~0.2 us). The results are bit-identical in
 * every case, so any estimate (the previous batch's count, the mask's
 * expected density) is safe: a wrong one only costs time. rows_hint < 0 is
 * HC_ERR_INVALID_ARG.
 */
hc_status hc_sparse_conv_rulebook_fwd_hint(const void* x, hc_dtype dt, int x_rows,
                                           const int32_t* rulebook, const int32_t* count,
                                           int capacity, int L, int C_in, int C_out,
                                           const void* W, const float* bias, hc_act act, void* y,
                                           const int32_t* coords, int B, int V, void* out,
                                           long long rows_hint, hc_stream_t stream);

/*
 * hc_sparse_linear_fwd -- linear layer on compact rows (Eq. 6), row-wise
 *   y[n, o] = act( bias[o] + sum_{c<C_in} x[n, c] * W[c*C_out + o] ),  n < N'
 * The coordinates are unchanged (C' = C).
 *   x [capacity, C_in], y [capacity, C_out], W [C_in, C_out] of dtype dt;
 *   count: one int32 on the device (N'), must not exceed `capacity`
 *   (clamped, HC_ERR_CAPACITY).
 */
hc_status hc_sparse_linear_fwd(const void* x, hc_dtype dt, const int32_t* count, int capacity,
                               int C_in, int C_out, const void* W, const float* bias, hc_act act,
                               void* y, hc_stream_t stream);

/*
 * hc_sparse_group_norm_fwd -- group normalisation of compact rows (Eqs. 7-9),
 * statistics taken over each frame's active rows only. Frame b owns the rows
 * [batch_offsets[b], batch_offsets[b+1]) (as written by hc_mask_compact); the
 * C channels form G groups of C/G consecutive channels. For every (b, g), over
 * the n = rows(b) * C/G values of the group:
 *   mu = sum / n,  var = sum((v - mu)^2) / n,  out = (v - mu) / sqrt(var + eps)
 * then out * gamma[c] + beta[c] (each optional: NULL = 1 / 0) and the
 * activation act (Eq. 10). G = 1 is layer normalisation.
 *   x, y      [capacity, C] of dtype dt; y may be x (in place). Rows outside
 *             every frame's range are not touched.
 *   batch_offsets [B+1] int32 on the device, non-decreasing, within
 *             [0, capacity]; otherwise HC_ERR_INVALID_INDEX is reported
 *             (hc_get_device_status) and the output is unspecified, but no
 *             access leaves x, y or the library's workspace.
 * Statistics in fp32 by pairwise (count, mean, M2) merging; the variance is
 * taken around the mean, never as E[x^2] - mean^2. Uses the library's
 * per-stream workspace ((B + 2 * SMs) * G * 16 bytes at most).
 */
hc_status hc_sparse_group_norm_fwd(const void* x, hc_dtype dt, const int32_t* batch_offsets, int B,
                                   int capacity, int C, int G, float eps, const float* gamma,
                                   const float* beta, hc_act act, void* y, hc_stream_t stream);

/*
 * hc_sparse_conv_gn_fwd -- a convolution layer followed by group
 * normalisation and the activation, the order of a block of the encoder
 * (Eqs. 5-6, then Eqs. 7-9, then Eq. 10):
 *   z = conv(x) + bias            as hc_sparse_conv_rulebook_fwd with act
 *                                 NONE, stored in y (dtype dt)
 *   y = act(GN(z) * gamma + beta) as hc_sparse_group_norm_fwd on y in place
 * The group statistics are those of z as stored (bf16-rounded for bf16).
 *   x, rulebook, count, capacity, L, C_in, C_out, W, bias as for
 *             hc_sparse_conv_rulebook_fwd; y [capacity, C_out] of dtype dt
 *   coords    [capacity, 2] int32 from hc_mask_compact (frame of row n is
 *             coords[2n]), batch_offsets [B+1] from the same call: the frame
 *             table must start at 0, end at *count and agree with coords
 *             (HC_ERR_INVALID_INDEX otherwise, output unspecified)
 *   G, eps, gamma, beta, act as for hc_sparse_group_norm_fwd (G divides C_out)
 * bf16 with C_out/G a power of two from 8 to the tensor-core tile (64
 * channels when C_out <= 64, else 128), C_out/8 a power of two: the
 * tensor-core epilogue writes one partial (count, mean, M2) per (frame,
 * 32-row block inside the frame, group), and one per (row, group) for blocks
 * shared by two frames, and a single normalising pass merges them (two
 * launches, y written once by each). Otherwise the two operations run one
 * after the other. Uses the library's per-stream workspace
 * ((B + capacity/32 + 1) * G * 16 + capacity * G * 8 bytes, or that of
 * hc_sparse_group_norm_fwd).
 */
hc_status hc_sparse_conv_gn_fwd(const void* x, hc_dtype dt, int x_rows, const int32_t* rulebook,
                                const int32_t* count, int capacity, int L, int C_in, int C_out,
                                const void* W, const float* bias, const int32_t* coords,
                                const int32_t* batch_offsets, int B, int G, float eps,
                                const float* gamma, const float* beta, hc_act act, void* y,
                                hc_stream_t stream);

/*
 * hc_conv_rulebook_transpose -- the Eq. 4 mapping read backwards, for the
 * input gradient: for every input row j, the taps (n, l) with
 * rulebook[l][n] == j, n < *count, as keys n*L + l in ascending order.
 *   rulebook  [L, capacity] from hc_conv_rulebook (capacity = its stride)
 *   row_ptr   [x_rows + 1] int32: row j's keys are taps[row_ptr[j] ..
 *             row_ptr[j+1])
 *   taps      [L * capacity] int32
 * Entries outside [-1, x_rows) are skipped and reported
 * (HC_ERR_INVALID_INDEX). Computed once per mask and reused by every layer.
 * Uses the library's per-stream workspace (2 int32 per input row).
 */
hc_status hc_conv_rulebook_transpose(const int32_t* rulebook, const int32_t* count, int capacity,
                                     int L, int x_rows, int32_t* row_ptr, int32_t* taps,
                                     hc_stream_t stream);

/*
 * hc_sparse_conv_rulebook_bwd -- gradients of the sparse spiral convolution
 * computed by hc_sparse_conv_rulebook_fwd. The paper gives the forward only
 * (Eqs. 4-5, 6, 10); these follow from it by the chain rule:
 *   dz[n][o]  = dy[n][o] * act'(y[n][o])   (ELU: 1 if y > 0 else y + 1;
 *                                           ReLU: 1 if y > 0 else 0)
 *   dbias[o]  = sum_n dz[n][o]
 *   dW[l*C_in + c][o] = sum_n x[j(n,l)][c] * dz[n][o]
 *   dx[j][c]  = sum over taps (n, l) reading row j of sum_o dz[n][o] W[l*C_in + c][o]
 * over output rows n < *count, with j(n,l) = rulebook[l][n] (absent taps -1
 * contribute nothing).
 *   x        [x_rows, C_in] input rows the forward read (dense B*V rows or
 *            compact), dtype dt; needed for dW
 *   y, dy    [capacity, C_out] forward output and upstream gradient, dt
 *   W        [L*C_in, C_out], dt; needed for dx
 *   row_ptr, taps  from hc_conv_rulebook_transpose; needed for dx
 *   dx       [x_rows, C_in], dt, every row written (0 where no tap reads
 *            it), or NULL
 *   dW       [L*C_in, C_out] fp32 or NULL;  dbias [C_out] fp32 or NULL
 * bf16: dW on tensor cores (tcgen05, fp32 accumulation); dz and the
 * per-tap products dz W^T are rounded to bf16 once before the input-gradient
 * sums. fp32: CUDA cores throughout. Every sum runs in a fixed order
 * (deterministic). Uses the library's per-stream workspace.
 */
hc_status hc_sparse_conv_rulebook_bwd(const void* x, hc_dtype dt, int x_rows,
                                      const int32_t* rulebook, const int32_t* count, int capacity,
                                      int L, int C_in, int C_out, const void* W, const void* y,
                                      const void* dy, hc_act act, const int32_t* row_ptr,
                                      const int32_t* taps, void* dx, float* dW, float* dbias,
                                      hc_stream_t stream);

/*
 * hc_mask_score_update -- the mask-score update of Eq. 3 (Sec. 3.1, Sparse
 * Mask Selection). O holds the outputs of K masks, [K, N, D] row-major (mask
 * k's N rows of D features). With S[i][k] = || O_i^T O_k ||_F^2:
 *   sim[i][k]    = S[i][k] / (|| O_k^T O_k ||_F * || O_i^T O_i ||_F)
 *   alpha_out[k] = alpha_in[k] + 1/(K-1) * sum over i != k of (1 - sim[i][k])
 * Readings: a mask whose output is all zero has similarity 0 to every mask;
 * with K = 1 alpha is copied unchanged.
 *   O          [K, N, D] of dtype dt (bf16: tensor cores, fp32 accumulation;
 *              fp32: CUDA cores, fp32 accumulation)
 *   alpha_in, alpha_out  [K] fp32 on the device; may be the same buffer
 *   sim        [K, K] fp32 or NULL
 * K*D at most HC_MASK_SCORE_MAX_FEATURES (else HC_ERR_UNSUPPORTED). Uses the
 * library's per-stream workspace: 64 KiB per work item (upper-triangle
 * 128 x 128 tiles of the [K*D]^2 Gram matrix times row splits, about the
 * SM count), plus N * K*D (rounded to 128) bf16 when D is not a multiple of 8.
 */
#define HC_MASK_SCORE_MAX_FEATURES 8192
hc_status hc_mask_score_update(const void* O, hc_dtype dt, int K, int N, int D,
                               const float* alpha_in, float* alpha_out, float* sim,
                               hc_stream_t stream);

/*
 * hc_mask_select_topk -- the kappa masks kept at inference (Sec. 3.1, Sparse
 * Mask Selection): indices of the kappa highest scores of alpha [K] (fp32,
 * device), highest first; equal scores lowest index first; a NaN score ranks
 * below every number. selected: [kappa] int32 on the device.
 * K at most HC_TOPK_MAX_MASKS.
 */
#define HC_TOPK_MAX_MASKS 32768
hc_status hc_mask_select_topk(const float* alpha, int K, int kappa, int32_t* selected,
                              hc_stream_t stream);

/*
 * hc_kappa_masks -- every kept mask applied to every sample (Eq. 1 per kept
 * mask, Sec. 3.1): out [B*kappa, V] with frame b*kappa + j equal to
 * masks[selected[j]] ([K, V] uint8). The result feeds hc_mask_compact; a
 * selected index outside [0, K) gives an all-zero frame and
 * HC_ERR_INVALID_INDEX.
 */
hc_status hc_kappa_masks(const uint8_t* masks, int K, int V, const int32_t* selected, int kappa,
                         int B, uint8_t* out, hc_stream_t stream);

/*
 * hc_gather_rows -- the feature matrix S' of Eq. 2: y[n] = x[f / fps, v] for
 * the n-th active coordinate (f, v) = coords[n], n < *count, where x is the
 * dense [B_in, V, C] input of dtype dt and fps = frames_per_sample (kappa
 * after hc_kappa_masks, else 1). Rows are copied bit for bit; y is
 * [capacity, C]. A coordinate outside the input is reported
 * (HC_ERR_INVALID_INDEX) and its row left untouched; *count above capacity
 * is clamped (HC_ERR_CAPACITY). x may be pinned host memory (cudaHostAlloc,
 * the same pointer on the device under unified addressing): the kernel then
 * reads only the active rows across the host link (zero-copy), which is how
 * a dense host-side input becomes compact device rows without copying the
 * whole tensor.
 * coords may be NULL: y[n] = row n of x (x viewed as B_in * V rows of C;
 * frames_per_sample unused) for n < *count, rows n >= B_in * V reported
 * (HC_ERR_INVALID_INDEX) and left untouched: a copy of the first N' rows
 * sized on the device. With y in pinned host memory this reads compact
 * results back without the host learning N' first (no host wait between
 * the producing call and the copy).
 */
hc_status hc_gather_rows(const void* x, hc_dtype dt, int B_in, int V, int C, const int32_t* coords,
                         const int32_t* count, int capacity, int frames_per_sample, void* y,
                         hc_stream_t stream);

/*
 * hc_scatter_dense -- inverse of the decomposition (Eq. 2): compact rows back
 * into a dense [B, V, C] tensor.
 *   zero_fill == 0: out[coords[n]] = y[n] for n < N'; other rows untouched.
 *   zero_fill != 0: every row of out is written: y[n] at coords[n], zeros
 *                   elsewhere (the masked tensor of Eq. 1).
 *   y [N', C] of dtype dt (elements are copied bit for bit), coords/count as
 *   written by hc_mask_compact, out [B, V, C].
 *   row_of   [B, V] as written by hc_mask_compact, or NULL. Optional: with
 *            zero_fill it lets one pass write every dense row exactly once
 *            (coords may then be NULL); without it the zero fill is a
 *            separate pass over out before the scatter. Ignored when
 *            zero_fill == 0. (The problem statement's call has no row_of;
 *            passing NULL gives exactly that call.)
 */
hc_status hc_scatter_dense(const void* y, hc_dtype dt, const int32_t* coords,
                           const int32_t* row_of, const int32_t* count, int B, int V, int C,
                           int zero_fill, void* out, hc_stream_t stream);

/*
 * hc_spiral_conv_fwd -- the dense spiral-conv layer the sparse one replaces
 * (Sec. 3.2), used as the speed-up denominator: every (b, v) is an output row,
 *   y[(b*V+v), o] = act( bias[o] + sum_l sum_c x[b, spiral[v*L+l], c] *
 *                                            W[(l*C_in + c)*C_out + o] )
 * with -1 spiral entries skipped. x [B, V, C_in], y [B, V, C_out].
 */
hc_status hc_spiral_conv_fwd(const void* x, hc_dtype dt, const int32_t* spiral, int B, int V,
                             int L, int C_in, int C_out, const void* W, const float* bias,
                             hc_act act, void* y, hc_stream_t stream);

/*
 * Token operators
 * ---------------
 * A token is a row of a compact [capacity, C] matrix; the operators below are
 * the parts of a network over such rows (row embedding, layer norm,
 * root-mean-square norm with the residual's addition, the 8-bit form of the
 * linear layer) and their gradients. The paper has no counterpart.
 * In all of them `count` is N' on the device (clamped to [0, capacity],
 * HC_ERR_CAPACITY / HC_ERR_INVALID_INDEX reported when it was outside) or
 * NULL, which means all `capacity` rows; rows n >= N' are not written, and
 * what they hold has no effect (the 8-bit product copies whole tiles: it reads
 * up to 127 of them). Pointers need the alignment of their element type; rows that are
 * 16-byte aligned (pointer and row size) move in 16-byte pieces. Rows of more
 * than 2^31 - 8193 channels are refused (HC_ERR_INVALID_ARG), and so is a weight
 * of more than 65535 * 128 output channels (HC_ERR_UNSUPPORTED). Sums are
 * taken in fp32 and in a fixed order: results are the same from run to run.
 */

/*
 * hc_layer_norm_fwd -- layer norm of every row over its own C channels (the
 * per-frame norm is hc_sparse_group_norm_fwd):
 *   mean = sum x / C,  rstd = 1 / sqrt(sum (x - mean)^2 / C + eps)
 *   y[n][c] = (x[n][c] - mean) * rstd * gamma[c] + beta[c],  n < N'
 *   x, y      [capacity, C] of dtype dt; y may be x (in place)
 *   gamma, beta  [C] fp32, or NULL (1 / 0)
 *   mean, rstd   [capacity] fp32, or NULL: what hc_layer_norm_bwd reads
 * C >= 1, eps >= 0. A row of one value (C = 1 too) has that value as its mean
 * and y = beta exactly, whatever its size; with eps = 0 the row is NaN.
 */
hc_status hc_layer_norm_fwd(const void* x, hc_dtype dt, const int32_t* count, int capacity, int C,
                            float eps, const float* gamma, const float* beta, void* y, float* mean,
                            float* rstd, hc_stream_t stream);

/*
 * hc_layer_norm_bwd -- its gradient. With xh = (x - mean) * rstd and
 * g = dy * gamma, over rows n < N':
 *   dx[n][c]  = rstd * (g - (sum_c g) / C - xh * (sum_c g * xh) / C)
 *   dgamma[c] = sum_n dy * xh,  dbeta[c] = sum_n dy   (0 when N' = 0)
 *   x, dy     [capacity, C] of dtype dt; mean, rstd as the forward wrote them
 *   dx        [capacity, C] of dtype dt, or NULL; may be x or dy (in place)
 *   dgamma, dbeta  [C] fp32, or NULL each; at least one output is required
 * Uses the library's per-stream workspace (channel sums of 8 * C bytes for
 * each of at most three blocks per SM; rows of more than 8192 channels: 8 bytes
 * per row besides).
 */
hc_status hc_layer_norm_bwd(const void* x, const void* dy, hc_dtype dt, const int32_t* count,
                            int capacity, int C, const float* gamma, const float* mean,
                            const float* rstd, void* dx, float* dgamma, float* dbeta,
                            hc_stream_t stream);

/*
 * hc_rms_norm_fwd -- the residual's addition and the root-mean-square norm of
 * the sum, in the rows' type and/or in 8 bits for hc_fp8_linear_fwd:
 *   h = x + res, rounded to dt (h = x where res is NULL)
 *   rstd = 1 / sqrt(sum h^2 / C + eps)
 *   v = h * rstd * gamma;  y = v rounded to dt;  q, scales = the 8-bit form of
 *   v (as hc_quantize_fp8_rows makes it of fp32 rows),  n < N'
 *   x, res    [capacity, C] of dtype dt; res may be NULL
 *   gamma     [C] fp32, or NULL (1)
 *   h         [capacity, C] of dtype dt, or NULL: the residual stream after
 *             this layer, and what hc_rms_norm_bwd reads; may be x or res
 *   y         [capacity, C] of dtype dt, or NULL; may be x or res (h may not
 *             be the same one)
 *   rstd      [capacity] fp32, or NULL: for hc_rms_norm_bwd
 *   q         [capacity, HC_FP8_PITCH(C)], 16-byte aligned, and scales
 *             [ceil(C / 128), capacity] fp32, or both NULL
 * One of y and q is required. C >= 1, eps >= 0. Rows whose squares would pass
 * the range of fp32 are summed with their values scaled by a power of two. A
 * row of zeros gives zeros. With eps = 0 it is NaN, and a row whose root mean
 * square is below 2^-128 has an infinite rstd, outputs and gradients that are
 * infinite or NaN.
 */
hc_status hc_rms_norm_fwd(const void* x, const void* res, hc_dtype dt, const int32_t* count,
                          int capacity, int C, float eps, const float* gamma, void* h, void* y,
                          float* rstd, uint8_t* q, float* scales, hc_stream_t stream);

/*
 * hc_rms_norm_bwd -- its gradient. With hh = h * rstd and g = dy * gamma, over
 * rows n < N':
 *   dx[n][c]  = dres[n][c] + rstd * (g - hh * (sum_c g * hh) / C)
 *   dgamma[c] = sum_n dy * hh   (0 when N' = 0)
 * dx is the gradient of x and of res alike.
 *   h, dy     [capacity, C] of dtype dt; rstd as the forward wrote it
 *   dres      [capacity, C] of dtype dt: the gradient that reaches h on the
 *             residual stream, or NULL (0)
 *   dx        [capacity, C] of dtype dt, or NULL; may be h, dy or dres
 *   dgamma    [C] fp32, or NULL; at least one output is required
 * Uses the library's per-stream workspace (channel sums of 4 * C bytes for
 * each of at most four blocks per SM; rows of more than 8192 channels: 4 bytes
 * per row besides).
 */
hc_status hc_rms_norm_bwd(const void* h, const void* dy, const void* dres, hc_dtype dt,
                          const int32_t* count, int capacity, int C, const float* gamma,
                          const float* rstd, void* dx, float* dgamma, hc_stream_t stream);

/*
 * hc_embedding_fwd -- a table row for every token:
 *   y[n] = scale * table[ids[n * ids_stride]],  n < N'; zero for the id -1
 * (padding). Any other id outside [0, V) is reported (HC_ERR_INVALID_INDEX)
 * and treated as -1.
 *   table     [V, C] of dtype dt;  y [capacity, C] of dtype dt, rounded once
 *   ids       int32, ids_stride >= 1 elements apart: 1 for a list of ids, 2
 *             with ids = coords + 1 for the vertex of every active row of
 *             hc_mask_compact (a learned vector per vertex)
 */
hc_status hc_embedding_fwd(const void* table, hc_dtype dt, int V, int C, const int32_t* ids,
                           int ids_stride, const int32_t* count, int capacity, float scale,
                           void* y, hc_stream_t stream);

/*
 * hc_embedding_sort -- the token positions in ascending order of their id,
 * equal ids in ascending order of position:
 *   row_ptr   [V + 1] int32: the tokens of table row v are
 *             order[row_ptr[v]] .. order[row_ptr[v + 1] - 1]
 *   order     [capacity] int32, a permutation of the positions; entries from
 *             row_ptr[V] on (padding, ids out of range, then n >= N') belong
 *             to no row
 * Computed once per batch and reused by every table indexed with these ids.
 * Ids out of range other than -1 are reported (HC_ERR_INVALID_INDEX). The
 * result is unique (bit-exact). Uses the library's per-stream workspace (16
 * bytes per token and 512 KiB).
 */
hc_status hc_embedding_sort(const int32_t* ids, int ids_stride, const int32_t* count, int capacity,
                            int V, int32_t* row_ptr, int32_t* order, hc_stream_t stream);

/*
 * hc_embedding_bwd -- the table's gradient:
 *   dtable[v][c] = scale * sum of dy[order[i]][c], row_ptr[v] <= i < row_ptr[v + 1]
 * every row written (0 where no token reads it).
 *   dy        [capacity, C] of dtype dt;  dtable [V, C] fp32
 *   row_ptr, order  from hc_embedding_sort (same capacity). A range of row_ptr
 *             that is not inside [0, capacity], or an entry of order that is
 *             not below capacity, is reported (HC_ERR_INVALID_INDEX) and
 *             skipped; with a row_ptr that decreases, other rows that have more
 *             than 64 tokens, or share them with up to 15 neighbours in a
 *             large table, are unspecified. No access leaves the buffers.
 * A row of more than 64 tokens is cut into pieces summed by blocks of their
 * own and joined in order. Uses the library's per-stream workspace (8 * C
 * + 4 bytes for each 64 tokens, at most for eight pieces per SM).
 */
hc_status hc_embedding_bwd(const void* dy, hc_dtype dt, const int32_t* row_ptr,
                           const int32_t* order, int capacity, int V, int C, float scale,
                           float* dtable, hc_stream_t stream);

/*
 * The 8-bit form of a matrix: e4m3 values in rows of HC_FP8_PITCH(C) bytes
 * (C rounded up to 16, the bytes beyond C zero) and one fp32 scale per block
 * of HC_FP8_BLOCK channels; a value is q * scale.
 */
#define HC_FP8_BLOCK 128
#define HC_FP8_PITCH(C) (((C) + 15) / 16 * 16)

/*
 * hc_quantize_fp8_rows -- rows into the 8-bit form, a scale per row and block:
 *   scale = max(amax / 448, 2^-126),  q = e4m3(x / scale)
 * with amax the largest magnitude of the block's channels, both quotients in
 * fp32 and each rounding to nearest even. A block that holds a NaN or an
 * infinity gets a scale that is not finite, so that every product of that row
 * is NaN.
 *   x         [capacity, C] of dtype dt
 *   q         [capacity, HC_FP8_PITCH(C)], 16-byte aligned
 *   scales    [ceil(C / 128), capacity] fp32 (block-major)
 */
hc_status hc_quantize_fp8_rows(const void* x, hc_dtype dt, const int32_t* count, int capacity,
                               int C, uint8_t* q, float* scales, hc_stream_t stream);

/*
 * hc_quantize_fp8_weight -- a layer weight W [C_in, C_out] of dtype dt into
 * the 8-bit form that hc_fp8_linear_fwd reads, a scale per 128 x 128 block:
 *   wq        [C_out, HC_FP8_PITCH(C_in)], 16-byte aligned (W transposed)
 *   ws        [ceil(C_out / 128), ceil(C_in / 128)] fp32
 * Done once per weight. For the input gradient of the layer, quantise W's
 * transpose: the layer's input gradient is the same product with it.
 */
hc_status hc_quantize_fp8_weight(const void* W, hc_dtype dt, int C_in, int C_out, uint8_t* wq,
                                 float* ws, hc_stream_t stream);

/*
 * hc_fp8_linear_fwd -- hc_sparse_linear_fwd with both operands in 8 bits:
 *   y[n][o] = act( bias[o] + sum_b xs[b][n] * ws[o / 128][b] *
 *                  sum_{c in block b} xq[n][c] * wq[o][c] ),  n < N'
 *   xq, xs    as hc_quantize_fp8_rows wrote them (same capacity and C_in)
 *   wq, ws    as hc_quantize_fp8_weight wrote them
 *   bias      [C_out] fp32, or NULL for zero
 *   y         [capacity, C_out] of dtype y_dt
 * A NaN stays one behind either activation. Sums in fp32: a block's products
 * are added in the tensor cores' accumulators, the scaled block sums in
 * registers.
 */
hc_status hc_fp8_linear_fwd(const uint8_t* xq, const float* xs, const int32_t* count, int capacity,
                            int C_in, int C_out, const uint8_t* wq, const float* ws,
                            const float* bias, hc_act act, hc_dtype y_dt, void* y,
                            hc_stream_t stream);

/*
 * hc_linear_cross_entropy_fwd -- softmax cross entropy of the logits of a
 * linear layer, which are never kept. For n < N' with targets[n] >= 0:
 *   l[v] = sum_c x[n][c] * W[v][c] + bias[v]
 *   lse[n] = log sum_v exp(l[v]),  loss[n] = lse[n] - l[targets[n]]
 * A token with the target -1 takes no part: its loss and lse are 0. Any other
 * target outside [0, V) is reported (HC_ERR_INVALID_INDEX) and treated as -1.
 *   x         [capacity, C] of dtype dt
 *   W         [V, C] of dtype dt: a row per class, as an embedding table has
 *             (the same table may serve both)
 *   bias      [V] fp32, or NULL (0); -infinity excludes a class, whose row of W
 *             has to be finite all the same (a token whose classes are all
 *             excluded has the loss NaN)
 *   targets   [capacity] int32
 *   loss, lse [capacity] fp32, or NULL each; at least one is required. lse is
 *             what hc_linear_cross_entropy_bwd reads
 * fp32 operands keep fp32's precision: each is split into three bf16 numbers,
 * and the products that matter are summed (one with an infinity is NaN). Up to four rows, up to eight where
 * they or W are short, and few classes of few channels are summed in plain fp32.
 * Uses the library's per-stream workspace: with planes = 1 (bf16) or 3 (fp32),
 * 2 * planes * C + 16 bytes a row of the capacity (rounded up to 256 rows), 8
 * bytes a row and 64 classes, and 2 * planes * C bytes a class for fp32 and for
 * rows of W that are not 16-byte aligned; in plain fp32 less than a megabyte.
 */
hc_status hc_linear_cross_entropy_fwd(const void* x, const void* W, hc_dtype dt, const float* bias,
                                      const int32_t* targets, const int32_t* count, int capacity,
                                      int C, int V, float* loss, float* lse, hc_stream_t stream);

/*
 * hc_linear_cross_entropy_bwd -- its gradients. With
 *   G[n][v] = dloss[n] * (exp(l[v] - lse[n]) - (v == targets[n]))
 * for the tokens that take part, 0 for the others:
 *   dx[n][c] = sum_v G[n][v] * W[v][c]          (n < N')
 *   dW[v][c] = sum_n G[n][v] * x[n][c],  dbias[v] = sum_n G[n][v]
 * Every row of dW and dbias is written (0 where no token takes part).
 *   lse       [capacity] fp32, as the forward wrote it
 *   dloss     [capacity] fp32: the gradient of each token's loss (1 / tokens for
 *             their mean); not read where the target is -1
 *   dx        [capacity, C] of dtype dt, or NULL; may be x
 *   dW        [V, C] of dtype dt, or NULL; may not overlap W
 *   dbias     [V] fp32, or NULL; at least one output is required
 * G is held in bf16 for bf16 operands (a rounding of 2^-8 at most), in three bf16
 * numbers for fp32, in fp32 where the forward is plain fp32. Sums are in fp32; those
 * of bf16 operands stay in one accumulator of the tensor cores, which cuts off 2^-25
 * or so of a sum for every 16 terms (tokens for dW, classes of a piece for dx).
 * The workspace follows the capacity, not N': besides the forward's rows and W,
 * the vocabulary is taken in pieces whose G, 2 * planes bytes a row and class, takes
 * at most 512 MiB (but 2048 classes at least: 4.1 GB for 335200 rows of fp32); the
 * sums of dx take 4 * C bytes a row of the capacity and 30 MB, those of dW 20 MB,
 * those of dbias 4 bytes for 32 rows and a class of a piece (34 MB while G is
 * within 512 MiB). In plain fp32 all of it is at most 15 MB.
 */
hc_status hc_linear_cross_entropy_bwd(const void* x, const void* W, hc_dtype dt, const float* bias,
                                      const int32_t* targets, const float* lse, const float* dloss,
                                      const int32_t* count, int capacity, int C, int V, void* dx,
                                      void* dW, float* dbias, hc_stream_t stream);

/*
 * A list of tensors of any sizes and either type, gone over as one: a table in
 * device memory, made once for tensors that stay where they are.
 * hc_tensor_list_fill writes the table of n tensors, hc_tensor_list_bytes(n)
 * bytes, to host memory and fills in *list for the copy of it that the caller
 * then makes at device_table (both 8-byte aligned); the copy has to be there
 * before the first call with the list, and to stay. No GPU call is made.
 *   in, out   n device addresses each, aligned to their element type; out NULL:
 *             in place. No output may overlap another output or another
 *             tensor's input (HC_ERR_INVALID_ARG), or its own unless it is it
 *   numel     elements of each, 0 allowed;  dt  an hc_dtype each
 */
typedef struct hc_tensor_list {
    const void* table; /* the device copy */
    long long units;
    int tensors;
} hc_tensor_list;
size_t hc_tensor_list_bytes(int n);
hc_status hc_tensor_list_fill(const void* const* in, void* const* out, const long long* numel,
                              const int* dt, int n, void* host_table, const void* device_table,
                              hc_tensor_list* list);

/*
 * hc_grad_norm -- the norm over all inputs of a list:
 *   norm = sqrt(sum over all tensors of in^2)      (one fp32; 0 for no elements)
 * Sums of more than 32 squares are taken in more than fp32 and in a fixed
 * order; squares and sums above the range of fp32 are taken in 64 bits, what is
 * smaller than 2^-75 counts as 0. Uses the library's per-stream workspace (8 bytes
 * for each of at most 32 blocks per SM).
 */
hc_status hc_grad_norm(const hc_tensor_list* list, float* norm, hc_stream_t stream);

/*
 * hc_grad_clip -- the list's inputs scaled so that their norm is at most
 * max_norm, rounded once:
 *   out = in * (norm <= max_norm ? 1 : max_norm / norm)
 * norm is read on the device: hc_grad_norm's, or one that a caller has combined
 * from several. An infinite norm gives 0 (NaN where in is infinite), a NaN fills
 * all outputs. Tensors in place whose norm is not above max_norm are not touched.
 * norm may not lie in one of the list's tensors.
 */
hc_status hc_grad_clip(const hc_tensor_list* list, const float* norm, float max_norm,
                       hc_stream_t stream);

/*
 * hc_get_device_status -- synchronises `stream`, then reads and clears the
 * current device's sticky status word. Returns HC_OK if no kernel reported a
 * problem since the last read, else the lowest-numbered device error seen
 * (HC_ERR_CAPACITY, HC_ERR_INVALID_INDEX or HC_ERR_TIMEOUT), or HC_ERR_CUDA
 * if the synchronisation itself failed.
 */
hc_status hc_get_device_status(hc_stream_t stream);

/*
 * hc_test_set_option -- hooks for this library's own tests; the paper has no
 * counterpart and the operators never need them. They reach code paths that
 * ordinary inputs do not select. Settings stay until changed.
 *   HC_TEST_GROUP_NORM_PATH (process-wide): 0 = the library's own choice
 *       (default); 1 = always the per-(frame, group) kernel; 2 = the
 *       row-range kernels wherever the layout allows them.
 *   HC_TEST_WAIT_LIMIT_NS (current device): how long the pipelined kernels
 *       (tensor-core conv, mask score, weight gradient) wait on any one
 *       pipeline barrier before they give up, report HC_ERR_TIMEOUT and
 *       unwind. value > 0 sets it in nanoseconds; 0 restores the default
 *       (2 s). The unwind's own waits, for copies and MMAs already issued,
 *       always keep the default. A lowered limit makes ordinary calls fail
 *       with HC_ERR_TIMEOUT and unspecified outputs: it exists to test that
 *       path. Synchronous (a small host-to-device copy).
 * Returns HC_ERR_INVALID_ARG for an unknown option or a value out of range.
 */
typedef enum { HC_TEST_GROUP_NORM_PATH = 1, HC_TEST_WAIT_LIMIT_NS = 2 } hc_test_option;
hc_status hc_test_set_option(int option, long long value);

/* Text of the last host-side error on the calling thread ("" if none). */
const char* hc_last_error_string(void);

/* Library version, "major.minor.patch". */
const char* hc_version(void);

#ifdef __cplusplus
}
#endif

#endif /* HC_H */
