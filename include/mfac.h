/*
 * mfac.h - C ABI of the MI355X M-FAC IHVP library (gfx950, HIP).
 *
 * Matrix-free inverse-Hessian-vector products under the damped empirical
 * Fisher of a window of m gradients g_1..g_m in R^d (Frantar, Kurtic, Alistarh,
 * "M-FAC: Efficient Matrix-Free Approximations of Second-Order Information"):
 *
 *     F = lambda * I_d + (1/m) * sum_i g_i g_i^T            (Theorem 1)
 *
 * Two families of calls:
 *   - the dynamic sliding window (Section 3.2; optimizer of Section 4.2):
 *     replace one gradient, refresh the Gram row, recompute the m x m
 *     coefficients, and return F^-1 applied to the new gradient (and to up to
 *     max_queries extra vectors in the same two passes over the window);
 *   - the static block-wise precompute (Section 3.1, block-wise paragraph;
 *     Appendix C) with the inverse-diagonal query and the OBD keep-mask
 *     (Section 4.1).
 *
 * Conventions for every call:
 *   - Pointers are HIP device pointers unless marked (host).
 *   - Vectors of length d are fp32 and contiguous; a batch of n vectors is n
 *     rows of length d with row stride d (row-major). The window calls accept
 *     4-byte aligned vectors and take 128-bit accesses when every vector is
 *     16-byte aligned (and d % 4 == 0 for batches); the static calls state
 *     their own alignment below.
 *   - The library never allocates or frees device memory. Window storage,
 *     workspaces and outputs are owned by the caller and must outlive the
 *     handle (storage/workspace) or the call's stream work (inputs/outputs).
 *   - Calls only enqueue work on the handle's stream and return at once; the
 *     *_status calls and mfac_window_get_rows synchronise that stream.
 *   - Argument errors are detected on the host before anything is enqueued:
 *     the call returns MFAC_EINVAL or MFAC_EWORKSPACE and the handle is
 *     unchanged. A failed HIP launch returns MFAC_EHIP. A non-finite or
 *     non-positive pivot met on the device latches an error word in the
 *     workspace, reported as MFAC_ENONFINITE by the next *_status call.
 *   - A handle is used by one host thread and one stream at a time.
 *   - Calls are not meant for stream capture into HIP graphs: the ring head,
 *     the step count and the refactor counter advance on the host when a call
 *     is made, so a replayed graph would repeat the captured slot and policy.
 */
#ifndef MFAC_H
#define MFAC_H

#include <stddef.h>
#include <stdint.h>
#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    MFAC_OK = 0,
    MFAC_EINVAL = -1,      /* invalid argument (null pointer, size, range, alignment) */
    MFAC_EWORKSPACE = -2,  /* storage or workspace smaller than the *_bytes query   */
    MFAC_EHIP = -3,        /* a HIP runtime call or kernel launch failed              */
    MFAC_ENONFINITE = -4,  /* non-finite data or non-positive pivot seen on device    */
    MFAC_ESTATE = -5,      /* call not valid in the handle's current state            */
    MFAC_EPRECISION = -6,  /* fast static mode: the keep-mask could not be certified   */
    /* not a status: widens the enum to the full int32 range, so any code a C
       caller passes (e.g. to mfac_status_string) is a valid value of the type */
    MFAC_STATUS_INT32_ = 0x7fffffff
} mfac_status;

typedef struct mfac_window_s* mfac_window;
typedef struct mfac_static_s* mfac_static;

/* Text for a status code (static storage, never NULL). */
const char* mfac_status_string(mfac_status s);

/* Library version as MAJOR*10000 + MINOR*100 + PATCH. */
int32_t mfac_version(void);

/* ======================================================================
 * Dynamic sliding window (Section 3.2; Appendix B; Section 4.2)
 * ====================================================================== */

/* Bytes of window storage for an m x d window. The storage holds the m
 * gradients in a library-chosen layout (column slabs of the window, each slab
 * m rows x a fixed width, zero padded past d); read rows back with
 * mfac_window_get_rows. Returns 0 for d < 1 or m < 1. */
size_t mfac_window_storage_bytes(int64_t d, int32_t m);

/* Bytes of device workspace for the window (Gram matrix and coefficient
 * factor in fp64, per-call partial sums, error word). max_queries bounds the
 * n of mfac_window_replace (n extra queries) and mfac_ihvp. Returns 0 on
 * invalid sizes. */
size_t mfac_window_workspace_bytes(int64_t d, int32_t m, int32_t max_queries);

/* Create a window handle.
 *   1 <= d <= 2^34, m >= 1, lambda > 0 finite (kept in fp64: the
 *   coefficient phase runs in fp64), 0 <= max_queries <= 16,
 *   m * (max_queries + 1) <= 16384.
 *   storage:   >= mfac_window_storage_bytes(d, m), 256-byte aligned.
 *   workspace: >= mfac_window_workspace_bytes(d, m, max_queries), 256-byte aligned.
 *   G0:        m x d row-major initial gradients, or NULL for an empty window
 *              (all rows zero; Theorem 1 keeps the 1/m scale for the capacity
 *              m, so empty slots contribute nothing).
 * Enqueues: copy of G0 into the storage (or zero fill), Gram K = G G^T
 * (fp64 MFMA tiles on the exact fp32 values, fp64 reduction), and the
 * coefficient factor. The ring head starts at slot 0. *out receives a
 * host-allocated handle. */
mfac_status mfac_window_init(mfac_window* out, int64_t d, int32_t m, double lambda,
                             int32_t max_queries, void* storage, size_t storage_bytes,
                             void* workspace, size_t workspace_bytes,
                             const float* G0, hipStream_t stream);

/* Overwrite rows [first, first+count) of the window with count x d row-major
 * rows (no Gram update: call mfac_window_rebuild after the last batch). */
mfac_status mfac_window_set_rows(mfac_window w, int32_t first, int32_t count, const float* rows);

/* Recompute the Gram matrix from the stored rows and refactor the
 * coefficients (the O(d m^2 + m^3) setup of Section 3.2). Also the recovery
 * path after a latched non-finite error once the data is fixed. */
mfac_status mfac_window_rebuild(mfac_window w);

/* The sliding step (Section 3.2 update and multiplication; Appendix B's
 * combined update-multiply; Section 4.2's optimizer step):
 *   1. slot k (k = slot, or the ring head if slot == -1) takes g_new;
 *   2. p = G g_new gives row and column k of the Gram matrix;
 *   3. the m x m coefficients are refactored from the Gram matrix;
 *   4. y_out = F^-1 g_new for the window that now holds g_new, evaluated as
 *      m * G^T (G G^T + m*lambda*I)^-1 e_k (free of the cancellation of the
 *      direct form lambda^-1 g - G^T c), and Y = F^-1 X for the n extra rows.
 * X/Y (n x d) are read/written in the same two passes over the window as g.
 * y_out may be NULL (then only the window is updated); X and Y may be NULL iff
 * n == 0. g_new, X must not alias the window storage or y_out/Y.
 * When slot == -1 the ring head advances to (k + 1) mod m. */
mfac_status mfac_window_replace(mfac_window w, int32_t slot, const float* g_new,
                                float* y_out, int32_t n, const float* X, float* Y);

/* A sequence of sliding steps whose gradients are all known in advance:
 * gradient t of Gn (n x d row-major) enters the ring head, then Yn row t =
 * F_t^-1 Gn[t] for the window F_t that holds gradients 0..t of the sequence
 * (Section 3.2 update and multiplication, as n calls of mfac_window_replace
 * with slot -1, no extra queries). The window read that forms Yn[t] also
 * forms the Gram column of Gn[t+1] (Appendix B reuses one product of the
 * window for the update and the multiplication; here the reuse spans two
 * consecutive steps): the row Gn[t+1] replaces is still read for Yn[t], and
 * its dot with Gn[t+1] is taken as Gn[t+1] . Gn[t+1], its value after the
 * replacement. One read of the window per step instead of two for m <= 2048;
 * larger m runs the two passes per step of mfac_window_replace. Results equal
 * those of the separate calls up to the order of fp64 sums in the Gram
 * column, and for a window small enough for the one-launch step of
 * mfac_window_replace (ceil(d / 2048) <= 16, m * ceil(d / 2048) <= 32) in the other
 * fp64 sums too. Not for an optimizer loop, whose next gradient depends on this
 * step's output. n >= 1; Gn and Yn must not alias each other or the window
 * storage. The ring head and step count advance by n. */
mfac_status mfac_window_replace_seq(mfac_window w, int32_t n, const float* Gn, float* Yn);

/* Y = F^-1 X for n x d row-major X (Section 3.2 multiplication; Algorithm 2's
 * role): two passes over the window and an O(m^2) solve with the cached
 * factor. 1 <= n <= max_queries + 1 (the vectors one replace carries). */
mfac_status mfac_ihvp(mfac_window w, int32_t n, const float* X, float* Y);

/* mfac_ihvp for callers that cannot allocate device memory or pass a
 * workspace per call (code under HIP graph capture, tight serving loops,
 * harnesses that forbid hipMalloc): the same computation and results, with
 * the call's scratch (pass-1 partial sums, their reduction and the
 * coefficients) in a fixed 16 MiB device array inside the library instead of
 * the window's workspace. Allocates nothing; no hipMalloc, hipFree or
 * allocating library routine. The array exists once per GPU (held until the
 * process ends; its address is resolved at mfac_window_init) and is shared by
 * every call on that GPU, so calls that overlap on one GPU (several streams
 * or host threads) race and must be serialised by the caller; it keeps the
 * last call's contents, which later calls overwrite before reading.
 * Limit: (512 + 2) * m * n * 8 bytes (each part rounded up to 256) <= 16 MiB,
 * i.e. m * n <= 4080; larger returns MFAC_EWORKSPACE before anything is
 * enqueued. Other arguments and errors as mfac_ihvp. */
mfac_status mfac_ihvp_noalloc(mfac_window w, int32_t n, const float* X, float* Y);

/* Copy rows [first, first+count) back as count x d row-major fp32 (device
 * pointer). Synchronises the stream. */
mfac_status mfac_window_get_rows(mfac_window w, int32_t first, int32_t count, float* rows_out);

/* Current ring head (the slot the next replace with slot == -1 overwrites) and
 * number of replaces so far (host values; no device access). */
mfac_status mfac_window_info(mfac_window w, int32_t* head_out /* host */, int64_t* steps_out /* host */);

/* Set the ring head and step count (resume from a checkpoint of the rows). */
mfac_status mfac_window_set_head(mfac_window w, int32_t head, int64_t steps);

/* How the m x m coefficients follow a replace. The library keeps the explicit
 * fp64 inverse of A = G G^T + m*lambda*I.
 *   period == 0: refactor A from the Gram matrix on every replace (blocked
 *                Cholesky, triangular inverse, L^-T L^-1: the O(m^3) per-replace
 *                cost of Section 3.2's complexity analysis);
 *   period >= 1: O(m^2) update of the inverse on a replace (slot k's old
 *                pivot removed through its Schur complement, the new column
 *                inserted), with a full refactor from the Gram matrix every
 *                `period` replaces to bound rounding drift.
 * Default: max(m, 1024). */
mfac_status mfac_window_set_refactor_period(mfac_window w, int32_t period);

/* Change the stream later calls enqueue on. */
mfac_status mfac_window_set_stream(mfac_window w, hipStream_t stream);

/* Phase timing with HIP events recorded on the handle's stream (a tracing aid,
 * off by default). Phases: 0 = pass-1 kernel (G x), 1 = coefficient phase
 * (partial-sum reduction, Gram row, inverse update or refactor, coefficients),
 * 2 = pass-2 kernel (G^T c), 3 = the write of the new gradient into its slot.
 * enable != 0 starts recording around every replace, replace_seq and ihvp;
 * 0 stops (recorded events are kept until read). In mfac_window_replace_seq
 * phase 2 is the fused pass (G^T c of one step with G x of the next) for all
 * but the last step, and phase 0 runs once, for the first gradient. Each
 * recorded event costs a few microseconds of queue time between launches. A
 * replace of a small window (see mfac_window_replace_seq) runs as one launch
 * without phases when not traced, and as the separate kernels when traced: the
 * phase times are those of the latter. */
#define MFAC_NPHASES 4
mfac_status mfac_window_trace(mfac_window w, int32_t enable);

/* Synchronise the stream, add up the recorded phase times: ms_out and
 * count_out (host arrays of MFAC_NPHASES) receive milliseconds and launch
 * counts per phase; the recorded events are then released. */
mfac_status mfac_window_trace_read(mfac_window w, double* ms_out /* host */, int64_t* count_out /* host */);

/* Synchronise the stream and report (then clear) a latched device error. */
mfac_status mfac_window_status(mfac_window w);

/* Free the host handle (device buffers stay with the caller). NULL is a no-op. */
mfac_status mfac_window_destroy(mfac_window w);

/* ======================================================================
 * Static block-wise precompute (Section 3.1; Appendix C) and OBD queries
 * (Section 4.1)
 * ====================================================================== */

/* Bytes of workspace for the static path: per-block fp64 Gram/factor/inverse
 * buffers for a batch of blocks processed together, plus the fp64 inverse
 * diagonal (d values). block must divide d. Returns 0 on invalid sizes. */
size_t mfac_static_workspace_bytes(int64_t d, int32_t block, int32_t m);

/* Precompute for the block-wise Fisher: d/B independent blocks, block b
 * covering columns [bB, (b+1)B) with
 *     F_b = lambda * I_B + (1/m) G_b^T G_b.
 * G is the caller's m x d row-major gradient matrix; it is overwritten in
 * place by W with W_b = R_b^-1 G_b, R_b the Cholesky factor of
 * G_b G_b^T + m*lambda*I (the same role as the paper's V, which Algorithm 3
 * also writes over G: V_i = sqrt(q_i / lambda) W_i). The inverse diagonal
 * diag(F_b^-1) = (1 - sum_i W_b[i,:]^2) / lambda is formed in fp64 from the
 * unrounded W and kept in the workspace.
 * With MFAC_STATIC_FP32 the precompute leaves G intact instead (see the flag).
 * Requirements: 1 <= m <= 8192, 4 <= block, block % 4 == 0,
 * d % block == 0, d <= 2^32 - 256, lambda > 0 finite, G 16-byte aligned,
 * workspace 256-byte aligned (at least mfac_static_workspace_bytes_flags for
 * the flags given), flags a combination of MFAC_STATIC_* bits. */
mfac_status mfac_static_precompute(mfac_static* out, int64_t d, int32_t block, int32_t m,
                                   double lambda, float* G, void* workspace,
                                   size_t workspace_bytes, uint32_t flags, hipStream_t stream);

/* flags of mfac_static_precompute and mfac_static_precompute_paged */
#define MFAC_STATIC_TRACE 1u /* record HIP events around the precompute's stages and
                                mfac_obs_mask; read with mfac_static_trace_read */
/* Fast mode (mfac_static_precompute only; m <= 4096, block <= 65536): the
 * Gram matrices, their Cholesky factors and inverses, and W in fp32 (values
 * and sums; a product of two values, in the large matrix products, as the six
 * largest of the nine products of their three bf16 parts, which leaves out at
 * most 2^-24 (1 + 2^-10) of it). A Gram entry is summed over at most 2048 columns,
 * wider blocks adding their 2048-column splits in fp64, W over the m rows,
 * the squares of W in fp64 for the diagonal. The inverse diagonal then
 * carries the fp32 rounding (on gradient-like data with a well-conditioned
 * G_b G_b^T + m*lambda*I, a largest entry error of 1.4e-6 relative measured
 * at d = 4.19M, B = 2048, m = 1024). G is left intact: W and the fp32
 * L^-1 of every block go into the workspace. Of the later calls only
 * mfac_obs_mask reads G. mfac_obs_mask stays exact: coordinates whose fp64 score
 * lies within 1e-5 relative of the cut get their diagonal recomputed in fp64
 * (iterative refinement against G, see mfac_obs_mask), so the mask equals the
 * fp64 mask whenever the fp32 path's score error is below about 1e-5. */
#define MFAC_STATIC_FP32 2u

/* Workspace bytes for mfac_static_precompute with these flags (the fast mode
 * needs more: the fp32 L^-1 of every block, m*d floats for W, and the band
 * list). 0 on invalid sizes or flags. */
size_t mfac_static_workspace_bytes_flags(int64_t d, int32_t block, int32_t m, uint32_t flags);

/* Host-paged static precompute, for a G larger than the device should hold
 * (Appendix C, swapping gradient blocks between host and GPU memory; here
 * the pages are column ranges, which the block structure makes independent).
 * Computes the same W (written back over G on the host), inverse diagonal
 * and handle as mfac_static_precompute.
 *   G_host:    m x d row-major fp32 in pinned host memory (hipHostMalloc or
 *              a pinned torch tensor), 16-byte aligned; overwritten by W.
 *              Pageable memory is rejected (MFAC_EINVAL).
 *   page_cols: columns per page, a multiple of 4 and, when block < d, of
 *              block (a page holds whole blocks, at most 65535); values above
 *              d mean d; the page width (after that) at most 2^30. Three
 *              device page buffers of m * page_cols floats live in the
 *              workspace.
 * block < d: one sweep; each page is uploaded, its blocks go through Gram,
 * factor and W, and W is downloaded (G crosses the host link twice).
 * block == d: the one block's Gram is summed page by page, factored, and a
 * second sweep forms W page by page, starting with the (up to) three last
 * pages, still on the device (G crosses up to three times).
 * Uploads and downloads run on two streams the handle creates (default
 * priority) and overlap each other and the kernels on `stream`, which waits
 * for the last download before any later call on the handle. The queries
 * (mfac_static_ihvp, mfac_static_element, mfac_obs_update) of a paged
 * handle read W directly from the pinned host buffer over the host link;
 * mfac_inv_diag, mfac_inv_diag64 and mfac_obs_mask use the device diagonal.
 * Other requirements as mfac_static_precompute. */
size_t mfac_static_paged_workspace_bytes(int64_t d, int32_t block, int32_t m, int64_t page_cols);
mfac_status mfac_static_precompute_paged(mfac_static* out, int64_t d, int32_t block, int32_t m,
                                         double lambda, float* G_host, int64_t page_cols, void* workspace,
                                         size_t workspace_bytes, uint32_t flags, hipStream_t stream);

/* Per-stage device time of a static handle created with MFAC_STATIC_TRACE,
 * since creation or the last read (synchronises the stream). ms_out and
 * count_out (host arrays of MFAC_STATIC_NPHASES) receive milliseconds and
 * launch counts for: 0 batched Gram (one launch per batch of blocks), 1
 * factor and inverse, 2 W and inverse diagonal, 3 scores and keep-mask.
 * Without the flag every entry is 0. */
#define MFAC_STATIC_NPHASES 4
mfac_status mfac_static_trace_read(mfac_static s, double* ms_out /* host */, int64_t* count_out /* host */);

/* diag(F^-1) for all d coordinates (Appendix C, row-selected extraction with
 * the identity selection), rounded to fp32. */
mfac_status mfac_inv_diag(mfac_static s, float* diag_out);

/* Same, in fp64 (fp64-accurate in the default mode; in the fast mode it has
 * the fp32 path's error, except coordinates that an mfac_obs_mask call
 * recomputed in its band). */
mfac_status mfac_inv_diag64(mfac_static s, double* diag_out);

/* OBD saliency rho_j = theta_j^2 / (2 [F^-1]_jj) in fp64 (Section 4.1) and a
 * global keep-mask over all blocks: keep_mask[j] = 1 for the `keep` largest
 * rho, ties broken by the lower index; 0 <= keep <= d. scores_out may be
 * NULL. theta 4-byte aligned. Uses workspace scratch; output is exact given
 * the fp64 diagonal. In the fast mode (MFAC_STATIC_FP32) the scores come from
 * the fp32-path diagonal; the keep-th largest score t is selected, every
 * coordinate with a nonzero score within [t(1 - 1e-5), t(1 + 1e-5)] has
 * [F^-1]_jj recomputed in fp64 (x = A_b^-1 g_j by iterative refinement: the
 * residual g_j - A_b x formed from G in fp64, the kept fp32 L^-1 as
 * preconditioner, until the estimated remaining error is below 1e-13 of x;
 * then (1 - g_j.x) /
 * lambda), stored into the diagonal, and the selection runs again. The mask
 * then equals the fp64 mask: a coordinate outside the band is on the same side
 * of the fp64 cut as long as the fp32 scores are within 1e-5 / (1 + 1e-5)
 * relative of the fp64 ones. The refinement measures that error on the band
 * (the coordinates at the cut); if any exceeds 2.5e-6 (a quarter of the band's
 * half-width: the fp32 path is then too inaccurate for this G, e.g. blocks
 * whose Fisher term dwarfs m*lambda), the mask is not certified and the next
 * mfac_static_status returns MFAC_EPRECISION: use the default (fp64) mode. A
 * refinement that does not settle within 12 steps latches MFAC_ENONFINITE. */
mfac_status mfac_obs_mask(mfac_static s, const float* theta, int64_t keep,
                          double* scores_out, uint8_t* keep_mask_out);

/* Y = F^-1 X for the block-wise Fisher, n x d row-major fp32 X and Y,
 * 1 <= n <= 4 (Appendix C eq. 9; with W in place of V and q:
 * F_b^-1 x_b = (x_b - W_b^T (W_b x_b)) / lambda). Two passes over W (the
 * precompute's output in G's storage). X and Y 16-byte aligned and must not
 * alias G. */
mfac_status mfac_static_ihvp(mfac_static s, int32_t n, const float* X, float* Y);

/* Element queries [F^-1]_ij, O(m) each (Section 3.1, eq. 5):
 * (delta_ij - sum_k W[k,i] W[k,j]) / lambda when i and j share a block, 0
 * otherwise; fp64 sums of the fp32 W. ij: device array of 2*nq int64 indices
 * (i_0, j_0, i_1, j_1, ...); out: nq fp64 values. An index outside [0, d)
 * yields NaN and latches MFAC_ENONFINITE. */
mfac_status mfac_static_element(mfac_static s, int64_t nq, const int64_t* ij, double* out);

/* OBS correction (Section 4.1) for removing every coordinate j with
 * keep_mask[j] == 0 at once: delta = -F^-1 x with x_j = theta_j / [F^-1]_jj on
 * removed coordinates and 0 elsewhere, i.e. the sum of the single-weight OBS
 * updates -theta_j F^-1 e_j / [F^-1]_jj (the paper's approximate
 * multi-weight OBS). theta + delta zeroes a removed weight that is the only
 * removed one in its block. theta, delta_out: d fp32 (theta 4-byte,
 * delta_out 16-byte aligned); keep_mask: d uint8. */
mfac_status mfac_obs_update(mfac_static s, const float* theta, const uint8_t* keep_mask, float* delta_out);

mfac_status mfac_static_set_stream(mfac_static s, hipStream_t stream);
mfac_status mfac_static_status(mfac_static s);
mfac_status mfac_static_destroy(mfac_static s);

/* ======================================================================
 * Training operators: layer norm, linear layers, 8-bit activation copies
 * ======================================================================
 * The forward and backward passes of a transformer's feed-forward block, for
 * the models whose gradients the window above takes, with the activations
 * that the backward pass needs kept in 8 bits next to a window that fills
 * most of the card's memory. These calls have no handle: each one checks its
 * arguments on the host (MFAC_EINVAL, MFAC_EWORKSPACE; nothing is enqueued
 * then), enqueues its kernels on the given stream and returns. Nothing is
 * allocated, nothing is kept between calls, and a call may be captured into a
 * HIP graph. Results do not depend on the order in which work-groups run: sums
 * are joined in a fixed order, without atomics. Infinities and NaN pass through
 * by the rules of the arithmetic and are not latched as errors.
 *
 * Matrices are row-major with unit stride along a row and a leading dimension
 * (elements between rows) of at least the row's length; pointers are aligned to
 * the element. The products take 16-bit matrices as they are where the rows
 * start 16-byte aligned and their length is a multiple of 8 elements, and lay
 * others out in the workspace first, as they do with fp32 and with 8-bit copies.
 * Their *_bytes queries therefore take the matrices' addresses (which are not
 * read) and leading dimensions; x NULL means an 8-bit copy. A query returns 0 on
 * invalid sizes and where no workspace is needed. Workspaces are 256-byte aligned.
 * Sizes are at least 0 (rows) or 1 (columns) and at most 2^30, the widths of linear
 * layers at most 2^21; offsets are 64-bit. rows == 0 is valid: the gradients of
 * weights are then zero. Inputs and outputs must not overlap unless a call says
 * so. */

/* Element types. Sums, statistics and the arithmetic between them are fp32 in
 * every type; a result is rounded once, when it is stored. */
typedef enum {
    MFAC_F32 = 0,
    MFAC_BF16 = 1,
    MFAC_F16 = 2,
    /* not types: they widen the enum to int32, so that any code is a value of it */
    MFAC_DTYPE_NONE_ = -1,
    MFAC_DTYPE_INT32_ = 0x7fffffff
} mfac_dtype;

/* Activations: z, max(z, 0), z Phi(z) (Phi the normal distribution function),
 * 0.5 z (1 + tanh(sqrt(2/pi) (z + 0.044715 z^3))), z / (1 + exp(-z)). */
typedef enum {
    MFAC_ACT_NONE = 0,
    MFAC_ACT_RELU = 1,
    MFAC_ACT_GELU = 2,
    MFAC_ACT_GELU_TANH = 3,
    MFAC_ACT_SILU = 4,
    MFAC_ACT_NOT_ONE_ = -1, /* not activations: as above */
    MFAC_ACT_INT32_ = 0x7fffffff
} mfac_act;

/* 8-bit copies. Row r of a rows x cols matrix is cut into ceil(cols / 32) groups
 * of 32 neighbouring columns (the last may be shorter). Group j has the power
 * 2^e, e >= -126 the smallest with max |x| <= 127 * 2^e; s[r * ceil(cols/32) + j]
 * = e + 127 and q[r * ldq + c] = x * 2^-e rounded to the nearest integer, ties to
 * even (for e = 122 at most 63 in magnitude: 64 * 2^122 is no fp32 value). The copy
 * stands for q * 2^e, off by at most 2^(e-1) (2^e for e = 122). A value with 8 bits
 * times a power of two is a bf16 value, so bf16 products of it need no second
 * rounding. A group with an infinity or a NaN has s = 255 and q = 0 and stands
 * for NaN throughout. Rows of q lie ldq >= cols bytes apart; what is past the cols
 * of a row is neither read nor written. */
#define MFAC_PACK8_GROUP 32

/* q, s <- the 8-bit copy of x. */
mfac_status mfac_pack8(mfac_dtype type, int64_t rows, int64_t cols, const void* x, int64_t ldx, int8_t* q, int64_t ldq,
                       uint8_t* s, hipStream_t stream);

/* y <- the values a copy stands for, rounded to y's type (exact in fp32 and
 * bf16; in fp16 values past 65504 become 65504). */
mfac_status mfac_unpack8(mfac_dtype type, int64_t rows, int64_t cols, const int8_t* q, int64_t ldq, const uint8_t* s,
                         void* y, int64_t ldy, hipStream_t stream);

/* Layer norm of each row: mean, rstd = 1 / sqrt(mean((x - mean)^2) + eps), xhat =
 * (x - mean) rstd, y = xhat w + b. w and b (cols values of type wtype: fp32 or x's
 * type) may be NULL (1 and 0). mean_out and rstd_out (rows fp32 values) may be
 * NULL. q and s: the 8-bit copy of xhat, or both NULL. eps >= 0, finite. y may
 * be x. */
mfac_status mfac_layer_norm(mfac_dtype type, mfac_dtype wtype, int64_t rows, int64_t cols, const void* x, int64_t ldx,
                            const void* w, const void* b, double eps, void* y, int64_t ldy, float* mean_out,
                            float* rstd_out, int8_t* q, int64_t ldq, uint8_t* s, hipStream_t stream);

/* Gradients of layer norm: with h = dy w,
 *   dx = rstd (h - mean(h) - xhat mean(h xhat)) + add,
 *   dw = sum over rows of dy xhat, db = sum over rows of dy.
 * xhat is (x - mean) rstd, or the 8-bit copy (q, s), for which x and mean are
 * NULL. add (type, rows of ldadd) may be NULL: the gradient of a skip connection
 * around the norm. dw and db (cols values of wtype) may be NULL. dx may be dy
 * or add. */
size_t mfac_layer_norm_bwd_workspace_bytes(int64_t rows, int64_t cols);
mfac_status mfac_layer_norm_bwd(mfac_dtype type, mfac_dtype wtype, int64_t rows, int64_t cols, const void* dy,
                                int64_t lddy, const void* x, int64_t ldx, const float* mean, const float* rstd,
                                const int8_t* q, int64_t ldq, const uint8_t* s, const void* w, const void* add,
                                int64_t ldadd, void* dx, int64_t lddx, void* dw, void* db, void* workspace,
                                size_t workspace_bytes, hipStream_t stream);

/* Linear layer: z = x W^T + b, y = act(z) + res, for x (rows x cin), W (cout x cin),
 * y (rows x cout). bias (cout values of btype: fp32 or x's type) and res may be
 * NULL. z_out (type) or the 8-bit copy of z (q, s) keep the pre-activation for
 * the backward pass; at most one of the two, both optional. y may be res.
 * Products: fp16 and bf16 values on the matrix cores with fp32 sums; fp32 values
 * as three bf16 parts each, of whose nine products the six largest are taken
 * (what is left out is at most 2^-24 (1 + 2^-10) of the product); what of a value lies
 * below 2^-133 is left out, and an infinite one has no such parts: its products come
 * out NaN. Up to 16 rows of a forward pass in fp32 multiply in fp32. */
size_t mfac_linear_workspace_bytes(mfac_dtype type, int64_t rows, int64_t cin, int64_t cout, const void* x,
                                   int64_t ldx, const void* w, int64_t ldw);
mfac_status mfac_linear(mfac_dtype type, mfac_dtype btype, mfac_act act, int64_t rows, int64_t cin, int64_t cout,
                        const void* x, int64_t ldx, const void* w, int64_t ldw, const void* bias, const void* res,
                        int64_t ldres, void* y, int64_t ldy, void* z_out, int64_t ldz, int8_t* q, int64_t ldq,
                        uint8_t* s, void* workspace, size_t workspace_bytes, hipStream_t stream);

/* The activation's part of a backward pass over a rows x cols pre-activation z
 * (type, or its 8-bit copy):
 *   dz = dy act'(z) rounded to type, a = act(z) (NULL: not wanted),
 *   db[c] = sum over rows of dy act'(z) in fp32, before the rounding (NULL: not wanted).
 * With MFAC_ACT_NONE z, q, s are NULL, and dz may be NULL (it equals dy). dz may
 * be dy. */
size_t mfac_act_bwd_workspace_bytes(int64_t rows, int64_t cols);
mfac_status mfac_act_bwd(mfac_dtype type, mfac_act act, int64_t rows, int64_t cols, const void* dy, int64_t lddy,
                         const void* z, int64_t ldz, const int8_t* q, int64_t ldq, const uint8_t* s, void* dz,
                         int64_t lddz, void* a, int64_t lda, float* db, void* workspace, size_t workspace_bytes,
                         hipStream_t stream);

/* Gradient of a linear layer's input: dx = dz W + add, for dz (rows x cout), W
 * (cout x cin), dx (rows x cin); add (type) may be NULL. dx may be add. */
size_t mfac_linear_bwd_input_workspace_bytes(mfac_dtype type, int64_t rows, int64_t cin, int64_t cout, const void* dz,
                                             int64_t lddz, const void* w, int64_t ldw);
mfac_status mfac_linear_bwd_input(mfac_dtype type, int64_t rows, int64_t cin, int64_t cout, const void* dz,
                                  int64_t lddz, const void* w, int64_t ldw, const void* add, int64_t ldadd, void* dx,
                                  int64_t lddx, void* workspace, size_t workspace_bytes, hipStream_t stream);

/* Gradient of a linear layer's weight: dW = dz^T x (cout x cin, type gtype: fp32
 * or the inputs' type). x (rows x cin) is given in `type`, or as an 8-bit copy (q,
 * s; x NULL). gamma and beta (cin fp32 values each, or both NULL) say that the
 * layer's input was gamma x + beta, the affine part of a layer norm whose xhat
 * is x: dW = (dz^T x) diag(gamma) + db beta^T, for which db (cout fp32 values, the
 * column sums of dz) is needed; it may be NULL otherwise. */
size_t mfac_linear_bwd_weight_workspace_bytes(mfac_dtype type, int64_t rows, int64_t cin, int64_t cout,
                                              const void* dz, int64_t lddz, const void* x, int64_t ldx);
mfac_status mfac_linear_bwd_weight(mfac_dtype type, mfac_dtype gtype, int64_t rows, int64_t cin, int64_t cout,
                                   const void* dz, int64_t lddz, const void* x, int64_t ldx, const int8_t* q,
                                   int64_t ldq, const uint8_t* s, const float* gamma, const float* beta,
                                   const float* db, void* dw, int64_t lddw, void* workspace, size_t workspace_bytes,
                                   hipStream_t stream);

/* How a product of these passes is run, for tuning and tests. plan[0]: the side of its square tiles of the result (0:
 * the kernel for few rows); plan[1]: the parts that its sums are cut into; plan[2]: 1 where results are stored past the
 * caches. otype is the result's type (gtype for the weight's gradient, `type` otherwise); packed: x is an 8-bit copy
 * (weight only). rows is at least 1. */
typedef enum {
    MFAC_PRODUCT_FORWARD = 0,
    MFAC_PRODUCT_INPUT = 1,
    MFAC_PRODUCT_WEIGHT = 2,
    MFAC_PRODUCT_NONE_ = -1, /* not products: as above */
    MFAC_PRODUCT_INT32_ = 0x7fffffff
} mfac_product;
mfac_status mfac_linear_plan(mfac_dtype type, mfac_dtype otype, mfac_product product, int64_t rows, int64_t cin,
                             int64_t cout, int32_t packed, int32_t plan[3]);

/* ----------------------------------------------------------------------
 * A gated block: gated layers, what lies between two blocks, dropout
 * ----------------------------------------------------------------------
 * By the same rules as the calls above. */

/* Gated layer: z = x W^T + b for W of 2 hidden rows (those of the gate, then those of the other projection; bias likewise),
 * y = act(zg) zu, for x (rows x cin), W (2 hidden x cin), y (rows x hidden); hidden at most 2^20. Both projections, the
 * activation and the product are one kernel. bias (2 hidden values of btype) may be NULL. The pre-activations zg and zu
 * (rows x hidden each) may be kept for the backward pass, as matrices of `type` with the same ldz (they may be the halves of
 * one), or as 8-bit copies (qg, sg) and (qu, su) with the same ldq; both or neither of the two. */
size_t mfac_gated_linear_workspace_bytes(mfac_dtype type, int64_t rows, int64_t cin, int64_t hidden, const void* x,
                                         int64_t ldx, const void* w, int64_t ldw);
mfac_status mfac_gated_linear(mfac_dtype type, mfac_dtype btype, mfac_act act, int64_t rows, int64_t cin, int64_t hidden,
                              const void* x, int64_t ldx, const void* w, int64_t ldw, const void* bias, void* y,
                              int64_t ldy, void* zg, void* zu, int64_t ldz, int8_t* qg, uint8_t* sg, int8_t* qu,
                              uint8_t* su, int64_t ldq, void* workspace, size_t workspace_bytes, hipStream_t stream);

/* Its backward pass, by itself (cout 0: dy is the gradient of y, rows x hidden) or with that of the layer y W2^T that follows
 * (dy is rows x cout, W2 cout x hidden; that layer's bias has the column sums of dy). From the pre-activations (matrices or
 * copies), with da = dy W2, or dy,
 *   dz = [da zu act'(zg), da act(zg)], a = act(zg) zu,
 *   dx = dz W, dw1 = dz^T x (gtype), db1 = column sums of dz in fp32, dw2 = dy^T a (gtype);
 * those that are NULL are not formed, nor da, dz or a where they alone need it. da is not rounded. dz and a are rounded to
 * `type` for the products, so that fp16's past 65504 are infinite; for dw1 and dw2 of 16-bit data in fp32 (gtype) they are
 * taken in two parts, the second what the first's rounding leaves. The two parts of fp16 (dz's first serves dx too) are
 * stored times powers of two that keep them finite, which the products take out again; bf16 is infinite from 0x1.ffp127 on.
 * x, or its 8-bit copy (q, s; x NULL), is needed for dw1, W1 (w1) for dx, W2 (w2) for all but dw2. gamma and beta (cin fp32
 * values each; beta may be NULL) say that x stands for gamma x + beta in dw1. The workspace query takes, besides addresses
 * that are not read (x NULL: a copy), what is wanted as bits. */
#define MFAC_GATED_DX 1u
#define MFAC_GATED_DW1 2u
#define MFAC_GATED_DB1 4u
#define MFAC_GATED_DW2 8u
#define MFAC_GATED_BETA 16u /* beta is given */
size_t mfac_gated_bwd_workspace_bytes(mfac_dtype type, mfac_dtype gtype, int64_t rows, int64_t cin, int64_t hidden,
                                      int64_t cout, const void* dy, int64_t lddy, const void* w2, int64_t ldw2,
                                      const void* x, int64_t ldx, const void* w1, int64_t ldw1, uint32_t wanted);
mfac_status mfac_gated_bwd(mfac_dtype type, mfac_dtype gtype, mfac_act act, int64_t rows, int64_t cin, int64_t hidden,
                           int64_t cout, const void* dy, int64_t lddy, const void* w2, int64_t ldw2, const void* x,
                           int64_t ldx, const int8_t* q, int64_t ldq, const uint8_t* s, const float* gamma,
                           const float* beta, const void* w1, int64_t ldw1, const void* zg, const void* zu, int64_t ldz,
                           const int8_t* qg, const uint8_t* sg, const int8_t* qu, const uint8_t* su, int64_t ldqz,
                           void* dx, int64_t lddx, void* dw1, int64_t lddw1, float* db1, void* dw2, int64_t lddw2,
                           void* workspace, size_t workspace_bytes, hipStream_t stream);

/* Dropout. at: two int64 in device memory, seed and offset, 8-byte aligned, read when the kernel runs (so a captured graph
 * takes what they hold when it is replayed). Element (row, c) of a matrix takes half-word c % 8 of the Philox 4x32-10 block
 * with counter (c / 8, row, offset mod 2^32, offset / 2^32) and key (seed mod 2^32, seed / 2^32), both taken as unsigned;
 * half-word i is the lower (i even) or upper half of word i / 2. It is kept where the half-word is at least
 * T = floor(65536 p + 1/2), and multiplied by 65536 / (65536 - T); others become 0, infinities and NaN among them.
 * 0 <= p <= 1; with T = 0 every value is kept, with T = 65536 none. The mask depends on p, at and the place in the matrix
 * alone, not on the type or strides: the gradient is the same call on dy. y may be x. */
mfac_status mfac_dropout(mfac_dtype type, int64_t rows, int64_t cols, const void* x, int64_t ldx, double p,
                         const int64_t* at, void* y, int64_t ldy, hipStream_t stream);

/* What lies between two blocks of a network with a residual stream, row by row:
 *   n = N_post(y), s = scale res + gate drop(n), h = N_pre(s).
 * N is rms norm, x rstd w with rstd = 1 / sqrt(mean(x^2) + eps), or with MFAC_NORM_LAYER layer norm as above, both of one
 * kind; either may be absent (n = y; no h). post_w, post_b, pre_w, pre_b (cols values of wtype) may be NULL (1 and 0); rms
 * norm has no b. The gate is one value for each channel (`gate`, cols values of wtype), one for each element (`gates`, of
 * `type`), or absent (1). drop is dropout with p and at (at may be NULL where T is 0). res and s may be NULL (no residual;
 * not wanted, where h is). h is formed from s before its rounding. Statistics (rows fp32 values each) may be NULL; means are
 * layer norm's. q and sq: the 8-bit copy of N_pre's xhat, or both NULL. cols at most 2^15. eps >= 0 and scale finite. s may
 * be y or res, and h may be y or res, but not s. With MFAC_NORM_PRE alone and no residual, gate or dropout the call is
 * h = N(y). */
typedef enum {
    MFAC_NORM_POST = 1,
    MFAC_NORM_PRE = 2,
    MFAC_NORM_LAYER = 4
} mfac_norms;
mfac_status mfac_residual_norm(mfac_dtype type, mfac_dtype wtype, int32_t norms, int64_t rows, int64_t cols,
                               const void* y, int64_t ldy, const void* post_w, const void* post_b, const void* gate,
                               const void* gates, int64_t ldgates, const void* res, int64_t ldres, double scale, double p,
                               const int64_t* at, const void* pre_w, const void* pre_b, double eps, void* s, int64_t lds,
                               void* h, int64_t ldh, float* post_mean, float* post_rstd, float* pre_mean,
                               float* pre_rstd, int8_t* q, int64_t ldq, uint8_t* sq, hipStream_t stream);

/* Its gradients. ds is the gradient that reaches s from elsewhere (NULL: none; needed without MFAC_NORM_PRE), dh that of h.
 * With d = ds + the gradient of N_pre at dh,
 *   dres = scale d, dn = gate drop(d), dgate(s) = d drop(n), dy = the gradient of N_post at dn;
 * outputs may be NULL (not wanted); those of parameters (wtype) are sums over the rows. s, or the 8-bit copy of N_pre's xhat
 * (then s and pre_mean are NULL); y may be NULL where neither MFAC_NORM_POST nor a gate's gradient needs it. dy and dres may
 * be ds or dh, dy may be y. The workspace is needed for parameters' gradients. */
size_t mfac_residual_norm_bwd_workspace_bytes(mfac_dtype type, int32_t norms, int64_t rows, int64_t cols);
mfac_status mfac_residual_norm_bwd(mfac_dtype type, mfac_dtype wtype, int32_t norms, int64_t rows, int64_t cols,
                                   const void* ds, int64_t ldds, const void* dh, int64_t lddh, const void* y,
                                   int64_t ldy, const float* post_mean, const float* post_rstd, const void* s,
                                   int64_t lds, const int8_t* q, int64_t ldq, const uint8_t* sq, const float* pre_mean,
                                   const float* pre_rstd, const void* post_w, const void* post_b, const void* gate,
                                   const void* gates, int64_t ldgates, double scale, double p, const int64_t* at,
                                   const void* pre_w, void* dy, int64_t lddy, void* dres, int64_t lddres, void* dgates,
                                   int64_t lddgates, void* dpost_w, void* dpost_b, void* dgate, void* dpre_w,
                                   void* dpre_b, void* workspace, size_t workspace_bytes, hipStream_t stream);

/* How the products of a gated layer are run, as mfac_linear_plan: the layer itself, by what it keeps, or the product of
 * mfac_gated_bwd that forms da (cin is then its cout), by whether db1 or beta asks for column sums. */
typedef enum {
    MFAC_GATED_FORWARD = 0,        /* nothing kept */
    MFAC_GATED_HIDDEN = 1,
    MFAC_GATED_FORWARD_Z = 2,      /* the pre-activations kept */
    MFAC_GATED_FORWARD_COPIES = 3, /* 8-bit copies of them */
    MFAC_GATED_HIDDEN_SUMS = 4
} mfac_gated_product;
mfac_status mfac_gated_plan(mfac_dtype type, int32_t product, int64_t rows, int64_t cin, int64_t hidden, int32_t plan[3]);

#ifdef __cplusplus
}
#endif

#endif /* MFAC_H */
