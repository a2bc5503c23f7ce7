/*
 * lsp.h -- C ABI of the MI355X (gfx950) library for the GPU hot path of LSP-Offload
 * (arXiv 2406.10181): compressing a weight gradient through two learned sparse projectors
 * and expanding the CPU-computed subspace update back onto the weight; beside the per-step
 * calls, the two GPU-side pieces of the projector refresh (MaybeUpdate, Alg. 1): the estimation
 * bias of Def. 2 and the re-projection of the optimiser state.
 *
 * Letters.  G and W are m x n, row-major, leading dimension n.  r is the subspace size
 * (number of columns of P and Q; S is r x r).  d is the number of stored entries per
 * projector row.  The paper names these the other way round: its "(d,r)-sparse projector"
 * (Def. 1) has subspace size d and r nonzeros per row.
 *
 * Projectors.  P (m x r) and Q (n x r) are (d,r)-sparse in the sense of Def. 1 and are passed
 * in ELL layout: idx[row][k] (int32, a column in [0, r)) and val[row][k] (fp32), k < d,
 * row-major.  The dense meaning is  Phat[i][a] = sum of val[i][k] over k with idx[i][k] == a:
 * duplicate columns within a row add up, and an entry with val == 0 is padding (its index
 * must still be in range).  Indices are NOT range-checked by the compute calls; an index
 * outside [0, r) is undefined behaviour.  lsp_validate_projector() checks them on request.
 *
 * Memory.  Every pointer named "device" is device memory of the current HIP device, owned by
 * the caller for the whole call and until the enqueued work has finished.  The library never
 * allocates, frees or copies device memory in the compute calls, never synchronises the
 * stream, and keeps no state between calls.  Buffers must not alias one another.
 * All base pointers must be aligned to 16 bytes.
 *
 * Execution.  Compute calls only enqueue kernels on `stream` (a hipStream_t passed as
 * void*; NULL = the default stream) and return; work on one stream runs in call order
 * (Alg. 3 issues these per layer, in backward order, asynchronously).
 *
 * Errors.  Every call returns LSP_OK (0) or a negative lsp_status.  All argument checks are
 * made before the first HIP call: on LSP_ERR_NULL / SHAPE / DTYPE / WORKSPACE / ALIGN nothing has
 * been enqueued and no output has been touched.  LSP_ERR_LAUNCH means the HIP runtime refused a
 * launch (or, in the set-up calls, a copy, or the host ran out of memory); a call that consists of
 * several kernels may then have enqueued part of its work already, and its outputs are undefined.
 */
#ifndef LSP_H
#define LSP_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    LSP_F32  = 0,   /* IEEE binary32 */
    LSP_F16  = 1,   /* IEEE binary16 */
    LSP_BF16 = 2    /* bfloat16 */
} lsp_dtype;

typedef enum {
    LSP_OK            =  0,
    LSP_ERR_NULL      = -1,  /* a required pointer is NULL */
    LSP_ERR_SHAPE     = -2,  /* m, n, r or d not positive, d > r, size overflow, r or d above the supported maximum */
    LSP_ERR_DTYPE     = -3,  /* dtype is not one of lsp_dtype */
    LSP_ERR_WORKSPACE = -4,  /* workspace / plan buffer missing, misaligned or too small */
    LSP_ERR_LAUNCH    = -5,  /* the HIP runtime refused a launch or a copy (see lsp_last_hip_error) */
    LSP_ERR_INDEX     = -6,  /* lsp_validate_projector found an index outside [0, r) */
    LSP_ERR_ALIGN     = -7,  /* a base pointer is not 16-byte aligned */
    LSP_ERR_SKEW      = -8,  /* lsp_plan_build: the columns of Q are used too unevenly for a plan; use lsp_compress */
    LSP_ERR_TOO_LARGE = -9,  /* lsp_compress_planned_static: the problem needs more than LSP_STATIC_SCRATCH_BYTES of scratch */
    LSP_ERR_VALUE     = -10  /* a number is out of its range: a dropout, a beta or a smoothing not in [0, 1), a scale that is not finite, a negative eps */
} lsp_status;

#define LSP_MAX_R 2048       /* largest supported subspace size (the paper's largest setting) */
#define LSP_MAX_D 64         /* largest supported number of entries per projector row */
#define LSP_MAX_GROUP 16     /* most problems in one grouped call */
#define LSP_MAX_HEAD_DIM 128 /* widest head of the attention calls */
#define LSP_MAX_WIDTH 8192   /* longest row of the residual-norm calls */
#define LSP_MAX_ROWS (1 << 22)   /* most rows of one residual-norm call */
#define LSP_MAX_TENSORS (1 << 16)    /* most tensors of one optimizer step */
#define LSP_STATIC_SCRATCH_BYTES (24u << 20)   /* scratch held inside the library image, per GPU (lsp_compress_planned_static) */

/* ------------------------------------------------------------------------------------------
 * Compress:  S := P^T G Q.
 * The step "grad <- SendToCPU(P^T grad_W Q)" of Alg. 1 and the step that forms the projected
 * gradient of layer l in Alg. 3.  S is OVERWRITTEN (not accumulated); gradient accumulation
 * happens on G before the call.  G is widened exactly to fp32; all sums are fp32.
 *
 *   G          device, m*n elements of `dtype`, row-major
 *   P_idx/val  device, [m][d]
 *   Q_idx/val  device, [n][d]
 *   S          device, r*r fp32, row-major, written
 *   workspace  device scratch of at least lsp_compress_workspace_bytes(m,n,r,d) bytes,
 *              16-byte aligned; contents are clobbered; may be reused by later calls on
 *              the same stream
 *
 * This entry takes raw ELL projectors and needs no preparation: it builds the plan on the
 * device into the workspace and runs the planned kernels on it, all asynchronously; only
 * projectors too skewed for a plan are served by a scatter form (LDS and global fp32 atomics, far
 * slower, not bit-reproducible), chosen on the device.  An index outside [0, r) makes S NaN.
 * When the projectors stay fixed over many steps -- the paper refreshes them only every CheckFreq
 * steps in MaybeUpdate, Alg. 1 -- build a plan once with lsp_plan_build and call
 * lsp_compress_planned, which saves the build in every step.
 */
int lsp_compress(const void* G,
                 const int32_t* P_idx, const float* P_val,
                 const int32_t* Q_idx, const float* Q_val,
                 int64_t m, int64_t n, int32_t r, int32_t d,
                 float* S, lsp_dtype dtype,
                 void* workspace, size_t workspace_bytes, void* stream);

/* Bytes of device scratch lsp_compress needs (0 on invalid shapes). */
size_t lsp_compress_workspace_bytes(int64_t m, int64_t n, int32_t r, int32_t d);

/* One size that serves every call of this header on an (m, n, r, d) problem: the largest of the
 * per-call workspace queries below (0 on invalid shapes or dtype).  The library holds no
 * workspace of its own: scratch is always an argument of the call that uses it. */
size_t lsp_workspace_bytes(int64_t m, int64_t n, int32_t r, int32_t d, lsp_dtype dtype);

/* ------------------------------------------------------------------------------------------
 * Projector plan: a device-resident, column-sorted copy of P and Q for one (m, n, r, d)
 * problem, valid until the projector arrays change (every CheckFreq steps at most, Alg. 1).
 * It lives entirely in a caller-owned device buffer of lsp_plan_bytes() bytes; there is no
 * host handle.  Building a plan only sorts and packs the projector entries (no arithmetic on
 * G, W or S) and happens on the device, where the projectors live: three small kernels (about
 * 25 microseconds; nothing is copied to the host).
 *
 * lsp_plan_build_async only enqueues that work on `stream`; it needs device scratch of
 * lsp_plan_build_workspace_bytes() and reports what only the data can show -- an index outside
 * [0, r) (LSP_ERR_INDEX) or columns too skewed for a plan (LSP_ERR_SKEW) -- in `status` (device,
 * one int32, may be NULL), written when the build has run; a failed build also leaves the buffer
 * marked as "no plan", so that compress calls with it fill S with NaN.
 * lsp_plan_build is the synchronous form: it allocates and frees the scratch itself (a set-up call,
 * NOT part of the per-step path), waits for `stream` and returns the build's status.
 * lsp_plan_build_host makes the same bytes with every pointer in HOST memory and no HIP call; the
 * result can be copied to the device by the caller.  lsp_plan_refresh_values (below) drops new
 * values into a plan whose positions are unchanged.
 */
size_t lsp_plan_bytes(int64_t m, int64_t n, int32_t r, int32_t d);

int lsp_plan_build(const int32_t* P_idx, const float* P_val,
                   const int32_t* Q_idx, const float* Q_val,
                   int64_t m, int64_t n, int32_t r, int32_t d,
                   void* plan, size_t plan_bytes, void* stream);

size_t lsp_plan_build_workspace_bytes(int64_t m, int64_t n, int32_t r, int32_t d);
int lsp_plan_build_async(const int32_t* P_idx, const float* P_val,
                         const int32_t* Q_idx, const float* Q_val,
                         int64_t m, int64_t n, int32_t r, int32_t d,
                         void* plan, size_t plan_bytes,
                         void* workspace, size_t workspace_bytes,
                         int32_t* status, void* stream);

int lsp_plan_build_host(const int32_t* P_idx, const float* P_val,
                        const int32_t* Q_idx, const float* Q_val,
                        int64_t m, int64_t n, int32_t r, int32_t d,
                        void* plan_host, size_t plan_bytes);

/* Same sums as lsp_compress, with the projectors given as a plan; gather form, no global
 * atomics unless a row of P^T has more than 256 entries (heavily skewed projectors), and
 * bit-reproducible from run to run whenever no row of P^T had to be cut for that reason
 * (columns of Q that are shared among several lanes are summed in a fixed order).
 * workspace: at least lsp_compress_planned_workspace_bytes(m,n,r,d) bytes.
 * The plan lives in device memory, so the host cannot check it: the kernels compare the (m, n, r,
 * d) recorded in the plan with those of the call, and when they differ (a plan built for another
 * problem, or a buffer that holds no plan) they follow none of its offsets, touch nothing but S
 * and fill S with NaN -- the call still returns LSP_OK, the mistake shows in S. */
int lsp_compress_planned(const void* G, const void* plan,
                         int64_t m, int64_t n, int32_t r, int32_t d,
                         float* S, lsp_dtype dtype,
                         void* workspace, size_t workspace_bytes, void* stream);

size_t lsp_compress_planned_workspace_bytes(int64_t m, int64_t n, int32_t r, int32_t d);

/* lsp_compress_planned for callers that cannot allocate device memory or hand in scratch: code
 * running under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same
 * arguments, results (bit for bit) and errors as lsp_compress_planned, without the workspace: the
 * m x r fp32 intermediate lives in an array of LSP_STATIC_SCRATCH_BYTES (24 MiB) that is part of
 * the library image; every GPU the library runs on holds one copy of it until the process ends.
 * The call makes no allocation of any kind.  A problem whose intermediate does not fit (m * r * 4
 * bytes, rounded up to 256, above the limit; 11008 x 512 fits) is refused with LSP_ERR_TOO_LARGE
 * and nothing is enqueued.
 * All calls on one GPU share the array: calls on one stream are ordered and safe, calls whose
 * kernels can overlap in time (different streams, different host threads' streams) race on it and
 * give undefined S.  The array keeps the previous call's contents; nothing in it needs clearing. */
int lsp_compress_planned_static(const void* G, const void* plan,
                                int64_t m, int64_t n, int32_t r, int32_t d,
                                float* S, lsp_dtype dtype, void* stream);
size_t lsp_static_scratch_bytes(void);   /* LSP_STATIC_SCRATCH_BYTES */

/* ------------------------------------------------------------------------------------------
 * Decompress and apply:  W := rn( W - P S Q^T ), in place.
 * The step "W <- W - eta_t P Delta_W Q^T" of Alg. 1 and the last step of the layer loop of
 * Alg. 3.  The learning rate is already folded into S by the CPU optimiser (P (eta S) Q^T =
 * eta P S Q^T), so there is no scale argument.  Each W element is widened exactly to fp32,
 * the update is accumulated in fp32, and the result is rounded once (nearest, ties to even)
 * to `dtype`.  Needs no workspace and no plan (the ELL rows are read as they are).
 *
 *   W          device, m*n elements of `dtype`, row-major, read and written
 *   S          device, r*r fp32, row-major, read
 */
int lsp_decompress_apply(void* W, const float* S,
                         const int32_t* P_idx, const float* P_val,
                         const int32_t* Q_idx, const float* Q_val,
                         int64_t m, int64_t n, int32_t r, int32_t d,
                         lsp_dtype dtype, void* stream);

/* ------------------------------------------------------------------------------------------
 * Grouped calls: several independent matrices in one call.
 * Alg. 3 walks the model layer by layer, and the weight matrices of one layer (their gradients
 * are all there when the layer's backward pass ends) are independent problems with the same
 * subspace size: a grouped call serves them with one launch per kernel, so that workgroups of
 * different matrices fill the GPU together.  Results are those of the single calls, matrix by
 * matrix, bit for bit.
 *
 *   items      HOST array of `count` descriptors (1 <= count <= LSP_MAX_GROUP); read during the
 *              call only; every pointer inside is a device pointer with the meaning, layout and
 *              alignment of the same-named argument of the single call
 *   r, d, dtype  shared by all problems of the group; m and n are per problem
 * Problems of a group run concurrently: every item needs its own S and its own workspace
 * (LSP_ERR_WORKSPACE otherwise), and a W may appear only once (LSP_ERR_SHAPE).  Errors are
 * those of the single calls; on any error nothing is enqueued.  The kernel variant is one that all
 * problems can use: an n that is no multiple of 4 (compress; bf16: of 8) or odd (apply) takes the whole group
 * to the variant for such rows (which gives the same results).
 */
typedef struct {
    const void* G;            /* device, m*n elements of `dtype` */
    const void* plan;         /* device, from lsp_plan_build for this problem's projectors */
    float*      S;            /* device, r*r fp32, written */
    void*       workspace;    /* device, >= lsp_compress_planned_workspace_bytes(m,n,r,d) */
    size_t      workspace_bytes;
    int64_t     m, n;
} lsp_compress_item;

typedef struct {
    void*          W;         /* device, m*n elements of `dtype`, read and written */
    const float*   S;         /* device, r*r fp32 */
    const int32_t* P_idx;     /* device, [m][d] */
    const float*   P_val;
    const int32_t* Q_idx;     /* device, [n][d] */
    const float*   Q_val;
    int64_t        m, n;
} lsp_apply_item;

int lsp_compress_planned_grouped(const lsp_compress_item* items, int32_t count,
                                 int32_t r, int32_t d, lsp_dtype dtype, void* stream);

int lsp_decompress_apply_grouped(const lsp_apply_item* items, int32_t count,
                                 int32_t r, int32_t d, lsp_dtype dtype, void* stream);

/* Optional preparation for the expand side (lsp_decompress_apply*, lsp_estimation_bias): a copy
 * of an ELL projector in which the d entries of every row are put in an order that makes the
 * kernels' LDS gathers collide less.  The projector is the same matrix (Def. 1 fixes which entries
 * a row has, not their order; they are summed), so the copy can be passed wherever Q is expected;
 * results differ only by the order of fp32 additions.  Meant for Q (the kernels gather by the
 * rows of Q); harmless for P.  Like the plan it is made once per change of projectors.
 *   idx, val           HOST, [rows][d]
 *   idx_out, val_out   HOST, [rows][d], distinct from the inputs
 * Returns LSP_OK, LSP_ERR_NULL, LSP_ERR_SHAPE or LSP_ERR_INDEX (an index outside [0, r)). */
int lsp_projector_reorder_host(const int32_t* idx, const float* val, int64_t rows, int32_t d, int32_t r,
                               int32_t* idx_out, float* val_out);
/* The same for DEVICE arrays: a set-up call like lsp_plan_build -- it waits for `stream`, copies the
 * arrays to the host (allocating host memory), reorders there and copies the result into the
 * device arrays idx_out / val_out; synchronous.  Adds LSP_ERR_LAUNCH to the errors above. */
int lsp_projector_reorder(const int32_t* idx, const float* val, int64_t rows, int32_t d, int32_t r,
                          int32_t* idx_out, float* val_out, void* stream);

/* ------------------------------------------------------------------------------------------
 * Dense-projector ablation of compress:  S := P^T G Q with DENSE projectors, on the matrix cores.
 * Def. 1 makes the projectors (d, r)-sparse, and the calls above never multiply by the zeros.  This call
 * is the yardstick for that choice: the same contraction with dense m x r and n x r projectors (what a
 * subspace method without the sparsity would run), as two matrix-core products in the storage type with
 * fp32 accumulation, T = G Q rounded to the storage type in between.  Its cost does not depend on d.
 *
 *   G          device, m*n elements of `dtype` (LSP_F16 or LSP_BF16; LSP_ERR_DTYPE otherwise), row-major
 *   Pt, Qt     device, the TRANSPOSED dense projectors P^T [r][m] and Q^T [r][n], row-major, in `dtype`
 *   S          device, r*r fp32, written
 *   workspace  device scratch of at least lsp_compress_dense_workspace_bytes(m, n, r) bytes, 16-byte aligned
 * Shapes: m a multiple of 128, n of 64, r of 128 (LSP_ERR_SHAPE otherwise; the size query then returns 0).
 * Asynchronous, three kernels, no atomics (bit-reproducible); all pointers 16-byte aligned.
 */
size_t lsp_compress_dense_workspace_bytes(int64_t m, int64_t n, int32_t r);
int lsp_compress_dense(const void* G, const void* Pt, const void* Qt,
                       int64_t m, int64_t n, int32_t r, float* S, lsp_dtype dtype,
                       void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------------------------
 * Estimation bias of the projector pair on a gradient (Def. 2):
 *     b(P, Q; G) = || P P^T G Q Q^T - G ||_F / || G ||_F ,
 * the quantity MaybeUpdate in Alg. 1 compares with its threshold alpha to decide whether the
 * projectors are fitted again.  It composes the two steps above: the caller first compresses G
 * (lsp_compress or lsp_compress_planned: S = P^T G Q, which the training step computes anyway),
 * then this call rebuilds P S Q^T tile by tile in registers in one more streaming pass over G,
 * subtracts G and adds up the squares; no m x n temporary exists.  fp32 arithmetic; the
 * workgroups' sums are added in a fixed order in fp64, so the result is bit-reproducible.
 *
 *   G          device, m*n elements of `dtype`, row-major, read only
 *   S          device, r*r fp32: P^T G Q of the same G and projectors, read only
 *   out        device, 3 floats, overwritten: out[0] = || P S Q^T - G ||_F^2,
 *              out[1] = || G ||_F^2, out[2] = sqrt(out[0] / out[1]) (NaN by IEEE rules if G = 0)
 *   workspace  device scratch of at least lsp_estimation_bias_workspace_bytes(m,n,r,d) bytes,
 *              16-byte aligned; contents undefined afterwards
 * Errors as for lsp_decompress_apply, plus LSP_ERR_WORKSPACE.  Asynchronous on `stream`.
 */
int lsp_estimation_bias(const void* G, const float* S,
                        const int32_t* P_idx, const float* P_val,
                        const int32_t* Q_idx, const float* Q_val,
                        int64_t m, int64_t n, int32_t r, int32_t d, float* out,
                        void* workspace, size_t workspace_bytes,
                        lsp_dtype dtype, void* stream);
size_t lsp_estimation_bias_workspace_bytes(int64_t m, int64_t n, int32_t r, int32_t d);

/* ------------------------------------------------------------------------------------------
 * Optimiser-state re-projection: the last two assignments of MaybeUpdate in Alg. 1.  When the
 * projectors (P_prev, Q_prev) of a matrix are replaced by (P, Q), the first and second moments
 * kept in the subspace follow:
 *     M := (P^T P_prev) M (Q_prev^T Q)         V := (P^T P_prev)^2 V (Q_prev^T Q)^2
 * with the squares taken element by element (the reading under which V is the second moment of
 * the re-projected first-moment terms and stays non-negative).  Runs once per change of
 * projectors, on the device copy of the moments.
 *
 *   P_*, Pprev_*   device, [m][d] ELL pairs of the new and the previous left projector
 *   Q_*, Qprev_*   device, [n][d] ELL pairs of the new and the previous right projector
 *   M              device, r*r fp32, row-major, read and overwritten
 *   V              device, r*r fp32, read and overwritten; may be NULL (no second moment); not M
 *   workspace      device scratch of at least lsp_reproject_state_workspace_bytes(r) bytes,
 *                  16-byte aligned; contents undefined afterwards
 * The two r x r products of sparse matrices are summed in fp64 in an order that is not fixed, and
 * rounded to fp32 once: the result can differ in the last bits from run to run.  The dense r x r products run in fp32 on the matrix
 * cores.  Errors as for the other calls; asynchronous on `stream`.
 */
int lsp_reproject_state(const int32_t* P_idx, const float* P_val,
                        const int32_t* Pprev_idx, const float* Pprev_val,
                        const int32_t* Q_idx, const float* Q_val,
                        const int32_t* Qprev_idx, const float* Qprev_val,
                        int64_t m, int64_t n, int32_t r, int32_t d,
                        float* M, float* V,
                        void* workspace, size_t workspace_bytes, void* stream);
size_t lsp_reproject_state_workspace_bytes(int32_t r);

/* ------------------------------------------------------------------------------------------
 * Projector fitting (the minimisation in MaybeUpdate, Alg. 1; Eq. 2): gradient of the data term
 *     F(P, Q) = 1/2 || P P^T G Q Q^T - G ||_F^2      (half the squared numerator of Def. 2's bias)
 * with respect to the stored projector values,
 *     gP[i][k] = dF / dP_val[i][k],      gQ[j][k] = dF / dQ_val[j][k]
 * (a stored value enters the dense projector linearly at its position, duplicates add; so two stored
 * entries of a row with the same column get the same derivative).  The paper's objective is
 * ||b||_F + beta * regulariser: its data term is sqrt(2 F), whose gradient is this one divided by ||b||_F
 * (lsp_estimation_bias gives the norm), and the regulariser -- written with different exponents in
 * Alg. 1 and in Eq. 2 -- is an element-wise function of the values; both are left to the caller's
 * optimiser.  fp32 arithmetic; G is streamed twice; no m x n temporary.
 *
 *   G            device, m*n elements of `dtype`, read only
 *   plan         device, the plan of these projectors WITH THEIR CURRENT VALUES (lsp_plan_build, or
 *                lsp_plan_refresh_values after the values changed); a plan of another problem makes
 *                every output NaN (see lsp_compress_planned)
 *   P_*, Q_*     device, the same projectors as ELL arrays
 *   gP, gQ       device, [m][d] and [n][d] fp32, overwritten
 *   workspace    device scratch of at least lsp_bias_gradient_workspace_bytes(m,n,r,d) bytes, 16-byte
 *                aligned; afterwards its first m*r floats hold T = G Q and the next r*r floats S = P^T G Q
 * The r x r products of sparse matrices inside are summed in fp64 in an order that is not fixed, and rounded
 * to fp32 once (results can differ in the last bits from run to run).  Errors as for lsp_estimation_bias.  Asynchronous on `stream`.
 */
int lsp_bias_gradient(const void* G, const void* plan,
                      const int32_t* P_idx, const float* P_val,
                      const int32_t* Q_idx, const float* Q_val,
                      int64_t m, int64_t n, int32_t r, int32_t d,
                      float* gP, float* gQ,
                      void* workspace, size_t workspace_bytes,
                      lsp_dtype dtype, void* stream);
size_t lsp_bias_gradient_workspace_bytes(int64_t m, int64_t n, int32_t r, int32_t d);

/* New values into an existing plan: for projectors whose positions (idx arrays) are unchanged since
 * the plan was built and whose values changed -- every iteration of projector fitting.  One small
 * kernel on `stream`; nothing is sorted again, the host is not involved, no synchronisation.
 *   plan         device, a plan built for (m, n, r, d) with the same P_idx / Q_idx; updated in place
 *                (a plan of another problem is left untouched)
 *   P_val/Q_val  device, [m][d] / [n][d], the new values
 */
int lsp_plan_refresh_values(void* plan, const float* P_val, const float* Q_val,
                            int64_t m, int64_t n, int32_t r, int32_t d, void* stream);

/* ------------------------------------------------------------------------------------------
 * The operators of a training step that are no plain matrix products: what a transformer block
 * does between its weights on the GPU ("forwardBackward", Alg. 1) and so what makes the weight
 * gradients that compress takes.  They follow the rules above (device pointers, no allocation, no
 * synchronisation, checks before the first HIP call).  Descriptors are HOST structures, read during
 * the call only.
 *
 * Dropout.  A mask is a function of (seed, offset, place) and is never stored, so the backward pass
 * makes the same one again.  Philox4x32 with 7 rounds (Salmon, Moraes, Dror and Shaw, "Parallel random
 * numbers: as easy as 1, 2, 3", SC 2011) under the key (low half of seed, high half) turns a counter
 * of four 32-bit words into eight 16-bit words, lower half of each output word first: one for each of
 * eight elements that follow one another.  An element is dropped when its word is below
 * t = round(65536 dropout) and otherwise scaled by 65536 / (65536 - t).  Counters: for an element of a
 * matrix, (low half, high half of row * ceil(width / 8) + column / 8, 0, offset); for a probability,
 * (key / 8, query, batch * heads + head, offset).  Calls whose masks have to be independent use
 * different offsets (or seeds); dropout 0 keeps everything as it is.
 *
 * lsp_dropout:  y := drop(x), element by element; its backward pass is the same call on the gradient.
 *   x, y   device, [rows][width] of `dtype`, rows one behind the other; y may be x; at most 2^31 blocks of eight
 */
int lsp_dropout(const void* x, void* y, int64_t rows, int64_t width, float dropout, uint64_t seed, uint32_t offset,
                lsp_dtype dtype, void* stream);

/* Attention:  O = drop(P) V,  P = softmax(scale Q K^T) over the keys that a query sees,
 *             L = log of the sum of exp(scale q . k) over these keys (fp32, kept for the backward pass).
 * Query i of batch b counts when i < q_lens[b], key j when j < k_lens[b] (lengths outside [0, q_len] and
 * [0, k_len] are taken as the nearer end; NULL: all count).  Query i sees key j when both count and,
 * if causal, j - k_lens[b] <= i - q_lens[b] (the last query sees every key).  A query that does not count
 * or sees nothing has O = 0, L = -infinity and gets and gives no gradient; rows that do not count are
 * not read (they may hold anything), but those of O, dQ, dK and dV are written (zeros).
 * Query head h reads key head h / (heads / kv_heads).
 *   Q, O, dO, dQ    device, [batch][q_len][heads][head_dim] of `dtype`; K, V, dK, dV  [batch][k_len][kv_heads][head_dim];
 *                   each with the strides given (of batch, position and head, in elements; the last axis is
 *                   contiguous), so views into a joint projection serve as they are.  Strides are multiples of
 *                   16 bytes and a position's is below 8 MiB.  In O, dQ, dK and dV every row has a place of its own: the stride of an
 *                   axis is at least what the axes of smaller strides span; and none of them overlaps another operand
 *   L               device, [batch][heads][q_len] fp32
 *   head_dim        a multiple of 8, at most LSP_MAX_HEAD_DIM;  scale > 0, at most 2^127;  batch * heads * (q_len or k_len) below 2^27
 *   and no launch of 2^24 workgroups or more: batch * heads * ceil(q_len / 128) below 2^24 (forward: batch * kv_heads, where the query heads of
 *   a key head have 128 rows or fewer together; backward: together with batch * kv_heads * ceil(k_len / 128))
 * The products run on the matrix cores in `dtype` with fp32 accumulation (fp32: in fp32); scores, softmax
 * statistics and sums are fp32; probabilities and the gradients of the scores are rounded to `dtype` as
 * operands of the second products, and dO . O is made of O as it is stored.  So in 16 bits O and dV are 1.3 to 1.4
 * times, dQ and dK 1.5 times as far from the exact ones as these rounded once; fp32 has no such roundings.  No
 * atomics: results are the same bits from run to run.
 * The backward pass computes the probabilities again from Q, K and L; it needs the same problem with O and L
 * as the forward pass left them.  Non-finite elements of a row that counts reach the rows that see it, and may
 * reach others.
 * Workspaces: 16-byte aligned, as large as the queries say (0 bytes needed: may be NULL). */
typedef struct {
    const void*    Q;
    const void*    K;
    const void*    V;
    void*          O;
    float*         L;
    const int32_t* q_lens;         /* device, [batch], or NULL */
    const int32_t* k_lens;
    int64_t q_stride[3], k_stride[3], v_stride[3], o_stride[3];   /* batch, position, head */
    int32_t batch, heads, kv_heads, q_len, k_len, head_dim;
    int32_t causal;                /* 0 or 1 */
    float   scale, dropout;
    uint32_t offset;
    uint64_t seed;
} lsp_attention_problem;

typedef struct {
    const void* dO;
    void*       dQ;
    void*       dK;
    void*       dV;
    int64_t do_stride[3], dq_stride[3], dk_stride[3], dv_stride[3];
} lsp_attention_gradients;

size_t lsp_attention_forward_workspace_bytes(const lsp_attention_problem* problem, lsp_dtype dtype);
int    lsp_attention_forward(const lsp_attention_problem* problem, lsp_dtype dtype, void* workspace, size_t workspace_bytes, void* stream);
size_t lsp_attention_backward_workspace_bytes(const lsp_attention_problem* problem, lsp_dtype dtype);
int    lsp_attention_backward(const lsp_attention_problem* problem, const lsp_attention_gradients* gradients, lsp_dtype dtype,
                              void* workspace, size_t workspace_bytes, void* stream);

/* Between two blocks:  u = norm(f) (after a block),  y = residual_scale x + branch_scale gate * drop(u)
 * (the residual stream),  h = norm(y) (before the next block), each row by itself:
 *   LSP_NORM_NONE   norm(v) = v                        (weight and bias are ignored)
 *   LSP_NORM_RMS    norm(v) = v / sqrt(mean(v^2) + eps) * weight [+ bias]
 *   LSP_NORM_LAYER  norm(v) = (v - mean(v)) / sqrt(mean((v - mean(v))^2) + eps) * weight [+ bias]
 * All in fp32; y and h are rounded once each (h is made from the y before rounding).
 *   x, f, y, h      device, [rows][width] of `dtype` with the row strides given (elements, at least width).  y and h may each be x or
 *                   f, row on row, or one the other (h stays); h may be NULL, with pre = LSP_NORM_NONE
 *   weights, biases, gate   device, [width] of `dtype`; NULL: ones, zeros, ones
 *   stats           device, [4][rows] fp32, kept for the backward pass: mean of f, 1 / deviation of f, the same of y
 * The backward pass takes the gradients of y (dy) and h (dh; NULL where h is) and gives those of x and f and,
 * where asked for (not NULL), of the weights, biases and gate (fp32, [width], overwritten; sums over the rows in an
 * order that does not change from run to run).  It needs x and f as the forward pass had them (so neither y nor h
 * may be one of them then), and its stats.  dx and df may each be dy, dh, x or f, row on row, or one the other (df stays).
 * Otherwise what is written overlaps nothing else. */
typedef enum { LSP_NORM_NONE = 0, LSP_NORM_RMS = 1, LSP_NORM_LAYER = 2 } lsp_norm;

typedef struct {
    const void* x;
    const void* f;
    void*       y;
    void*       h;
    float*      stats;
    const void* post_weight;       /* of the norm of f */
    const void* post_bias;
    const void* gate;
    const void* pre_weight;        /* of the norm of y */
    const void* pre_bias;
    int64_t x_stride, f_stride, y_stride, h_stride;
    int64_t rows;
    int32_t width;
    int32_t post, pre;             /* lsp_norm */
    float   eps, residual_scale, branch_scale, dropout;
    uint32_t offset;
    uint64_t seed;
} lsp_residual_norm_problem;

typedef struct {
    const void* dy;
    const void* dh;
    void*       dx;
    void*       df;
    float*      post_weight;
    float*      post_bias;
    float*      gate;
    float*      pre_weight;
    float*      pre_bias;
    int64_t dy_stride, dh_stride, dx_stride, df_stride;
} lsp_residual_norm_gradients;

int    lsp_residual_norm_forward(const lsp_residual_norm_problem* problem, lsp_dtype dtype, void* stream);
size_t lsp_residual_norm_backward_workspace_bytes(const lsp_residual_norm_problem* problem, lsp_dtype dtype);
int    lsp_residual_norm_backward(const lsp_residual_norm_problem* problem, const lsp_residual_norm_gradients* gradients, lsp_dtype dtype,
                                  void* workspace, size_t workspace_bytes, void* stream);

/* Rotary positions with norms of the heads, between the joint projection and attention:
 *   Qr = rotate(norm(Q)),  Kr = rotate(norm(K)),  and, where it is asked for, Vr = V,
 * each head of each token by itself.  norm: lsp_norm over the head_dim elements of a head, with weight [+ bias] as below (LSP_NORM_NONE: not
 * read).  rotate: pair j < rotated / 2 of a head turns by the angle position * frequencies[j],
 *   (a, b) -> (a cos - b sin, a sin + b cos);   elements from `rotated` on stay.
 * A pair is elements (j, rotated / 2 + j) or, with neighbours = 1, (2 j, 2 j + 1).  Angles are computed in fp64 with what its roundings
 * take off (a far position keeps all digits, as long as position * frequency is below 2^70), their sines, the norms and the turning in fp32; the result is rounded once.
 * Token i of text b counts when i < lens[b] (lengths outside [0, length] are taken as the nearer end; NULL: all count).  Its position is
 * positions[b][i] or, where that is NULL, starts[b] + i (starts NULL: i).  Its key goes to place starts[b] + i of the text's `cache` places in Kr, and its
 * value there in Vr, so that the caches that lsp_attention_forward reads are filled by the call that turns the keys (cache = length and starts =
 * NULL: tensors like K).  Tokens that do not count are not read, and their rows not written; nor are places outside [0, cache).
 *   Q, Qr, dQr, dQ  device, [batch][length][heads][head_dim] of `dtype`; K, V, dK  [batch][length][kv_heads][head_dim];
 *   Kr, Vr, dKr     [batch][cache][kv_heads][head_dim]; each with strides as in attention (multiples of 16 bytes, a position's below 8 MiB, and here a
 *                   head's below 256 MiB; in what is written every row has a place of its own).  V and Vr may be NULL, both.
 *   Qr may be Q and, where starts is NULL, Kr may be K and Vr V, row on row.  Otherwise what is written overlaps nothing else.
 *   q_weight, k_weight, q_bias, k_bias   device, [head_dim] of `dtype`; NULL: ones, zeros
 *   frequencies     device, [rotated / 2] fp32, radians a position; NULL only where rotated = 0
 *   head_dim, rotated   multiples of 8, rotated <= head_dim <= LSP_MAX_HEAD_DIM;  batch * length * (heads + 2 kv_heads) below 2^31
 * The backward pass gives dQ and dK from dQr and dKr (of tokens that do not count zeros, without reading anything; a key whose place is outside the
 * cache has gradient zero) and, where asked for (not NULL), the gradients of weights and biases (fp32, [head_dim], overwritten; sums over tokens and
 * heads in an order that does not change from run to run).  It needs Q and K as the forward pass had them where there is a norm (so Qr and Kr may
 * not be on them then).  dQ may be dQr or Q, row on row, and, where starts is NULL, dK may be dKr or K. */
typedef struct {
    const void*    Q;
    const void*    K;
    const void*    V;
    void*          Qr;
    void*          Kr;
    void*          Vr;
    const void*    q_weight;
    const void*    k_weight;
    const void*    q_bias;
    const void*    k_bias;
    const float*   frequencies;
    const int32_t* positions;      /* device, [batch][length], or NULL */
    const int32_t* starts;         /* device, [batch], or NULL */
    const int32_t* lens;
    int64_t q_stride[3], k_stride[3], v_stride[3], qr_stride[3], kr_stride[3], vr_stride[3];   /* batch, position, head */
    int32_t batch, length, cache, heads, kv_heads, head_dim, rotated;
    int32_t neighbours;            /* 0 or 1 */
    int32_t norm;                  /* lsp_norm */
    float   eps;
} lsp_rotary_problem;

typedef struct {
    const void* dQr;
    const void* dKr;
    void*       dQ;
    void*       dK;
    float*      q_weight;
    float*      k_weight;
    float*      q_bias;
    float*      k_bias;
    int64_t dqr_stride[3], dkr_stride[3], dq_stride[3], dk_stride[3];
} lsp_rotary_gradients;

int    lsp_rotary_forward(const lsp_rotary_problem* problem, lsp_dtype dtype, void* stream);
size_t lsp_rotary_backward_workspace_bytes(const lsp_rotary_problem* problem, lsp_dtype dtype);
int    lsp_rotary_backward(const lsp_rotary_problem* problem, const lsp_rotary_gradients* gradients, lsp_dtype dtype,
                           void* workspace, size_t workspace_bytes, void* stream);

/* Softmax cross entropy over a vocabulary, from the last hidden states:  z = H W^T (never stored),
 *   L = log(sum over the vocabulary of exp(z)),
 *   losses = L - (1 - smoothing) z[target] - smoothing mean(z) + z_loss L^2,  row by row.
 * A row whose target is outside [0, vocab) does not count: it is not read, its loss and L are 0, and it gets and gives no gradient.
 *   H        device, [rows][width] of `dtype`;  W  [vocab][width]; with row strides (elements), multiples of 16 bytes below 8 MiB
 *   targets  device, [rows] int64
 *   losses   device, [rows] fp32;  logs: the same for L, or NULL
 *   all of them, and weights, 16-byte aligned;  width    a multiple of 8, at most 2^16;  rows at most LSP_MAX_ROWS;  vocab at most 2^20;  0 <= smoothing < 1;  0 <= z_loss <= 1
 * lsp_cross_entropy_backward gives losses and logs too (it needs no forward call before it), and the gradients of
 *   scale * sum over the rows of weights * losses
 * with respect to H (dH, rows that do not count: zeros) and W (dW), overwritten; either may be NULL.  What is written overlaps nothing else.  weights: device, [rows] fp32, or NULL: ones (of rows that
 * do not count not used); scale is finite.
 * The products run on the matrix cores in `dtype` with fp32 accumulation (fp32: in fp32).  Rows are taken in blocks; for a block the
 * exponentials are kept in 16 bits (fp32: in 32), each relative to the largest of its row in a piece of the vocabulary (what is below 2^-29 of that loses digits, and is 0 below
 * 2^-40), and become the gradient of z in place, rounded to `dtype` before the second products; a target's is p - 1 of z in fp32, and dH has it without that rounding.  No atomics that add:
 * results are the same bits from run to run.  A logit that is not finite reaches its row's loss and dH, and all of dW.
 * fp16: the gradients of z have one scale, by the largest |weight|; a row whose weight is 2^-18 of that loses digits of its small probabilities' gradients, and one of 2^-38 has none of them left.
 * Workspaces: 16-byte aligned, as large as the queries say: bounded but for 4 bytes a row, however many there are. */
typedef struct {
    const void*    H;
    const void*    W;
    const int64_t* targets;
    float*         losses;
    float*         logs;
    int64_t h_stride, w_stride;
    int64_t rows;
    int32_t width, vocab;
    float   smoothing, z_loss;
} lsp_cross_entropy_problem;

typedef struct {
    void*        dH;
    void*        dW;
    const float* weights;
    int64_t dh_stride, dw_stride;
    float   scale;
} lsp_cross_entropy_gradients;

size_t lsp_cross_entropy_forward_workspace_bytes(const lsp_cross_entropy_problem* problem, lsp_dtype dtype);
int    lsp_cross_entropy_forward(const lsp_cross_entropy_problem* problem, lsp_dtype dtype, void* workspace, size_t workspace_bytes, void* stream);
size_t lsp_cross_entropy_backward_workspace_bytes(const lsp_cross_entropy_problem* problem, lsp_dtype dtype);
int    lsp_cross_entropy_backward(const lsp_cross_entropy_problem* problem, const lsp_cross_entropy_gradients* gradients, lsp_dtype dtype,
                                  void* workspace, size_t workspace_bytes, void* stream);

/* One step of AdamW (Loshchilov and Hutter, "Decoupled weight decay regularization", ICLR 2019) over many tensors, for the parameters that have no projector:
 *   g = grad_scale grad,  m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2,
 *   param -= rate * rate_factor * (decay param + (m / (1 - beta1^step)) / (sqrt(v / (1 - beta2^step)) + eps)),   all in fp32, in place.
 * Each tensor has its own types, decay and factor of the rate.  Where there is a master (fp32), it is what is updated, and param becomes it rounded; otherwise
 * param itself is read and rounded once.
 * LSP_STATE_F32: m and v are fp32.  LSP_STATE_8BIT: bytes; 256 elements that follow one another (the last ones of a tensor: fewer) share an fp32 scale.  m is e4m3 (4 bits
 * of exponent, 3 of mantissa, largest 448) times m_scale; v is without sign, 5 bits of exponent and 3 of mantissa: code 0 is 0 and code c otherwise
 * 2^((c >> 3) - 31) * (1 + (c & 7) / 8) (largest 1.875), times v_scale.  The step takes m and v before they are rounded (to nearest, ties to even; a v
 * that is not 0 never becomes 0 (but below 2^-149 of the largest), so that no small v makes a large step); a scale is the block's largest magnitude over 448 or 1.875.  State that is all zeros,
 * codes and scales, is where training begins.  A gradient that is not finite, or whose
 * square is not in fp32, spoils its element and, in 8 bits, can spoil its block's states.
 *   items       HOST array of `count` descriptors, 1 <= count <= LSP_MAX_TENSORS, read during the call only; no tensor twice, no overlaps
 *   step        number of this step, from 1 on (a captured call repeats it);  0 <= beta < 1, eps >= 0 (an element whose m and v are 0 gets no update but decay, whatever eps is)
 *   grad_scale  device, one fp32 (of clipping, or of a scaled loss), or NULL: 1.  Where it is not finite the step does nothing
 * At most 2^35 elements a tensor, and in all, each tensor padded to a multiple of 4096, fewer than 2^36.  Tensors are 16-byte aligned, scales and grad_scale 4-byte. */
typedef enum { LSP_STATE_F32 = 0, LSP_STATE_8BIT = 1 } lsp_state;

typedef struct {
    void*       param;             /* device, [elements] of `dtype` */
    const void* grad;              /* device, [elements] of `grad_dtype` */
    void*       m;                 /* device, [elements] fp32, or bytes */
    void*       v;
    float*      m_scale;           /* device, [ceil(elements / 256)]; LSP_STATE_8BIT only */
    float*      v_scale;
    float*      master;            /* device, [elements] fp32, or NULL */
    int64_t     elements;
    float       rate_factor, decay;
    int32_t     dtype, grad_dtype; /* lsp_dtype */
} lsp_adamw_item;

int lsp_adamw(const lsp_adamw_item* items, int32_t count, lsp_state states, double rate, double beta1, double beta2, double eps, int64_t step,
              const float* grad_scale, void* stream);

/* ------------------------------------------------------------------------------------------
 * Utilities.
 */

/* Checks every idx[row][k] against [0, r).  Enqueues a kernel on `stream`, then WAITS for it
 * (this call synchronises the stream).  Returns LSP_OK or LSP_ERR_INDEX.
 * flag: device, one int32 of scratch. */
int lsp_validate_projector(const int32_t* idx, int64_t rows, int32_t d, int32_t r,
                           int32_t* flag, void* stream);

/* Measurement aids (not part of the method): one plain streaming pass over `bytes` bytes of device
 * memory (a multiple of 16; fp32 data for the second call), to find out what a kernel with nothing
 * but the stream in it reaches on this GPU.  lsp_hbm_probe_read reads every byte once (compress reads G
 * once) and leaves one float per workgroup in `workspace` (>= lsp_hbm_probe_workspace_bytes(bytes));
 * lsp_hbm_probe_rmw does y[i] -= c on fp32 data (decompress-apply reads and writes W once).  Asynchronous
 * on `stream`; errors as above. */
size_t lsp_hbm_probe_workspace_bytes(size_t bytes);
int    lsp_hbm_probe_read(const void* buf, size_t bytes, void* workspace, size_t workspace_bytes, void* stream);
int    lsp_hbm_probe_rmw(void* buf, size_t bytes, float c, void* stream);

const char* lsp_strerror(int code);      /* static string for an lsp_status */
int         lsp_last_hip_error(void);    /* raw hipError_t of the last LSP_ERR_LAUNCH on this thread */
int         lsp_version(void);           /* major*10000 + minor*100 + patch */

#ifdef __cplusplus
}
#endif
#endif /* LSP_H */
