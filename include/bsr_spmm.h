/*
 * bsr_spmm -- block-sparse times dense product for AMD MI355X (gfx950).
 *
 *     Y = X * W^T        X dense (m, k), W block-sparse (n, k) in BSR, Y dense (m, n)
 *
 * The operation and the storage format are those of the paper's Background
 * section (the three arrays block_data / block_indices / index_pointer, W kept
 * as (n, k) so that a block-row of W produces a run of consecutive columns of
 * Y) and of the unnumbered equation in its Approaches section (X W_B^T = Y
 * with b_r | n and b_c | k):
 *
 *     block_data[p][a][c] = W[r*bs_r + a][block_indices[p]*bs_c + c]
 *         for p in [index_pointer[r], index_pointer[r+1])
 *     Y[i][r*bs_r + a]    = sum_p sum_c X[i][block_indices[p]*bs_c + c] * block_data[p][a][c]
 *
 * Conventions for every entry point
 *   - plain C ABI; every function returns a bsr_status, never throws or aborts;
 *   - "host" pointers are ordinary CPU memory, "device" pointers are GPU
 *     memory of the current HIP device; the library never allocates or frees
 *     device memory (the caller does, e.g. with PyTorch) and never takes
 *     ownership of a caller's buffer;
 *   - dense matrices are row-major and contiguous; index arrays are int32;
 *   - `hip_stream` is a hipStream_t passed as void* (NULL = the default stream);
 *     device work is queued on it and the call returns without waiting.
 *
 * Debug mode.  A handle created while the environment variable BSR_SPMM_DEBUG is set to anything but "0"
 * re-checks, on the device and before every product (bsr_spmm, bsr_spmm_ex, bsr_spmm_static, bsr_spmm_epilogue, bsr_sddmm,
 * bsr_sddmm_ws), the arrays every kernel address derives from: index_pointer and block_indices as they are in device
 * memory at that moment (BSR_ERR_INDPTR, BSR_ERR_INDEX) and the plan in the workspace
 * (BSR_ERR_WORKSPACE when it no longer holds what bsr_create() wrote, or the first product that wanted more of
 * it).  On a failure nothing else is launched.  The check waits for the stream (one extra launch, a 16-byte copy, a synchronisation), so
 * such a call is NOT asynchronous; it is skipped while the stream is being captured into a graph.
 */
#ifndef BSR_SPMM_H
#define BSR_SPMM_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of X, block_data and Y.  Accumulation is always fp32. */
typedef enum { BSR_F32 = 0, BSR_F16 = 1, BSR_BF16 = 2 } bsr_dtype;

typedef enum {
    BSR_OK = 0,
    BSR_ERR_NULL = 1,        /* a required pointer is NULL */
    BSR_ERR_SHAPE = 2,       /* negative size, bs_r <= 0, bs_c <= 0, bs_r !| n, bs_c !| k (Approaches: b_r | n, b_c | k),
                                or a size that does not fit the int32 index arithmetic */
    BSR_ERR_INDPTR = 3,      /* index_pointer[0] != 0, decreasing, or last entry != nnzb */
    BSR_ERR_INDEX = 4,       /* a block_indices entry outside [0, k/bs_c) */
    BSR_ERR_DTYPE = 5,       /* unknown dtype, or y_dtype neither the input type nor BSR_F32 */
    BSR_ERR_ALIGN = 6,       /* a device pointer is not 16-byte aligned */
    BSR_ERR_WORKSPACE = 7,   /* workspace smaller than bsr_workspace_size() reports, or the chosen kernel needs
                                scratch (bsr_scratch_size) that has not been lent with bsr_set_scratch */
    BSR_ERR_HIP = 8,         /* a HIP runtime call failed (launch, copy), or bsr_create() found no host memory for its plan */
    BSR_ERR_UNSUPPORTED = 9, /* the requested kernel path cannot handle this block shape */
    BSR_ERR_SCRATCH_LIMIT = 10,/* bsr_spmm_static(): the product needs more scratch than the library's built-in
                                  BSR_STATIC_SCRATCH_BYTES */
    BSR_ERR_OVERLAP = 11,    /* a buffer that is written overlaps another one of the call */
    BSR_ERR_DEVICE = 12      /* the handle was created on another device than the current one (bsr_spmm_epilogue, bsr_adamw_*) */
} bsr_status;

/* Which kernel family bsr_spmm_ex() uses. */
typedef enum {
    BSR_PATH_AUTO = 0,   /* the library's choice for this matrix and m */
    BSR_PATH_WAVE = 1,   /* wavefront-reduction kernels: lanes split the reduction inside and across the
                            stored blocks of a block-row, cross-lane sum at the end (the paper's
                            "parallelize within blocks" + "aggregate partial results", Sections 4.4.2-4.4.3);
                            any block shape */
    BSR_PATH_MFMA = 2    /* matrix-core kernels: one workgroup owns an (m-tile, block-row) tile of Y and walks
                            the stored blocks of the block-row (the tile-per-thread-block design of the paper's
                            "Utilizing shared memory" section, with run-time indices); block shapes listed at
                            bsr_spmm_ex() */
} bsr_path;

typedef struct bsr_matrix bsr_matrix;   /* opaque handle: shape, device pointers (not owned), plan */

/*
 * Structural check of a BSR pattern (Background: the three arrays).  HOST pointers.
 *   n, k        rows / columns of W;   bs_r, bs_c  block shape (bs_r | n, bs_c | k)
 *   nnzb        number of stored blocks
 *   index_pointer_host  n/bs_r + 1 entries: starts at 0, non-decreasing, ends at nnzb
 *   block_indices_host  nnzb entries in [0, k/bs_c); any order inside a block-row, duplicates allowed
 *                       (duplicates are summed, as the definition sums over stored blocks)
 * Returns BSR_OK or the first problem found (NULL, SHAPE, INDPTR, INDEX in that order).
 */
bsr_status bsr_validate(int64_t n, int64_t k, int32_t bs_r, int32_t bs_c, int64_t nnzb,
                        const int32_t* index_pointer_host, const int32_t* block_indices_host);

/*
 * Bytes of DEVICE workspace bsr_create() needs for its plan (block-row order and work lists).
 * Always > 0 and a multiple of 256.  Errors: NULL, SHAPE.
 */
bsr_status bsr_workspace_size(int64_t n, int64_t k, int32_t bs_r, int32_t bs_c, int64_t nnzb,
                              size_t* bytes);

/*
 * Build a handle for W.  Validates the pattern (as bsr_validate), bins the block-rows by
 * their number of stored blocks and orders them longest first (the paper's Discussion: rows
 * with very different block counts make equal-sized work units diverge), and copies that
 * plan into `workspace_dev` on `hip_stream` (asynchronous; the host staging copy is owned by
 * the handle).
 *   block_data_dev     DEVICE, nnzb*bs_r*bs_c elements of `dtype`, [nnzb][bs_r][bs_c] row-major
 *   block_indices_dev  DEVICE, nnzb int32          index_pointer_dev  DEVICE, n/bs_r+1 int32
 *   block_indices_host / index_pointer_host        HOST copies of the same two arrays, read during
 *                                                  this call only
 *   workspace_dev      DEVICE, at least bsr_workspace_size() bytes, 16-byte aligned
 * The four device buffers stay owned by the caller and must outlive the handle, the products that are
 * still to run (on any stream) and the graphs that hold some; their contents (block values included) may
 * change between products as long as the pattern does not.
 * nnzb == 0 is valid (Y becomes all zeros); then block_data_dev / block_indices_* may be NULL.
 * On error *out is set to NULL.
 */
bsr_status bsr_create(bsr_matrix** out, int64_t n, int64_t k, int32_t bs_r, int32_t bs_c, int64_t nnzb,
                      bsr_dtype dtype, const void* block_data_dev,
                      const int32_t* block_indices_dev, const int32_t* index_pointer_dev,
                      const int32_t* block_indices_host, const int32_t* index_pointer_host,
                      void* workspace_dev, size_t workspace_bytes, void* hip_stream);

/* Frees the handle's host memory only (after waiting for a plan upload that may still read it).
 * NULL is accepted. */
void bsr_destroy(bsr_matrix* W);

/*
 * Y[m][n] = X[m][k] * W^T  (Approaches, the equation; overwrite, not accumulate).
 *   X_dev   DEVICE, m*k elements of W's dtype, row-major      Y_dev  DEVICE, m*n elements of y_dtype
 *   y_dtype W's dtype or BSR_F32; the fp32 accumulator is rounded to nearest-even on store
 *   m       any value >= 0 (m == 0 returns BSR_OK without device work)
 * Every element of Y is written; columns of an empty block-row are exact zeros.  Asynchronous on
 * `hip_stream`; no hidden synchronisation.  A product may be queued on any stream: until the plan
 * upload that bsr_create() queued on its own stream has finished, products make their stream wait
 * for it (an event wait on the device, not on the host).  Products on one handle may run
 * concurrently (unless they use lent scratch, see bsr_set_scratch): some kernels read a per-m work
 * list that the first product of that m uploads into the workspace (the handle keeps the lists of
 * the 4 most recent values of m; other streams wait for that upload the same way).  With more than
 * 4 distinct m in flight at once on one handle a list may be replaced while an earlier product still
 * reads it: keep such products ordered on one stream.
 * A product recorded into a graph uses such a list only if an eager product of that m has uploaded it before and the
 * upload is over; the list is then kept for the graph's replays (up to 3 values of m per handle, as long as the handle
 * or its workspace lives).  Otherwise it is recorded without one: the same result, less evenly spread over the CUs.
 * Likewise the kernel that sweeps blocks with sides of 8 or 16 has a plan that the first product that wants it builds (host
 * time: 0.05 ms for 3000 stored blocks, 0.7 ms for 50000) and uploads; a product recorded before that runs on another kernel.
 * (16-bit blocks with one side of 8, n and k multiples of 16: built by bsr_create().)
 * NaN or Inf in X: kernels that fill their last, partial group of blocks with zero-valued dummy
 * blocks multiply those zeros by real entries of X (the thin-block kernels: by column 0 of X), so a
 * non-finite entry there can reach outputs it does not belong to; so do kernels that multiply blocks of 8 rows or columns
 * in 16x16 tiles or two block-rows at a time (n and k multiples of 16: for other sizes such outputs are summed again from
 * their own blocks).  Finite inputs are unaffected.
 * Errors: NULL, SHAPE (m < 0 or m*max(k,n) >= 2^31), DTYPE, ALIGN, HIP.
 */
bsr_status bsr_spmm(const bsr_matrix* W, int64_t m, const void* X_dev, void* Y_dev,
                    bsr_dtype y_dtype, void* hip_stream);

/*
 * The product with what a layer does to it before it is stored (bsr_spmm_epilogue), in the same launches:
 *     z = (X W^T)[i][j] + bias[j]            Z[i][j] = z                       if z_dev
 *     y = act(z)                             or z * act'(Z0[i][j])             with through_dev = Z0
 *     Y[i][j] = y + R[i][j]                                                    if residual_dev = R
 * In training, Z is what the activation's gradient is taken at (bsr_epilogue_backward); `through` takes a gradient through
 * the activation in front of the layer whose W^T is multiplied: Y = (G W) * act'(Z0).  All of it is fp32 arithmetic on the
 * accumulated sum; what is stored is rounded once, to nearest-even, and act(z) sees the z before that rounding.
 *   act             BSR_ACT_*: none; max(z, 0); z Phi(z), Phi the normal distribution's integral (relative error below
 *                   1.5e-6 + 2^-23 z^2 down to z = -12.9, where Phi is below fp32's normal numbers, and below 1.5e-6 for
 *                   positive z); z (1 + tanh(sqrt(2 / pi) (z + 0.044715 z^3))) / 2; z / (1 + exp(-z))
 *   bias_dev        DEVICE, n elements of bias_dtype (W's dtype or BSR_F32), or NULL
 *   residual_dev    DEVICE, m rows of n elements of y_dtype, `residual_ld` elements apart (0: n, contiguous), or NULL
 *   through_dev     DEVICE, Z0, m*n elements of y_dtype, or NULL; not read where act is BSR_ACT_NONE (slope 1)
 *   z_dev           DEVICE, m*n elements of y_dtype, every one written, or NULL
 * Fill unused members with zeros.  A NaN stays a NaN; at an infinite z the activations' and slopes' limits are taken.
 */
typedef enum { BSR_ACT_NONE = 0, BSR_ACT_RELU = 1, BSR_ACT_GELU = 2, BSR_ACT_GELU_TANH = 3, BSR_ACT_SILU = 4 } bsr_act;
typedef struct {
    bsr_act act;
    bsr_dtype bias_dtype;
    const void* bias_dev;
    const void* residual_dev;
    int64_t residual_ld;
    const void* through_dev;
    void* z_dev;
} bsr_epilogue;

/*
 * As bsr_spmm() -- the same kernels, choices, streams and captures; those of bsr_tune(), which times the product alone, too, but
 * three or four blocks in flight are two here -- with `epilogue` (HOST, read during the call).  Y and Z must overlap neither
 * each other nor any input (a residual is not added in place), nor the handle's arrays, its workspace and what has been lent
 * as scratch.
 * Errors: as bsr_spmm(), plus NULL (epilogue), DTYPE (act, bias_dtype), SHAPE (residual_ld below n, or m * residual_ld
 * >= 2^37), ALIGN (a pointer not 16-byte aligned, or rows of a residual that are neither contiguous nor multiples of
 * 16 bytes apart), OVERLAP, DEVICE.
 */
bsr_status bsr_spmm_epilogue(const bsr_matrix* W, int64_t m, const void* X_dev, void* Y_dev, bsr_dtype y_dtype,
                             const bsr_epilogue* epilogue, void* hip_stream);

/*
 * The gradient of that epilogue, from G = dL/dY:
 *     dZ[i][j] = G[i][j] * act'(Z[i][j])          db[j] = sum over i of dZ[i][j]
 * dZ is what the layer's own gradients are taken of -- bsr_sddmm(W, dZ, X), bsr_spmm(handle of W^T, dZ) -- and db is the
 * bias's.  (The residual's gradient is G itself.)  One pass over G and Z; the sums are fp32, of dZ before its rounding, and
 * added in a fixed order (no atomics).
 *   G_dev, Z_dev   DEVICE, m*n elements of g_dtype, row-major; Z_dev is not read where act is BSR_ACT_NONE (may be NULL)
 *   DZ_dev         DEVICE, m*n elements of dz_dtype (g_dtype, or any type where g_dtype is BSR_F32), or NULL; it may be
 *                  G_dev or Z_dev itself where the types are the same
 *   DB_dev         DEVICE, n floats, or NULL (not both NULL); m == 0: zeros
 *   workspace_dev  DEVICE, bsr_epilogue_backward_workspace_size() bytes (0: none, it may be NULL), overwritten; read only
 *                  where DB_dev is given.  Calls that may run at the same time, replayed graphs among them, need one each.
 * Asynchronous on hip_stream.  Errors: NULL, SHAPE (m or n negative, m >= 2^30, n >= 2^28, or m*n >= 2^40), DTYPE,
 * ALIGN (a pointer not 16-byte aligned), WORKSPACE, OVERLAP, HIP.
 */
bsr_status bsr_epilogue_backward_workspace_size(int64_t m, int64_t n, size_t* bytes);
bsr_status bsr_epilogue_backward(int64_t m, int64_t n, bsr_act act, bsr_dtype g_dtype, const void* G_dev, const void* Z_dev,
                                 bsr_dtype dz_dtype, void* DZ_dev, float* DB_dev, void* workspace_dev, size_t workspace_bytes,
                                 void* hip_stream);

/*
 * Scratch.  Some kernels need device memory beyond X, W and Y for the duration of one product:
 * for thin blocks (bs_r = 16, bs_c = 1, fp32) one matrix-core path first writes a transposed copy of
 * X, m*k floats, so that the columns of X that the stored blocks select (Background: the block's
 * column index picks the part of X) become contiguous rows.  The library does not allocate it.
 *   bsr_scratch_size  bytes such a product with m rows would use (0 when no kernel for this W
 *                     needs scratch); multiple of 256.
 *   bsr_set_scratch   lends `bytes` of DEVICE memory (16-byte aligned) to the handle, or takes it
 *                     back with NULL.  The memory stays owned by the caller and must outlive its
 *                     use; products that use it must not overlap in time on one handle (they
 *                     share it), i.e. keep them on one stream.
 * A thin-block W whose block-rows store their blocks in non-decreasing block-column order (k a
 * multiple of 4, at most 64512) needs none: its product runs in one launch that gathers the columns
 * from rows of X staged in LDS, and is preferred unless the block-rows are dense (more than 80 blocks
 * per 1024 columns on average).  For any other thin-block W, without (enough) scratch BSR_PATH_AUTO
 * uses the wavefront-reduction kernels and BSR_PATH_MFMA returns BSR_ERR_WORKSPACE.
 */
bsr_status bsr_scratch_size(const bsr_matrix* W, int64_t m, size_t* bytes);
bsr_status bsr_set_scratch(bsr_matrix* W, void* scratch_dev, size_t bytes);

/*
 * As bsr_spmm() with the kernel family fixed.  BSR_PATH_MFMA needs bs_r and bs_c in {16, 32, 64};
 * or bs_r and bs_c in {8, 16} with n and k multiples of 16 (the blocks are grouped into 16x16
 * tiles), with other n and k where bsr_query_path() answers BSR_PATH_MFMA for this m; or the thin shape bs_c == 1 with bs_r == 16 and fp32; or its transpose, bs_r == 1 with bs_c == 16,
 * fp32, fp32 output and no block stored twice; otherwise BSR_ERR_UNSUPPORTED.
 * BSR_PATH_WAVE takes any shape.
 */
bsr_status bsr_spmm_ex(const bsr_matrix* W, int64_t m, const void* X_dev, void* Y_dev,
                       bsr_dtype y_dtype, bsr_path path, void* hip_stream);

/*
 * Plan-time tuning by timed trials ("Automatic parameter tuning": the paper picks its kernels'
 * parameters per input shape by running the candidates).  Runs the product for every candidate
 * kernel and setting the library has for this W, this m and this output type -- 2 warm-up and
 * `trials` timed launches each (trials < 1: 20), timed with events on `hip_stream` -- and remembers
 * the fastest in the handle: later bsr_spmm() / BSR_PATH_AUTO calls with the same m and y_dtype use
 * it.  Every candidate computes the same product, so Y_dev holds Y = X * W^T afterwards.
 *   X_dev, Y_dev  as for bsr_spmm(); their values do not change which kernel is fastest
 *   tried_out     (may be NULL) number of candidates that ran
 *   best_us_out   (may be NULL) microseconds per product of the one remembered
 * Waits for the stream (it is not asynchronous) and must not run concurrently with other calls on
 * the same handle.  Lend scratch first (bsr_set_scratch) if kernels that need it should compete.
 * Errors: as bsr_spmm(); on error nothing is remembered.
 */
bsr_status bsr_tune(bsr_matrix* W, int64_t m, const void* X_dev, void* Y_dev, bsr_dtype y_dtype,
                    int trials, void* hip_stream, int* tried_out, float* best_us_out);

/*
 * What bsr_tune() remembered for (m, y_dtype): settings_out = {kernel family (bsr_path), matrix-core
 * kernel variant (0 the library's choice, 1 direct, 2 k-split, 3 LDS tiles, 4 LDS stripe, 5 row groups for
 * the longest block-rows and LDS tiles for the others, 6 the sweep kernel for sides of 8 and 16, 7 16x16 tiles of
 * 8-wide blocks), wavefronts (variant 6: groups of 64 outputs) per workgroup, tile setting, two per-variant settings}, 0 = the kernel's default; us_out (may be
 * NULL) its measured microseconds per product.  BSR_ERR_UNSUPPORTED if nothing is remembered.
 */
bsr_status bsr_tune_result(const bsr_matrix* W, int64_t m, bsr_dtype y_dtype, int32_t settings_out[6], float* us_out);

/* The path BSR_PATH_AUTO resolves to for this handle, m and an output of W's type (never AUTO; what bsr_tune()
 * remembered is not consulted).  Below 16 rows, and with 8-wide blocks where n or k is no multiple of 16, a 16-bit W may
 * resolve to another one for a BSR_F32 output, whose sums are kept as exact as the wavefront-reduction kernels'.
 * Errors: NULL. */
bsr_status bsr_query_path(const bsr_matrix* W, int64_t m, bsr_path* path_out);

/*
 * The sibling product Z = G * W (the gradient of the layer's input when Y = X * W^T is a sparse
 * layer's forward pass, the use the paper's Introduction names) is the same product with W^T in
 * place of W:  Z = G * (W^T)^T.  These two calls build W^T in the same storage format -- a (k, n)
 * matrix of bs_c x bs_r blocks -- from which bsr_create() makes a handle; then
 * bsr_spmm(handle of W^T, m, G, Z, ...) is the sibling product.
 *
 * bsr_transpose_pattern (HOST pointers): validates the pattern as bsr_validate and writes
 *   t_index_pointer_host  k/bs_c + 1 entries      t_block_indices_host  nnzb entries (block-rows of W)
 *   perm_host             nnzb entries: stored block q of W^T is the transpose of block perm[q] of W
 * The blocks of a block-row of W^T come by ascending block-row of W.
 *
 * bsr_transpose_values (DEVICE pointers, asynchronous on hip_stream):
 *   t_block_data[q][c][a] = block_data[perm[q]][a][c],  q in [0, nnzb)
 * t_block_data_dev has nnzb*bs_c*bs_r elements of `dtype`, caller-owned; call it again whenever
 * the values of W change.  Errors: NULL, SHAPE, DTYPE, INDPTR, INDEX, UNSUPPORTED (a block larger
 * than 64 KiB), HIP.
 */
bsr_status bsr_transpose_pattern(int64_t n, int64_t k, int32_t bs_r, int32_t bs_c, int64_t nnzb,
                                 const int32_t* index_pointer_host, const int32_t* block_indices_host,
                                 int32_t* t_index_pointer_host, int32_t* t_block_indices_host, int32_t* perm_host);
bsr_status bsr_transpose_values(bsr_dtype dtype, int32_t bs_r, int32_t bs_c, int64_t nnzb, const int32_t* perm_dev,
                                const void* block_data_dev, void* t_block_data_dev, void* hip_stream);

/*
 * The sampled sibling: the gradient of the stored blocks.  With Y = X * W^T a layer's forward pass
 * and G = dL/dY, Y is linear in block_data[p][a][c] with coefficient X[i][col*bs_c + c] in
 * Y[i][r*bs_r + a], so
 *     D[p][a][c] = sum over i of  G[i][r*bs_r + a] * X[i][block_indices[p]*bs_c + c]
 * for every stored block p of block-row r: the entries of G^T X at the positions W stores.
 *   G_dev   DEVICE, m*n elements of W's dtype, row-major     X_dev  DEVICE, m*k elements, row-major
 *   D_dev   DEVICE, nnzb*bs_r*bs_c elements of d_dtype (W's dtype or BSR_F32), the layout of
 *           block_data; every element is written; fp32 accumulation, rounded to nearest-even
 * Block shapes with bs_r, bs_c in {8, 16, 32, 64} run on the matrix cores (with a side of 8 from 256 rows on, fp32 from
 * 512 rows and many blocks on); blocks of 1, 2, 4, 8 or 16 rows and any width else on a kernel that gives a lane one
 * column of one block; any other shape on a plain loop.  Thin blocks (16 x 1, fp32): in block-column order (k a multiple
 * of 4) on a matrix-core kernel that turns rows of X over in LDS, where that is the quicker; else, with scratch lent for
 * this m (bsr_scratch_size, bsr_set_scratch) and 32 rows or more, X is transposed into the scratch, which is
 * overwritten, and another matrix-core kernel runs; else the kernel of a lane per column.
 * Asynchronous on hip_stream; reads W's pattern only, not its values.
 * Errors: NULL, SHAPE (m < 0 or m*max(k,n) >= 2^31), DTYPE, ALIGN, HIP.
 */
bsr_status bsr_sddmm(const bsr_matrix* W, int64_t m, const void* G_dev, const void* X_dev, void* D_dev,
                     bsr_dtype d_dtype, void* hip_stream);

/*
 * bsr_sddmm() with memory for this one call: a W of few blocks keeps all CUs busy only if the rows of G and X are
 * split, and the partial results (fp32) of the splits need a place until they are added.
 *   bsr_sddmm_workspace_size  bytes a product with m rows would use (0: none); multiple of 256.  The first call of
 *                             these on a handle builds the product's plan on the host (milliseconds for tens of
 *                             thousands of stored blocks)
 *   workspace_dev             DEVICE, 16-byte aligned, or NULL; overwritten.  With fewer bytes than that the rows are
 *                             not split (the result is as good, the call slower: 4096 rows, 1843 bf16 16x16 blocks of
 *                             (3072, 768) 50 us instead of 21).  Calls with memory of their own may
 *                             run concurrently on one handle.
 */
bsr_status bsr_sddmm_workspace_size(const bsr_matrix* W, int64_t m, size_t* bytes);
bsr_status bsr_sddmm_ws(const bsr_matrix* W, int64_t m, const void* G_dev, const void* X_dev, void* D_dev,
                        bsr_dtype d_dtype, void* workspace_dev, size_t workspace_bytes, void* hip_stream);

/*
 * bsr_spmm() for callers that can neither allocate nor lend device memory: code under HIP graph capture,
 * tight serving loops, harnesses that forbid hipMalloc.  (No passage of the paper defines this call; it is
 * the product of bsr_spmm_ex(..., BSR_PATH_MFMA, ...) for the one kernel family that needs per-call scratch.)
 * For thin blocks (bs_r = 16, bs_c = 1, fp32, y_dtype BSR_F32) the matrix-core path keeps a transposed copy
 * of X in scratch; here that scratch is an array of BSR_STATIC_SCRATCH_BYTES bytes inside the library's code
 * object instead of memory lent with bsr_set_scratch().  Every GPU the library is loaded on holds its own
 * copy of the array until the process ends; its address is looked up once per device (at bsr_create(), else
 * at the first call).  The call itself allocates and frees nothing, on the device or through any library.
 *   Arguments as bsr_spmm().  m >= 1 rows need bsr_scratch_size(W, m) bytes: beyond the built-in size the
 *   call returns BSR_ERR_SCRATCH_LIMIT and does no device work (256 x 4096: 4 MiB + 256 bytes).
 *   Any other block shape or output type: BSR_ERR_UNSUPPORTED (no other kernel needs per-call scratch; use
 *   bsr_spmm()).
 * All calls on one GPU share that GPU's array, whatever the handle or stream: calls that overlap in time on
 * one GPU race; keep them ordered on one stream.  The array keeps the last call's contents; nothing in it
 * has to start at zero (each call first overwrites every entry it later reads for rows below m).
 * Errors: as bsr_spmm(), plus SCRATCH_LIMIT and UNSUPPORTED.
 */
#define BSR_STATIC_SCRATCH_BYTES (8u << 20)
bsr_status bsr_spmm_static(const bsr_matrix* W, int64_t m, const void* X_dev, void* Y_dev,
                           bsr_dtype y_dtype, void* hip_stream);

/*
 * One AdamW step over many tensors in as few launches as they have kinds (type, gradient's type, master copy or not): the
 * step from the gradients that bsr_sddmm() and bsr_epilogue_backward() make to the block values that bsr_spmm() reads, those
 * of W^T with them.  With g the gradient times grad_scale, t the step's number (from 1):
 *     m = beta1 m + (1 - beta1) g        v = beta2 v + (1 - beta2) g^2
 *     p = p (1 - lr weight_decay) - lr / (1 - beta1^t) * m / (sqrt(v) / sqrt(1 - beta2^t) + eps)
 * in fp32 whatever the types.  Where eps does not keep the quotient finite (it may be 0): with fp32 states sqrt(v) is at least
 * 2^-63, the root of the smallest normal number, so that 0 / 0 is 0; with 8-bit states and eps below 2^-40 an element
 * whose v is below 2^-120, which is held as 0, gets no update.
 *   param_dev      DEVICE, count elements of dtype (block_data of a W, a bias, ...), updated
 *   master_dev     DEVICE, count floats, or NULL: the parameter in fp32 (16-bit types only); it is updated and param_dev is
 *                  its nearest-even rounding.  Without one a 16-bit parameter is rounded up or down at random so that its mean
 *                  is kept: most updates are below half its last place
 *   grad_dev       DEVICE, count elements of grad_dtype (dtype or BSR_F32), read
 *   exp_avg_dev, exp_avg_sq_dev
 *                  DEVICE, m and v, updated: count floats each or, with 8-bit states, count bytes each.  Zeros to begin with
 *   scales_dev     8-bit states: DEVICE, three floats for each 256 elements begun, updated; zeros to begin with
 *   bs_r, bs_c, t_param_dev, t_perm_host
 *                  with t_param_dev (else all 0): the tensor is a W's blocks [stored blocks][bs_r][bs_c], t_param_dev
 *                  (DEVICE) the blocks of its transpose as bsr_transpose_values() orders them, written anew by every step;
 *                  t_perm_host (HOST, read during bsr_adamw_create only) is bsr_transpose_pattern()'s perm
 * 8-bit states, in groups of 256 elements from a tensor's start.  m: an e4m3 number times a scale, rounded to nearest-even; 0
 * where the group's largest is below 2^-100.  v: 0 for v below 2^-120, else 2^(start + (code - 1) spacing), code 1 .. 255, from
 * the group's smallest such v (at least 2^-40 of the largest) to its largest, rounded up or down at random so that its mean is kept (a step changes v by less than half the spacing:
 * rounded to nearest it would stop).  The random numbers are a hash of seed, step, the tensor's place in the list and the
 * element's in the tensor: the same call on the same values gives the same bits.  The update itself sees m and v before
 * their rounding.
 * Not finite gradients: they reach p, and with 8-bit states the moments of their whole group; a loop that scales its loss
 * looks for them and sets grad_scale_dev to 0, for which parameters and moments stay as they are.
 */
typedef struct bsr_adamw bsr_adamw;     /* opaque handle: the list of tensors (device pointers not owned) */
typedef struct {
    int64_t count;
    bsr_dtype dtype, grad_dtype;
    void* param_dev;
    float* master_dev;
    const void* grad_dev;
    void* exp_avg_dev;
    void* exp_avg_sq_dev;
    float* scales_dev;
    float weight_decay;
    int32_t bs_r, bs_c;
    void* t_param_dev;
    const int32_t* t_perm_host;
} bsr_adamw_tensor;

/* A step's settings.  The *_dev members (DEVICE scalars, or NULL) take the place of the values beside them when the step runs:
 * a step captured into a graph reads its number, rate and scale at every replay.  Where the number is below 1 there, or the
 * scale 0, the step is skipped. */
typedef struct {
    double lr, beta1, beta2, eps;       /* 0 <= beta < 1, lr and eps >= 0 */
    int64_t step;                       /* t >= 1 */
    float grad_scale;                   /* 1: gradients as they are; 0: the step is skipped (else 2^-40 to 2^40 in size) */
    uint32_t seed;
    const float* lr_dev;
    const int64_t* step_dev;
    const float* grad_scale_dev;
} bsr_adamw_hyper;

/*
 * bsr_adamw_workspace_size  bytes of DEVICE workspace for the tables of a list (> 0, a multiple of 256)
 * bsr_adamw_create          checks the list (`tensors`, HOST) and uploads its tables to workspace_dev on hip_stream; the
 *                           device buffers and the workspace stay the caller's, must outlive the handle, the steps that are
 *                           still to run (on any stream) and the graphs that hold some, and keep their places; everything a step writes must be apart from every other buffer of the list.  Not for a
 *                           stream that is being captured.  state_bits: 32 or 8, of all its tensors.  *out is NULL on error
 * bsr_adamw_step            one step, asynchronous on hip_stream (steps on other streams wait for the upload on the device);
 *                           steps of one handle must not overlap in time.  A captured step may be replayed
 * bsr_adamw_moments         m and v as values of `dtype`: exp_avg_out[i], exp_avg_sq_out[i] (HOST arrays of DEVICE pointers,
 *                           count elements each, or NULL: not wanted) for tensor i of the list; apart from one another and
 *                           from the list's buffers
 * bsr_adamw_destroy         frees the handle's host memory (after waiting for the upload); NULL is accepted
 * Errors: NULL; SHAPE (sizes, blocks that do not make up a tensor, settings out of range, 2^36 elements in all); DTYPE
 * (state_bits too); ALIGN (16 bytes, scales and scalars their own size); INDEX (t_perm_host is no permutation);
 * WORKSPACE; OVERLAP; UNSUPPORTED (a block that bsr_transpose_values refuses); DEVICE; HIP.
 */
bsr_status bsr_adamw_workspace_size(int64_t n_tensors, const bsr_adamw_tensor* tensors, int32_t state_bits, size_t* bytes);
bsr_status bsr_adamw_create(bsr_adamw** out, int64_t n_tensors, const bsr_adamw_tensor* tensors, int32_t state_bits,
                            void* workspace_dev, size_t workspace_bytes, void* hip_stream);
bsr_status bsr_adamw_step(const bsr_adamw* opt, const bsr_adamw_hyper* hyper, void* hip_stream);
bsr_status bsr_adamw_moments(const bsr_adamw* opt, bsr_dtype dtype, void* const* exp_avg_out, void* const* exp_avg_sq_out,
                             void* hip_stream);
void bsr_adamw_destroy(bsr_adamw* opt);

/*
 * A pair of projections whose results gate one another: Wg and Wu, (n, k) each, in blocks of the same shape, as ONE handle W
 * of 2n rows in which block-row 2r is block-row r of Wg and block-row 2r + 1 that of Wu.  The halves of a result are then made
 * by neighbouring block-rows, and W stays a matrix like any other: bsr_sddmm(W, dZ, X) is the gradient of its blocks,
 * bsr_spmm(handle of W^T, dZ) that of X, bsr_adamw_step and bsr_muon_step update it.
 *     z_g = X Wg^T + bias_g      z_u = X Wu^T + bias_u      H[i][j] = act(z_g[i][j]) z_u[i][j]
 * z, biases and gradients of both are kept in W's order, bs_r columns of one half and bs_r of the other in turn: with u = bs_r
 * and j = r u + a, column 2 r u + a is z_g's, column 2 r u + u + a z_u's.  All of it is fp32 arithmetic on the sums; H and Z
 * are rounded once, to nearest-even, and H is made of the z before that rounding.
 *   H_dev          DEVICE, m*n elements of h_dtype (W's dtype or BSR_F32), every one written
 *   gated (HOST)   act; bias_dev: DEVICE, 2n elements of bias_dtype (W's dtype or BSR_F32), or NULL; z_dev: DEVICE, Z, m*2n
 *                  elements of h_dtype, every one written, or NULL
 *   workspace_dev  DEVICE, bsr_spmm_gated_workspace_size() bytes (0: none, it may be NULL; blocks with a side of 8 may need one
 *                  until a product has run, and none from then on), overwritten.  Calls that may run at the same time, replayed
 *                  graphs among them, need one each
 * Streams and captures as bsr_spmm().  The kernel is the library's choice by W and m; what bsr_tune() remembered is for the other
 * products, and for a gated one where it leaves its sums in the workspace or in Z.  H, Z and the workspace must overlap neither one
 * another nor an input, nor the handle's arrays, its workspace and what has been lent as scratch.
 * Errors: as bsr_spmm_epilogue(), plus SHAPE (an odd number of block-rows) and WORKSPACE.
 */
typedef struct {
    bsr_act act;
    bsr_dtype bias_dtype;
    const void* bias_dev;
    void* z_dev;
} bsr_gated;
bsr_status bsr_spmm_gated_workspace_size(const bsr_matrix* W, int64_t m, bsr_dtype h_dtype, size_t* bytes);
bsr_status bsr_spmm_gated(const bsr_matrix* W, int64_t m, const void* X_dev, void* H_dev, bsr_dtype h_dtype, const bsr_gated* gated,
                          void* workspace_dev, size_t workspace_bytes, void* hip_stream);

/*
 * Its gradient, from G = dL/dH and the Z that was kept:
 *     dz_g = G z_u act'(z_g)      dz_u = G act(z_g)      db[j] = sum over i of dZ[i][j]
 * One pass over G and Z; the sums are fp32, of dZ before its rounding, and added in a fixed order (no atomics).
 *   unit           columns of a half that stand together in Z and dZ: W's bs_r; it divides n
 *   G_dev          DEVICE, m*n elements of g_dtype      Z_dev  DEVICE, m*2n elements of g_dtype
 *   DZ_dev         DEVICE, m*2n elements of dz_dtype (g_dtype, or any type where g_dtype is BSR_F32), or NULL; it may be Z_dev
 *                  itself where the types are the same
 *   DB_dev         DEVICE, 2n floats, or NULL (not both NULL); m == 0: zeros
 *   workspace_dev  DEVICE, bsr_gated_backward_workspace_size() bytes (0: none), overwritten; read only where DB_dev is given.
 *                  Calls that may run at the same time, replayed graphs among them, need one each.
 * Asynchronous on hip_stream.  Errors: NULL, SHAPE (m or n negative, unit below 1 or no divisor of n, m >= 2^30, n >= 2^27, or
 * m*n >= 2^39), DTYPE, ALIGN (a pointer not 16-byte aligned), WORKSPACE, OVERLAP, HIP.
 */
bsr_status bsr_gated_backward_workspace_size(int64_t m, int64_t n, int32_t unit, size_t* bytes);
bsr_status bsr_gated_backward(int64_t m, int64_t n, int32_t unit, bsr_act act, bsr_dtype g_dtype, const void* G_dev, const void* Z_dev,
                              bsr_dtype dz_dtype, void* DZ_dev, float* DB_dev, void* workspace_dev, size_t workspace_bytes,
                              void* hip_stream);

/*
 * The norms around a block of a network whose blocks add to a stream S of hidden states: what the block's result B meets on
 * its way into the stream, and what the next block is given, in one pass.
 *     b = post(B)        S'[i][j] = stream_scale S[i][j] + branch_scale gate[j] b[i][j]        U = pre(S')
 * post, pre: none; x / sqrt(mean(x^2) + eps); (x - mean(x)) / sqrt(mean((x - mean(x))^2) + eps), over a row, times a weight, plus
 * a bias.  fp32 arithmetic; U is made of S' before its rounding; each result is rounded once, to nearest-even.
 *   S_dev          DEVICE, m*n elements of s_dtype (b_dtype or BSR_F32)
 *   B_dev          DEVICE, m*n elements of b_dtype, or NULL: no block has run yet (S' = stream_scale S; post and gate are not looked at)
 *   S_out_dev      DEVICE, S', m*n elements of s_dtype, or NULL; it may be S_dev itself
 *   U_dev          DEVICE, U, m*n elements of b_dtype, or NULL (always where pre is none; not both NULL); it may be B_dev itself
 *   how (HOST)     weights, biases and gate: DEVICE, n elements of w_dtype (b_dtype or BSR_F32), or NULL (1, 0 and 1)
 * A NaN or an infinity reaches its own row only.  Mean squares are fp32 numbers: values beyond 2^63 in size count as infinite
 * there, and with eps = 0 rows whose mean square is below 2^-126 have no defined norm.
 * Asynchronous on hip_stream.  Errors: NULL, SHAPE (m or n negative, m >= 2^30, n > 16384, eps negative), DTYPE (an unknown norm
 * too), ALIGN (a pointer not 16-byte aligned), UNSUPPORTED (U_dev without pre), OVERLAP, HIP.
 */
typedef enum { BSR_NORM_NONE = 0, BSR_NORM_RMS = 1, BSR_NORM_LAYER = 2 } bsr_norm;
typedef struct {
    bsr_norm post, pre;
    bsr_dtype w_dtype;
    const void* post_weight_dev;
    const void* post_bias_dev;
    const void* gate_dev;
    const void* pre_weight_dev;
    const void* pre_bias_dev;
    double eps;
    float stream_scale, branch_scale;
} bsr_residual;
bsr_status bsr_residual_norm(int64_t m, int64_t n, bsr_dtype s_dtype, const void* S_dev, bsr_dtype b_dtype, const void* B_dev,
                             void* S_out_dev, void* U_dev, const bsr_residual* how, void* hip_stream);

/*
 * Its gradient, from GS = dL/dS' (what reaches S' otherwise) and GU = dL/dU, at S' as it was stored: with g = GS + pre'(GU),
 *     dS = stream_scale g      dB = post'(branch_scale gate g)
 * and, summed over the rows, the gradients of the five vectors.
 *   S_dev          DEVICE, S', m*n elements of s_dtype (not read, may be NULL, where pre is none)
 *   B_dev          as given to bsr_residual_norm(); NULL: DB_dev and the gradients of post and gate have to be NULL
 *   GS_dev, GU_dev DEVICE, m*n elements of s_dtype and b_dtype, or NULL (zeros; GU_dev always where pre is none)
 *   DS_dev, DB_dev DEVICE, m*n elements of s_dtype and b_dtype, or NULL: not wanted; DS_dev may be GS_dev or S_dev itself, DB_dev
 *                  GU_dev or B_dev
 *   grads (HOST)   DEVICE, n floats each, or NULL: not wanted (also for a vector that is not there: it counts as 1 or 0); m == 0:
 *                  zeros.  fp32 sums in a fixed order (no atomics)
 *   workspace_dev  DEVICE, bsr_residual_norm_backward_workspace_size() bytes, overwritten; it may be NULL where no sum is
 *                  wanted and n <= 8192.  Calls that may run at the same time, replayed graphs among them, need one each.
 * Asynchronous on hip_stream.  Errors: as bsr_residual_norm(), plus WORKSPACE, UNSUPPORTED (what belongs to a norm or a branch
 * that is not there) and NULL (nothing wanted).
 */
typedef struct {
    float* post_weight_dev;
    float* post_bias_dev;
    float* gate_dev;
    float* pre_weight_dev;
    float* pre_bias_dev;
} bsr_residual_grads;
bsr_status bsr_residual_norm_backward_workspace_size(int64_t m, int64_t n, size_t* bytes);
bsr_status bsr_residual_norm_backward(int64_t m, int64_t n, bsr_dtype s_dtype, const void* S_dev, bsr_dtype b_dtype, const void* B_dev,
                                      const void* GS_dev, const void* GU_dev, void* DS_dev, void* DB_dev, const bsr_residual* how,
                                      const bsr_residual_grads* grads, void* workspace_dev, size_t workspace_bytes, void* hip_stream);

/*
 * One step over the stored blocks of many matrices whose update is orthogonalised block by block: every singular value of a
 * block's update is brought near 1 by Newton-Schulz steps, products alone, on the matrix cores with fp32 sums: of numbers in two
 * fp16 parts, to 2^-23 of their powers of two, where |a| >= 1 and a, b, c keep X's singular values below 3.9; in three bf16 parts (24
 * bits) or fp32 elsewhere.  With the parts of fp16 an update's root mean square error is 1.0 to 1.5 times that of the same steps in
 * plain fp32 arithmetic, its largest up to 1.8 times.
 * With g the gradient times grad_scale,
 *     M = momentum M + g                 V = g + momentum M (nesterov) or M
 *     X = V / (|V| + eps), |V| the block's Frobenius norm;  ns_steps times  X = a X + b (X X^T) X + c (X X^T)^2 X
 *     p = p (1 - lr weight_decay) - lr scale X
 * Biases and other tensors that are not blocks take bsr_adamw_step().
 *   blocks, bs_r, bs_c   the tensor: a W's block_data, sides from 1 to 64 (a side of 1: V / |V| times what the steps make of 1)
 *   param_dev, master_dev, grad_dev, t_param_dev, t_perm_host, weight_decay   as in bsr_adamw_tensor: a 16-bit parameter without
 *                        a master copy is rounded at random so that its mean is kept, by a hash of seed, step, the tensor's
 *                        place in the list and the element's in the tensor
 *   momentum_dev         DEVICE, M, a float an element, updated; zeros to begin with
 *   scale                of the update
 * Not finite gradients reach M there and p in their whole block; a loop that scales its loss looks for them and sets
 * grad_scale_dev to 0, for which everything stays as it is.  A block of zeros has an update of 0 (eps > 0).
 */
typedef struct bsr_muon bsr_muon;       /* opaque handle: the list of tensors (device pointers not owned) */
typedef struct {
    int64_t blocks;
    int32_t bs_r, bs_c;
    bsr_dtype dtype, grad_dtype;
    void* param_dev;
    float* master_dev;
    const void* grad_dev;
    float* momentum_dev;
    void* t_param_dev;
    const int32_t* t_perm_host;
    float weight_decay, scale;
} bsr_muon_tensor;

/* A step's settings; the *_dev members as in bsr_adamw_hyper (step: of the random roundings alone). */
typedef struct {
    double lr, momentum, eps;           /* lr >= 0, 0 <= momentum < 1, eps > 0 (2^-100 to 1) */
    float a, b, c;                      /* of the Newton-Schulz steps */
    int32_t ns_steps, nesterov;         /* 0 to 16 steps */
    int64_t step;                       /* t >= 1 */
    float grad_scale;                   /* 1: gradients as they are; 0: the step is skipped (else 2^-40 to 2^40 in size) */
    uint32_t seed;
    const float* lr_dev;
    const int64_t* step_dev;
    const float* grad_scale_dev;
} bsr_muon_hyper;

/*
 * bsr_muon_workspace_size, bsr_muon_create, bsr_muon_step, bsr_muon_destroy: as bsr_adamw_*.  Errors: as there; SHAPE for sides
 * beyond 64, too.
 */
bsr_status bsr_muon_workspace_size(int64_t n_tensors, const bsr_muon_tensor* tensors, size_t* bytes);
bsr_status bsr_muon_create(bsr_muon** out, int64_t n_tensors, const bsr_muon_tensor* tensors, void* workspace_dev, size_t workspace_bytes,
                           void* hip_stream);
bsr_status bsr_muon_step(const bsr_muon* opt, const bsr_muon_hyper* hyper, void* hip_stream);
void bsr_muon_destroy(bsr_muon* opt);

/*
 * Measurement helper for the benchmark, not part of the product (no passage of the paper defines it): one
 * launch of a kernel that only issues independent matrix-core instructions of the given input type
 * (8 accumulator chains per wavefront, 32 wavefronts per CU, `iters` rounds, no memory traffic), so that
 * roofline fractions can be quoted against the rate this chip delivers as well as the published peak.
 *   sink_dev   DEVICE, 4 bytes, never written in practice     flops_out  HOST: the flops the launch performs
 * Asynchronous on hip_stream; time it with events.  Errors: NULL, SHAPE (iters outside [1, 2^20]), DTYPE, HIP.
 */
bsr_status bsr_probe_mfma(bsr_dtype dtype, int32_t iters, void* sink_dev, void* hip_stream, double* flops_out);

/* Static, human-readable text for a status code.  (Like bsr_workspace_size(), bsr_destroy(), bsr_query_path(),
 * bsr_scratch_size() and bsr_set_scratch(), a housekeeping call that no passage of the paper defines.) */
const char* bsr_status_string(bsr_status s);

#ifdef __cplusplus
}
#endif
#endif /* BSR_SPMM_H */
