/*
 * ftc.h -- C ABI of libftc: sparse neighbour aggregation for GCN / AGNN on AMD gfx950,
 * after FTC-GNN (arXiv 2412.12218).
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 *  - Every array pointer inside the structs and in the argument lists is a DEVICE
 *    pointer owned by the caller; the structs themselves and all scalars live on the
 *    host.  The library never allocates or frees device memory, never synchronises and
 *    never prints: a call validates its arguments on the host and enqueues kernels on
 *    `stream` (a hipStream_t passed as void*, NULL = the default stream).  Scratch
 *    memory comes from a caller-provided workspace whose size is returned by the
 *    matching *_workspace_bytes query (a pure host function).  The library keeps no state
 *    between calls apart from the thread-local error text (and the built-in scratch buffer of
 *    ftc_spmm_noalloc); a call may be recorded into a HIP graph, the first one included.
 *  - Return value: FTC_OK or a negative ftc_status; ftc_last_error() returns a
 *    thread-local description of the last failure.
 *  - The graph is a CSR adjacency with int32 indices (`nodePointer` / `edgeList` in the
 *    paper, Section V.A).  Column indices within a row may be unsorted and may repeat;
 *    repeated entries are separate edges whose contributions add.  Index validity
 *    (monotone row_ptr, 0 <= col < n) is the caller's responsibility and can be checked
 *    with ftc_validate_csr.
 *  - Dense matrices are row-major with a leading dimension in ELEMENTS.  The vector
 *    kernels need the base pointer 16-byte aligned and ld * sizeof(element) a multiple of
 *    16 with D a multiple of 8 (16-bit types) or 4 (fp32).  Other shapes are taken too: by
 *    kernels of the same kind at element alignment in ftc_spmm (with a window index), the
 *    dense update and the weight gradient, by slower row-wise kernels elsewhere.  Outputs
 *    never alias inputs unless stated.
 *  - n == 0 or nnz == 0 is legal.  A row without stored entries produces a zero output row
 *    (SpMM / layers) and no softmax output.
 */
#ifndef FTC_H
#define FTC_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    FTC_OK = 0,
    FTC_EINVAL = -1,       /* null pointer, negative size, inconsistent sizes          */
    FTC_EUNSUPPORTED = -2, /* dtype / dimension / tile combination not implemented      */
    FTC_EALIGN = -3,       /* pointer or leading dimension violates a stated alignment  */
    FTC_EWORKSPACE = -4,   /* workspace missing or smaller than *_workspace_bytes says  */
    FTC_EHIP = -5          /* the HIP runtime reported an error at launch               */
} ftc_status;

typedef enum { FTC_F32 = 0, FTC_F16 = 1, FTC_BF16 = 2 } ftc_dtype;

/* Kernel family used by ftc_spmm / ftc_sddmm and the layers built on them. */
typedef enum {
    FTC_PATH_AUTO = 0, /* per row window: matrix-core tiles where the condensed window is
                          dense enough, vector gather elsewhere                          */
    FTC_PATH_VALU = 1, /* vector gather path for every window                           */
    FTC_PATH_MFMA = 2  /* matrix-core condensed-tile path for every window (16-bit only) */
} ftc_path;

/* CSR adjacency: row_ptr[n+1], col_idx[nnz]; row_ptr[0] == 0, row_ptr[n] == nnz. */
typedef struct {
    int32_t n;
    int32_t nnz;
    const int32_t *row_ptr;
    const int32_t *col_idx;
} ftc_csr;

/*
 * Output of the sparse graph transformation (Section V.A).  Rows are cut into windows
 * of blk_h consecutive rows (the last one may be short); S_w is the ascending list of
 * distinct column ids used by window w.
 *   edge_to_row[e]      global row of edge e                              [nnz]
 *   edge_to_col[e]      position of col_idx[e] in S_w of the edge's window [nnz]
 *   block_partition[w]  ceil(|S_w| / blk_w): TC blocks of window w        [n_windows]
 *   win_col_ptr[w]      start of S_w inside win_cols                      [n_windows+1]
 *   win_cols            S_0, S_1, ... back to back; capacity nnz entries  [nnz]
 *   summary[0]          sum of |S_w|;  summary[1] = sum of block_partition
 *                       (`block_counter`)                                 [2]
 * All arrays are allocated by the caller before ftc_build_windows fills them.
 */
typedef struct {
    int32_t blk_h;
    int32_t blk_w;
    int32_t n_windows; /* ceil(n / blk_h) */
    int32_t *edge_to_row;
    int32_t *edge_to_col;
    int32_t *block_partition;
    int32_t *win_col_ptr;
    int32_t *win_cols;
    int64_t *summary;
} ftc_windows;

/* Library version: major * 10000 + minor * 100 + patch. */
int32_t ftc_version(void);

/* Description of the last error on this host thread ("" if none). Never NULL. */
const char *ftc_last_error(void);

/*
 * Checks on the device that row_ptr is non-decreasing with row_ptr[0] == 0 and
 * row_ptr[n] == nnz, and that every column index lies in [0, n).  *flag (device int32)
 * is set to 0 when the graph is valid, otherwise to a bit mask: 1 = row_ptr, 2 = col_idx.
 */
int32_t ftc_validate_csr(const ftc_csr *g, int32_t *flag, void *stream);

/*
 * Sparse graph transformation (Section V.A, `edgeToRow`, `edgeToColumn`,
 * `blockPartition`, `block_counter`; TC_BLK_H = 16 and TC_BLK_W = 8 in the paper, both
 * free here with 1 <= blk_h <= 64 and blk_w >= 1).  Fills every array of `out`;
 * out->blk_h, blk_w and n_windows are inputs and must be consistent with g->n.  The
 * result is uniquely determined (ascending order, strict de-duplication).
 */
size_t ftc_build_windows_workspace_bytes(int32_t n, int32_t nnz, int32_t blk_h, int32_t blk_w);
int32_t ftc_build_windows(const ftc_csr *g, ftc_windows *out, void *ws, size_t ws_bytes,
                          void *stream);

/*
 * The same transformation with its independent kernels side by side.  Windows of different sizes
 * are condensed by different kernels (Section V.A: the windows do not depend on each other), each of
 * which fills only part of the GPU; given three more streams they overlap (0.39 instead of 0.54 ms
 * on the R-MAT benchmark graph).  `side` holds three hipStream_t and four hipEvent_t (timing may be
 * disabled) created by the caller on the device of `stream`, all at the default priority: `stream`
 * forks into the side streams through `fork` after the classification and waits for `join[i]` of
 * each before the final scan, so for the caller everything still happens in stream order and nothing
 * waits on the host.  The handles are used only during the call; two calls that overlap in time need
 * two sets.  side == NULL is ftc_build_windows.  Small graphs (up to 2^18 nodes, depending on the
 * density) are transformed by one kernel after the other on `stream`, which is faster there; the side
 * streams are then left alone.
 */
typedef struct {
    void *stream[3]; /* hipStream_t */
    void *fork;      /* hipEvent_t  */
    void *join[3];   /* hipEvent_t  */
} ftc_side_streams;
int32_t ftc_build_windows_concurrent(const ftc_csr *g, ftc_windows *out, void *ws, size_t ws_bytes,
                                     const ftc_side_streams *side, void *stream);

/*
 * Symmetric GCN normalisation for a pattern that already contains the self-loops
 * (the paper names the GCN model in Section VI; the formula is the standard
 * A^ = D~^-1/2 (A+I) D~^-1/2).  d~_i = number of stored entries of row i,
 * dinv[i] = d~_i^-1/2 (0 for an empty row), vals[e] = dinv[row(e)] * dinv[col_idx[e]].
 * Either output may be NULL.  w may be NULL; when given, its edge_to_row is used to
 * find the row of an edge.
 */
int32_t ftc_gcn_norm(const ftc_csr *g, const ftc_windows *w, float *vals, float *dinv,
                     void *stream);

/*
 * Sparse neighbour aggregation (Section V.A; SpMM C = A x B of Section I.A.2):
 *   out[i, 0:D] = sum over stored entries e of row i of vals[e] * X[col_idx[e], 0:D]
 * accumulated in fp32.  vals == NULL means all ones.  X has g->n rows of dtype x_dtype;
 * out has g->n rows of dtype out_dtype.  out_scale (n floats, may be NULL) multiplies output
 * row i by out_scale[i]; relu != 0 then applies max(0, .) before the store.
 * w may be NULL (vector path on the CSR only).  `path` is an ftc_path.
 */
size_t ftc_spmm_workspace_bytes(int32_t n, int32_t nnz, int32_t D);
int32_t ftc_spmm(const ftc_csr *g, const ftc_windows *w, const float *vals, const void *X,
                 int32_t ldx, int32_t x_dtype, int32_t D, void *out, int32_t ldo,
                 int32_t out_dtype, const float *out_scale, int32_t relu, int32_t path, void *ws,
                 size_t ws_bytes, void *stream);

/*
 * ftc_spmm for callers that cannot allocate device memory and have no workspace to pass: code under
 * HIP graph capture, tight serving loops, harnesses that forbid allocation.  Same arguments, same
 * kernels and bit-identical results; the scratch memory is a buffer of FTC_NOALLOC_SCRATCH_MIB MiB
 * built into the library (one copy per GPU, held until the process ends).  The call allocates and
 * frees nothing.  FTC_EWORKSPACE when ftc_spmm_workspace_bytes(n, nnz, D) exceeds the buffer (about
 * nnz * D > 4e9 with 16-bit features).  The device that `stream` belongs to must be current.  All
 * calls on one GPU share the buffer: calls that overlap in time on one GPU (different streams, or
 * several host threads) race; calls in one stream are safe.  Nothing in the buffer has to be zero and
 * nothing is kept between calls.  The first call on a device looks up the buffer's address.
 */
#define FTC_NOALLOC_SCRATCH_MIB 64
int32_t ftc_spmm_noalloc(const ftc_csr *g, const ftc_windows *w, const float *vals, const void *X,
                         int32_t ldx, int32_t x_dtype, int32_t D, void *out, int32_t ldo,
                         int32_t out_dtype, const float *out_scale, int32_t relu, int32_t path,
                         void *stream);

/*
 * Sparse edge feature computation (Section V.A; SDDMM D = A o (B x C) of Section I.A.2,
 * A taken as the 0/1 pattern), result laid out like col_idx (`EdgeValList`):
 *   edge_out[e] = alpha * row_scale[i] * col_scale[j] * sum_k X[i,k] * Y[j,k],
 *   i = row of e, j = col_idx[e].
 * X and Y have g->n rows, the same dtype and leading dimension, and may be the same
 * matrix.  row_scale / col_scale may be NULL (1.0).
 * cosine != 0 selects the AGNN edge score instead: the scales are the inverse Euclidean norms of
 * the rows themselves,
 *   edge_out[e] = alpha * sum_k X[i,k] * Y[j,k] / (max(||X[i,:]||, 1e-12) * max(||Y[j,:]||, 1e-12)),
 * row_scale and col_scale must then be NULL; no array of norms has to exist, the vector
 * kernel recomputes them from the rows it has loaded.
 */
size_t ftc_sddmm_workspace_bytes(int32_t n, int32_t nnz, int32_t D);
int32_t ftc_sddmm(const ftc_csr *g, const ftc_windows *w, const void *X, const void *Y,
                  int32_t ld, int32_t dtype, int32_t D, const float *row_scale,
                  const float *col_scale, float alpha, int32_t cosine, float *edge_out,
                  int32_t path, void *ws, size_t ws_bytes, void *stream);

/*
 * Inverse Euclidean row norms used by the AGNN cosine: rinv[i] = 1 / max(||H[i,:]||, 1e-12).
 */
int32_t ftc_row_rnorm(int32_t n, const void *H, int32_t ld, int32_t dtype, int32_t D,
                      float *rinv, void *stream);

/*
 * Edge softmax over the stored entries of every row (the attention weights of AGNN,
 * which the paper names in Section VI):
 *   p[e] = exp(s[e] - m_i) / sum_{e' in row i} exp(s[e'] - m_i),  m_i = max over row i.
 * p_out may alias e_in.  Rows without entries write nothing.  w may be NULL; with a window
 * index the work is split by edges (edge_to_row), which keeps hub rows from serialising,
 * and a workspace of ftc_edge_softmax_workspace_bytes is needed (none when w is NULL).
 */
size_t ftc_edge_softmax_workspace_bytes(int32_t n, int32_t nnz);
int32_t ftc_edge_softmax(const ftc_csr *g, const ftc_windows *w, const float *e_in, float *p_out,
                         void *ws, size_t ws_bytes, void *stream);

/*
 * Dense update phase (Section I.A.2): Z = X * W, X n x d_in (dtype), W d_in x d_out
 * row-major of the same dtype, fp32 accumulation, Z n x d_out of z_dtype.
 * Any d_in, d_out >= 1: W stays on chip for d_in <= 256 and d_out <= 64 (the benchmark models);
 * wider inputs are contracted in chunks, wider outputs written in groups of 64 columns (X is read
 * once per group).  row_scale (n floats, may be NULL) multiplies row i of the product by
 * row_scale[i]; relu != 0 then applies max(0, .).
 */
int32_t ftc_update_gemm(int32_t n, const void *X, int32_t ldx, int32_t dtype, int32_t d_in,
                        const void *W, int32_t d_out, void *Z, int32_t ldz, int32_t z_dtype,
                        const float *row_scale, int32_t relu, void *stream);

/*
 * GCN layer forward: out = act(A^ * (X * W)) with A^ given by (g, vals); update first,
 * then aggregation (Eq. 1-2 of Section I).  W is d_in x d_out row-major, same dtype as X.
 * The intermediate X * W lives in the workspace: fp16 for fp16 inputs, fp32 otherwise.
 * dinv (n floats, may be NULL) selects the factored form of the symmetric normalisation:
 * the edge values are dinv[i] * dinv[j], `vals` is ignored (may be NULL), row j of X * W is
 * scaled by dinv[j] when it is written, the aggregation runs without edge values and output
 * row i is scaled by dinv[i].  No per-edge value array is read then.
 */
size_t ftc_gcn_layer_workspace_bytes(int32_t n, int32_t nnz, int32_t d_in, int32_t d_out);
int32_t ftc_gcn_layer(const ftc_csr *g, const ftc_windows *w, const float *vals,
                      const float *dinv, const void *X, int32_t ldx, int32_t dtype, int32_t d_in,
                      const void *W, int32_t d_out, int32_t relu, void *out, int32_t ldo,
                      int32_t out_dtype, int32_t path, void *ws, size_t ws_bytes, void *stream);

/*
 * AGNN propagation layer forward: s_ij = beta * cos(h_i, h_j) on the stored entries,
 * P = edge softmax of s, out = P * H (H not normalised).  edge_p, when not NULL,
 * receives P (nnz floats).  With a window index scores, softmax and aggregation run fused in one
 * pass over the edges (P follows from the pass's weights); the softmax is then shifted by |beta|,
 * an upper bound of every score, instead of by the row maximum.  Above |beta| = 16 when edge_p is
 * given, and from 43 on without it, the unfused chain with the row-wise softmax is used (the
 * weights of a row whose neighbours all point away are exp(-2 |beta|)).
 * row_z, when not NULL, receives the softmax denominators of that pass,
 * z_i = sum over row i of exp(beta * cos - |beta|) (n floats, 0 for a row without entries): what
 * ftc_agnn_layer_backward_fused needs instead of P.  out_f32, when not NULL, receives the result
 * once more, unrounded (n x D fp32, leading dimension ld_f32, a multiple of 4; rows 16-byte
 * aligned): the backward pass takes <dY_i, out_i> from it when `out` itself is 16-bit.  Only the
 * fused pass produces these two (FTC_EUNSUPPORTED together with edge_p, without a window index or
 * for shapes it does not cover).
 */
size_t ftc_agnn_layer_workspace_bytes(int32_t n, int32_t nnz, int32_t D);
int32_t ftc_agnn_layer(const ftc_csr *g, const ftc_windows *w, const void *H, int32_t ld,
                       int32_t dtype, int32_t D, float beta, void *out, int32_t ldo,
                       int32_t out_dtype, float *edge_p, float *row_z, float *out_f32,
                       int32_t ld_f32, int32_t path, void *ws, size_t ws_bytes, void *stream);

/*
 * ---- Backward pass ----------------------------------------------------------------------------
 * The paper speaks of GNN training as well as inference (Sections II and V) and gives no gradient
 * formulas; the entry points below compute the derivatives of the forward definitions above.
 * Gradient arrays are fp32.  The sparse products of the backward pass run on the forward SpMM /
 * SDDMM kernels.
 */

/*
 * Transposed index of a symmetric pattern: T[e] = position of the stored entry (j, i) for the
 * stored entry e = (i, j), -1 where the pattern does not hold it; *flag (device int32) becomes 1
 * if any entry has no partner, else 0.  Needs ascending, duplicate-free columns inside every row.
 * w may be NULL (its edge_to_row only saves a search).
 */
int32_t ftc_transpose_index(const ftc_csr *g, const ftc_windows *w, int32_t *T, int32_t *flag,
                            void *stream);

/*
 * Derivative of ftc_edge_softmax: ds[e] = p[e] * (dp[e] - sum over the row of p * dp).
 * ds may alias dp.  w and the workspace (ftc_edge_softmax_workspace_bytes) as in ftc_edge_softmax:
 * with the window index the work is split by entries, not rows (no long-row imbalance).
 */
int32_t ftc_edge_softmax_backward(const ftc_csr *g, const ftc_windows *w, const float *p,
                                  const float *dp, float *ds, void *ws, size_t ws_bytes,
                                  void *stream);

/*
 * Weight gradient of the update phase: dW = X^T * G, X n x d_in (x_dtype), G n x d_out (fp32),
 * dW d_in x d_out row-major (fp32).  Any d_in, d_out <= 504 (FTC_EUNSUPPORTED beyond).  Partial sums
 * of row blocks are added in a fixed order (reproducible); where the workspace holds few of them
 * (wide products) the rows are taken in several rounds.
 */
size_t ftc_weight_grad_workspace_bytes(int32_t n, int32_t d_in, int32_t d_out);
int32_t ftc_weight_grad(int32_t n, const void *X, int32_t ldx, int32_t x_dtype, int32_t d_in,
                        const float *G, int32_t ldg, int32_t d_out, float *dW, void *ws,
                        size_t ws_bytes, void *stream);

/*
 * Backward of ftc_update_gemm (Z = act(X * W), no row scale) for a loss with dL/dZ = dZ (n x d_out,
 * fp32): dP = dZ where the layer's output Z was positive (Z == NULL: no ReLU, dP = dZ),
 * dW = X^T * dP (d_in x d_out, fp32), dX = dP * W^T (n x d_in, of type dx_dtype; dX == NULL:
 * skipped).  Any d_in; d_out <= 504 (beyond 64 output columns dX is computed by the kernels of
 * ftc_update_gemm on the transposed weights).
 */
size_t ftc_update_gemm_backward_workspace_bytes(int32_t n, int32_t d_in, int32_t d_out);
int32_t ftc_update_gemm_backward(int32_t n, const void *X, int32_t ldx, int32_t dtype, int32_t d_in,
                                 const void *W, int32_t d_out, const void *Z, int32_t ldz,
                                 int32_t z_dtype, const float *dZ, int32_t lddz, void *dX,
                                 int32_t lddx, int32_t dx_dtype, float *dW, void *ws,
                                 size_t ws_bytes, void *stream);

/*
 * Backward of ftc_gcn_layer for a loss with dL/d(out) = dY (n x d_out, fp32):
 *   dP = dY where the layer's output Y was positive (Y == NULL: no ReLU, dP = dY),
 *   dZ = A^^T * dP,  dW = X^T * dZ (d_in x d_out),  dX = dZ * W^T (n x d_in; dX == NULL: skipped).
 * (gT, wT, valsT) describe A^^T: the transposed graph, its window index and its edge values; for
 * the symmetric GCN normalisation they are the forward graph itself.  dinv != NULL selects the
 * factored normalisation as in ftc_gcn_layer (valsT ignored).  X, W as in the forward call;
 * d_out <= 504.
 */
size_t ftc_gcn_layer_backward_workspace_bytes(int32_t n, int32_t nnz, int32_t d_in, int32_t d_out);
int32_t ftc_gcn_layer_backward(const ftc_csr *gT, const ftc_windows *wT, const float *valsT,
                               const float *dinv, const void *X, int32_t ldx, int32_t dtype,
                               int32_t d_in, const void *W, int32_t d_out, const void *Y,
                               int32_t ldy, int32_t y_dtype, const float *dY, int32_t lddy,
                               float *dX, int32_t lddx, float *dW, int32_t path, void *ws,
                               size_t ws_bytes, void *stream);

/*
 * Backward of ftc_agnn_layer for a loss with dL/d(out) = dY (n x D, same dtype and leading
 * dimension as H): dH (n x D, of type dh_dtype: fp32, or a 16-bit type when the layer below takes
 * its incoming gradient in that type) and *dbeta (device fp32).  p are the probabilities of the
 * forward pass (edge_p of ftc_agnn_layer), T the transposed index of the pattern, which must be
 * symmetric (ftc_transpose_index with flag 0).  With hn_i = h_i / max(|h_i|, 1e-12),
 * c_e = <hn_i, hn_j>:
 *   dp_e = <dY_i, h_j>,  ds = softmax backward of (p, dp),  dbeta = sum_e ds_e c_e,
 *   q_i = beta * sum_e (ds_e + ds_T(e)) hn_j,
 *   dH_i = sum_e p_T(e) dY_j  +  (q_i - hn_i <hn_i, q_i>) / |h_i|.
 */
size_t ftc_agnn_layer_backward_workspace_bytes(int32_t n, int32_t nnz, int32_t D);
int32_t ftc_agnn_layer_backward(const ftc_csr *g, const ftc_windows *w, const int32_t *T,
                                const void *H, int32_t ld, int32_t dtype, int32_t D, float beta,
                                const float *p, const void *dY, int32_t lddy, void *dH,
                                int32_t lddh, int32_t dh_dtype, float *dbeta, int32_t path,
                                void *ws, size_t ws_bytes, void *stream);

/*
 * The same gradients in one pass over the entries, for a symmetric pattern: every entry gathers
 * h_j and dY_j once and the per-node pair (1 / z_j, <dY_j, Y_j>); no edge array (probabilities,
 * transposed index) is read or written.  row_z are the denominators of the forward pass (row_z of
 * ftc_agnn_layer with the same H and beta), Y its output (n x D, any dtype; it enters through
 * <dY_i, Y_i> = sum over row i of p * dp, so a 16-bit Y costs accuracy -- a few 1e-3 of a row's
 * largest gradient entry with bf16 -- and out_f32 of the forward call is the better choice).
 * H and dY share dtype and leading dimension, rows 16-byte aligned; the window index is required;
 * (dtype, D) must be a width the single-pass forward covers, with at most 128 elements once
 * padded to its lane layout (ftc_plan_graph reports it), and |beta| < 43.  FTC_EUNSUPPORTED otherwise: use
 * ftc_agnn_layer_backward.  The formulas hold on a symmetric pattern only.  pattern_flag (device
 * int32, may be NULL) is the flag ftc_transpose_index wrote for this graph: when it is not zero
 * (some entry has no transposed partner) every element of dH and *dbeta is set to NaN instead of a
 * gradient of nothing.  NULL: the caller vouches for the symmetry.
 */
size_t ftc_agnn_layer_backward_fused_workspace_bytes(int32_t n, int32_t nnz, int32_t D);
int32_t ftc_agnn_layer_backward_fused(const ftc_csr *g, const ftc_windows *w, const void *H,
                                      int32_t ld, int32_t dtype, int32_t D, float beta,
                                      const float *row_z, const void *Y, int32_t ldy,
                                      int32_t y_dtype, const void *dY, int32_t lddy, void *dH,
                                      int32_t lddh, int32_t dh_dtype, float *dbeta,
                                      const int32_t *pattern_flag, void *ws, size_t ws_bytes,
                                      void *stream);

/*
 * ---- Graph transformer -------------------------------------------------------------------------
 * Layers of models that learn features per node id and attend between all nodes of a graph: the rows of a
 * table by id, the dense layer with its epilogue, and attention over a batch of graphs, each with its
 * gradients.  Matrices are row-major with a leading dimension at any alignment of an element (16-byte aligned
 * rows are fastest), sums and softmax statistics fp32, results the same in every run.  Counts and widths are at most 2^30, and
 * sizes that do not fit one launch (2^32 threads) are refused with FTC_EUNSUPPORTED.
 */

/*
 * Rows of a table: out[i, :] = scale * E[ids[i], :], E vocab x D (dtype), out n x D (out_dtype).  An id outside
 * [0, vocab) (a padded place, -1) gives a row of zeros.
 * Gradient: dE[v, :] = scale * sum over {i : ids[i] = v} of dOut[i, :], all vocab rows written (zeros without
 * an id), added up in fp32 by ascending i and rounded once; ids outside the table are left out.
 */
int32_t ftc_embedding(int32_t n, const int32_t *ids, int32_t vocab, const void *E, int32_t lde, int32_t dtype,
                      int32_t D, float scale, void *out, int32_t ldo, int32_t out_dtype, void *stream);
size_t ftc_embedding_backward_workspace_bytes(int32_t n, int32_t vocab, int32_t D);
int32_t ftc_embedding_backward(int32_t n, const int32_t *ids, int32_t vocab, const void *dOut, int32_t lddo,
                               int32_t dtype, int32_t D, float scale, void *dE, int32_t ldde, int32_t de_dtype,
                               void *ws, size_t ws_bytes, void *stream);

typedef enum {
    FTC_ACT_NONE = 0,
    FTC_ACT_RELU = 1,
    FTC_ACT_GELU = 2, /* p Phi(p), the exact form */
    FTC_ACT_SILU = 3  /* p / (1 + exp(-p)) */
} ftc_act;

/*
 * Dense layer: Z = act(X * W + bias) + residual, X n x d_in and W d_in x d_out (contiguous) of `dtype`,
 * bias (d_out numbers, may be NULL) and residual (n x d_out, may be NULL) of the same, Z n x d_out of z_dtype
 * (fp32 or `dtype`); sums, activation and residual in fp32, one rounding at the end.  Z may be the residual itself
 * (in place: same pointer, leading dimension and type).  fp32 products of more than four terms may
 * count an operand below 2^-110 with an error of up to 2^-134; larger ones, infinities and NaN are as in fp32.
 * slope (n x d_out, may be NULL) receives act'(X * W + bias), which is all the backward pass needs of the
 * activation: float for fp32 inputs, int16 for 16-bit ones (fixed point, 2^14 is 1; -2^15 is NaN).
 * ftc_linear differs from ftc_update_gemm in the epilogue, and in its kernels, which are for layers of any
 * width; narrow outputs of many rows with a row scale or ReLU alone are ftc_update_gemm's.
 */
size_t ftc_linear_workspace_bytes(int32_t n, int32_t d_in, int32_t d_out);
int32_t ftc_linear(int32_t n, const void *X, int32_t ldx, int32_t dtype, int32_t d_in, const void *W,
                   int32_t d_out, const void *bias, int32_t act, const void *residual, int32_t ldr, void *slope,
                   int32_t lds, void *Z, int32_t ldz, int32_t z_dtype, void *ws, size_t ws_bytes, void *stream);

/*
 * Backward of ftc_linear for dL/dZ = dZ (n x d_out, `dtype`): dP = dZ * slope (slope NULL: no activation),
 *   dX = dP * W^T + dX_add (n x d_in, dx_dtype),  dW = X^T * dP (d_in x d_out, contiguous),  db = column sums of dP;
 * dX, dW, db may each be NULL (not computed); dW and db are of dw_dtype; dx_dtype and dw_dtype are fp32 or `dtype`.
 * dX_add (n x d_in of `dtype`, may be NULL) is what reaches X on another way, as through a residual connection around
 * the layer; it may be dX itself (same pointer, leading dimension and type).  The gradient of the residual is dZ.
 * dP is rounded to `dtype` for the products, db sums it unrounded.
 */
size_t ftc_linear_backward_workspace_bytes(int32_t n, int32_t d_in, int32_t d_out);
int32_t ftc_linear_backward(int32_t n, const void *X, int32_t ldx, int32_t dtype, int32_t d_in, const void *W,
                            int32_t d_out, const void *slope, int32_t lds, const void *dZ, int32_t lddz,
                            const void *dX_add, int32_t ldda, void *dX, int32_t lddx, int32_t dx_dtype, void *dW,
                            void *db, int32_t dw_dtype, void *ws, size_t ws_bytes, void *stream);

/*
 * Dense layer with weights of their own for every group of rows (the types of nodes, experts): group g has the rows group_ptr[g] .. group_ptr[g+1] of X and Z
 * (device int32, n_groups + 1 entries, non-decreasing; a group may have no row), W[g] (W: n_groups x d_in x d_out, contiguous) and bias[g] (n_groups x d_out, contiguous, may
 * be NULL).  Otherwise as ftc_linear, for each group; rows in front of the first and behind the last group are neither read nor written, and
 * W of groups without a row is not read.  Offsets outside [0, n] are taken as the nearest end; d_in, d_out and n_groups at most 2^20.
 */
size_t ftc_grouped_linear_workspace_bytes(int32_t n, int32_t n_groups, int32_t d_in, int32_t d_out);
int32_t ftc_grouped_linear(int32_t n, const int32_t *group_ptr, int32_t n_groups, const void *X, int32_t ldx,
                           int32_t dtype, int32_t d_in, const void *W, int32_t d_out, const void *bias, int32_t act,
                           const void *residual, int32_t ldr, void *slope, int32_t lds, void *Z, int32_t ldz,
                           int32_t z_dtype, void *ws, size_t ws_bytes, void *stream);

/*
 * Backward of ftc_grouped_linear, as ftc_linear_backward for each group: dW (n_groups x d_in x d_out, contiguous) and db (n_groups x d_out,
 * contiguous) of groups without a row are zeros.  Sums over the rows are added in a fixed order.
 */
size_t ftc_grouped_linear_backward_workspace_bytes(int32_t n, int32_t n_groups, int32_t d_in, int32_t d_out);
int32_t ftc_grouped_linear_backward(int32_t n, const int32_t *group_ptr, int32_t n_groups, const void *X, int32_t ldx,
                                    int32_t dtype, int32_t d_in, const void *W, int32_t d_out, const void *slope,
                                    int32_t lds, const void *dZ, int32_t lddz, const void *dX_add, int32_t ldda,
                                    void *dX, int32_t lddx, int32_t dx_dtype, void *dW, void *db, int32_t dw_dtype,
                                    void *ws, size_t ws_bytes, void *stream);

/*
 * The norms before and after a block of a network (attention, a feed-forward block), its gate and its residual connection, over the n rows
 * of d numbers of the residual stream X and of the block's output F:
 *   p = Npost(F),  h = x_scale X + gate p,  u = Npre(h),
 *   N(t) = (t - mean(t)) / sqrt(mean((t - mean(t))^2) + eps) w + b  by rows; FTC_NORM_RMS: without mean(t); FTC_NORM_NONE: N(t) = t.
 * F may be NULL: h = x_scale X.  Weights and biases (d numbers each) may be NULL: ones and zeros.  gate may be NULL (ones), d numbers (ldg 0) or
 * n x d (ldg >= d); gate, post_w and post_b are of F, post_w and post_b of a norm, and refused without.  All matrices and vectors are of `dtype`;
 * everything in between is fp32, and u is that of the unrounded h.  1 <= d <= 16384, eps > 0.  With distances from the mean above 1e19, whose squares fp32 does not
 * hold, rows are normalised as in exact arithmetic all the same, as long as the distances themselves are numbers of fp32.  A layer norm's mean is right to a rounding of it and some of
 * the distances: equal numbers give the bias.
 */
typedef enum {
    FTC_NORM_NONE = 0,
    FTC_NORM_RMS = 1,
    FTC_NORM_LAYER = 2
} ftc_norm;

typedef struct {
    int32_t n, d, dtype;
    int32_t post, pre; /* ftc_norm */
    float eps, x_scale;
    const void *X, *F, *gate, *post_w, *post_b, *pre_w, *pre_b;
    int32_t ldx, ldf, ldg;
} ftc_block;

/*
 * H (n x d, may be NULL) receives h, U (n x d, may be NULL; needs `pre`) u; one of them is given.  H may be X itself (in place: same pointer
 * and leading dimension).  stats (n x 4 floats, 16-byte aligned, may be NULL) receives each row's mean and factor 1 / sqrt(..) of both norms, which
 * the backward pass needs.
 */
int32_t ftc_block_norm(const ftc_block *b, void *H, int32_t ldh, void *U, int32_t ldu, float *stats, void *stream);

/* What ftc_block_norm_backward computes: each may be NULL.  dX, dF and, for a gate of n x d, dgate are of the block's type; the others, d numbers each, of
 * dw_dtype (fp32 or the block's type). */
typedef struct {
    void *dX, *dF, *dgate, *dpost_w, *dpost_b, *dpre_w, *dpre_b;
    int32_t lddx, lddf, lddg, dw_dtype;
} ftc_block_grads;

/*
 * Gradients of ftc_block_norm for dL/dh = dH (what reaches h on other ways than u; NULL: nothing) and dL/du = dU (NULL: nothing; needs `pre`), the
 * block as the forward call was given it (X not overwritten) and stats as it wrote them; these may be NULL where there is no norm.  The gradient of a gate, a weight or a
 * bias is of one that the block has, but for biases of a norm, whose values the gradients do not need: dpre_b and dpost_b need the norm only.
 * dX may be dH itself (same pointer and leading dimension).  Sums over the rows are added in a fixed order.
 */
size_t ftc_block_norm_backward_workspace_bytes(int32_t n, int32_t d);
int32_t ftc_block_norm_backward(const ftc_block *b, const float *stats, const void *dH, int32_t lddh, const void *dU,
                                int32_t lddu, const ftc_block_grads *g, void *ws, size_t ws_bytes, void *stream);

/*
 * The norm over all gradients of a model and their clipping, for scale * g as the gradients (scale: what a scaled loss is divided by again):
 *   norm = |scale| sqrt(sum over all gradients of g^2),  out = scale min(1, max_norm / norm) g.
 * `grads` is an array of `count` descriptors on the HOST, read during the call: a matrix `grad` of rows x cols (ld; one row for what is contiguous) of any ftc_dtype, each
 * its own, and for ftc_clip_grad_norm `out` of the same type (ldo), which may be `grad` itself (same ld) and must not overlap anything else.  Tensors without a number are
 * skipped.  norm (device float) receives the norm before clipping.  Squares are summed in 64 bits, in a fixed order.  A norm that is infinite makes zeros of what is finite, and one
 * that is NaN makes everything NaN, as the formula has it; max_norm may be infinite (nothing is clipped but by scale) and is not negative.  At most 2^31 - 1 numbers in the rows of a
 * matrix that is not contiguous and 2^38 in a tensor.
 */
typedef struct {
    const void *grad;
    void *out;
    int64_t rows, cols, ld, ldo;
    int32_t dtype;
} ftc_grad;

size_t ftc_grad_norm_workspace_bytes(int32_t count);
int32_t ftc_grad_norm(const ftc_grad *grads, int32_t count, double scale, float *norm, void *ws, size_t ws_bytes,
                      void *stream);
int32_t ftc_clip_grad_norm(const ftc_grad *grads, int32_t count, double max_norm, double scale, float *norm, void *ws,
                           size_t ws_bytes, void *stream);

/*
 * Attention inside every graph of a packed batch.  Graph g has the query rows q_ptr[g] .. q_ptr[g+1] of Q and out,
 * and the rows kv_ptr[g] .. kv_ptr[g+1] of K and V (device int32, n_graphs + 1 entries, non-decreasing; the same
 * array where every node attends to every node; one query a graph: a readout).  Head h has columns h D .. of Q and
 * out, and columns (h / (heads / kv_heads)) D .. of K and V: kv_heads divides heads.  Q, K, V may be column ranges of one matrix.
 *   s_ij = scale <q_i, k_j> (scale: any finite number),  p = softmax over the keys j of the graph with kv_mask[j] != 0,  out_i = sum_j p_ij v_j.
 * kv_mask (n_kv bytes) may be NULL: all keys; K and V of masked keys are not read.  A query without a key gives
 * zeros.  Rows in front of the first and behind the last graph are neither read nor written.  lse (n_q x heads floats, may be NULL)
 * receives log sum_j exp(s_ij) (-inf without a key), what the backward pass needs.  All matrices are of `dtype`; D <= 128, kv_heads <= 65535,
 * n_q * heads and n_kv * kv_heads at most 2^30.  Offsets outside [0, n_q] ([0, n_kv]) are taken as the nearest end.
 * In 16 bits the probabilities are rounded to `dtype` before they multiply V (fp16: 2^15 times them).
 */
size_t ftc_graph_attention_workspace_bytes(int32_t n_q, int32_t n_kv, int32_t n_graphs, int32_t heads,
                                           int32_t kv_heads, int32_t D);
int32_t ftc_graph_attention(int32_t n_q, const int32_t *q_ptr, int32_t n_kv, const int32_t *kv_ptr,
                            int32_t n_graphs, int32_t heads, int32_t kv_heads, int32_t D, int32_t dtype,
                            const void *Q, int32_t ldq, const void *K, int32_t ldk, const void *V, int32_t ldv,
                            const uint8_t *kv_mask, float scale, void *out, int32_t ldo, float *lse, void *ws,
                            size_t ws_bytes, void *stream);

/*
 * Gradients of ftc_graph_attention for dL/d(out) = dOut; out and lse as the forward call wrote them, the other
 * arguments as it was given them.  The probabilities are computed again from lse, nothing of the size queries x keys is kept:
 *   dV_j = sum_i p_ij dOut_i,  ds_ij = p_ij (<dOut_i, v_j> - <dOut_i, out_i>),
 *   dQ_i = scale sum_j ds_ij k_j,  dK_j = scale sum_i ds_ij q_i   (sums over the heads that share a K/V head).
 * All matrices are of `dtype`; rows of dK and dV of masked keys are zeros.  dQ, dK, dV must not overlap an input.  In 16 bits
 * p (fp16: 2^15 p) and ds are rounded to `dtype` for their products (ds for D up to 32, and in graphs of one tile, to two numbers).  In fp16 a ds
 * below 2^-14 is held in steps of 2^-24, and sums of many such, dQ and dK, keep what they lost: scale the loss so that p times a gradient is well
 * above that.
 * With D above 32 in 16 bits <dOut_i, out_i> is that of `out` as it was rounded: where V has a mean of once (ten times) its spread, dQ is
 * 2 to 3 (11 to 24) and dK 2 (11 to 14) times as far off as results that are only rounded, without a mean 1.5 times.  (A row that all of V
 * have in common adds itself to out and nothing to dQ and dK: it can be taken off before.)
 */
size_t ftc_graph_attention_backward_workspace_bytes(int32_t n_q, int32_t n_kv, int32_t n_graphs, int32_t heads,
                                                    int32_t kv_heads, int32_t D);
int32_t ftc_graph_attention_backward(int32_t n_q, const int32_t *q_ptr, int32_t n_kv, const int32_t *kv_ptr,
                                     int32_t n_graphs, int32_t heads, int32_t kv_heads, int32_t D, int32_t dtype,
                                     const void *Q, int32_t ldq, const void *K, int32_t ldk, const void *V,
                                     int32_t ldv, const uint8_t *kv_mask, float scale, const void *out, int32_t ldo,
                                     const float *lse, const void *dOut, int32_t lddo, void *dQ, int32_t lddq,
                                     void *dK, int32_t lddk, void *dV, int32_t lddv, void *ws, size_t ws_bytes,
                                     void *stream);

/*
 * ---- Locality reordering (preprocessing) ------------------------------------------------------
 * The sparse graph transformation (Section IV.A) condenses the columns that the rows of a window
 * share; how many they share, and how often a gathered feature row is still in cache, depends on
 * the numbering of the nodes, which the paper takes as given.  These calls relabel the nodes before
 * the transformation and keep a permutation-in / permutation-out contract:
 *   perm[new] = old id, inv[old] = new id (device, int32, n entries each);
 *   features enter the new numbering with ftc_permute_rows(map = perm), results leave it with
 *   ftc_permute_rows(map = inv); the layers themselves run on the relabelled graph unchanged.
 * All results are unique (stable sorts) and reproducible.
 */
enum {
    FTC_ORDER_NONE = -1,          /* keep the numbering (a value of ftc_plan.reorder only) */
    FTC_ORDER_DEGREE = 0,         /* descending number of stored entries of the row, ties: ascending id */
    FTC_ORDER_DEGREE_CLASSES = 1, /* descending bit length of that number (power-of-two classes), ties:
                                     ascending id -- keeps the given order inside a class */
    FTC_ORDER_COMMUNITIES = 2     /* a value of ftc_plan.reorder only: ftc_label_propagation +
                                     ftc_order_by_key are worth a trial (keep the result if the window
                                     build's sum_uniq drops) */
};

/* Workspace of ftc_degree_order, ftc_order_by_key, ftc_label_propagation and ftc_permute_graph. */
size_t ftc_reorder_workspace_bytes(int32_t n, int32_t nnz);

/* perm and inv of the ordering `mode` of g's nodes. */
int32_t ftc_degree_order(const ftc_csr *g, int32_t mode, int32_t *perm, int32_t *inv, void *ws,
                         size_t ws_bytes, void *stream);

/*
 * perm and inv of the ascending order of keys[0 .. n) (device, int32, >= 0), ties by ascending id:
 * nodes with equal keys -- the same community label, say -- become neighbours in the new numbering.
 * *flag (device int32) becomes 1 if a key is negative (it is then ordered as 0), else 0.
 */
int32_t ftc_order_by_key(int32_t n, const int32_t *keys, int32_t *perm, int32_t *inv,
                         int32_t *flag, void *ws, size_t ws_bytes, void *stream);

/*
 * Community labels by synchronous label propagation, for a community ordering with
 * ftc_order_by_key: every node starts with its own id; in each of `rounds` rounds every node takes
 * the label that occurs most often among the stored entries of its row (duplicates count, a
 * self-loop counts the node's own label; the smallest label on a tie), all nodes at once from the
 * labels of the round before; a row without entries keeps its label.  labels: device int32[n].
 * Ten rounds recover the blocks of the stochastic-block-model benchmark graph.  Unique result.
 */
int32_t ftc_label_propagation(const ftc_csr *g, int32_t rounds, int32_t *labels, void *ws,
                              size_t ws_bytes, void *stream);

/*
 * Relabelled graph: row `new` of the output holds the entries of row perm[new] of g with every
 * column c replaced by inv[c], ascending inside the row, duplicates kept.  row_ptr_out has n + 1
 * entries, col_idx_out nnz.  (perm, inv) may come from ftc_degree_order or from the caller (e.g. a
 * community ordering); *flag (device int32) becomes 1 if they are not a permutation and its
 * inverse -- no index is followed unchecked, the output is then unspecified -- else 0.
 */
int32_t ftc_permute_graph(const ftc_csr *g, const int32_t *perm, const int32_t *inv,
                          int32_t *row_ptr_out, int32_t *col_idx_out, int32_t *flag, void *ws,
                          size_t ws_bytes, void *stream);

/*
 * out[r, :] = X[map[r], :] for r in [0, n): X and out are n x D matrices of the same dtype; a map
 * entry outside [0, n) gives a row of zeros.  out must not alias X.
 */
int32_t ftc_permute_rows(int32_t n, const void *X, int32_t ldx, int32_t dtype, int32_t D,
                         const int32_t *map, void *out, int32_t ldo, void *stream);

/*
 * ---- Per-graph plan ---------------------------------------------------------------------------
 * The paper's outlook (Section VII) names a framework that adapts its use of the hardware to the
 * input graph.  Here the adaptation has two levels.  Per window: FTC_PATH_AUTO sends a window to the
 * matrix cores or to the vector kernels by its density, with measured crossovers (ftc_spmm,
 * ftc_sddmm).  Per graph: ftc_plan_graph turns a few statistics, gathered once at build time, into
 * the choices that hold for the whole graph.  The statistics live on the device (ftc_degree_stats,
 * and summary[0] of ftc_build_windows); the caller copies them to the host once per graph.
 */

/* stats[0] = sum over the rows of (stored entries)^2, stats[1] = longest row (device, int64[2]). */
int32_t ftc_degree_stats(const ftc_csr *g, int64_t *stats, void *stream);

typedef struct {
    double skew;          /* n * sum_deg_sq / nnz^2: mean popularity of the node an entry points to, relative to
                             the mean row length (1 for a regular graph; row lengths stand in for column counts,
                             exact on symmetric patterns) */
    double reuse;         /* nnz / sum_uniq: stored entries per condensed column, averaged over the windows */
    int32_t reorder;      /* the ordering to apply, for a feature matrix (n * D elements) larger than one L2
                             (4 MiB): FTC_ORDER_DEGREE_CLASSES when skew >= 2, FTC_ORDER_COMMUNITIES (a trial
                             of the community ordering) for flatter degrees with at least 8 entries per row on
                             average; else FTC_ORDER_NONE */
    int32_t agnn_single_pass;           /* ftc_agnn_layer without edge_p runs as one pass for this (dtype, D) */
    int32_t agnn_backward_single_pass;  /* ftc_agnn_layer_backward_fused covers this (dtype, D) */
    int32_t spmm_mfma_windows;   /* FTC_PATH_AUTO may send windows of this (dtype, D) to the matrix cores ... */
    int32_t sddmm_mfma_windows;  /* ... for SpMM / for SDDMM */
    float mfma_min_reuse;        /* entries per condensed column from which a window goes there (< 0: never) */
} ftc_plan;

/* Host-only, pure.  sum_deg_sq from ftc_degree_stats, sum_uniq = summary[0] of ftc_build_windows. */
int32_t ftc_plan_graph(int32_t n, int32_t nnz, int64_t sum_deg_sq, int64_t sum_uniq, int32_t D,
                       int32_t dtype, ftc_plan *plan);

#ifdef __cplusplus
}
#endif
#endif /* FTC_H */
