/*
 * gnn.h - C ABI of the MI355X (gfx950) GCN / GAT layer library.
 *
 * The library computes forward and backward passes of GCN and GAT layers
 * with adaptive operator reordering and caching (arXiv 2308.12093, Sec. 3).
 *
 * General rules, valid for every entry point below
 * ------------------------------------------------
 *  - Pointers named in a "device" position are DEVICE pointers (HIP global
 *    memory); they are borrowed for the duration of the enqueued work and are
 *    never freed or retained by the library.  gnn_plan_desc_t, gnn_plan_info_t,
 *    gnn_graph_t themselves are HOST structs (holding device pointers).
 *  - The library allocates no device memory.  Every scratch byte comes from the
 *    caller's `workspace` (size reported by gnn_plan_query / the *_workspace_bytes
 *    helpers; must be 256-byte aligned).  Every call that takes a `cache` or a
 *    `workspace` also takes its size in bytes and returns GNN_ERR_BUFFER_TOO_SMALL,
 *    before any launch, when that is below what gnn_plan_query reported for the plan.
 *  - Every call only enqueues kernels on `hip_stream` (a hipStream_t passed as
 *    void*; NULL = the default stream) and returns; there is no host
 *    synchronisation unless the entry point says otherwise.
 *  - All argument checks run before the first launch, so a call that returns
 *    an error has had no side effect.  No entry point aborts or throws.
 *  - Dense tensors are row-major fp32.  Index arrays are int32.  Outputs are
 *    overwritten, not accumulated into, unless an entry point's flag asks for it.
 *  - Sparse matrices are square n x n in CSR (App. D.1, 0-based): rowptr[0] = 0,
 *    rowptr[n] = nnz, column indices strictly ascending inside a row.  Row i is
 *    the aggregating node, col[e] the neighbour whose features it reads.
 */
#ifndef GNN_H
#define GNN_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    GNN_OK = 0,
    GNN_ERR_INVALID_ARG = 1,      /* NULL where a pointer is required, negative size, bad enum, misalignment */
    GNN_ERR_BAD_GRAPH = 2,        /* graph struct inconsistent with the plan (n / nnz mismatch, missing arrays) */
    GNN_ERR_BUFFER_TOO_SMALL = 3, /* a caller buffer is smaller than the size the library reported */
    GNN_ERR_STATE = 4,            /* backward asked to read a cache that no forward has filled */
    GNN_ERR_UNSUPPORTED = 5,      /* shape outside what the kernels handle */
    GNN_ERR_HIP = 6               /* a HIP call or launch failed */
} gnn_status_t;

typedef enum { GNN_LAYER_GCN = 0, GNN_LAYER_GAT = 1, GNN_LAYER_SAGE = 2 } gnn_layer_t;

/* How an AUTO order / backward scheme is chosen for GCN. */
typedef enum {
    GNN_SELECT_PAPER_RULE = 0,    /* the usage conditions of the tables of Sec. 3.1: SpMM cost is taken
                                     to be proportional to the dense width                              */
    GNN_SELECT_CALIBRATED = 1     /* same candidates, compared by gnn_spmm_time_model_us: the time of this
                                     library's SpMM on an MI355X, which is flat below ~32 columns and has a
                                     fixed launch cost (Sec. 4.1 reports that the proportional rule misses
                                     the best scheme where the two widths are close)                    */
} gnn_select_t;

/* Order of the two products of X' = A' X Theta (Sec. 3.1, Table "GCN schemes"). */
typedef enum {
    GNN_ORDER_AUTO = 0,
    GNN_ORDER_TRANSFORM_FIRST = 1, /* A' (X Theta): GEMM, then SpMM of width F_out */
    GNN_ORDER_PROPAGATE_FIRST = 2  /* (A' X) Theta: SpMM of width F_in, then GEMM  */
} gnn_order_t;

/* Backward scheme (Sec. 3.1, Table "GCN schemes"). */
typedef enum {
    GNN_BWD_AUTO = 0,
    GNN_BWD_FUSED_PROPAGATE = 1,  /* H = A'^T G once (width F_out); dTheta = X^T H; dX = H Theta^T       */
    GNN_BWD_SPLIT_PROPAGATE = 2   /* dTheta = (A'X)^T G; dX = A'^T (G Theta^T): SpMMs of width F_in       */
} gnn_bwd_t;

/* What forward keeps for backward (Sec. 3.1 "Caching intermediate values"; Table "GAT caching"). */
typedef enum {
    GNN_CACHE_AUTO = 0,
    GNN_CACHE_NONE = 1,
    GNN_CACHE_AX = 2,                /* GCN: P = A' X                                                    */
    GNN_CACHE_GAT_FEAT = 3,          /* GAT: M = X Theta                                  (4nhk bytes)   */
    GNN_CACHE_GAT_FEAT_NODEATT = 4,  /* GAT: M, s, d                                      (4nh(k+2))     */
    GNN_CACHE_GAT_FEAT_EDGE = 5      /* GAT: M, edge weights alpha, LeakyReLU mask        (4nhk + 5qh)   */
} gnn_cache_t;

/*
 * A graph: host struct of device arrays.
 *   csr_*      the matrix by rows (always required).  csr_val may be NULL for GAT
 *              (attention ignores edge weights, Sec. 3.2) - never for GCN.
 *   csr_erow   optional for GCN, required for GAT: row index of every stored entry (erow[e] = i for
 *              rowptr[i] <= e < rowptr[i+1]), as written by gnn_expand_ptr.  With it
 *              the sparse kernels split work by equal numbers of entries, which
 *              keeps hub rows from serialising (products of a few thousand rows go
 *              by rows all the same); without it a row is the work of one or eight
 *              wavefronts (sums in another order, slower on skewed graphs).
 *   csc_*      the same matrix by columns, i.e. the CSR arrays of its transpose:
 *              colptr[n+1], row[nnz] ascending inside a column, perm[nnz] mapping a
 *              CSC slot to the CSR slot of the same entry, val = csr_val[perm]
 *              (may be NULL: then values are fetched through perm), ecol = the
 *              expanded column index per CSC slot (like csr_erow: optional for GCN,
 *              required by gat_layer_bwd).
 *              Needed by every backward pass unless `symmetric` is set.
 *   symmetric  nonzero promises A'^T == A' (pattern and values); the CSC arrays
 *              are then ignored and may be NULL.  Only meaningful for GCN and SAGE.
 */
typedef struct {
    int32_t n, nnz;
    const int32_t *csr_rowptr, *csr_col;
    const float *csr_val;
    const int32_t *csr_erow;
    const int32_t *csc_colptr, *csc_row, *csc_perm;
    const float *csc_val;
    const int32_t *csc_ecol;
    int32_t symmetric;
} gnn_graph_t;

typedef struct {
    gnn_layer_t layer;
    int32_t n, nnz;           /* nodes, stored entries (self-loops included)                    */
    int32_t f_in;             /* m                                                              */
    int32_t f_out;            /* k, per head for GAT                                            */
    int32_t heads;            /* GAT only (GCN, SAGE: 1)                                        */
    int32_t need_input_grad;  /* 0: backward skips dX (first layer of a network)                */
    int32_t has_bias;         /* forward adds b, backward writes db                             */
    int32_t fuse_relu;        /* GCN, SAGE: forward applies ReLU, backward masks dY by [Y > 0]  */
    float leaky_slope;        /* GAT only: beta of LeakyReLU                                    */
    gnn_order_t order;        /* AUTO or a forced choice                                        */
    gnn_bwd_t bwd;
    gnn_cache_t cache;
    gnn_select_t selection;   /* how AUTO decides (GCN, SAGE: order and scheme; GAT: the cache variant) */
    int32_t constant_input;   /* GCN, SAGE with the A'X cache: the caller promises that X and the graph
                                 are the same in every forward call until gnn_plan_reset_cache
                                 (a first layer whose input features never change).  Forward then
                                 computes A'X only while the cache is empty, and AUTO counts that
                                 SpMM as free.  A GCN layer reads X only in that first call.       */
    int32_t fuse_elu;         /* GAT only: forward applies ELU (alpha = 1) after the bias, backward
                                 multiplies dY by its derivative taken from the output Y            */
} gnn_plan_desc_t;

typedef struct {
    gnn_order_t order;        /* resolved, never AUTO */
    gnn_bwd_t bwd;
    gnn_cache_t cache;
    size_t cache_bytes;       /* size of the `cache` buffer fwd writes and bwd reads            */
    size_t workspace_bytes;   /* max over fwd and bwd                                           */
    int64_t transient_fwd;    /* number of fp32 transients of the paper's tables (nk / nm ...)  */
    int64_t transient_bwd;
    int64_t spmm_width_fwd;   /* summed dense widths of the SpMMs the scheme runs               */
    int64_t spmm_width_bwd;
} gnn_plan_info_t;

typedef struct gnn_plan gnn_plan_t;

/*
 * gnn_plan_create - choose ordering, backward scheme and cache policy (host only, no device work).
 *
 * GCN, caching allowed (cache = AUTO or AX)        [Table "GCN schemes with caching"]:
 *     with dX:  F_out <  F_in    -> transform-first + fused-propagate, no cache
 *               F_out >= F_in    -> propagate-first caching A'X + split-propagate reading it
 *     no dX:    F_out <  F_in/2  -> transform-first + fused-propagate
 *               F_out >= F_in/2  -> propagate-first with cache + split-propagate with cache
 * GCN, caching forbidden (cache = NONE)            [Table "GCN schemes"]:
 *     forward:  F_out < F_in -> transform-first, else propagate-first
 *     backward: with dX: F_out < 2 F_in -> fused-propagate, else split-propagate
 *               no dX:   F_out <   F_in -> fused-propagate, else split-propagate
 * With selection = CALIBRATED the same candidate schemes are compared by the summed model time
 * of their SpMMs instead (the GEMMs are the same in every scheme); ties go to the rule's choice.
 * With constant_input (and caching allowed) the forward SpMM of the cached scheme costs nothing.
 * Forced `order` / `bwd` values override the rule; cache = AX needs order = PROPAGATE_FIRST
 * (else GNN_ERR_INVALID_ARG).  GAT: order is fixed (node-attention form, App. B);
 * cache AUTO -> GNN_CACHE_GAT_FEAT_EDGE, the fastest variant of Sec. 4.2; with selection = CALIBRATED ->
 * GNN_CACHE_GAT_FEAT_NODEATT, the fastest measured on an MI355X (the edge passes rebuild alpha from four
 * floats per node for less than reading five bytes per entry and head costs).
 * The plan is a host object owned by the caller until gnn_plan_destroy.
 */
gnn_status_t gnn_plan_create(const gnn_plan_desc_t *desc, gnn_plan_t **out);
gnn_status_t gnn_plan_query(const gnn_plan_t *plan, gnn_plan_info_t *out);
void gnn_plan_destroy(gnn_plan_t *plan);

/* Forget that a forward pass has filled the cache (constant_input: the next forward recomputes A'X). */
gnn_status_t gnn_plan_reset_cache(gnn_plan_t *plan);

/*
 * gnn_spmm_time_model_us - the time model behind GNN_SELECT_CALIBRATED (host only): microseconds of
 * one SpMM of dense width f on a graph of n nodes and nnz entries with this library's kernels on an
 * MI355X:  t = 12 + nnz * max(13, c * f) * 1e-6,  c = 0.32 ps per entry and column while the dense
 * operand (D = 4 n f bytes) is below 70 MB, else 0.32 + 0.045 log2(D / 70 MB), at most 0.53.
 * Fitted to measurements on R-MAT graphs of 2^11 .. 2^22 nodes; within about 20 % of them.
 */
double gnn_spmm_time_model_us(int64_t n, int64_t nnz, int32_t f);

/*
 * gcn_layer_fwd - Y = A' X W + 1 b^T (Eq. gcn-fwd), optionally ReLU.
 *   X [n, f_in], W [f_in, f_out], b [f_out] or NULL, Y [n, f_out]           (device)
 *   cache      cache_bytes >= the plan's; written when the plan caches A'X, may be NULL (size 0) otherwise
 *   workspace  workspace_bytes >= the plan's
 * Errors: INVALID_ARG (NULL X / W / Y, b missing while has_bias), BAD_GRAPH
 * (n / nnz differ from the plan, csr arrays or csr_val NULL), BUFFER_TOO_SMALL (cache or
 * workspace smaller than gnn_plan_query reports).
 */
gnn_status_t gcn_layer_fwd(gnn_plan_t *plan, const gnn_graph_t *graph, const float *X, const float *W,
                           const float *b, float *Y, void *cache, size_t cache_bytes,
                           void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * gcn_layer_bwd - dW = X^T A'^T dY, db = dY^T 1, dX = A'^T dY W^T (Eqs. gcn-bwd-*).
 *   X   [n, f_in]; may be NULL when the plan caches A'X (App. A: the input is then not needed)
 *   Y   [n, f_out] forward output; required iff fuse_relu (its sign gives the ReLU mask)
 *   dY  [n, f_out]; dW [f_in, f_out]; db [f_out] (required iff has_bias);
 *   dX  [n, f_in]  (required iff need_input_grad, ignored otherwise)
 * Errors: as forward, plus STATE when the plan caches A'X and no forward has run
 * on this plan since creation, BAD_GRAPH when the graph is not symmetric and
 * the CSC arrays are missing.
 */
gnn_status_t gcn_layer_bwd(gnn_plan_t *plan, const gnn_graph_t *graph, const float *X, const float *W,
                           const float *Y, const float *dY, float *dW, float *db, float *dX,
                           void *cache, size_t cache_bytes, void *workspace, size_t workspace_bytes,
                           void *hip_stream);

/*
 * sage_layer_fwd / sage_layer_bwd - a GraphSAGE layer, the other layer that Sec. 3.1 "Generalizability"
 * names for the same chained product:  Y = X W_self + A' X W_neigh + 1 b^T  (optionally ReLU), with A'
 * the row-normalised pattern (gnn_aggregator_weights, GNN_AGG_MEAN) or any other entry values.
 * The plan is made with layer = GNN_LAYER_SAGE; order, backward scheme, cache (A'X) and their AUTO
 * choice are those of GCN, since the SpMM widths are the same (F_out transform-first, F_in propagate-first).
 *   X [n, f_in], W_self / W_neigh [f_in, f_out], b [f_out] or NULL, Y [n, f_out]
 *   backward: dW_self = X^T G, dW_neigh = (A'X)^T G, db = G^T 1, dX = G W_self^T + A'^T G W_neigh^T
 *   (G = dY, masked by [Y > 0] with fuse_relu).  X is needed by backward in every scheme.
 *   dX and dY may share memory with fuse_relu only (in gcn_layer_bwd always): without it dY is read after dX is written.
 * cache / workspace sizes: gnn_plan_query.  Errors as gcn_layer_fwd / gcn_layer_bwd.
 */
gnn_status_t sage_layer_fwd(gnn_plan_t *plan, const gnn_graph_t *graph, const float *X, const float *W_self,
                            const float *W_neigh, const float *b, float *Y, void *cache, size_t cache_bytes,
                            void *workspace, size_t workspace_bytes, void *hip_stream);
gnn_status_t sage_layer_bwd(gnn_plan_t *plan, const gnn_graph_t *graph, const float *X, const float *W_self,
                            const float *W_neigh, const float *Y, const float *dY, float *dW_self,
                            float *dW_neigh, float *db, float *dX, void *cache, size_t cache_bytes,
                            void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * gat_layer_fwd - multi-head GAT forward (Eqs. gat-fwd, gat-fwd-att), heads concatenated.
 *   X [n, f_in], W [f_in, heads*f_out], a_src / a_dst [heads, f_out], b [heads*f_out] or NULL,
 *   Y [n, heads*f_out] laid out [n][head][f_out] (head is the middle axis, Sec. 3.2);
 *   with fuse_elu, Y = ELU(aggregate + b) (the activation of the paper's two-layer GAT, Sec. 4).
 *   a_src multiplies the features of the row (aggregating) node, a_dst those of
 *   the column (neighbour) node: logit(i, j) = <a_src, m_i> + <a_dst, m_j>.
 *   The softmax runs over the stored entries of row i; csr_val is ignored.
 *   cache layout (all fp32 unless noted, each block 256-byte aligned, in this order):
 *     GAT_FEAT:         M [n][h][k]
 *     GAT_FEAT_NODEATT: M, s [n][h], d [n][h]
 *     GAT_FEAT_EDGE:    M, alpha [nnz][h], mask [nnz][h] uint8 (1 where the logit is > 0)
 */
gnn_status_t gat_layer_fwd(gnn_plan_t *plan, const gnn_graph_t *graph, const float *X, const float *W,
                           const float *a_src, const float *a_dst, const float *b, float *Y,
                           void *cache, size_t cache_bytes, void *workspace, size_t workspace_bytes,
                           void *hip_stream);

/*
 * gat_layer_bwd - gradients of Sec. "GAT Backward Pass": dW [f_in, h*k], da_src / da_dst [h, k],
 *   db [h*k] (iff has_bias), dX [n, f_in] (iff need_input_grad).  Needs the CSC arrays and perm.
 *   Y [n, h*k]: the forward output; required iff fuse_elu (ELU'(x) = 1 for x > 0, else Y + 1).
 *   Whatever the cache variant did not keep is recomputed with the forward kernels.
 */
gnn_status_t gat_layer_bwd(gnn_plan_t *plan, const gnn_graph_t *graph, const float *X, const float *W,
                           const float *a_src, const float *a_dst, const float *Y, const float *dY,
                           float *dW, float *da_src, float *da_dst, float *db, float *dX,
                           void *cache, size_t cache_bytes, void *workspace, size_t workspace_bytes,
                           void *hip_stream);

/* ---- preprocessing: integer kernels and the normalisation (Sec. "GCN Forward Pass") ---- */

/*
 * gnn_add_self_loops_degree - pattern of A + I and its row degrees.
 *   in:  rowptr [n+1], col [nnz] (ascending rows; a diagonal entry may already be there)
 *   out: rowptr_out [n+1], col_out [capacity nnz + n], deg_out [n] = entries per row of A + I
 *   nnz_out_host: HOST pointer; receives rowptr_out[n].  This call synchronises the stream.
 *   workspace: gnn_scan_workspace_bytes(n) bytes.
 */
gnn_status_t gnn_add_self_loops_degree(int32_t n, int32_t nnz, const int32_t *rowptr, const int32_t *col,
                                       int32_t *rowptr_out, int32_t *col_out, int32_t *deg_out,
                                       int32_t *nnz_out_host, void *workspace, size_t workspace_bytes,
                                       void *hip_stream);
size_t gnn_scan_workspace_bytes(int32_t n);

/* val_out[e] = 1 / sqrt(deg[i] * deg[col[e]]) for every stored entry e of row i. */
gnn_status_t gnn_gcn_normalize(int32_t n, const int32_t *rowptr, const int32_t *col, const int32_t *deg,
                               float *val_out, void *hip_stream);

/*
 * gnn_aggregator_weights - entry values for the other layers with the same chained product A' X Theta
 * (Sec. 3.1 "Generalizability"; App. "GCN Forward Pass": mean aggregation is D A X Theta), on the
 * pattern of A + I with the degrees written by gnn_add_self_loops_degree:
 *   GNN_AGG_GCN_SYM  1 / sqrt(deg_i deg_j)            (what gnn_gcn_normalize writes)
 *   GNN_AGG_MEAN     1 / deg_i                         (row-normalised: mean over N(i) and i itself)
 *   GNN_AGG_GIN_SUM  1, and 1 + eps on the diagonal    (the sum aggregation of a GIN layer)
 * The mean weights are not symmetric: the graph then needs its CSC arrays (symmetric = 0) for backward.
 */
typedef enum { GNN_AGG_GCN_SYM = 0, GNN_AGG_MEAN = 1, GNN_AGG_GIN_SUM = 2 } gnn_aggregator_t;
gnn_status_t gnn_aggregator_weights(gnn_aggregator_t kind, float eps, int32_t n, const int32_t *rowptr,
                                    const int32_t *col, const int32_t *deg, float *val_out, void *hip_stream);

/*
 * gnn_csr_transpose - CSC arrays of a CSR matrix (App. D.1): colptr_out [n+1], row_out [nnz]
 * ascending inside every column, perm_out [nnz] (CSC slot -> CSR slot).  Deterministic:
 * a stable radix sort of the row-major entries by column.
 */
gnn_status_t gnn_csr_transpose(int32_t n, int32_t nnz, const int32_t *rowptr, const int32_t *col,
                               int32_t *colptr_out, int32_t *row_out, int32_t *perm_out,
                               void *workspace, size_t workspace_bytes, void *hip_stream);
size_t gnn_transpose_workspace_bytes(int32_t n, int32_t nnz);

/* out[e] = i for ptr[i] <= e < ptr[i+1]  (the COO row array of App. D.2, from CSR). */
gnn_status_t gnn_expand_ptr(int32_t n, int32_t nnz, const int32_t *ptr, int32_t *out, void *hip_stream);

/* out[p] = in[perm[p]] (e.g. csc_val from csr_val). */
gnn_status_t gnn_gather_f32(int64_t count, const float *in, const int32_t *perm, float *out, void *hip_stream);

/* ---- the sparse and dense operators on their own (App. E) ---- */

/*
 * gnn_spmm_csr - C = A B (App. E.1).  B, C [n, f].  val NULL = all ones.
 *   erow: optional expanded row index (see gnn_graph_t).  Products of more than a few thousand rows are then split by entries
 *   instead of by rows; smaller ones go by rows with it or without.
 *   bias [f] or NULL, relu (0 or 1; anything else is GNN_ERR_INVALID_ARG): fused epilogue C = relu(A B + 1 b^T).
 *   workspace: gnn_spmm_workspace_bytes(n, nnz, f) bytes (only used with erow): partial rows of the
 *   blocks, when f is not a multiple of 4 a copy of B with rows padded to the next multiple of 4, and for
 *   products of 2e9 multiplications and more the lists and partial rows of long rows computed in pieces.
 *   B and C may start at any 4-byte aligned address; 16-byte aligned rows take the fastest kernel.
 */
gnn_status_t gnn_spmm_csr(int32_t n, int32_t nnz, const int32_t *rowptr, const int32_t *col, const float *val,
                          const int32_t *erow, const float *B, int32_t f, float *C,
                          const float *bias, int32_t relu,
                          void *workspace, size_t workspace_bytes, void *hip_stream);
size_t gnn_spmm_workspace_bytes(int32_t n, int32_t nnz, int32_t f);

/*
 * gnn_spmm_csr_static - gnn_spmm_csr for callers that cannot allocate device memory and have no workspace
 * to pass: code under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same
 * arguments, kernels and results as gnn_spmm_csr; the scratch (partial rows, padded operand) is a device
 * array of GNN_STATIC_SCRATCH_BYTES bytes inside the library, one copy per GPU, held until the process ends.
 * The call allocates nothing and frees nothing.
 *   Errors: as gnn_spmm_csr; GNN_ERR_BUFFER_TOO_SMALL when those two exceed GNN_STATIC_SCRATCH_BYTES (then use
 *   gnn_spmm_csr with a workspace).  Large products whose long rows gnn_spmm_csr computes in pieces, with a workspace for
 *   those, are computed without pieces here: results equal to rounding.
 *   The first call on a device looks up the array's address there (make it outside a graph capture).
 *   All calls on one GPU share that GPU's array: calls that may overlap in time on one GPU (different
 *   streams, or several host threads) race; calls on one stream are ordered and safe.  Nothing in the
 *   array needs clearing between calls: every partial row is written before it is read.
 */
#define GNN_STATIC_SCRATCH_BYTES (32u << 20)
gnn_status_t gnn_spmm_csr_static(int32_t n, int32_t nnz, const int32_t *rowptr, const int32_t *col, const float *val,
                                 const int32_t *erow, const float *B, int32_t f, float *C,
                                 const float *bias, int32_t relu, void *hip_stream);

/*
 * Storage formats other than CSR (App. D.2 coordinate, D.3 ELLPACK, D.4 hybrid) and SpMM on them, for the
 * format comparison of App. E.1.  The layers never use them.
 *   ELLPACK arrays ell_col / ell_val [t][n] are slot-major: slot j of row i at [j * n + i]; a row's stored
 *   entries fill its slots from the front, padding has column -1 and value 0.  With t >= the longest row this
 *   is plain ELLPACK (p = t); with a smaller t it is the hybrid format: the first t entries of every row in
 *   the ELLPACK arrays, the others row-major in coordinate arrays coo_row / coo_col / coo_val [rest_nnz].
 *
 * gnn_csr_hyb_count - rest_ptr_out [n+1] (device) = exclusive scan of max(0, row length - t);
 *   rest_nnz_out_host / max_row_out_host: HOST pointers receiving rest_ptr_out[n] and the longest row
 *   (either may be NULL).  Synchronises the stream.  workspace: gnn_hyb_workspace_bytes(n).
 * gnn_csr_to_hyb - fills the arrays; val NULL = all ones.  rest_ptr NULL: no coordinate part is written
 *   (entries beyond slot t are dropped, so pass t >= the longest row).  t = 0: everything goes to the
 *   coordinate arrays (ell_* may be NULL).
 * gnn_spmm_ell - C = A B from the ELLPACK arrays.  Deterministic.
 * gnn_spmm_coo - C = A B (accumulate = 0: C is cleared first) or C += A B (accumulate != 0) from
 *   coordinate arrays in any order; val NULL = all ones.  Uses fp32 atomic additions: the result is
 *   reproducible only up to fp32 rounding.
 * gnn_spmm_hyb - gnn_spmm_ell on the first t slots, then gnn_spmm_coo accumulating the rest.
 *   B, C [n, f] row-major.  Errors: GNN_ERR_INVALID_ARG for negative sizes / NULL required pointers.
 */
size_t gnn_hyb_workspace_bytes(int32_t n);
gnn_status_t gnn_csr_hyb_count(int32_t n, const int32_t *rowptr, int32_t t, int32_t *rest_ptr_out,
                               int32_t *rest_nnz_out_host, int32_t *max_row_out_host,
                               void *workspace, size_t workspace_bytes, void *hip_stream);
gnn_status_t gnn_csr_to_hyb(int32_t n, int32_t t, const int32_t *rowptr, const int32_t *col, const float *val,
                            const int32_t *rest_ptr, int32_t *ell_col, float *ell_val,
                            int32_t *coo_row, int32_t *coo_col, float *coo_val, void *hip_stream);
gnn_status_t gnn_spmm_ell(int32_t n, int32_t t, const int32_t *ell_col, const float *ell_val,
                          const float *B, int32_t f, float *C, void *hip_stream);
gnn_status_t gnn_spmm_coo(int32_t n, int64_t nnz, const int32_t *row, const int32_t *col, const float *val,
                          const float *B, int32_t f, float *C, int32_t accumulate, void *hip_stream);
gnn_status_t gnn_spmm_hyb(int32_t n, int32_t t, const int32_t *ell_col, const float *ell_val,
                          int64_t rest_nnz, const int32_t *coo_row, const int32_t *coo_col, const float *coo_val,
                          const float *B, int32_t f, float *C, void *hip_stream);

/*
 * gnn_sddmm_csr - D_e = val_e * <B_i, Ct_j> for every stored entry e = (i, j) (App. E.2),
 *   batched over `heads` with the head as the middle axis: B, Ct [n][heads][f], D [nnz][heads].
 *   Ct is the transpose of the paper's C (row j = column j of C).  val NULL = all ones.
 *   erow [nnz]: the row i of every entry (gnn_expand_ptr of the row pointers); the kernel is
 *   one thread per (entry, head), so it needs no row pointers.
 */
gnn_status_t gnn_sddmm_csr(int32_t n, int32_t nnz, const int32_t *erow, const int32_t *col, const float *val,
                           const float *B, const float *Ct, int32_t heads, int32_t f, float *D,
                           void *hip_stream);

/*
 * gnn_gat_aggregate_csr - the edge phase of the GAT forward pass as one operator (Eqs. gat-fwd-att, gat-fwd):
 *   alpha_e = softmax over the stored entries of row i of LeakyReLU(s_i + d_j)   per head,
 *   Y_{i,p,:} = sum_e alpha_{e,p} M_{col e,p,:} (+ bias, then ELU if elu != 0),
 * in a single pass over the entries: the logits, the running softmax and the weighted sum stay in registers,
 * no per-edge array is written.  M, Y [n][heads][f]; s, d [n][heads] (App. B: s_i = <a_src, m_i>,
 * d_j = <a_dst, m_j>); bias [heads * f] or NULL;
 * stat_out [n][heads][2] receives (row maximum of the LeakyReLU'd logits, sum of exp(. - maximum)), from which
 * alpha_e = exp(w_e - max) / sum.  erow [nnz]: row of every entry (gnn_expand_ptr).
 *   f: a multiple of 4 with f / 4 a power of two, at most 256; M, Y and bias 16-byte aligned; n below 2^24,
 *   M below 4 GiB and nnz * heads below 2^30 (the gathers use 32-bit byte offsets)
 *   (GNN_ERR_UNSUPPORTED otherwise: gat_layer_fwd then runs the steps as separate kernels).
 *   workspace: gnn_gat_aggregate_workspace_bytes(nnz, heads, f).
 */
gnn_status_t gnn_gat_aggregate_csr(int32_t n, int32_t nnz, const int32_t *rowptr, const int32_t *erow,
                                   const int32_t *col, const float *M, const float *s, const float *d,
                                   int32_t heads, int32_t f, float leaky_slope, const float *bias, int32_t elu,
                                   float *Y, float *stat_out, void *workspace, size_t workspace_bytes,
                                   void *hip_stream);
size_t gnn_gat_aggregate_workspace_bytes(int32_t nnz, int32_t heads, int32_t f);

/*
 * gnn_gemm - C = op(A) op(B) on the matrix cores: fp32 operands and results; fp32 accumulation,
 *   except that the transposed-A form accumulates in fp64 (its reduction runs over all nodes).
 *   trans_a == 0: A is [M, K] else A is [K, M] and used transposed (then K may be huge:
 *   the product is split along K and reduced in a fixed order; deterministic).
 *   trans_b == 0: B is [K, N] else B is [N, K].  C is [M, N].  All row-major, dense (ld = columns).
 *   bias [N] or NULL, relu: fused epilogue.  Supported: (0,0), (0,1), (1,0).
 *   relu is a flag word: GNN_GEMM_RELU (1) applies max(., 0); GNN_GEMM_ACCUMULATE (4) adds the
 *   product (and bias) to what C holds before the ReLU, trans_a == 0 only (GNN_ERR_UNSUPPORTED
 *   otherwise); any other bit is GNN_ERR_INVALID_ARG.
 *   workspace: gnn_gemm_workspace_bytes(trans_a, trans_b, M, N, K); required for (0,0) (holds B in the
 *   form the product reads) and (1,0) (holds the partial products); (0,1) runs without, faster with.
 *   A workspace for K serves every smaller K.
 */
enum { GNN_GEMM_RELU = 1, GNN_GEMM_ACCUMULATE = 4 };
gnn_status_t gnn_gemm(int32_t trans_a, int32_t trans_b, int64_t M, int64_t N, int64_t K,
                      const float *A, const float *B, float *C, const float *bias, int32_t relu,
                      void *workspace, size_t workspace_bytes, void *hip_stream);
size_t gnn_gemm_workspace_bytes(int32_t trans_a, int32_t trans_b, int64_t M, int64_t N, int64_t K);

/*
 * gnn_softmax_xent - sum-reduced softmax cross-entropy over the rows of Z [n, c] with
 * integer labels [n]; writes dZ = softmax(Z) - onehot [n, c] and loss_out[0] (device, fp32).
 * (The loss used on the two-layer GCN workload; not part of a layer.)
 *   workspace: 4 * ceil(n / 256) bytes.
 */
gnn_status_t gnn_softmax_xent(int32_t n, int32_t c, const float *Z, const int32_t *labels, float *dZ,
                              float *loss_out, void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * gnn_sum_squared_error - loss_out[0] = 1/2 sum (Z - T)^2 over `count` elements and dZ = Z - T
 * (the squared-error loss of the paper's full-network runs, Sec. 4, sum-reduced so that the
 * gradient entries are O(1)).  Deterministic two-stage sum.  workspace: 4096 bytes.
 */
gnn_status_t gnn_sum_squared_error(int64_t count, const float *Z, const float *T, float *dZ, float *loss_out,
                                   void *workspace, size_t workspace_bytes, void *hip_stream);

/* ---- between the layers: dropout, layer norm, residual connections, gated feed-forward blocks ---- */

/*
 * gnn_dropout_t - which elements of an [n, f] array are dropped: a HOST struct that names the generator.
 *   p      probability of an element to be dropped, 0 <= p < 1; the others are multiplied by 1 / (1 - p)
 *   site   which dropout of a network this is: calls with different sites drop independently
 *   state  DEVICE pointer to {seed, step}, 8-byte aligned; may be NULL where p is 0.  Read by the kernels, so that a captured
 *          graph draws anew on every replay once the step is advanced (gnn_rng_advance, on the stream, after the backward pass).
 * Element (i, c) is dropped where word c % 4 of the Philox4x32-10 block (Salmon, Moraes, Dror, Shaw, "Parallel random
 * numbers: as easy as 1, 2, 3", SC 2011) with key = seed and counter = (c / 4, i, site, low 32 bits of step) is below
 * round(p 2^32).  The mask depends on nothing else and is never stored: backward forms it again from the same struct, and every
 * operator below that is given the same struct and shape drops the same elements.  What is dropped becomes 0, infinities and NaN too.
 */
typedef struct {
    float p;
    uint32_t site;
    const uint64_t *state;
} gnn_dropout_t;

/* step += by, in device memory. */
gnn_status_t gnn_rng_advance(uint64_t *state, uint64_t by, void *hip_stream);

/*
 * gnn_dropout - Y = R + dropout(X), all [n, f]; R NULL: Y = dropout(X).  drop NULL (or p = 0): nothing is dropped.
 *   The gradient with respect to X is the same call on dY without R, that with respect to R is dY.
 *   Y may be X or R.  Errors: INVALID_ARG (NULL X / Y, negative n, f < 1, p outside [0, 1), state NULL or misaligned),
 *   UNSUPPORTED (f beyond 2^30).
 */
gnn_status_t gnn_dropout(int32_t n, int32_t f, const float *X, const float *R, const gnn_dropout_t *drop, float *Y,
                         void *hip_stream);

/*
 * ELU with alpha = 1; the last three are those of gnn_gate_t, for the products below (gnn_linear_..): a layer norm takes the first three.
 * In these products a sigmoid and the normal distribution's integral are off by what one unit in the last place of their argument is worth
 * and a few units of their own; arguments beyond some 87 (of GELU some 13) below zero give 0.
 */
typedef enum {
    GNN_ACT_NONE = 0, GNN_ACT_RELU = 1, GNN_ACT_ELU = 2, GNN_ACT_SIGMOID = 3, GNN_ACT_SILU = 4, GNN_ACT_GELU = 5
} gnn_act_t;

/*
 * gnn_layer_norm_fwd - Y = dropout(act(gamma xhat + beta)), xhat = (x - mean) rstd over the f columns of a row,
 *   rstd = 1 / sqrt(variance + eps) with the variance divided by f.  X, Y [n, f]; gamma, beta [f] or NULL (1 and 0);
 *   ELU with alpha = 1; drop NULL: no dropout; stat_out [n][2] = (mean, rstd), which backward reads.  Y may be X (where no
 *   backward pass follows: that needs X).
 * gnn_layer_norm_bwd - from X, stat and dY [n, f] the gradients dX [n, f], dgamma and dbeta [f]; any of them may be NULL.  The
 *   activation's derivative is taken from gamma xhat + beta, formed again as in forward (ReLU' = 0 at 0, NaN at NaN), the mask of dropout
 *   likewise: act, drop, gamma and beta as in forward.  dX may be dY.  The sums over the rows have a fixed order.
 *   workspace: gnn_layer_norm_workspace_bytes(n, f), which does not fall as n grows; not used where dgamma and dbeta are NULL
 *   (then it may be NULL).
 * Errors: INVALID_ARG (NULL X / Y / stat / dY, negative n, f < 1, eps below the least normal float or not finite, act no
 *   gnn_act_t, drop as in gnn_dropout, workspace NULL or not 256-byte aligned), BUFFER_TOO_SMALL, UNSUPPORTED (f beyond 2^24, or
 *   2^24 rows and more of f beyond 4096).
 */
gnn_status_t gnn_layer_norm_fwd(int32_t n, int32_t f, const float *X, const float *gamma, const float *beta, float eps,
                                gnn_act_t act, const gnn_dropout_t *drop, float *Y, float *stat_out, void *hip_stream);
gnn_status_t gnn_layer_norm_bwd(int32_t n, int32_t f, const float *X, const float *stat, const float *gamma,
                                const float *beta, gnn_act_t act, const gnn_dropout_t *drop, const float *dY, float *dX,
                                float *dgamma, float *dbeta, void *workspace, size_t workspace_bytes, void *hip_stream);
size_t gnn_layer_norm_workspace_bytes(int32_t n, int32_t f);

/*
 * gnn_add_layer_norm_fwd - the end of one residual block and the norm that begins the next:
 *   H = R + dropout(X), Y = gamma xhat(H) + beta.  X, R, H, Y [n, f]; H may be X or R; stat_out as above, of H.
 * gnn_add_layer_norm_bwd - dR = dH + (gradient of the norm at H, from dY), dX = dropout(dR); dH [n, f] is what flows back
 *   into H from elsewhere, NULL: nothing.  dX NULL: not written (without dropout it is dR).  dR and dX may each be dY or dH, but
 *   not the same array.  dgamma and dbeta may be NULL.  workspace: gnn_layer_norm_workspace_bytes(n, f).
 * Errors: as gnn_layer_norm_fwd / _bwd; NULL R, H, dR are INVALID_ARG as well.
 */
gnn_status_t gnn_add_layer_norm_fwd(int32_t n, int32_t f, const float *X, const float *R, const gnn_dropout_t *drop,
                                    const float *gamma, const float *beta, float eps, float *H, float *Y, float *stat_out,
                                    void *hip_stream);
gnn_status_t gnn_add_layer_norm_bwd(int32_t n, int32_t f, const float *H, const float *stat, const float *gamma,
                                    const gnn_dropout_t *drop, const float *dY, const float *dH, float *dR, float *dX,
                                    float *dgamma, float *dbeta, void *workspace, size_t workspace_bytes, void *hip_stream);

/* The activation of a gate: 1 / (1 + exp(-a)), a / (1 + exp(-a)), a Phi(a) with Phi the normal distribution (by erf). */
typedef enum { GNN_GATE_SIGMOID = 0, GNN_GATE_SILU = 1, GNN_GATE_GELU = 2 } gnn_gate_t;

/*
 * gnn_gated_fwd - the two projections of a gated feed-forward block, the activation and the product:
 *   [A | U] = X W + 1 b^T,  H = act(A) .* U.   X [n, f_in], W [f_in, 2 f_out] = [W_gate | W_up], b [2 f_out] or NULL, H [n, f_out].
 *   (The projection back is gnn_gemm, or the product of the next layer.)
 *   Z [n, 2 f_out] or NULL: receives [A | U], which backward may read instead of forming it again.
 * gnn_gated_bwd - with D = [dH .* U .* act'(A) | dH .* act(A)]:  dW = X^T D [f_in, 2 f_out], db = D^T 1 [2 f_out] (NULL: not
 *   wanted), dX = D W^T [n, f_in] (NULL: not wanted).  Z as forward left it, or NULL: [A | U] is formed again from X, W and b.
 *   Sums are fp32 or better everywhere.  Products of many rows over 32 and more indices (f_in of them forward, 2 f_out in dX, n
 *   in dW) take a float as two fp16 numbers: one is off by up to 8 u (u = 2^-24; a float product by u), and by an operand's
 *   loss of 2^-50 of the largest of its row (of X, D) or column (of W; of X and D in dW, in chunks of 4096 rows), which shows where
 *   operands lie below 2^-27 of it.  Root mean square errors are no larger than those of a chain of float multiplications and
 *   additions.  Shorter products are those of floats.  Few rows: float products forward, gnn_gemm's for dX, doubles for dW, but for
 *   dW of 2^19 elements and more the two fp16 numbers again, or floats below 32 rows.
 *   Outputs must not overlap inputs or each other.
 *   workspace: gnn_gated_workspace_bytes(backward, n, f_in, f_out), backward 0 or 1; what it returns does not fall as n grows.
 * Errors: INVALID_ARG (NULL X / W / H / dH / dW, negative n, f_in < 1 or f_out < 1, gate no gnn_gate_t, workspace NULL or not
 *   256-byte aligned), BUFFER_TOO_SMALL, UNSUPPORTED (f_in or f_out beyond 2^21; ceil(n / 32) ceil(max(f_in, f_out) / 64) from 2^24
 *   on, of f_in below 4 or f_out 1 ceil(n / 32) ceil(f_out / 32); backward also (f_in + 1) f_out from 2^28 on, and 64 x 64 tiles of
 *   dW times n / 4096 from 2^24 on).
 */
gnn_status_t gnn_gated_fwd(gnn_gate_t gate, int32_t n, int32_t f_in, int32_t f_out, const float *X, const float *W,
                           const float *b, float *H, float *Z, void *workspace, size_t workspace_bytes, void *hip_stream);
gnn_status_t gnn_gated_bwd(gnn_gate_t gate, int32_t n, int32_t f_in, int32_t f_out, const float *X, const float *W,
                           const float *b, const float *Z, const float *dH, float *dW, float *db, float *dX,
                           void *workspace, size_t workspace_bytes, void *hip_stream);
size_t gnn_gated_workspace_bytes(int32_t backward, int32_t n, int32_t f_in, int32_t f_out);

/* ---- rows in 8 bits; root-mean-square norm; products with their epilogue ---- */

/*
 * gnn_rows8_t - an [n, f] array held in 8 bits, a scale for each row: a HOST struct of device arrays.
 *   q        integers from -127 to 127, rows gnn_rows8_stride(f) bytes apart (f rounded up to a multiple of 16); 16-byte aligned.  The
 *            bytes behind a row's f may hold anything
 *   scale    [n]
 *   columns  [f], or NULL: all ones.  Read where the array is an input that says so
 * Element (i, c) is q[i][c] * scale[i] * columns[c].
 */
typedef struct {
    int8_t *q;
    float *scale;
    const float *columns;
} gnn_rows8_t;
int64_t gnn_rows8_stride(int32_t f);

/*
 * gnn_quantize_rows - out = X .* columns in 8 bits.  X [n, f], columns [f] or NULL.  With x a row of X .* columns and a its largest
 *   magnitude: q = round(x * (127 / a)), ties to even, scale = a / 127; the product with columns, the quotients and the product are each
 *   rounded to a float (with the exponent range of one extended below, so that rows of the least floats keep their digits; a scale
 *   below the least normal float does not).  An element is off by at most (0.5 + 127 x 2^-23) scale.  A row of zeros has scale 0; a
 *   row with an infinity or a NaN in it has integers 0 and scale NaN, so that every element of it is NaN.  out->columns has to be NULL.
 * gnn_dequantize_rows - Y [n, f] = the elements of `in`, in->columns included.
 * Errors: INVALID_ARG (NULL X / Y / struct / q / scale, q not 16-byte aligned, out->columns not NULL, negative n, f < 1), UNSUPPORTED
 *   (f beyond 2^24, or 2^24 rows and more of f beyond 4096).
 */
gnn_status_t gnn_quantize_rows(int32_t n, int32_t f, const float *X, const float *columns, const gnn_rows8_t *out, void *hip_stream);
gnn_status_t gnn_dequantize_rows(int32_t n, int32_t f, const gnn_rows8_t *in, float *Y, void *hip_stream);

/*
 * gnn_rms_norm_fwd - H = R + dropout(X), Y = gamma xhat with xhat = h rstd, rstd = 1 / sqrt(mean of h^2 over the f columns + eps).
 *   X, R, H, Y [n, f]; gamma [f] or NULL (1).  R NULL: H is X, and H and drop have to be NULL (or p = 0).  H may be X or R; Y may be X where
 *   R is NULL.
 *   xhat8 or NULL: receives xhat (without gamma) in 8 bits.  Its integers are those of H (gnn_quantize_rows), its scale that of H times
 *   rstd.  gnn_rms_norm_bwd reads them instead of H; with `columns` set to gamma the same rows are Y, for gnn_linear_bwd.
 *   Y NULL: not wanted (xhat8 is then).  rstd_out [n] or NULL: for backward.
 *   A row whose squares add up to more than the largest float has xhat = 0.
 * gnn_rms_norm_bwd - dR = dH + rstd (g - xhat mean(g xhat)) with g = gamma dY, dX = dropout(dR), dgamma = sum over the rows of dY xhat;
 *   any of them may be NULL.  dH [n, f] is what flows back into H from elsewhere, NULL: nothing.  xhat from H and rstd, or from xhat8
 *   (whose columns are not read): one of them is NULL.  dR and dX may each be dY or dH, but not the same array.  The sums over the rows
 *   have a fixed order.
 *   workspace: gnn_rms_norm_workspace_bytes(n, f), which does not fall as n grows; not used where dgamma is NULL (then it may be NULL).
 * Errors: INVALID_ARG (NULL X; with R NULL H or a dropout, with R H NULL or Y; Y and xhat8 both NULL; a bad xhat8 as in
 *   gnn_quantize_rows; backward: NULL rstd / dY, H and xhat8 both or neither; dR == dX; negative n, f < 1, eps below the least normal
 *   float or not finite, drop as in gnn_dropout, workspace NULL or not 256-byte aligned), BUFFER_TOO_SMALL, UNSUPPORTED (as
 *   gnn_quantize_rows).
 */
gnn_status_t gnn_rms_norm_fwd(int32_t n, int32_t f, const float *X, const float *R, const gnn_dropout_t *drop, const float *gamma,
                              float eps, float *H, float *Y, const gnn_rows8_t *xhat8, float *rstd_out, void *hip_stream);
gnn_status_t gnn_rms_norm_bwd(int32_t n, int32_t f, const float *H, const gnn_rows8_t *xhat8, const float *rstd, const float *gamma,
                              const gnn_dropout_t *drop, const float *dY, const float *dH, float *dR, float *dX, float *dgamma,
                              void *workspace, size_t workspace_bytes, void *hip_stream);
size_t gnn_rms_norm_workspace_bytes(int32_t n, int32_t f);

/*
 * gnn_linear_fwd - Y = act(Z) + R, Z = X W + 1 b^T.  X [n, f_in], W [f_in, f_out], b [f_out] or NULL, R [n, f_out] or NULL, Y [n, f_out].
 *   Z [n, f_out] or NULL: receives X W + b, which backward may read instead of forming it again.  Y may be R.
 * gnn_linear_bwd - with D = dY .* act'(Z):  dW = X^T D [f_in, f_out], db = D^T 1 [f_out] (NULL: not wanted), dX = D W^T [n, f_in] (NULL: not
 *   wanted).  (The gradient of R is dY.)  ReLU' = 0 at 0, NaN at NaN.
 *   X, or X8: the rows in 8 bits, columns included; one of them is NULL.
 *   Z as forward left it, or Z8: the same in 8 bits, columns included, or neither: Z is formed again from X, W and b, and X8 will not do.
 *   GNN_ACT_NONE reads neither of them.
 *   Sums are fp32 or better everywhere.  Products of many rows over 32 and more indices (f_in of them forward, f_out in dX, n in dW)
 *   take a float as two fp16 numbers: one is off by up to 8 u (u = 2^-24; a float product by u), and by an operand's loss of 2^-40 of the
 *   largest of its row (of X, D) or column (of W; of X and D in dW, in chunks of 4096 rows), or of 2^-151 where that is more.  The loss
 *   shows where operands lie below 2^-16 of that largest; above it root mean square errors are no larger than those of a chain of float
 *   multiplications and additions.  (Some of them lose 2^-50, from 2^-27 on: those of few columns, and X W where an X whose f_in is a
 *   multiple of four is not 16-byte aligned.)  Few rows and shorter products: those of floats, in chains of 1024 rows at most in dW, or
 *   doubles.  From X8 dW is as exact: an integer is one fp16 number, and its row's scale goes to the row of D.
 *   Outputs must not overlap inputs or each other, but for Y and R.
 *   workspace: gnn_linear_workspace_bytes(backward, n, f_in, f_out), backward 0 or 1; what it returns does not fall as n grows.
 * Errors: INVALID_ARG (NULL X / W / Y / dY / dW, X and X8 both or neither, Z and Z8 both, X8 without Z or Z8 where act is not
 *   GNN_ACT_NONE, q not 16-byte aligned or NULL, scale NULL, negative n, f_in < 1 or f_out < 1, act no gnn_act_t, workspace NULL or not
 *   256-byte aligned), BUFFER_TOO_SMALL, UNSUPPORTED (as gnn_gated_fwd / _bwd, f_out in place of 2 f_out).
 */
gnn_status_t gnn_linear_fwd(gnn_act_t act, int32_t n, int32_t f_in, int32_t f_out, const float *X, const float *W, const float *b,
                            const float *R, float *Y, float *Z, void *workspace, size_t workspace_bytes, void *hip_stream);
gnn_status_t gnn_linear_bwd(gnn_act_t act, int32_t n, int32_t f_in, int32_t f_out, const float *X, const gnn_rows8_t *X8,
                            const float *W, const float *b, const float *Z, const gnn_rows8_t *Z8, const float *dY, float *dW,
                            float *db, float *dX, void *workspace, size_t workspace_bytes, void *hip_stream);
size_t gnn_linear_workspace_bytes(int32_t backward, int32_t n, int32_t f_in, int32_t f_out);

/*
 * gnn_linear8_fwd - Y = act(X W^T + 1 b^T) + R of two arrays in 8 bits: X [n, f_in], W [f_out, f_in], a row for each column of Y (gnn_quantize_rows
 *   of the transposed weights, once); b [f_out] or NULL, R and Y [n, f_out], R or NULL.  The sums over f_in are of integers and exact.
 *   Behind an RMS norm X is its xhat8, and gamma goes into the weights (gnn_quantize_rows' columns): both `columns` have to be NULL here.
 *   Y may be R.  No workspace.
 * Errors: INVALID_ARG (NULL Y, X or W or one of their arrays, columns not NULL, q not 16-byte aligned, negative n, f_in < 1 or f_out < 1, act
 *   no gnn_act_t), UNSUPPORTED (f_in beyond 2^17, whose sums 32 bits hold, f_out beyond 2^21, ceil(n / 32) ceil(f_out / 32) from 2^24 on).
 */
gnn_status_t gnn_linear8_fwd(gnn_act_t act, int32_t n, int32_t f_in, int32_t f_out, const gnn_rows8_t *X, const gnn_rows8_t *W,
                             const float *b, const float *R, float *Y, void *hip_stream);

const char *gnn_status_string(gnn_status_t status);

#ifdef __cplusplus
}
#endif
#endif /* GNN_H */
