/*
 * bpt.h -- C ABI of the B200 (sm_100a) implementation of BP-Transformer's graph
 * self-attention (arXiv 1911.04070).
 *
 * The library builds the binary-partition attention graph of Sec. 3.2 on the
 * device and evaluates graph self-attention with tree relative positions
 * (Sec. 3.1 and 3.4) forward and backward over it.
 *
 * Conventions (0-indexed): n tokens (a power of two), L = log2 n, node (l, m)
 * is the m-th node of level l and covers tokens [m*2^l, (m+1)*2^l); level 0 are
 * the tokens, level L is the root.  Node ids are level-major:
 *     id(l, m) = 2n - (2n >> l) + m        (tokens 0..n-1, root 2n-2).
 * An edge v -> u means "u attends to v".
 *
 * Ownership: the caller owns every buffer.  Unless a comment says "host", every
 * pointer is a DEVICE pointer valid on the current device.  Calls enqueue work on
 * `cuda_stream` (a cudaStream_t passed as void*, NULL = legacy default stream) and
 * return without synchronising.  Nothing is allocated or kept between calls, so the attention calls
 * (bpt_attn_fwd / bpt_attn_bwd and their _varlen, _ex, _rows forms) can be captured in a CUDA graph.
 * The library reads no environment variable and keeps no process-wide setting (the exceptions, the
 * benchmark trace and the failure record, are described at bpt_trace_begin and bpt_check_device).
 * Argument errors are detected on the host before anything is launched.
 *
 * Device-side failure report.  A non-empty attention workspace begins with a 256-byte status block
 * that every attention call clears on its stream before its kernels run.  Kernels that wait on
 * hardware barriers (the tensor-memory kernels) bound every wait to about a second; if one expires
 * the kernel winds down, the results of the call are invalid and BPT_ERR_TIMEOUT is stored in the
 * block.  bpt_check reads it.  The gated feed-forward calls take a separate, optional block, and store
 * BPT_ERR_TIMEOUT in a record of the device besides, which no call clears: bpt_check_device reads it.  A token id
 * outside its table (bpt_embed_fwd, bpt_embed_bwd) is stored there too, as BPT_ERR_INDEX.
 */
#ifndef BPT_H
#define BPT_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    BPT_OK = 0,
    BPT_ERR_INVALID_ARG = 1,  /* null pointer, non-positive size, unknown flag, ...          */
    BPT_ERR_UNSUPPORTED = 2,  /* head size / dtype / range the kernels do not cover; n not  */
                              /* a power of two                                             */
    BPT_ERR_WORKSPACE = 3,    /* workspace missing or smaller than the size query says      */
    BPT_ERR_CUDA = 4,         /* a CUDA runtime call or launch failed                       */
    BPT_ERR_TIMEOUT = 5,      /* a bounded device-side wait expired (see bpt_attn_fwd)      */
    BPT_ERR_OVERFLOW = 6,     /* edge count does not fit the 32-bit index arrays            */
    BPT_ERR_SCRATCH_LIMIT = 7,/* problem needs more scratch than the built-in static array  */
    BPT_ERR_INDEX = 8         /* a token id outside the table (see bpt_embed_fwd)           */
} bpt_status;

/* flags of a graph */
enum {
    BPT_BIDIR = 0,      /* contextual edges from both sides (Sec. 3.2.2)                          */
    BPT_LEFT_ONLY = 1,  /* only the left context, for autoregressive use (Sec. 4.2); self and      */
                        /* affiliated edges are kept                                               */
    BPT_MODE_PAD = 0,   /* default: k nodes per level plus the alignment node of Sec. 3.2.2 -- one  */
                        /* more when the level's last node is a left child, so that the next level  */
                        /* starts on a whole parent                                                 */
    BPT_MODE_ALG1 = 2   /* Algorithm 1 taken literally: exactly k nodes per level, no extra node   */
};

typedef enum { BPT_F32 = 0, BPT_BF16 = 1 } bpt_dtype;

typedef struct {
    int32_t n, k;
    uint32_t flags;
    int32_t n_levels;             /* L = log2 n                                     */
    int32_t n_nodes;              /* 2n - 1 (Sec. 3.2.1)                            */
    int32_t n_rel;                /* rows of the relation table, see bpt_build_graph */
    int64_t n_edges;              /* E                                              */
    size_t build_workspace_bytes; /* workspace bpt_build_graph needs                */
} bpt_graph_dims;

typedef struct {
    const int32_t* row_ptr; /* [n_nodes + 1] CSR by destination                              */
    const int32_t* col;     /* [E] source node of each edge, ascending inside a row          */
    const int32_t* rel;     /* [E] relation id of each edge                                  */
    const int32_t* t_ptr;   /* [n_nodes + 1] by-source lists (needed by the backward), or NULL */
    const int32_t* t_dst;   /* [E] destination node, ascending inside a source's list        */
    const int32_t* t_eid;   /* [E] position of that edge in col/rel                          */
    bpt_graph_dims dims;
} bpt_graph;

/*
 * Sizes of the graph for (n, k, flags) -- host only, no device work.
 * Sec. 3.2: 2n-1 nodes; per token a self loop (Algorithm 1, N <- {u}), k (or k+1
 * with the pad rule) contextual nodes per level and side, fine to coarse; per span
 * one affiliated edge from every token it contains.
 * Requires n a power of two (Sec. 3.2.1 builds a perfect binary tree; shorter sequences are served
 * by the length arguments of the attention calls), 2 <= n <= 2^20, 1 <= k <= 2^20.  `out` is a host pointer.
 * Errors: INVALID_ARG, UNSUPPORTED (range, n not a power of two), OVERFLOW (E >= 2^31).
 */
bpt_status bpt_graph_dims_query(int32_t n, int32_t k, uint32_t flags, bpt_graph_dims* out);

/*
 * Build the graph on the device (Sec. 3.2.2 edge construction, Sec. 3.4 labels).
 *
 * Outputs (device, caller-allocated): row_ptr[n_nodes+1], col[E], rel[E] and, unless
 * all three are NULL, the by-source lists t_ptr[n_nodes+1], t_dst[E], t_eid[E].
 * Rows are destinations in node-id order, sources ascending by node id.
 * Relation ids, with W = k+1:  self = 0;  o-th node (nearest first) joining on the
 * left at level j: 1 + j*W + o;  on the right: 1 + L*W + j*W + o;  token -> its
 * ancestor at level j (1..L): 1 + 2*L*W + (j-1);  n_rel = 1 + 2*L*W + L.
 * `dims` (host) must come from bpt_graph_dims_query.  `workspace` (device) must hold
 * dims->build_workspace_bytes.  `out` (host) receives the pointers and dims.
 * Errors: INVALID_ARG, WORKSPACE, CUDA.
 */
bpt_status bpt_build_graph(const bpt_graph_dims* dims, int32_t* row_ptr, int32_t* col, int32_t* rel,
                           int32_t* t_ptr, int32_t* t_dst, int32_t* t_eid,
                           void* workspace, void* cuda_stream, bpt_graph* out);

/*
 * Bytes of device workspace bpt_attn_fwd (backward == 0) or bpt_attn_bwd
 * (backward != 0) should be given for this problem; 0 on invalid arguments.  Host only.
 * The same sizes serve the _varlen and _ex forms.
 *
 * The backward accepts any workspace of at least bpt_attn_bwd_min_workspace_bytes: where its
 * kernels keep per-(batch entry, head) scratch they work through the pairs in passes, as many pairs
 * per pass as the given bytes hold (the size returned here plans at most 10 GiB per pass).  dq, dk
 * and dv do not depend on the number of passes; d_rel is summed pass by pass, in a fixed order
 * for a given workspace size.
 */
size_t bpt_attn_workspace_bytes(const bpt_graph* g, int32_t B, int32_t H, int32_t d, bpt_dtype dtype, int backward);
size_t bpt_attn_bwd_min_workspace_bytes(const bpt_graph* g, int32_t B, int32_t H, int32_t d, bpt_dtype dtype);

/*
 * Waits for `cuda_stream` and reports what the last attention call that used `workspace` (device
 * pointer, the one passed to that call; NULL is allowed and reports BPT_OK) left in the status
 * block: BPT_OK, or BPT_ERR_TIMEOUT when a bounded device-side wait expired and the call's results
 * are invalid.  BPT_ERR_CUDA when the synchronisation or the copy fails.  Host-synchronous: not for
 * use inside a stream capture.
 */
bpt_status bpt_check(const void* workspace, void* cuda_stream);

/*
 * Waits for `cuda_stream` and reports whether a bounded device-side wait of any gated feed-forward call
 * (bpt_gated_ff_fwd, bpt_gated_ff_bwd, with or without a status block) or of the wait self-test expired on
 * the current device since the last such report: BPT_OK, or BPT_ERR_TIMEOUT; or BPT_ERR_INDEX, where a token id was outside
 * its table.  What is reported is cleared; of both, the timeout is reported first and the id by the next call.  For
 * training loops: once per step, where the step's calls ran inside an autograd engine that keeps no status
 * blocks.  Covers the work that `cuda_stream` has waited for; work that still runs on other streams
 * is reported by a later call.  BPT_ERR_CUDA when the synchronisation, a copy or a launch fails.  Host-synchronous: not
 * for use inside a stream capture.
 */
bpt_status bpt_check_device(void* cuda_stream);

/*
 * Forward graph self-attention with relative positions (Sec. 3.4 equation, built on
 * the GSA equations of Sec. 3.1).  For every batch entry b, node u, head h:
 *     s_e = scale * q[b,u,h,:] . (k[b,v,h,:] + rel_emb[rel_e,:])   over edges e = (v -> u)
 *     P   = softmax_e(s),   out[b,u,h,:] = sum_e P_e v[b,v,h,:],   lse[b,u,h] = log sum_e exp(s_e)
 * q, k, v, out: [B, n_nodes, H, d] contiguous, element type `dtype`; rel_emb: [n_rel, d],
 * same type, shared by all heads; lse: [B, n_nodes, H] fp32.  Accumulation is fp32.
 * `scale` is explicit (the paper divides by sqrt(d); callers pass 1/sqrt(d)).
 * d must be 32 or 64.  `g` is a host pointer to a struct of device pointers.
 * `workspace` may be NULL when the size query returns 0.
 * Errors: INVALID_ARG, UNSUPPORTED, WORKSPACE, CUDA; device-side: see bpt_check.
 */
bpt_status bpt_attn_fwd(const bpt_graph* g, int32_t B, int32_t H, int32_t d, bpt_dtype dtype,
                        const void* q, const void* k, const void* v, const void* rel_emb, float scale,
                        void* out, float* lse, void* workspace, size_t workspace_bytes, void* cuda_stream);

/*
 * Backward of the same equation: given d_out = dLoss/d out, with P_e = exp(s_e - lse_u),
 *     dP_e = d_out_u . v_v,   dS_e = P_e (dP_e - d_out_u . out_u),
 *     dq_u = scale * sum_{e into u} dS_e (k_v + rel_emb[rel_e]),
 *     dk_v = scale * sum_{e out of v} dS_e q_u,      dv_v = sum_{e out of v} P_e d_out_u,
 *     d_rel[r] = scale * sum_{b,h} sum_{e: rel_e = r} dS_e q_u     (the table is shared, Sec. 3.4).
 * out and lse are the forward's results.  dq, dk, dv: [B, n_nodes, H, d] in `dtype`;
 * d_rel: [n_rel, d] fp32.  All four are overwritten, not accumulated into.  The sums are
 * taken in a fixed order without atomics, so results are bit-reproducible.
 * The d_rel rows of the ancestor relations are written as exact zeros: all edges into a
 * span share one relation, so that embedding shifts every score of the row alike and
 * the softmax (hence the loss) does not depend on it.
 * d_out_u . out_u is evaluated with the stored `out`, so for bf16 the gradients carry the
 * rounding of `out` (relative 2^-9 per element) on top of the fp32 arithmetic.
 * The graph must carry the by-source lists.  Errors as for the forward.
 */
bpt_status bpt_attn_bwd(const bpt_graph* g, int32_t B, int32_t H, int32_t d, bpt_dtype dtype,
                        const void* q, const void* k, const void* v, const void* rel_emb, float scale,
                        const void* out, const float* lse, const void* d_out,
                        void* dq, void* dk, void* dv, float* d_rel,
                        void* workspace, size_t workspace_bytes, void* cuda_stream);

/*
 * The same two operations for sequences shorter than n (Sec. 3.2.1 defines the tree over a
 * power-of-two number of tokens and is silent about other lengths; this is the library's reading).
 * lengths: device array [B], 1 <= lengths[b] <= n (values outside are clamped).  Batch entry b has
 * its real tokens in the first lengths[b] leaves; a node is real when it covers at least one real
 * token.  Every edge whose source or destination is not real is dropped; node ids, relation ids and
 * offsets stay those of the full graph, so the same bpt_graph and relation table serve all lengths.
 * Rows of nodes that are not real: out = 0, lse = 0, dq = dk = dv = 0.
 * The q, k, v, d_out rows of nodes that are not real never influence a result, but they must hold
 * finite values (they may be multiplied by an exact zero weight): initialise the padding.
 * Everything else is as for bpt_attn_fwd / bpt_attn_bwd; the forward of the backward's `out`, `lse`
 * must have been computed with the same lengths.
 */
bpt_status bpt_attn_fwd_varlen(const bpt_graph* g, int32_t B, int32_t H, int32_t d, bpt_dtype dtype,
                               const void* q, const void* k, const void* v, const void* rel_emb, float scale,
                               const int32_t* lengths, void* out, float* lse,
                               void* workspace, size_t workspace_bytes, void* cuda_stream);
bpt_status bpt_attn_bwd_varlen(const bpt_graph* g, int32_t B, int32_t H, int32_t d, bpt_dtype dtype,
                               const void* q, const void* k, const void* v, const void* rel_emb, float scale,
                               const int32_t* lengths, const void* out, const float* lse, const void* d_out,
                               void* dq, void* dk, void* dv, float* d_rel,
                               void* workspace, size_t workspace_bytes, void* cuda_stream);

/*
 * The general form of the two operations: optional sequence lengths (as for the _varlen entry points,
 * NULL = all n) and attention dropout (App. A.1 of the paper lists an attention dropout rate for
 * every experiment; the way the masks are drawn is the library's).  With 0 < dropout_p < 1 every edge
 * weight of every (batch entry, head) is kept with probability 1 - dropout_p and divided by
 * 1 - dropout_p, after the softmax and before the product with v; lse is that of the softmax.
 * The mask is a pure function of (dropout_seed, batch entry, head, destination node, source node):
 * Philox4x32 with 10 rounds, key = (low, high) word of the seed, counter = (destination, source,
 * batch entry * H + head, 0x42505431), edge kept iff the first output word >= floor(dropout_p * 2^32).
 * The backward rebuilds it from the same options (nothing is stored); pass the options the forward had.
 * `path` picks the kernels of the token rows where the tiled tensor-core path applies (bf16, head
 * size 64, n >= 64, k <= 64): BPT_PATH_AUTO lets the library choose by k; BPT_PATH_MMA forces the
 * warp-level (mma.sync) kernels, BPT_PATH_TC5 the tensor-memory (tcgen05) kernels wherever they cover
 * the shape -- for comparison runs and tests.  Other values: INVALID_ARG.
 * `opt` is a host pointer; NULL means no lengths, no dropout, automatic path.  dropout_p outside
 * [0, 1): INVALID_ARG.
 */
enum { BPT_PATH_AUTO = 0, BPT_PATH_MMA = 1, BPT_PATH_TC5 = 2 };
typedef struct {
    const int32_t* lengths; /* device [B] or NULL */
    float dropout_p;
    uint64_t dropout_seed;
    uint32_t path;          /* BPT_PATH_* */
} bpt_attn_options;

bpt_status bpt_attn_fwd_ex(const bpt_graph* g, int32_t B, int32_t H, int32_t d, bpt_dtype dtype,
                           const void* q, const void* k, const void* v, const void* rel_emb, float scale,
                           const bpt_attn_options* opt, void* out, float* lse,
                           void* workspace, size_t workspace_bytes, void* cuda_stream);
bpt_status bpt_attn_bwd_ex(const bpt_graph* g, int32_t B, int32_t H, int32_t d, bpt_dtype dtype,
                           const void* q, const void* k, const void* v, const void* rel_emb, float scale,
                           const bpt_attn_options* opt, const void* out, const float* lse, const void* d_out,
                           void* dq, void* dk, void* dv, float* d_rel,
                           void* workspace, size_t workspace_bytes, void* cuda_stream);

/*
 * Forward for a few destination rows only -- the building block of step-by-step decoding with the
 * left-only graph (Sec. 4.2 uses BPT autoregressively): when token i arrives, the rows that change in
 * a layer are token i and its L ancestors, and with lengths[b] = i + 1 the ancestors attend exactly
 * the tokens seen so far.  rows: device array [B][n_rows] of node ids (one list per batch entry;
 * ids outside [0, n_nodes) are skipped); only those rows of out and lse are written.  Same equation,
 * options and layouts as bpt_attn_fwd_ex; runs on the general row kernel, needs no workspace.
 * Errors: INVALID_ARG, UNSUPPORTED, CUDA.
 */
bpt_status bpt_attn_fwd_rows(const bpt_graph* g, int32_t B, int32_t H, int32_t d, bpt_dtype dtype,
                             const void* q, const void* k, const void* v, const void* rel_emb, float scale,
                             const bpt_attn_options* opt, const int32_t* rows, int32_t n_rows,
                             void* out, float* lse, void* cuda_stream);

/*
 * Output projection, residual and layer normalisation of a layer in one kernel (Algorithm 2 of Sec. 3.3:
 * Z = norm(H + GSA(H) W^O), with the output projection W^O of Sec. 3.1):
 *     z[r, :] = LayerNorm(h[r, :] + a[r, :] w_o^T) * gamma + beta        for every row r,
 * where a is the attention output with the heads concatenated ([B, n_nodes, H, d] seen as [rows, D], D = H * d),
 * w_o is [D, D] with row o holding the weights of output channel o (the layout of a linear layer's weight),
 * h the layer's input states [rows, D], gamma / beta the normalisation's scale and shift [D] (fp32), z the
 * result [rows, D].  a, w_o, h, z are bf16, contiguous and 16-byte aligned; the product accumulates in fp32 and
 * mean / variance (biased, about the mean) are taken in fp32 over the D channels; one rounding to bf16.
 * D must be 128, 256 or 512; rows >= 1.  `workspace` is NULL or a device buffer of at least 256 bytes that
 * receives the status block (see bpt_check).  Forward only: training goes through the separate operators.
 * Errors: INVALID_ARG, UNSUPPORTED, CUDA.
 */
bpt_status bpt_out_proj_norm(const void* a, const void* w_o, const void* h, const float* gamma, const float* beta,
                             void* z, int64_t rows, int32_t D, float eps, void* workspace, void* cuda_stream);

/*
 * Gated feed-forward block (the position-wise half of Algorithm 2, Sec. 3.3, with a gated inner layer):
 *     y = (act(x w_gate^T) * (x w_up^T)) w_down^T          for every row of x
 * x, y: [rows, D]; w_gate, w_up: [F, D]; w_down: [D, F] (the layout of a linear layer's weight); all bf16, contiguous and
 * 16-byte aligned.  act: BPT_ACT_RELU, BPT_ACT_SILU (g / (1 + exp(-g))) or BPT_ACT_GELU (g/2 (1 + erf(g / sqrt 2))), the
 * last to 0.75e-7 |g| beside fp32 rounding; relative to its own vanishing tail 0.4 % at g = -6, 1 % at -8.
 * Both projections, the activation and the product run in one kernel, which rounds the inner row act(..) * (..) once
 * to bf16 (the second product's operand type); products accumulate in fp32; y is rounded once.  Calls for which
 * bpt_gated_ff_few_rows (host) says 1 -- few rows for the size of the weights, as in decoding -- keep the inner row to about
 * 16 bits instead, and their kernels wait for nothing.
 * rows >= 0, D and F multiples of 8 (16-byte rows).  x and y must not overlap.  An infinite weight makes the results that it
 * enters infinite or, where a value is kept as two terms, NaN.
 *
 * Backward: from x, the weights and dy = dLoss/dy (nothing else of the forward is needed: both projections are computed
 * again, in fp32), dx [rows, D] and dw_gate, dw_up [F, D], dw_down [D, F], all bf16, overwritten.  dx may be NULL; the
 * three weight gradients are given together or are all NULL.  The inner row and the gradients of the two projections are rounded once to bf16
 * (operands of the products that follow); calls of at most 64 rows keep them to about 16 bits.  Sums over rows are taken in a fixed order without atomics: bit-reproducible.
 *
 * `workspace`: bpt_gated_ff_workspace_bytes bytes (host query; 0 on invalid arguments and for rows == 0, where NULL
 * will do), 256-byte aligned; two calls whose GPU work overlaps need one each.  `status`: NULL, or a device buffer of at
 * least 256 bytes that receives the status block (see bpt_check; apart from the workspace, which is large and need not
 * outlive the call's work); either way a wait that expired also shows in bpt_check_device.
 * Errors: INVALID_ARG, UNSUPPORTED (sizes), WORKSPACE, CUDA; device-side: see bpt_check, bpt_check_device.
 */
enum { BPT_ACT_RELU = 0, BPT_ACT_SILU = 1, BPT_ACT_GELU = 2 };
int32_t bpt_gated_ff_few_rows(int64_t rows, int32_t D, int32_t F);
size_t bpt_gated_ff_workspace_bytes(int64_t rows, int32_t D, int32_t F, int backward);
bpt_status bpt_gated_ff_fwd(const void* x, const void* w_gate, const void* w_up, const void* w_down, void* y,
                            int64_t rows, int32_t D, int32_t F, int32_t act, void* status, void* workspace,
                            size_t workspace_bytes, void* cuda_stream);
bpt_status bpt_gated_ff_bwd(const void* x, const void* w_gate, const void* w_up, const void* w_down, const void* dy,
                            void* dx, void* dw_gate, void* dw_up, void* dw_down, int64_t rows, int32_t D, int32_t F, int32_t act,
                            void* status, void* workspace, size_t workspace_bytes, void* cuda_stream);

/*
 * The seam between two blocks of a layer: norm after a block, gate, scaled residual, norm before the next block.
 * Algorithm 2 (Sec. 3.3) has Z = norm(H + GSA(H)) and H' = norm(Z + FFN(Z)); with everything but `norm` off this is
 * that step.  For every row of D channels, in one pass over the data:
 *     n = post(b),    r = alpha h + gate n,    y = norm(r)
 * norm and post: BPT_NORM_NONE (the identity), BPT_NORM_LAYER ((x - mean) / sqrt(var + eps), biased variance about the
 * mean) or BPT_NORM_RMS (x / sqrt(mean(x^2) + eps)), each times its weight plus its bias where those are not NULL.
 * h, b, y, r: [rows, D] contiguous, element type `dtype`; b may be NULL (r = alpha h; no post norm, no gate).
 * weight, bias, post_weight, post_bias: [D] of type param_dtype, or NULL; only with the norm they belong to.
 * gate: [gate_groups, D] of type gate_dtype, or NULL (1): row i takes gate row i / (rows / gate_groups), so that one
 * row gates everything, one per sequence, or one per row; gate_groups must divide rows.
 * Arithmetic and statistics are fp32; y is computed from the unrounded r; one rounding per stored value.
 * rows >= 0, 1 <= D <= 8192.  Rows whose D * sizeof(element) is not a multiple of 16 bytes, and tensors that are not
 * 16-byte aligned, are served element by element.  y must be given exactly when norm is not NONE; r may be NULL
 * then.  y or r may be the same buffer as h or b.  `stats`: NULL, or [rows][4] fp32 (16-byte aligned) that receives mean
 * and reciprocal deviation of the post norm and of the norm (0 and 1 for an absent norm), for the backward.
 *
 * Backward: given dy = dLoss/dy (NULL: zero) and dr = dLoss/dr (NULL: zero), writes those of dh, db [rows, D] (dtype),
 * d_weight, d_bias, d_post_weight, d_post_bias [D] (param_dtype), d_gate [gate_groups, D] (gate_dtype) that are not
 * NULL:  dR = dr + norm'(dy),  dh = alpha dR,  dn = gate dR,  db = post'(dn),  and the column sums that belong to the
 * parameters.  Everything is recomputed from h, b and the forward's `stats` (which may be NULL when neither norm is
 * there).  Outputs are overwritten; the sums are taken in a fixed order
 * without atomics, so results are bit-reproducible.  Results must not overlap inputs.
 * `workspace`: bpt_res_norm_bwd_workspace_bytes bytes (host query; 0 on invalid arguments), plain scratch without a
 * status block (nothing here waits), 16-byte aligned; two calls whose GPU work overlaps need one each.
 * Errors: INVALID_ARG, UNSUPPORTED (D, rows >= 2^31), WORKSPACE, CUDA.
 */
enum { BPT_NORM_NONE = 0, BPT_NORM_LAYER = 1, BPT_NORM_RMS = 2 };
typedef struct {
    int64_t rows;
    int64_t gate_groups;
    int32_t D;
    bpt_dtype dtype, param_dtype, gate_dtype;
    int32_t norm, post_norm;    /* BPT_NORM_* */
    float alpha, eps;
    const void *h, *b;
    const void *weight, *bias, *post_weight, *post_bias, *gate;
} bpt_res_norm_args;
bpt_status bpt_res_norm_fwd(const bpt_res_norm_args* args, void* y, void* r, float* stats, void* cuda_stream);
size_t bpt_res_norm_bwd_workspace_bytes(const bpt_res_norm_args* args);
bpt_status bpt_res_norm_bwd(const bpt_res_norm_args* args, const float* stats, const void* dy, const void* dr, void* dh, void* db,
                            void* d_weight, void* d_bias, void* d_post_weight, void* d_post_bias, void* d_gate,
                            void* workspace, size_t workspace_bytes, void* cuda_stream);

/*
 * Token ids to node states (Sec. 3.3: token nodes start from their embeddings, span nodes from zero), and the gradient of the table.
 *     out[b, t, :] = scale * weight[ids[b, t], :]   for t < lengths[b];      zeros for the other rows t < out_rows
 * ids: [batch, tokens] of id_bytes 4 or 8, contiguous; lengths: [batch] (clamped to 0 .. tokens) or NULL (all tokens); ids
 * behind a sequence's length are not looked at.  weight: [vocab, D] of weight_dtype, contiguous; out: [batch, out_rows, D] of out_dtype, contiguous,
 * out_rows >= tokens (2n - 1 for the nodes of a tree over n tokens).  The product is taken in fp32 and rounded once.
 * An id outside 0 .. vocab - 1 reads nothing: its row is zeros, it adds nothing to the gradient, and BPT_ERR_INDEX shows in
 * bpt_check_device.
 *
 * Backward: d_weight[v, :] = scale * sum of d_out[b, t, :] over the places with ids[b, t] = v, in weight_dtype; zeros for ids that stand
 * nowhere and for padding_idx (-1: none; the forward pays no attention to it).  Every row is overwritten.  d_out: [batch, out_rows, D] of out_dtype;
 * rows behind the tokens add nothing, whatever stands there.  `weight` is not looked at.  Sums are taken in fp32 in a fixed order without
 * atomics: bit-reproducible.
 * Tensors may start at any element; widths that are multiples of 8 on 16-byte boundaries take the shortest kernels.
 * `workspace`: bpt_embed_bwd_workspace_bytes bytes (host query; 0 on invalid arguments), plain scratch without a status
 * block, 16-byte aligned; two calls whose GPU work overlaps need one each.
 * batch, tokens >= 0; vocab, batch * out_rows < 2^30; D <= 2^20.  Errors: INVALID_ARG, UNSUPPORTED (sizes), WORKSPACE, CUDA; device-side: INDEX.
 */
typedef struct {
    int64_t batch, tokens, out_rows, vocab, padding_idx;
    int32_t D, id_bytes;
    bpt_dtype weight_dtype, out_dtype;
    float scale;
    const void* ids;
    const int32_t* lengths;
    const void* weight;
} bpt_embed_args;
bpt_status bpt_embed_fwd(const bpt_embed_args* args, void* out, void* cuda_stream);
size_t bpt_embed_bwd_workspace_bytes(const bpt_embed_args* args);
bpt_status bpt_embed_bwd(const bpt_embed_args* args, const void* d_out, void* d_weight, void* workspace, size_t workspace_bytes,
                         void* cuda_stream);

/*
 * The norm over all gradients of a model, and clipping.
 *     norm = sqrt(sum of squares over all elements of all tensors)   (BPT_GRAD_NORM_L2),   or the largest |element|   (BPT_GRAD_NORM_MAX)
 *     c = min(1, max_norm / (norm + eps)),      out <- c * grad   for every tensor
 * `grads` is a HOST array of n entries, read before the call returns; entry i has numel elements of `dtype` at `grad`, contiguous.  out NULL: the
 * tensor is scaled in place, and not written at all where c = 1; otherwise c * grad goes to `out` (out_dtype), which may be
 * the gradient itself in its own type, also where c = 1.  Nothing that is written may overlap anything else of the call -- the same
 * tensor given twice, for one; refused.  bpt_grad_norm writes no tensor (out is not looked at) and counts a tensor given twice twice.
 * norm: device, fp32 [1].  A NaN among the gradients, or an infinity with BPT_GRAD_NORM_L2, makes norm NaN or infinite as it would by
 * the formula, and c NaN or 0; nothing is hidden.  Squares are summed in fp64 where fp32 would lose them, so
 * the norm is right for gradients of any size; c and the products are fp32, one rounding.  A norm that fp32 has no number for comes out
 * infinite in `norm`; c is that of the sum itself.  Fixed order, no atomics: bit-reproducible.
 * n = 0, or nothing in any tensor: norm 0.  max_norm >= 0 (infinite: nothing is scaled, whatever the norm), eps >= 0.
 * `workspace`: bpt_grad_norm_workspace_bytes bytes (host query; 0 on invalid arguments), plain scratch without a status block, 16-byte
 * aligned; two calls whose GPU work overlaps need one each.  Two launches for up to 960 tensors.
 * Errors: INVALID_ARG, UNSUPPORTED (numel > 2^40, 2^42 elements in all), WORKSPACE, CUDA.
 */
enum { BPT_GRAD_NORM_L2 = 0, BPT_GRAD_NORM_MAX = 1 };
typedef struct {
    void* grad;
    void* out;
    int64_t numel;
    bpt_dtype dtype, out_dtype;
} bpt_grad;
size_t bpt_grad_norm_workspace_bytes(const bpt_grad* grads, int32_t n);
bpt_status bpt_grad_norm(const bpt_grad* grads, int32_t n, int32_t norm_type, float* norm, void* workspace, size_t workspace_bytes,
                         void* cuda_stream);
bpt_status bpt_clip_grads(const bpt_grad* grads, int32_t n, int32_t norm_type, float max_norm, float eps, float* norm, void* workspace,
                          size_t workspace_bytes, void* cuda_stream);

/*
 * What a decoding step (Sec. 4.2 uses BPT as a language model) does to its logits before a token is taken.  For row b and id v, with
 *     seen(v): v stands in history[b, 0 .. lengths[b]);    n(v): how often it stands in history[b, prompt_lengths[b] .. lengths[b])
 *     x = logits[b, v];   if seen(v): x = x > 0 ? x / repetition : x * repetition;   if n(v) > 0: x -= frequency n(v) + presence
 *     x += bias[b, v];    x += bias_values[b, j] for the last j with bias_ids[b, j] = v;     out[b, v] = allowed(b, v) ? x : -infinity
 * in fp32, rounded once.  What a mask forbids is -infinity whatever stands there (NaN too); a row without an allowed id is all -infinity.
 * logits: [rows, vocab] of `dtype`, rows logits_stride elements apart; out: of out_dtype, rows out_stride apart; out may be the logits
 * themselves (same address, type and stride) and must otherwise not overlap them, nor any other argument.
 * history: [rows, history_len] of history_bytes 4 or 8, rows history_stride apart; history_len 0: none.  lengths, prompt_lengths: [rows]
 * (clamped to 0 .. history_len and 0 .. lengths[b]) or NULL (history_len; 0).  Ids outside 0 .. vocab - 1 count for nothing.
 * repetition (> 0), presence, frequency: numbers, or where the _rows pointer is not NULL one fp32 value per row.
 * bias: of bias_dtype, rows bias_stride apart (0: one row for all), or NULL.  bias_ids, bias_values: [rows, bias_count] contiguous (ids of
 * bias_id_bytes 4 or 8; outside 0 .. vocab - 1: no effect); bias_count 0: none.
 * allowed: bit v % 32 of word v / 32 set where v is allowed, rows allowed_stride words apart (0: one row for all), or NULL.
 * `workspace`: bpt_adjust_logits_workspace_bytes bytes (host query; 0 where none is needed, and on invalid arguments), plain scratch
 * without a status block, 16-byte aligned; two calls whose GPU work overlaps need one each.
 * rows, vocab, history_len, bias_count < 2^30 (vocab >= 1).  Errors: INVALID_ARG, UNSUPPORTED (sizes), WORKSPACE, CUDA.
 */
typedef struct {
    int64_t rows, vocab, logits_stride, out_stride;
    bpt_dtype dtype, out_dtype;
    const void* logits;
    int64_t history_len, history_stride;
    const void* history;
    const int32_t *lengths, *prompt_lengths;
    const float *repetition_rows, *presence_rows, *frequency_rows;
    float repetition, presence, frequency;
    int32_t history_bytes, bias_id_bytes;
    bpt_dtype bias_dtype;
    const void* bias;
    int64_t bias_stride, bias_count;
    const void* bias_ids;
    const float* bias_values;
    const int32_t* allowed;
    int64_t allowed_stride;
} bpt_logits_args;
size_t bpt_adjust_logits_workspace_bytes(const bpt_logits_args* args);
bpt_status bpt_adjust_logits(const bpt_logits_args* args, void* out, void* workspace, size_t workspace_bytes, void* cuda_stream);

/*
 * Backward pass for callers that must not allocate device memory (the paper has no
 * counterpart; this is a deployment convenience).
 *
 * Who needs it: code that runs where cudaMalloc is off limits -- a plugin inside a host
 * application that hands out tensors but no raw allocator, a real-time or safety-reviewed
 * loop whose rules forbid allocation after start-up, a process whose memory pool already
 * owns the whole device.  Such callers can provide the inputs and outputs of the
 * backward, but have nowhere to get its workspace from.
 *
 * Same arguments, results and errors as bpt_attn_bwd, minus the workspace: the scratch
 * is a 32 MiB array that lives inside the library's device image (every GPU that loads
 * the library carries it until the process exits).  bpt_static_scratch_bytes() returns
 * that limit.  The backward fits its passes to the array (fewer (batch entry, head) pairs
 * per pass than with a large workspace, same results for dq, dk, dv); only a problem whose
 * bpt_attn_bwd_min_workspace_bytes exceeds the limit -- one pair alone does not fit -- is
 * refused with BPT_ERR_SCRATCH_LIMIT before anything is launched (use bpt_attn_bwd with
 * your own workspace then).  The call itself performs no cudaMalloc / cudaFree and calls
 * no allocating library routine.
 *
 * The first call on each device looks up the array's device address (with that device
 * current); make that first call outside of any stream capture.  The CUDA runtime loads the
 * part of the library that holds the array at that first look-up, and that is when the
 * driver sets the 32 MiB aside: a process that hands the rest of the device to a pool of its
 * own should make one call (any small problem) during start-up, before the pool takes the
 * memory.  All calls on a device
 * share the one array, and it keeps whatever the previous call left in it: the backward
 * overwrites every part before reading it, so nothing needs clearing, but two calls whose
 * GPU work overlaps (different streams, or different threads) would race on it -- keep
 * them ordered on one stream.
 */
size_t bpt_static_scratch_bytes(void);
bpt_status bpt_attn_bwd_static_scratch(const bpt_graph* g, int32_t B, int32_t H, int32_t d, bpt_dtype dtype,
                                       const void* q, const void* k, const void* v, const void* rel_emb, float scale,
                                       const void* out, const float* lse, const void* d_out,
                                       void* dq, void* dk, void* dv, float* d_rel, void* cuda_stream);

/*
 * Per-launch timing for benchmarks (no counterpart in the paper).  Between
 * bpt_trace_begin and bpt_trace_end every kernel the library launches is followed by
 * a CUDA event on its stream; bpt_trace_end waits for the last one and returns, for
 * the first min(*n_marks, capacity) launches, the milliseconds since the previous
 * mark (ms, host array, may be NULL) and a static name (names, host array, may be
 * NULL).  `capacity` of bpt_trace_begin bounds the number of launches recorded
 * (< 4096); later launches go unrecorded.  This is the one piece of process-global
 * state in the library: not thread-safe, off by default, one trace at a time.
 * Errors: INVALID_ARG (nesting, capacity), CUDA.
 */
bpt_status bpt_trace_begin(int32_t capacity, void* cuda_stream);
bpt_status bpt_trace_end(int32_t* n_marks, float* ms, const char** names, int32_t capacity);

/*
 * Test hook for the failure report (no counterpart in the paper): launches one tiny kernel in which
 * one thread waits, for at most `limit_cycles` clock cycles (1 .. 2^31), on a hardware barrier that
 * expects one arrival.  With arrive == 0 nobody arrives: the wait runs out, the kernel stores
 * BPT_ERR_TIMEOUT in the status block at `workspace` (device, >= 256 bytes, cleared first) and ends --
 * exactly the give-up path of the tensor-memory kernels; with arrive != 0 the thread arrives itself
 * and the block stays clear.  The device's record is set along with the block.  Nothing faults or hangs
 * either way.  Read the outcome with bpt_check and bpt_check_device.
 * Errors: INVALID_ARG, CUDA.
 */
bpt_status bpt_selftest_wait_timeout(void* workspace, int64_t limit_cycles, int32_t arrive, void* cuda_stream);

/*
 * Index checks (no counterpart in the paper).  The package builds the library twice: libbpt.so, and
 * libbpt_check.so compiled with -DBPT_BOUNDS_CHECK, in which every index a gather or an index-array
 * write uses (an offset into col / rel / t_dst / t_eid against E, a gathered or staged node row against
 * n_nodes, a relation row against n_rel, an edge id against E) is tested before the access.  A
 * violation is counted, the first one recorded, and the access skipped; nothing traps.
 * bpt_debug_bounds waits for `cuda_stream`, copies the record to `record` (host, four words:
 * number of violations, site code of the first one, its index, its limit) and clears it.
 * In libbpt.so the checks are compiled out and the call returns BPT_ERR_UNSUPPORTED.
 * Errors: INVALID_ARG, UNSUPPORTED, CUDA.
 */
bpt_status bpt_debug_bounds(uint32_t* record, void* cuda_stream);

/* Static description of a status code (host). */
const char* bpt_status_str(bpt_status s);

#ifdef __cplusplus
}
#endif
#endif /* BPT_H */
