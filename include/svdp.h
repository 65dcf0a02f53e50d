/*
 * libsvdp — decode step of a ReGLU FFN gated by a low-rank SVD sparsity
 * predictor, for AMD MI355X (gfx950).  C ABI; every pointer named "device" is
 * a device pointer owned by the caller, the library never frees or keeps it.
 *
 * Notation follows the paper: d = hidden size, D = intermediate size,
 * r = predictor rank, x in R^d a decode token, W_gate, W_up in R^{D x d},
 * W_down in R^{d x D} (Sec. 3).  The predictor A B x + b of Sec. 4.1, eq. (2)
 * is passed in row-vector form: P = B^T (d x r), Q = A (D x r), so that the
 * scores are s = (x P) Q^T + b.
 *
 * Common rules for every call that takes a stream:
 *  - asynchronous on `stream` (a hipStream_t passed as void*, NULL = default
 *    stream); the call never synchronises (svdp_whiten_factors, an offline step,
 *    is the one exception and says so), never allocates device memory and
 *    never copies device data to the host, so it can be captured in a HIP graph;
 *  - arguments are validated on the host first; on any error nothing is
 *    enqueued and a status other than SVDP_OK is returned;
 *  - `ws` is a device scratch buffer of at least svdp_workspace_bytes() bytes,
 *    256-byte aligned, owned by the caller; its contents are undefined between
 *    calls; two calls that may overlap in time need distinct workspaces;
 *  - the library keeps no mutable state between calls: everything a call does
 *    follows from its arguments, so calls on different streams and from
 *    different host threads are independent (given distinct workspaces);
 *  - B is the number of tokens decoded together, 1 <= B <= SVDP_MAX_BATCH; all
 *    tokens of a batch share ONE mask (the union of their masks) and one index
 *    list, and every token is computed exactly over that list;
 *  - results are deterministic: floating-point sums are formed in a fixed
 *    order that depends only on the shapes and on the index list (no
 *    floating-point atomics, as in the paper's App. C down projection).
 *
 * Shape limits (else SVDP_ERR_UNSUPPORTED): D % 64 == 0, and with
 * e = 4 (fp32) or 8 (bf16) elements per 16 bytes: d % e == 0, r % e == 0,
 * r <= 2048, d <= 16384; the tokens of a batch must also fit the 160 KB of
 * local memory of a compute unit next to a kernel's scratch (B * d storage
 * elements; svdp_workspace_bytes returns 0 for a shape and batch that do not).
 * Every matrix pointer must be 16-byte aligned.
 */
#ifndef SVDP_H
#define SVDP_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define SVDP_MAX_BATCH 8

typedef enum {
    SVDP_OK = 0,
    SVDP_ERR_INVALID_ARG = 1,  /* null pointer, bad size, misaligned pointer   */
    SVDP_ERR_UNSUPPORTED = 2,  /* shape or dtype outside the limits above       */
    SVDP_ERR_WORKSPACE = 3,    /* ws is NULL, misaligned or too small           */
    SVDP_ERR_HIP = 4           /* the HIP runtime refused a launch              */
} svdp_status;

typedef enum {
    SVDP_F32 = 0,  /* IEEE binary32 */
    SVDP_BF16 = 1, /* bfloat16 bit patterns (upper 16 bits of a binary32) */
    SVDP_E4M3 = 8  /* 8 bits, caches of K and V only: 1 sign, 4 exponent bits (bias 7), 3 bits of mantissa, no
                      infinities, all ones NaN; times a power of two (see svdp_kv_cache)   */
} svdp_dtype;

/* Flags of svdp_layer.flags */
enum {
    /* dReLU variant (paper Sec. 5.1, eq. 6): ReLU is applied to the up branch too. */
    SVDP_FLAG_DRELU = 1u,
    /* Sequential pipeline (paper Sec. 4.2, "Gate/up execution order"): the gate
     * product of a predicted-active neuron re-validates the prediction; when it is
     * <= 0 for every token of the batch, neither its W_up row nor its W_down row
     * is read.  The output is unchanged (such a neuron contributes exactly zero);
     * what changes is the bytes read: d*w per listed neuron for the gate, 2*d*w more
     * only for those that survive.  Pays when the predictor over-predicts (low rank,
     * cautious bias); costs one more dependent fetch per row otherwise.  A dedicated
     * row kernel runs (vector units).                                                */
    SVDP_FLAG_REVALIDATE = 2u,
    /* Which arithmetic units the batch-sensitive kernels use.  The paper's App. C gives a
     * row-at-a-time kernel (Alg. 3) and a gather-then-dense-contraction form (Alg. 4); its
     * Sec. 6 notes that batching lowers the sparsity the first can exploit.
     *  neither flag (default): per kernel and batch capacity, whichever was measured faster on
     *      MI355X: matrix cores for the scores from 3 tokens and for the rows from 5 tokens
     *      (bf16 layers of at least 2 M elements a matrix; over all rows above 1 M elements and 768
     *      rows), vector units below.
     *  SVDP_FLAG_ENGINE_VECTOR: fp32 vector arithmetic everywhere (any dtype, batch, flags).
     *  SVDP_FLAG_ENGINE_MATRIX: matrix cores wherever a kernel for them exists:
     *      - rows (gate, up, down over the list): taken 16 at a time as MFMA tiles straight
     *        from their place in the weight matrices (no gathered copy), bf16 x bf16 -> fp32
     *        for gate and up, fp32 outer products for the down projection; needs bf16 storage
     *        and no SVDP_FLAG_REVALIDATE;
     *      - scores (t Q^T + b): bf16 MFMAs with t split into three bf16 terms (exact to fp32), or
     *        fp32 MFMAs for fp32 storage; below three tokens bf16 storage with r a multiple of 32,
     *        r <= 512.
     *      Layers that do not qualify use the vector kernels.
     * Both engines give the same mask and list (up to scores within rounding of zero) and a y
     * that agrees to fp32 rounding (sums are cut differently).  Setting both is an error.     */
    SVDP_FLAG_ENGINE_VECTOR = 4u,
    SVDP_FLAG_ENGINE_MATRIX = 8u
};

/* One FFN layer with its predictor.  All pointers are device pointers.
 * Storage precision policy (paper App. C, "Precision"): weights, predictor
 * factors and tokens are stored in `wdtype`; all arithmetic, the rank-r
 * intermediate t = x P, the scores and y are fp32.                              */
typedef struct svdp_layer {
    int32_t d, D, r;
    int32_t wdtype;        /* svdp_dtype of P, Q, W_gate, W_up, W_downT and of x          */
    const void *P;         /* [d][r] row-major                                            */
    const void *Q;         /* [D][r] row-major                                            */
    const float *b;        /* [D] fp32 bias (= minus the calibrated threshold, Alg. 2)    */
    const void *W_gate;    /* [D][d] row-major: row i = neuron i                          */
    const void *W_up;      /* [D][d] row-major                                            */
    const void *W_downT;   /* [D][d] row-major: row i = column i of W_down (the paper's
                              column-major W_down, App. C "Memory")                       */
    uint32_t flags;        /* SVDP_FLAG_*                                                 */
} svdp_layer;

/* Bytes of device scratch any call below needs for this layer and up to
 * max_batch tokens.  Host-only, pure.  Returns 0 if the layer is unsupported.   */
size_t svdp_workspace_bytes(const svdp_layer *layer, int32_t max_batch);

/* Predictor scores (Sec. 4.1, eq. 2, before the step function; first line of
 * Alg. 3):  s[t][i] = sum_k (sum_j x[t][j] P[j][k]) Q[i][k] + b[i].
 * x: device [B][d] in layer->wdtype.  s: device [B][D] fp32, fully written.     */
svdp_status svdp_predict(const svdp_layer *layer, const void *x, int32_t B,
                         float *s, void *ws, size_t ws_bytes, void *stream);

/* Mask and index list (step function H of eq. 2; Alg. 4's nonzero):
 * neuron i is active iff s[t][i] > 0 (strictly; NaN is inactive) for at least
 * one token t < B.
 * s: device [B][D] fp32.  mask: device [D/64] 64-bit words, bit j of word k is
 * neuron 64k+j, fully written.  idx: device [D] int32, receives the active neurons
 * in ascending order in idx[0..nnz), the rest is left untouched.  nnz: device
 * [1] int32.  ws, ws_bytes: accepted for uniformity with the other calls; this
 * call needs no scratch, NULL and 0 are fine.                                   */
svdp_status svdp_compact(const float *s, int32_t B, int32_t D, uint64_t *mask,
                         int32_t *idx, int32_t *nnz, void *ws, size_t ws_bytes, void *stream);

/* Sparse ReGLU FFN over an index list (Sec. 3; Alg. 3's three kernels / Alg. 4):
 *   y[t][:] = sum_{n < nnz} ReLU(W_gate[i_n]·x[t]) * (W_up[i_n]·x[t]) * W_downT[i_n][:],
 * i_n = idx[n].  Only the listed rows of the three matrices are read.
 * idx: device int32, entries in [0, D), ascending not required but duplicates
 * are summed twice; an entry outside [0, D) is skipped on the device (it
 * contributes nothing and no row is read out of bounds).  nnz: device [1] int32,
 * clamped on the device to 0 <= *nnz <= D (never read on the host).  y: device [B][d] fp32, fully written (zeros
 * when *nnz == 0).                                                              */
svdp_status svdp_sparse_ffn(const svdp_layer *layer, const void *x, int32_t B,
                            const int32_t *idx, const int32_t *nnz, float *y,
                            void *ws, size_t ws_bytes, void *stream);

/* Dense ReGLU FFN (Sec. 3, eq. 1) over all D neurons: the same-GPU baseline
 * the sparse step is compared with.  y: device [B][d] fp32.                     */
svdp_status svdp_dense_ffn(const svdp_layer *layer, const void *x, int32_t B,
                           float *y, void *ws, size_t ws_bytes, void *stream);

/* The whole decode step of Alg. 3 for one batch: scores, union mask, index
 * list, sparse FFN.  Equivalent to svdp_predict + svdp_compact +
 * svdp_sparse_ffn without materialising the scores.
 * mask_out [D/64], idx_out [D], nnz_out [1]: device, each nullable; when given
 * they receive what svdp_compact would have produced.  y: device [B][d] fp32.   */
svdp_status svdp_ffn_step(const svdp_layer *layer, const void *x, int32_t B, float *y,
                          uint64_t *mask_out, int32_t *idx_out, int32_t *nnz_out,
                          void *ws, size_t ws_bytes, void *stream);

/* svdp_ffn_step for callers that cannot hand over or allocate scratch memory (code under HIP
 * graph capture that owns no buffer, tight serving loops, harnesses that forbid allocation):
 * the same step, with the scratch taken from an array of SVDP_STATIC_SCRATCH_BYTES that the
 * library's image holds on every GPU it runs on until the process ends.  Allocates nothing.
 * Layers and batches whose svdp_workspace_bytes() exceeds the array are refused with
 * SVDP_ERR_WORKSPACE (the 7B- and Mistral-shaped bf16 layers fit with one token).
 * All calls on one GPU share that GPU's array: two calls that may overlap in time on the same
 * GPU (different streams, different threads) race; serialise them or use svdp_ffn_step.
 * Nothing in the array needs to start at zero, and nothing is kept in it between calls.
 * Results are bit for bit those of svdp_ffn_step.                                              */
#define SVDP_STATIC_SCRATCH_BYTES (8u << 20)
svdp_status svdp_ffn_step_static(const svdp_layer *layer, const void *x, int32_t B, float *y,
                                 uint64_t *mask_out, int32_t *idx_out, int32_t *nnz_out, void *stream);

/* The sparse FFN of svdp_ffn_step from given mask words, without the predictor (Alg. 3 after its
 * first line): the row kernel scans the mask words, takes its share of the ascending list and
 * computes gate and up over the active rows; the down projection follows and y [B][d] is fully
 * written, bit for bit what svdp_ffn_step gives for the same mask.  With y == NULL everything but
 * the final sum of the partial results is enqueued (the row kernel; for batches on the matrix
 * cores the gate/up kernel and the down-projection kernel) and the partial results stay in the
 * workspace: that form exists so that the dominant kernels can be timed by themselves.
 * mask: device [D/64] words as written by svdp_compact or svdp_ffn_step.                        */
svdp_status svdp_active_rows(const svdp_layer *layer, const void *x, int32_t B, const uint64_t *mask,
                             float *y, void *ws, size_t ws_bytes, void *stream);

/* Glue between stacked layers used by the stacked benchmark (not from the
 * paper): v = x + y; x_next = v / sqrt(mean(v^2) + eps) + shift, rounded to
 * `dtype`.  x: device [d] in `dtype`; y: device [d] fp32; shift: device [d]
 * fp32; x_next: device [d] in `dtype` (may alias x).  d must be a multiple of 8
 * (bf16) or 4 (fp32), all four pointers 16-byte aligned.                       */
svdp_status svdp_stack_glue(const void *x, const float *y, const float *shift,
                            int32_t d, int32_t dtype, float eps, void *x_next,
                            void *stream);

/* ---- offline build: greedy bias calibration (Alg. 2; App. A "Greedy threshold selection") ----
 *
 * svdp_calib_bias runs Alg. 2 from its sort onward on given statistics of a calibration set:
 *   w [D][T] fp32  damage weights  |ReLU(W_gate[i,:] x_t) (W_up[i,:] x_t)|^2 ||W_down[:, i]||^2
 *   s [D][T] fp32  proxy scores    (A B x_t)_i  = the predictor's scores without bias
 * (row i = neuron i, column t = sample t; both device, read only; no NaN).
 * Per neuron the samples are sorted by score (equal scores keep sample order), the pointer starts at
 * the first positive weight (at T if there is none) with tau = the score there, and the greedy loop
 * advances the neuron whose next `eta` samples cost least (fp32 sum, left to right; smallest index
 * among equal costs; pointer update k <- min(k + eta, T)) until at least `need` of the D*T
 * (neuron, sample) pairs satisfy s <= tau, or no step is left.  For a sparsity level sp of Alg. 2,
 * need = the smallest integer >= sp*D*T.
 * Outputs (device): b [D] fp32 = -tau; k [D] int32 (nullable) the final pointers (counts, 1..T);
 * steps [1] int32 (nullable) the number of greedy steps taken; kendall [D] fp32 (nullable) App. A's
 * check 1 - K_d / (M (M-1)) of the eta-step sums' order, M = T / eta.
 * The result equals the sequential priority-queue loop exactly (integers and bit patterns).
 * Limits: 1 <= T <= 4096, eta >= 1, D >= 1; otherwise SVDP_ERR_UNSUPPORTED / SVDP_ERR_INVALID_ARG.
 * ws: device, 256-byte aligned, >= svdp_calib_workspace_bytes(D, T, eta) (0 for invalid sizes).
 * Asynchronous on `stream`, no allocation, no host read-back.                                     */
size_t svdp_calib_workspace_bytes(int32_t D, int32_t T, int32_t eta);

/* The integer `need` of svdp_calib_bias for a sparsity level sp of Alg. 2 ("while the sparsity is below
 * s"): the smallest integer n with n >= sp * D * T, the product taken in double precision from left to
 * right, clamped to [0, D * T].  Host-only, pure.  Returns -1 for D < 1, T < 1 or sp not a number.     */
int64_t svdp_calib_need(double sparsity, int32_t D, int32_t T);

/* The statistics svdp_calib_bias consumes, for T calibration tokens X [T][d] (device, in the
 * layer's storage type): w [D][T] and s [D][T] as defined above, with A B x evaluated the way
 * the runtime predictor does, (x P) Q^T in fp32 (the layer's bias b is not used).  Dense
 * contractions on the matrix cores.  bf16 storage only (SVDP_ERR_UNSUPPORTED otherwise).
 * ws: device, 256-byte aligned, >= svdp_calib_stats_workspace_bytes(layer, T).                     */
size_t svdp_calib_stats_workspace_bytes(const svdp_layer *layer, int32_t T);
svdp_status svdp_calib_stats(const svdp_layer *layer, const void *X, int32_t T, float *w, float *s,
                             void *ws, size_t ws_bytes, void *stream);
svdp_status svdp_calib_bias(const float *w, const float *s, int32_t D, int32_t T, int32_t eta, int64_t need,
                            float *b, int32_t *k, int32_t *steps, float *kendall,
                            void *ws, size_t ws_bytes, void *stream);

/* ---- offline build: predictor factors with data whitening (Sec. 4.1, Alg. 1) ----
 *
 * From the gate matrix W_gate [D][d] and T calibration tokens X [T][d] (both device, in `wdtype`):
 * with S any factor of the tokens' second moments, S S^T = X^T X, and U Sigma V^T the SVD of W_gate S,
 * the rank-r pair A = U_r Sigma_r, B = V_r^T S^-1 minimises ||(W_gate - A B) X^T||_F over rank-r products.
 * Outputs in the library's letters, fp32, device: Q = A [D][r], P = B^T [d][r], so that the predictor's
 * scores are (x P) Q^T; the caller rounds them to the layer's storage type.  sigma [r] (host, nullable):
 * the r leading singular values of W_gate S, descending.  sweeps [2] (host, nullable): sweeps[0] = 0,
 * sweeps[1] = block-Jacobi sweeps that the (last projected) eigen-decomposition took.
 * S is the lower Cholesky factor of X^T X, as Alg. 1 prints it (blocked factorisation, 64-wide blocks);
 * V and Sigma^2 are the r leading eigenpairs of (W_gate S)^T (W_gate S), by subspace iteration with Chebyshev
 * filters; directions that dominate are taken out of W_gate S, so that the others are accurate relative to themselves
 * (residuals of the wanted vectors together at most 1e-10 of the smallest wanted eigenvalue, as a rule below 2e-11).
 * Block Jacobi sweeps decompose the projections, and the whole matrix where d < 256, r is more than about 0.4 d, no gap
 * follows the r-th value or fewer than r are above rounding (off-diagonal norm of 1e-11 of the whole).  S^-1 is applied
 * to the r chosen vectors by block back-substitution.  All arithmetic is fp64, the contractions on the matrix cores.
 * Needs d a multiple of 64, T >= d and X^T X positive definite to working precision (every pivot of
 * the factorisation above 1e-13 of the largest diagonal element), r <= d; otherwise
 * SVDP_ERR_UNSUPPORTED.
 * Unlike the decode calls this one is an offline step: it SYNCHRONISES `stream` several times (it reads
 * the factorisation's verdict, convergence figures and eigenvalues on the host) and cannot be captured in a graph.  It allocates
 * nothing on the device.  ws: device, 256-byte aligned, >= svdp_whiten_workspace_bytes(d, D, T, r)
 * (0 for sizes it does not take).                                                                      */
size_t svdp_whiten_workspace_bytes(int32_t d, int32_t D, int32_t T, int32_t r);
svdp_status svdp_whiten_factors(const void *W_gate, const void *X, int32_t d, int32_t D, int32_t T, int32_t r,
                                int32_t wdtype, float *P, float *Q, float *sigma, int32_t *sweeps,
                                void *ws, size_t ws_bytes, void *stream);

/* svdp_ffn_step with svdp_stack_glue in front of it, in the same launches: the step's token is
 * x = RMSNorm(x_prev + y_prev) + shift rounded to `wdtype` (bit for bit what svdp_stack_glue writes),
 * formed inside the step's first kernel, which saves the glue's own launch between stacked layers.
 * x_prev [B][d] in `wdtype`, y_prev [B][d] fp32, shift [d] fp32 (shared by the tokens): device, read;
 * x_out [B][d] in `wdtype`: device, receives x (must not alias x_prev or y_prev; the row kernel reads it).
 * The other arguments as in svdp_ffn_step; y may alias y_prev.                                     */
svdp_status svdp_ffn_step_glued(const svdp_layer *layer, const void *x_prev, const float *y_prev,
                                const float *shift, float eps, void *x_out, int32_t B, float *y,
                                uint64_t *mask_out, int32_t *idx_out, int32_t *nnz_out,
                                void *ws, size_t ws_bytes, void *stream);

/* ---- decoding with drafted tokens ----
 *
 * A program that verifies drafted tokens decodes a small tree of tokens for each request in one pass and keeps the
 * branch that its own answers agree with.  Per step: svdp_tree_attn in every layer, svdp_tree_accept on the logits,
 * svdp_kv_plan for the slots of the accepted tokens, svdp_kv_commit for their K and V of all layers.  Only accepted
 * tokens ever enter the cache, so nothing in it has to be moved or taken back.
 *
 * Rows and trees.  T rows (tokens) of R requests, one request after the other: request r has the rows
 * starts[r] .. starts[r + 1], its nodes 0, 1, ...; starts: device [R + 1] int32, ascending, starts[0] = 0; rows from
 * starts[R] to T are padding.  tree: device [T] 64-bit words, bit j of tree[t]: row t sees node j of its own request;
 * NULL: every node sees the nodes before it and itself.  A request has up to max_nodes <= SVDP_MAX_NODES nodes; the host knows no
 * other number, so kernel and workspace go by it: 64 requests of one token take 1.2 to 2.8 times as long with 64 as with 1.
 * Nodes come after their ancestors (node 0 first: the newest certain token).
 *
 * Pages.  A request's tokens lie in pages of `page` tokens: token i in page table[r][i / page], at i % page.
 * table: device [R][max_pages] int32; entries past a request's length have no influence.  A slot is page id * page + place.
 *
 * Limits (else SVDP_ERR_UNSUPPORTED): page 32, 64, 128 or 256; dim 64, 128 or 256; R <= SVDP_MAX_REQUESTS; T <=
 * SVDP_MAX_ROWS; T * heads_q below 2^26; pages * page, R * max_pages and max_pages * page below 2^31; attention: R * heads *
 * ceil(rows / 16) * (max_pages * page / 128 + 2) below 2^31, where rows = max_nodes * heads_q / heads (some more are taken).  Values read
 * from device memory that lie outside their range never lead outside a buffer: lengths are clamped to the table's
 * width, a page id outside [0, pages) is skipped with its tokens.  What a call writes must not overlap anything else it is given. */
#define SVDP_MAX_NODES 64
#define SVDP_MAX_REQUESTS 4096
#define SVDP_MAX_ROWS (1 << 24)

/* K and V of the cached tokens, all layers.  With e = 16 bytes / element size (8 in 8 bits too), V holds e tokens of a channel side by
 * side: what a lane of the matrix cores multiplies the weights of e tokens with is then one 16-byte load.        */
typedef struct svdp_kv_cache {
    int32_t layers, pages, page, heads, dim;
    int32_t dtype;         /* svdp_dtype of K and V, and of q, k, v and out (SVDP_E4M3: those are bf16) */
    void *K;               /* [layers][pages][heads][page][dim], 16-byte aligned      */
    void *V;               /* [layers][pages][heads][page / e][dim][e], 16-byte aligned */
    uint8_t *K_scale;      /* SVDP_E4M3 only, else not looked at: [layers][pages][heads][page], 16-byte aligned: each token's   */
    uint8_t *V_scale;      /* head of K and of V is its codes times 2^(scale - 127), scale from 1 to 254, as bf16: exact from  */
                           /* 2^-126 on up to bf16's largest number; infinite beyond it, and below 2^-126 it may lose bits     */
} svdp_kv_cache;

/* Attention of every row over its request's cached tokens 0 .. lens[r] and over the nodes that it sees:
 *   out[t][h] = sum_j softmax_j(scale q[t][h] . k_j[c]) v_j[c],  c = h / (heads_q / heads).
 * q: device rows of [heads_q][dim], q_stride elements apart; k, v: device rows of [heads][dim], the step's own
 * tokens (not in the cache), k_stride and v_stride elements apart; the three pointers 16-byte aligned, the strides
 * whole 16-byte vectors.  scale: finite, and times log2(e) too.  lens: device [R] int32.  out: device
 * [T][heads_q][dim] in the cache's type, rows of requests written (padding and nodes past max_nodes are not).  lse:
 * device [T][heads_q] fp32, nullable: the natural logarithm of the softmax's denominator (with its maximum), for
 * joining with attention over other tokens.
 * A row that sees nothing: out 0, lse -inf; so too where every weight is zero (all scores -inf).  Tokens that a row
 * does not see have no influence on it, NaN and infinities included.  Scores, softmax and sums are fp32; for
 * their product with V the weights of a bf16 cache are two bf16 terms each, within 2^-15.
 * ws: >= svdp_tree_attn_workspace_bytes() (0 for arguments it does not take).                                      */
size_t svdp_tree_attn_workspace_bytes(const svdp_kv_cache *cache, int32_t heads_q, int32_t R, int32_t max_pages,
                                      int32_t max_nodes);
svdp_status svdp_tree_attn(const svdp_kv_cache *cache, int32_t layer, const void *q, int64_t q_stride, const void *k,
                           int64_t k_stride, const void *v, int64_t v_stride, const uint64_t *tree, const int32_t *table,
                           int32_t max_pages, const int32_t *lens, const int32_t *starts, int32_t R, int32_t T,
                           int32_t max_nodes, int32_t heads_q, float scale, void *out, float *lse, void *ws,
                           size_t ws_bytes, void *stream);

/* Greedy acceptance.  logits: device rows of [V] in `dtype`, `stride` elements apart (aligned to their elements).
 * best [T]: the index of a row's largest logit, the lowest one among equals; NaN counts as largest (as it does for
 * torch.argmax).  tokens: device [T] int32, the drafted tokens.  From node 0, which is always kept, the walk goes to the
 * lowest node whose parent (the last node before it that it sees) is the current one and whose token is best of the
 * current one, until there is none.  The sets of `tree` have to be trees: node j sees itself, its parent, and what its parent sees.
 * keep [T]: a row's place in the branch (0, 1, ...), -1 for a row that is not in it.  counts [R]: length of the branch
 * (0 for a request without rows).  next [R]: best of the branch's last node, the token that follows it (-1 without rows).
 * All outputs device int32, fully written.  ws: >= svdp_tree_accept_workspace_bytes() (0 for arguments it does not take). */
size_t svdp_tree_accept_workspace_bytes(int32_t T, int32_t V, int32_t dtype);
svdp_status svdp_tree_accept(const void *logits, int64_t stride, int32_t dtype, int32_t V, const int32_t *tokens,
                             const uint64_t *tree, const int32_t *starts, int32_t R, int32_t T, int32_t max_nodes,
                             int32_t *keep, int32_t *counts, int32_t *next, int32_t *best, void *ws, size_t ws_bytes,
                             void *stream);

/* Block tables and slots of a step, from the requests' lengths.  Free pages are the `pool[1]` entries of the ring
 * ring[pages] from place pool[0] on (cyclic).  add[r] >= 0: request r, of lens[r] tokens, takes the pages that add[r] more need, in the
 * order of the requests, from the ring's front, and its new entries of `table` are written.  add[r] = -1: the
 * request ends, its pages go to the ring's end in the order of the requests and of its table row (they are free from
 * the next call on).  Refused (refused[r] = 1, else 0; its length stays, its rows get no slots) is a request
 *  - whose tokens would not fit its row of the table: it asks for no pages, the requests after it are not touched by it;
 *  - whose pages are not there after those of the requests before it: so is every request after it that needs a page, even
 *    where there would be enough for that one.
 * lens_out [R] int32: the lengths after the step.  pool_out [2]: place and number of the free pages after it.
 * keep: device [T], the place of row t among its request's added tokens, -1 for a row that is not added (as
 * svdp_tree_accept writes it); NULL: row starts[r] + i has place i.  slots: device [T] 64-bit, the slot of each row, -1 where it has none.
 * table and ring are changed in place; no array that is written (they, slots, lens_out, pool_out, refused) may overlap another
 * one (else SVDP_ERR_INVALID_ARG).  Every other array is device int32.
 * A repeated call with the same inputs writes the same values.                                                        */
svdp_status svdp_kv_plan(int32_t *table, int32_t max_pages, int32_t *ring, int32_t pages, int32_t page, const int32_t *pool,
                         const int32_t *lens, const int32_t *add, const int32_t *starts, const int32_t *keep, int32_t R,
                         int32_t T, int64_t *slots, int32_t *lens_out, int32_t *pool_out, int32_t *refused, void *stream);

/* K and V of new tokens into their slots, all layers: k, v: device, row t of layer l is [heads][dim] at
 * l * layer_stride + t * row_stride elements (whole 16-byte vectors, pointers 16-byte aligned).  slots: device [T]; a
 * slot outside [0, pages * page) is skipped, no two rows may have the same one.  Rows are of the cache's type.
 * SVDP_E4M3: rows are bf16.  Each token's head gets the least power of two 2^b, b >= -96, at which none of its elements is above
 * 448 2^b, and its elements are divided by it and rounded to e4m3 (to the nearest, ties to even; where b is 120 to no more than 240, so
 * that every element is a finite bf16 number again).  Infinities and NaN become NaN, and do not count for the power.  */
svdp_status svdp_kv_commit(const svdp_kv_cache *cache, const void *k, int64_t k_layer_stride, int64_t k_row_stride,
                           const void *v, int64_t v_layer_stride, int64_t v_row_stride, const int64_t *slots, int32_t T,
                           void *stream);

/* The other way: row t of k and v, all layers, becomes K and V of slot slots[t]; zeros where that lies outside [0, pages * page).
 * Strides and types as above (SVDP_E4M3: bf16, exact for all that svdp_kv_commit writes).  The same slot may be read
 * by several rows; rows must not overlap each other or anything else (refused where rows of K meet, rows of V, or rows of
 * both whose strides are the same).                                                                                  */
svdp_status svdp_kv_read(const svdp_kv_cache *cache, const int64_t *slots, int32_t T, void *k, int64_t k_layer_stride,
                         int64_t k_row_stride, void *v, int64_t v_layer_stride, int64_t v_row_stride, void *stream);

/* ---- around attention and logits ---- */

/* Norms of the heads of q and k, and their rotation by the rows' positions:
 *   y = x / sqrt(mean(x^2) + eps) * weight (SVDP_ROPE_NORM; weight NULL: 1),  then for i < rot / 2
 *   (y_a, y_b) -> (y_a cos - y_b sin, y_b cos + y_a sin),  angle = places[t] * inv_freq[i],
 * (a, b) = (i, rot / 2 + i), or (2 i, 2 i + 1) with SVDP_ROPE_INTERLEAVED; channels from rot on are not turned.
 * q: device rows of [heads_q][dim], q_stride elements apart, k: of [heads][dim] (heads may be 0: no k), in `dtype`, SVDP_F32 or
 * SVDP_BF16; q_out and k_out likewise.  In place (q_out = q with the same stride, k_out = k likewise) is fine; otherwise they
 * overlap nothing (refused where rows of the same stride meet).  Pointers 16-byte aligned, strides whole 16-byte vectors.  places: device [T] int32; inv_freq: device [rot / 2]
 * fp32 (both may be NULL if rot is 0).  q_weight, k_weight: device [dim] fp32, with SVDP_ROPE_WEIGHT_EACH [heads][dim], 16-byte
 * aligned, NULL for none.  dim 64, 128 or 256; rot a multiple of 8, up to dim.  Angles are taken in 64 bits, so that far positions lose
 * nothing; all else is fp32, rounded once.                                                                          */
enum { SVDP_ROPE_INTERLEAVED = 1u, SVDP_ROPE_NORM = 2u, SVDP_ROPE_WEIGHT_EACH = 4u };
svdp_status svdp_qk_rope(int32_t dtype, int32_t dim, int32_t T, const void *q, int64_t q_stride, int32_t heads_q, const void *k,
                         int64_t k_stride, int32_t heads, const int32_t *places, const float *inv_freq, int32_t rot, uint32_t flags,
                         const float *q_weight, const float *k_weight, float eps, void *q_out, int64_t q_out_stride, void *k_out,
                         int64_t k_out_stride, void *stream);

/* A token for each row of logits, drawn with given random numbers.  logits: device rows of [V] in `dtype`, `stride` elements apart (aligned
 * to their elements; 0: all draws from one row), V <= SVDP_MAX_VOCABULARY.  A row's tokens stand in order, largest logit first, lowest index first among
 * equals, with weights w = 2^44 exp((x - x_first) / temperature) rounded to whole numbers.  Kept are the first tokens of the order: no more
 * than top_k (0 or less: all); the fewest whose weight is at least top_p of the weight of those (1 or more, NaN: all);
 * those with w >= min_p 2^44 (0 or less, NaN: all); always the first one.  Drawn is the first one at which the sum of
 * the weights, in order, exceeds u times the kept tokens' sum: u in [0, 1), what lies outside counts as its nearest end.
 * temperature 0 or less, or NaN: the first token.  A largest logit of +inf or NaN (NaN is above all): the lowest index that has
 * it.  All logits -inf: -1.  Sums are whole numbers and exact, so that nothing depends on how the work is divided.
 * u, temperature, top_p, min_p: device [T] fp32; top_k: device [T] int32; all but u may be NULL (1, all, all, all).
 * answers [T] int32.  logp [T] fp32, nullable: logarithm of the drawn token's share of the kept weight (0 for a first token that is not
 * drawn, -inf with -1).  No scratch memory is needed.                                                              */
#define SVDP_MAX_VOCABULARY (1 << 19)
svdp_status svdp_sample(const void *logits, int64_t stride, int32_t dtype, int32_t V, const float *u, const float *temperature,
                        const int32_t *top_k, const float *top_p, const float *min_p, int32_t T, int32_t *answers, float *logp,
                        void *stream);

/* The branch of each tree that agrees with given answers (drawn ones, e.g.): keep, counts and next as svdp_tree_accept forms them from its
 * `best`, here answers [T] int32.  An answer of -1 agrees with no token from 0 on.                                  */
svdp_status svdp_tree_walk(const int32_t *answers, const int32_t *tokens, const uint64_t *tree, const int32_t *starts, int32_t R,
                           int32_t T, int32_t max_nodes, int32_t *keep, int32_t *counts, int32_t *next, void *stream);

/* Static string for a status code.  Never NULL. */
const char *svdp_status_string(svdp_status st);

/* Library version, "major.minor". */
const char *svdp_version(void);

#ifdef __cplusplus
}
#endif
#endif /* SVDP_H */
