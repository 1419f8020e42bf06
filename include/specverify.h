/*
 * specverify.h -- C ABI of libspecverify: batched verification of a draft token tree on one GPU.
 *
 * The library implements the verification step of multi-path speculative decoding (paper
 * Section 2, step 3): given target and draft logits on the nodes of a draft tree, the tree, the
 * sampling parameters and caller-supplied uniforms, it selects one accepted node and one
 * correction ("bonus") token so that the emitted tokens follow the target distribution.
 *
 * General rules for every entry point
 *   - `extern "C"`, plain pointers and sizes.  Unless a parameter says "host", a data pointer is
 *     a DEVICE pointer owned by the caller; the library only borrows it until the work it
 *     enqueued on `stream` has finished.  `SpecIn` / `SpecOut` themselves are host structs, read
 *     during the call only.
 *   - `stream` is a `cudaStream_t` passed as `void*` (NULL = the legacy default stream).  Calls
 *     enqueue kernels and return; they never synchronise, allocate or free.
 *   - Scratch memory comes from the caller: `ws` (device, 256-byte aligned) of at least
 *     `spec_workspace_bytes()` bytes.  Two calls that may overlap on the GPU need two workspaces.
 *   - Return value: SPEC_OK or a negative SPEC_ERR_* found on the host before anything was
 *     enqueued.  Problems only visible on the device (bad topology or token, a non-finite row, a
 *     bounded wait that ran out) are reported per sequence in `SpecOut.status` (a SPEC_DEV_*
 *     code); that sequence gets accept_len = -1 and accepted_node = -1.  Nothing traps.
 *   - There is no CPU fallback.
 *
 * Tree layout (Definition 3.1, Definition 5.2): node 0 is the root (the current context);
 * parent[0] = -1 and parent[i] < i.  The child list of a node is the set of nodes naming it as
 * parent, in increasing index order; that is the order in which children are tried.  Equal tokens
 * under one parent stay separate nodes (multiplicity, Section 3.2).  At most SPEC_MAX_CHILDREN
 * children per node and SPEC_MAX_NODES nodes per sequence.
 *
 * Sampling distribution of a row (Section 4 names temperature and nucleus sampling; top-k is an
 * addition): y = z / T, softmax; top-k keeps every token whose logit is >= the k-th largest logit
 * value; top-p then keeps the fewest leading groups of equal-logit tokens whose mass (within the
 * top-k set) reaches top_p; renormalise.  The same transform is applied to target and draft rows.
 */
#ifndef SPECVERIFY_H
#define SPECVERIFY_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define SPEC_MAX_CHILDREN 16
#define SPEC_MAX_NODES 1024

/* host-side return codes */
#define SPEC_OK 0
#define SPEC_ERR_NULL (-1)        /* a required pointer is NULL                                  */
#define SPEC_ERR_SHAPE (-2)       /* B, N, V or a stride is out of range                         */
#define SPEC_ERR_DTYPE (-3)       /* a dtype that the call does not take                          */
#define SPEC_ERR_PARAM (-4)       /* temperature <= 0 or not finite, top_p outside (0,1], top_k < 0 */
#define SPEC_ERR_WORKSPACE (-5)   /* ws NULL, misaligned or too small                            */
#define SPEC_ERR_UNSUPPORTED (-6) /* vocabulary too large for the on-chip plan of this device    */
#define SPEC_ERR_CUDA (-7)        /* a CUDA runtime call failed (launch configuration, no device) */

/* per-sequence device status codes (SpecOut.status) */
#define SPEC_DEV_OK 0
#define SPEC_DEV_TOPOLOGY 1       /* parent[0] != -1, parent[i] outside [0,i), too many children */
#define SPEC_DEV_TOKEN 2          /* token outside [0,V)                                         */
#define SPEC_DEV_NONFINITE 3      /* a logit row holds NaN / +inf, or only -inf                  */
#define SPEC_DEV_TIMEOUT 4        /* a bounded on-device wait ran out                            */
#define SPEC_DEV_PAGE 5           /* a block id outside the cache, or a key beyond the block table */
#define SPEC_DEV_BLOCKS 6         /* no free block left, or no room for one in the block table   */

#define SPEC_F32 0
#define SPEC_BF16 1
#define SPEC_F16 2                /* the operators on projections and caches, and log probabilities */

typedef struct {
    int32_t B, N, V;              /* sequences, nodes per sequence (root included), vocabulary   */
    int32_t logits_dtype;         /* SPEC_F32 or SPEC_BF16                                        */
    const void *target_logits;    /* [B,N,V] row of node a of sequence b at b*seq_stride + a*node_stride */
    const void *draft_logits;     /* same layout; rows of nodes without children are never read  */
    int64_t seq_stride;           /* in elements                                                  */
    int64_t node_stride;          /* in elements, >= V; the V entries of a row are contiguous     */
    const int32_t *parent;        /* [N], or [B,N] with topo_seq_stride = N                       */
    int64_t topo_seq_stride;      /* 0: one topology shared by the batch                          */
    const int32_t *token;         /* [B,N] draft token of each node; token[b,0] is ignored        */
    float temperature;            /* > 0                                                          */
    int32_t top_k;                /* 0 = off                                                      */
    float top_p;                  /* in (0,1]; 1 = off                                            */
    const float *temperature_per_seq; /* optional [B]; overrides `temperature` when not NULL      */
    const float *u_accept;        /* [B,N] uniforms in [0,1): entry of node a decides a's test    */
    const float *u_bonus;         /* [B,N] uniforms in [0,1): the stop node's entry draws the bonus */
} SpecIn;

typedef struct {
    int32_t *accepted_node;       /* [B] index of the accepted node (0 = nothing accepted)        */
    int32_t *accept_len;          /* [B] tau = depth of the accepted node                          */
    int32_t *out_tokens;          /* [B,N] tokens on the accepted path, then the bonus, then -1   */
    int32_t *bonus_token;         /* [B]                                                           */
    int32_t *status;              /* [B] SPEC_DEV_*                                                */
    /* optional outputs: skipped when NULL */
    float *residual;              /* [B,V] the distribution the bonus token was drawn from         */
    float *node_thr;              /* [B,N] threshold node a is tested with as if it were reached:
                                     SpecInfer: min(1, P/q) after its earlier siblings were rejected
                                     (asking for it disables the early exit after an accepted
                                     sibling); Traversal: the final weight of a.  Root: 1          */
    float *node_w_in;             /* [B,N] Traversal only: weight handed to a by its parent        */
    float *node_features;         /* [B,N,4] entropy (nats) of the target and draft sampling
                                     distributions and their largest probability:
                                     H_p, H_q, top1_p, top1_q (q entries 0 for childless nodes)   */
    float *margin;                /* [B,N+1] |u_accept - threshold| per node (NaN where the node
                                     was not evaluated), last entry: distance of the bonus draw to
                                     the nearer CDF boundary, as a fraction of the total mass      */
} SpecOut;

/* Bytes of scratch the calls below need for these shapes (depends on B, N only).
 * host pointers.  Returns SPEC_OK or SPEC_ERR_NULL / SPEC_ERR_SHAPE. */
int32_t spec_workspace_bytes(const SpecIn *in, int64_t *bytes);

/*
 * Sampling distribution of every node's target (which = 0) or draft (which = 1) row, written to
 * HBM (Section 4: temperature / nucleus; tie rules above).
 *   probs      [B,N,V] float, contiguous.  May be NULL when only the statistics are wanted.
 *   row_stats  optional [B,N,6] float: max of z/T, sum of kept exp(z/T - max), kept count,
 *              entropy (nats), largest probability, smallest kept logit value.
 * Only B, N, V, dtype, the logits of the chosen side, strides and the sampling parameters of `in`
 * are read (every row of the chosen side is read, whatever the tree).  With truncating parameters
 * (top_k or top_p active) `ws` must be a workspace of spec_workspace_bytes(); otherwise it may be
 * NULL.  Rows that are not finite produce NaN statistics and zero probabilities.
 */
int32_t spec_tree_probs(const SpecIn *in, int32_t which, float *probs, float *row_stats,
                        void *ws, int64_t ws_bytes, void *stream);

/*
 * The first half of a verification call on its own: the statistics (reference, normaliser, top-k /
 * top-p cut) of every row the verifiers read -- the one pass over the logits in HBM (Section 4's
 * sampling transform, without materialising the distributions).  Results stay in `ws`; the entry point
 * exists so that this pass can be timed and profiled by itself.  Same arguments and checks as the
 * verifiers.
 */
int32_t spec_row_statistics(const SpecIn *in, void *ws, int64_t ws_bytes, void *stream);

/*
 * SpecInfer verification (Algorithm 4 used top-down, Section 3.2 "OT-based algorithms"):
 * starting at the root, try the children of the current node in list order; child x is accepted
 * when u_accept < min(1, P(x)/q(x)), where P is the node's target distribution after the residual
 * updates P <- norm((P - q)+) of the siblings rejected before it; on acceptance move to that
 * child, otherwise stop and draw the bonus token from P by inverse CDF with the node's u_bonus
 * (from the unmodified target distribution at a childless node).
 * Fused: logits in, decisions out; no [B,N,V] tensor is written.
 */
int32_t spec_verify_specinfer(const SpecIn *in, const SpecOut *out, void *ws, int64_t ws_bytes,
                              void *stream);

/*
 * Top-down verification with one of the other OTLP solvers the paper defines (Appendix B; composed as
 * Section 3.2 "OT-based algorithms" says: at a node the solver puts out one token; the walk moves to the
 * first child, in list order, that carries it, and stops when no child does -- that token is the
 * correction token).  solver: 0 = NSS (Algorithm 1: the token is drawn from p, the drafts are ignored),
 * 1 = NaiveTree (Algorithm 2: the first child is tested with min(1, p/q), otherwise a draw from
 * norm((p - q)+)), 2 = SpecTr K-SEQ (Algorithm 3: division factor rho* by root search, every child
 * tested with min(1, p / (rho q)), otherwise a draw from its residual).  A child's test uses its entry
 * of u_accept, a draw at node a the entry u_bonus[a].  Same inputs, workspace, stream and status rules
 * as spec_verify_specinfer; of SpecOut only accepted_node, accept_len, out_tokens, bonus_token and
 * status are written, and the optional outputs must be NULL (SPEC_ERR_UNSUPPORTED otherwise, and for
 * N > 128).  solver outside 0..2: SPEC_ERR_PARAM.
 */
int32_t spec_verify_otlp(const SpecIn *in, const SpecOut *out, int32_t solver, void *ws, int64_t ws_bytes,
                         void *stream);

/*
 * SpecInfer verification for callers that cannot allocate device memory.  The paper has no
 * counterpart to this entry point: it exists for hosts of this library that are handed their
 * device buffers by someone else and may not call cudaMalloc themselves -- a plugin running inside
 * an inference server whose memory pool is closed to it, a process under a fixed memory budget, or
 * code that runs where an allocation would stall or fail (a latency-critical decoding loop, a
 * region in which the allocator is locked).  Same inputs, outputs and results as
 * spec_verify_specinfer, but no `ws` argument: the scratch memory is an array of
 * SPEC_STATIC_WS_BYTES bytes inside the library image, present on every GPU that has loaded the
 * library until the process exits.
 *   - Limit: B * N <= SPEC_STATIC_MAX_NODES (tree nodes summed over the batch); larger shapes
 *     return SPEC_ERR_WORKSPACE and nothing is enqueued.  V is not limited by the scratch.
 *   - The first call on a device looks up the array's device address (once per device, with that
 *     device current) before it enqueues anything; make that first call outside any stream
 *     capture.  No call allocates or frees memory.
 *   - Every call uses the same array, which still holds the previous call's records when the next
 *     one starts; the call clears the parts that must start empty (the published weights and the
 *     arrival counters) on `stream` itself.  Two calls that can overlap on the GPU (different
 *     streams without an ordering between them) race on the array: serialise them, or give the
 *     others a workspace through spec_verify_specinfer.
 */
#define SPEC_STATIC_MAX_NODES 4096
#define SPEC_STATIC_WS_BYTES (1536 * 1024)
int32_t spec_verify_specinfer_static(const SpecIn *in, const SpecOut *out, void *stream);

/*
 * Traversal Verification (Section 3.2, bottom-up; block verification of Section 3.1 on one
 * path).  Weights flow down: a child with token x gets min(1, w P(x)/q(x)) from its parent's
 * current (w, P); a node is tested (u_accept < w) only after all its child subtrees were
 * rejected, each rejection updating the parent to S = sum (wP - q)+, w <- S / (S + 1 - w),
 * P <- (wP - q)+ / S.  The first node accepted in depth-first post-order wins; the root always
 * accepts.  The bonus token is drawn from the accepted node's final P with its u_bonus.
 */
int32_t spec_verify_traversal(const SpecIn *in, const SpecOut *out, void *ws, int64_t ws_bytes,
                              void *stream);

/*
 * Offline analysis of a batch of draft trees (Section 5 and Appendices C, D): for every node with
 * children, from its sampling distributions p, q (same transform as the verifiers) and its child list,
 *   acceptance  [B,N,4] acceptance rates alpha(f) of Definition 5.1 with k = the node's number of
 *               children: NSS (Algorithm 6), Naive (Algorithm 7), SpecTr (Algorithm 8), SpecInfer
 *               (Algorithm 9);
 *   divergence  [B,N,3] L1 distance sum |p - q| (Section 5), KL(p||q), KL(q||p) in nats (the selector's
 *               scalar features, Section 6; +inf where the second law has no mass under the first);
 *   branch      [5][B,N] branching probability B(f, ch(parent), token) of Definition 5.3 of moving from
 *               the parent into the node, for f = NSS (Algorithm 11), Naive (12), SpecTr (13), SpecInfer
 *               with children tried in list order (what spec_verify_specinfer runs), SpecInfer with the
 *               next child picked uniformly (Algorithm 14; NaN for more than 10 children); root: 1; a
 *               child whose token an earlier sibling carries is never moved to: 0;
 *   reach       [5][B,N] product of the branching probabilities along the node's path;
 *   block_eff   [5][B]  sum of reach over the tree's nodes = E[tau + 1 | tree], the inner sum of
 *               equation (3) (average it over sampled trees for the paper's estimator).
 * Rows of childless nodes are NaN in acceptance / divergence.  All outputs are device pointers, all
 * required.  `ws`: spec_analysis_workspace_bytes() bytes.  u_accept / u_bonus of `in` must be valid
 * but do not influence the outputs.  SpecTr's rho* is found to (k - 1) 2^-40 on [1, k].
 */
typedef struct {
    float *acceptance;
    float *divergence;
    float *branch;
    float *reach;
    float *block_eff;
} SpecAnalysisOut;
int32_t spec_analysis_workspace_bytes(const SpecIn *in, int64_t *bytes);
int32_t spec_tree_analysis(const SpecIn *in, const SpecAnalysisOut *out, void *ws, int64_t ws_bytes, void *stream);

/*
 * Forward-pass time of delayed-expansion actions (Appendix E, equation (8)): for action a = (K, L1, L2)
 * at context length ctx,
 *   T_hat[a] = sum_{j<L1} t_q(ctx + j) + sum_{j<L2} t_q(ctx + L1 + j K) + t_p(ctx + L1 + K L2),
 * t_q / t_p: measured draft / target forward times per context length (tables of n_len doubles; a length
 * beyond the table uses its last entry).  actions [n_actions,3] int32, T_hat [n_actions] double; all
 * device pointers.
 */
int32_t spec_latency_model(const double *t_q, const double *t_p, int32_t n_len, int32_t ctx, const int32_t *actions,
                           int32_t n_actions, double *T_hat, void *stream);

/*
 * Inverse-CDF draw (the "Sample Y ~ p" steps of Algorithms 1-4) from R rows of non-negative
 * weights that need not be normalised: token[r] = smallest t with w_0 + ... + w_t > u[r] * sum(w).
 *   weights [R,V] float contiguous, u [R] in [0,1), token [R] (-1 for an all-zero row),
 *   margin optional [R]: distance to the nearer CDF boundary as a fraction of the total.
 */
int32_t spec_sample_bonus(const float *weights, int32_t R, int32_t V, const float *u,
                          int32_t *token, float *margin, void *ws, int64_t ws_bytes, void *stream);

/*
 * Host-buffer form of the two verifiers (the verification step of Section 2 for a caller whose
 * logits sit in host memory).  Every data pointer of `in` and `out` is a HOST pointer (pinned
 * memory gives asynchronous copies); logits must be dense ([B,N,V] contiguous).  `dev_buf` is a
 * DEVICE buffer of at least spec_host_staging_bytes() bytes, 256-byte aligned, owned by the
 * caller; inputs are copied into it, the verifier (algorithm 0 = SpecInfer, 1 = Traversal) runs
 * on `stream`, the five required outputs are copied back and the stream is synchronised before
 * the call returns -- this is the one entry point that synchronises.  Optional outputs and
 * temperature_per_seq are not available here (SPEC_ERR_UNSUPPORTED when set).
 */
int32_t spec_host_staging_bytes(const SpecIn *in, int64_t *bytes);
int32_t spec_verify_host(const SpecIn *in, const SpecOut *out, int32_t algorithm, void *dev_buf,
                         int64_t dev_bytes, void *stream);

/* ------------------------------------------------------------------------------------------------
 * The operators around a verification in a decoding loop (the target model's pass over the draft tree of
 * Section 2, step 2, and what a paged cache of keys and values needs before and after it).
 *
 * A cache is num_blocks blocks of block_size slots; slot s is entry s % block_size of block s / block_size.  A request's token at
 * position j lies at entry j % block_size of the block that its row of the block table names in column j / block_size.
 * lengths[b] is the number of committed tokens.  The N nodes of a request's tree lie behind them: node i at entry lengths[b] + i
 * (node 0 is the root: the token emitted last, whose keys and values are not in the cache yet), at POSITION
 * lengths[b] + depth(i).  A request with lengths[b] < 0 takes no part: nothing of it matters but the length.  n_nodes (optional,
 * [B]): the request's tree has n_nodes[b] <= N nodes; what belongs to the others reaches no result, whatever it holds (the others'
 * rows of an array that is there may be read along with the tree's).  Status codes per request as
 * above; a request with n_nodes[b] outside [0,N] counts as one without nodes, with SPEC_DEV_TOPOLOGY.  N is at most
 * SPEC_MAX_NODES here too; a node may have any number of children.
 * ------------------------------------------------------------------------------------------------ */

/*
 * Blocks, slots and positions of a step, from the requests' lengths.  Request b needs ceil((lengths[b] + nodes) / block_size) blocks
 * and has the first owned[b] columns of its row of block_table.  What it lacks is taken, request by request, from a
 * ring of free blocks: the free_range[1] entries of free_blocks from index free_range[0] on (mod free_size).
 * The first request that the ring has too few blocks for, and every later one that lacks any, gets none
 * (SPEC_DEV_BLOCKS, slots and positions -1); so does one whose row is too short, which takes none from the ring either.
 * block_table is written in columns owned[b] .. only; owned and free_range are inputs and stay as they are, the new
 * values are owned_out and free_range_out (other arrays): the call can be repeated.
 * A bad tree leaves positions of -1 and SPEC_DEV_TOPOLOGY, a negative or too large block id slots of -1 and
 * SPEC_DEV_PAGE.  Idle requests and nodes beyond n_nodes[b]: slots and positions -1.
 */
typedef struct {
    int32_t B, N;
    int32_t block_size, table_width;  /* slots of a block; columns of block_table                     */
    const int32_t *lengths;           /* [B]                                                          */
    const int32_t *n_nodes;           /* optional [B]                                                 */
    const int32_t *parent;            /* [N], or [B,N] with topo_seq_stride = N                       */
    int64_t topo_seq_stride;
    int32_t *block_table;             /* row b at b * table_stride                                    */
    int64_t table_stride;
    const int32_t *owned;             /* [B]                                                          */
    const int32_t *free_blocks;       /* [free_size]                                                  */
    int32_t free_size;
    const int32_t *free_range;        /* [2]: index of the first free block, number of free blocks    */
    int32_t *slots, *positions;       /* [B,N]                                                        */
    int32_t *owned_out;               /* [B]                                                          */
    int32_t *free_range_out;          /* [2]                                                          */
    int32_t *status;                  /* [B]                                                          */
} SpecSlots;
int32_t spec_cache_slots(const SpecSlots *a, void *stream);

/*
 * Norm and rotation of queries and keys per head, and keys and values into the cache, in one pass: for a head's row x of a query or key,
 *   y = x / sqrt(mean(x^2) + eps) * weight   (no norm where the weight is NULL),
 *   (a, b) -> (a cos t - b sin t, b cos t + a sin t), t = positions[token] * inv_freq[i], for the i-th of the rot/2 pairs of the first
 *   rot entries: (y_i, y_{i + rot/2}) with pairs = 0 (halves), (y_{2i}, y_{2i+1}) with pairs = 1 (neighbours).
 * Queries go to q_out (may be q itself), keys and values (values as they are) to slot slots[token] of the caches.
 * Arithmetic in fp32, angles reduced in fp64, one rounding at the end.  A token whose slot is outside
 * [0, num_blocks * block_size) is padding: nothing of it is read or written.  No two tokens may share a slot.
 * D: a multiple of 8 up to 256; rot: a multiple of 16 up to D.  T: below 2^31 - 4096.  Strides in elements; the D entries of a head are contiguous.
 */
typedef struct {
    int32_t T, Hq, Hkv, D, rot, pairs, dtype;   /* tokens; heads; SPEC_F32, SPEC_BF16 or SPEC_F16     */
    int32_t num_blocks, block_size;
    const void *q, *k, *v;
    int64_t q_stride[2], k_stride[2], v_stride[2];              /* token, head                        */
    const void *q_weight, *k_weight;            /* optional [D], of the same type                     */
    float eps;
    const float *inv_freq;                      /* [rot/2]; may be NULL for rot = 0                     */
    const int32_t *positions, *slots;           /* [T]                                                */
    void *q_out;
    int64_t q_out_stride[2];
    void *k_cache, *v_cache;
    int64_t k_cache_stride[3], v_cache_stride[3];               /* block, slot, head                  */
} SpecNormRope;
int32_t spec_norm_rope_cache(const SpecNormRope *a, void *stream);

/*
 * Attention of the nodes of every request's tree over its committed tokens and the tree (Section 2, step 2: the target pass with
 * a tree mask).  Node i of request b, at position t = lengths[b] + depth(i), sees
 *   the committed tokens at positions j < lengths[b], and itself and its ancestors in the tree,
 *   with window > 0 of these only the ones at positions > t - window or < sinks;
 *   out[b,i,h] = sum_j softmax_j(scale q[b,i,h] . k_j) v_j over what it sees, k and v of head h / (Hq / Hkv).
 * N = 1, parent = {-1}: plain decoding; parent[i] = i - 1: a stretch of a prompt.
 * Scores, maxima and sums in fp32; probabilities are rounded to the type of the values for the product with them.
 * A row that sees nothing (a block id outside [0, num_blocks) hides its keys and gives SPEC_DEV_PAGE) is 0, its lse -inf; so are all
 * rows of a request with a bad tree (SPEC_DEV_TOPOLOGY).  A row whose scores are all -inf is NaN (0 / 0), its lse -inf.  Keys and values that
 * no node sees are not read; what a node does not see does not reach its row, whatever it holds (NaN and infinities too).  Rows of idle requests and of nodes beyond n_nodes[b] stay as they were.
 * SPEC_DEV_TIMEOUT (a wait ran out, in any request's part of the work): the rows of the call's requests are undefined.
 * D: 64, 128 or 256.  q, caches and out of one type, SPEC_BF16 or SPEC_F16.  Strides in elements, multiples of 8, and bases on 16 bytes;
 * the D entries of a head are contiguous; out overlaps no input.  lse: optional, log of sum_j exp(scale q.k_j) (natural).
 * `ws`: spec_tree_attention_workspace_bytes() bytes (a function of the sizes; contents do not matter).
 */
typedef struct {
    int32_t B, N, Hq, Hkv, D, dtype;
    int32_t num_blocks, block_size, table_width;
    int32_t window, sinks;            /* window 0: none                                               */
    float scale;                      /* >= 0, finite                                                 */
    const void *q;
    int64_t q_stride[3];              /* request, node, head                                          */
    const void *k_cache, *v_cache;
    int64_t k_cache_stride[3], v_cache_stride[3];               /* block, slot, head                  */
    const int32_t *block_table;
    int64_t table_stride;
    const int32_t *lengths;           /* [B]                                                          */
    const int32_t *n_nodes;           /* optional [B]                                                 */
    const int32_t *parent;            /* [N], or [B,N] with topo_seq_stride = N                       */
    int64_t topo_seq_stride;
    void *out;
    int64_t out_stride[3];            /* request, node, head                                          */
    float *lse;                       /* optional [B,N,Hq]                                            */
    int32_t *status;                  /* [B]                                                          */
} SpecAttention;
int32_t spec_tree_attention_workspace_bytes(const SpecAttention *a, int64_t *bytes);
int32_t spec_tree_attention(const SpecAttention *a, void *ws, int64_t ws_bytes, void *stream);

/*
 * After a verification: the accepted path's entries move behind the committed tokens, in every cache of a stack (keys and values of all
 * layers).  The path's node at depth d = 1, 2, ... goes from entry lengths[b] + node to entry lengths[b] + d; other entries
 * stay as they are.  lengths_out[b] = lengths[b] + depth(accepted) + 1 (the root is committed too; the correction token is the next
 * tree's root).  accepted_node[b] = -1 (a failed verification) or an idle request: nothing moves, the length stays.
 * accepted_node outside the tree: SPEC_DEV_TOPOLOGY, as with a bad tree; a bad block id on the path, also under entries that are in place
 * already, or a path that leaves the table: SPEC_DEV_PAGE; then nothing of the request moves and its length stays.  The blocks that hold a request's tree must be its own.
 */
typedef struct {
    int32_t B, N, caches;
    int32_t num_blocks, block_size, table_width;
    void *cache;                      /* row of slot e of block k of cache c: c * stride[0] + k * stride[1] + e * stride[2] bytes */
    int64_t stride[3];
    int64_t row_bytes;                /* below 2^31                                                   */
    const int32_t *block_table;
    int64_t table_stride;
    const int32_t *lengths;           /* [B]                                                          */
    const int32_t *n_nodes;           /* optional [B]                                                 */
    const int32_t *parent;            /* [N], or [B,N] with topo_seq_stride = N                       */
    int64_t topo_seq_stride;
    const int32_t *accepted_node;     /* [B]                                                          */
    int32_t *lengths_out;             /* [B], not `lengths`                                           */
    int32_t *status;                  /* [B]                                                          */
} SpecCommit;
int32_t spec_cache_commit(const SpecCommit *a, void *stream);

/*
 * Verification of drafted chains from probabilities (the single-path case of Section 3.1, for callers that have the laws
 * already: own logit processors, grammar masks).  Request b drafted the tokens token[cu_drafts[b] .. cu_drafts[b+1]); its i-th draft (0-based) is
 * judged by row cu_drafts[b] + b + i of target_probs and row cu_drafts[b] + i of draft_probs; the request's last
 * target row (index cu_drafts[b+1] + b) is the law behind all drafts.  Draft i is accepted when u_accept[its index] < min(1, p(x) / q(x)) (0 where
 * p(x) <= 0, 1 where q(x) <= 0 < p(x)); the first one rejected ends the chain, and a token is drawn by inverse CDF from
 * norm((p - q)+) of its rows, or from the last row where all were accepted, with u_bonus of that target row.
 * draft_probs NULL: the drafts were looked up, q is 1 at the drafted token and 0 elsewhere.
 * Rows need not be normalised for the draw; decisions and sums in fp64.  (p - q)+ without mass: the draw is from p.
 * A gathered probability that is negative or not finite, or a row without finite positive mass: SPEC_DEV_NONFINITE; a token outside [0,V):
 * SPEC_DEV_TOKEN; cu_drafts that decrease, leave [0, n_drafts], or give a request more than max_drafts:
 * SPEC_DEV_TOPOLOGY; then accept_len and tokens are -1.
 */
typedef struct {
    int32_t B, V, max_drafts, dtype;  /* SPEC_F32 or SPEC_BF16                                        */
    int64_t n_drafts;                 /* drafts of all requests                                       */
    const void *target_probs;         /* [n_drafts + B, V], rows target_stride elements apart         */
    const void *draft_probs;          /* [n_drafts, V], rows draft_stride elements apart, or NULL     */
    int64_t target_stride, draft_stride;
    const int32_t *token;             /* [n_drafts]                                                   */
    const int32_t *cu_drafts;         /* [B + 1]                                                      */
    const float *u_accept;            /* [n_drafts]                                                   */
    const float *u_bonus;             /* [n_drafts + B]                                               */
    int32_t *accept_len;              /* [B]                                                          */
    int32_t *out_tokens;              /* [B, max_drafts + 1]: accepted drafts, the drawn token, then -1 */
    int32_t *bonus_token;             /* [B]                                                          */
    int32_t *status;                  /* [B]                                                          */
} SpecChains;
int32_t spec_verify_probs(const SpecChains *a, void *stream);

/* ------------------------------------------------------------------------------------------------
 * Shared prefixes, bounded caches, and what a service answers with.  Caches, tables, lengths and trees as above.
 * ------------------------------------------------------------------------------------------------ */

/*
 * spec_tree_attention for requests that share prefixes: a group's prefix is attended to once for all of its members.  Group g has shared_blocks[g] whole
 * blocks, prefix_table[g][0 ..), and the members members[first[g] .. first[g+1]); group[b] is request b's group (negative: none) and place[b] its
 * place among that group's members.  A member's committed tokens begin with its prefix: lengths[b] counts it, and the first shared_blocks[g]
 * columns of its row of block_table are not read.  Every row has the result that spec_tree_attention gives for a row of block_table that begins with
 * the prefix's blocks, and a lse with it; window and sinks are 0.
 * A plan that does not fit together (first not rising within [0, n_members], members[first[group[b]] + place[b]] other than b, group[b] >= n_groups,
 * shared_blocks[g] outside [0, prefix_width]) or a length below the prefix: SPEC_DEV_TOPOLOGY for the requests concerned (a `first` that does not rise:
 * for all), whose rows are 0.  A bad block of a prefix hides its keys and gives its members SPEC_DEV_PAGE.
 * `ws`: spec_prefix_attention_workspace_bytes() bytes (a function of the sizes; contents do not matter).  With groups about 4 (B + n_members) N Hq D of them, for rows
 * whose two parts are put together at the end: up to four times the output.
 */
typedef struct {
    SpecAttention attention;          /* window and sinks 0                                           */
    int32_t n_groups, n_members, prefix_width;      /* n_members at most B                            */
    const int32_t *group;             /* [B]                                                          */
    const int32_t *members;           /* [n_members]                                                  */
    const int32_t *first;             /* [n_groups + 1]                                               */
    const int32_t *place;             /* [B]                                                          */
    const int32_t *shared_blocks;     /* [n_groups]                                                   */
    const int32_t *prefix_table;      /* row g at g * prefix_stride                                   */
    int64_t prefix_stride;
} SpecPrefixAttention;
int32_t spec_prefix_attention_workspace_bytes(const SpecPrefixAttention *a, int64_t *bytes);
int32_t spec_prefix_attention(const SpecPrefixAttention *a, void *ws, int64_t ws_bytes, void *stream);

/*
 * Log probabilities of given tokens under rows of logits, with the rows' entropy and their most probable tokens.  Row (b, i) is
 *   logits[b,i] where parent is NULL;
 *   the logits of the i-th node of the path to accepted_node[b], the root being the 0th, where parent is given: what a verification's
 *   out_tokens[b,i] was put out from.  Behind the path, and where accepted_node[b] is -1, there is no row.
 * With y = z / temperature:  logprob = y_token - log sum exp y;  entropy = -sum p log p, in nats;  top: the `top` largest by (logit, lower index
 * first), and their log probabilities.  A token of -1 is none: its logprob is 0.  Where there is no row, logprob, entropy and top_logprobs
 * are 0 and top_tokens -1.
 * A row with NaN or +inf, or only -inf: SPEC_DEV_NONFINITE, its values NaN and top_tokens -1.  A token outside [-1,V): SPEC_DEV_TOKEN and a
 * logprob of NaN.  accepted_node outside [-1,N) or a bad parent on its path: SPEC_DEV_TOPOLOGY, as without a row.
 * Exponentials and sums of up to a few hundred entries in fp32, everything above in fp64; the entropy is off by up to 5.5 times an exponential's 2^-22,
 * whatever it is.  One read of the rows, and a second of what comes near the most probable; rows of which hundreds of entries are equal there, or in fp32 and
 * fp16 no further apart than 2^-7 of their size, are read again up to `top` times: the same results in up to 50 times the time.
 */
#define SPEC_MAX_TOP 32
typedef struct {
    int32_t B, N, V, K, top, dtype;   /* K given tokens a row (with parent: 1); top up to SPEC_MAX_TOP and V; SPEC_F32, SPEC_BF16 or SPEC_F16 */
    const void *logits;               /* row of (b, i) at b * seq_stride + i * node_stride; its V entries are contiguous */
    int64_t seq_stride, node_stride;  /* in elements                                                  */
    const int32_t *parent;            /* optional [N], or [B,N] with topo_seq_stride = N              */
    int64_t topo_seq_stride;
    const int32_t *accepted_node;     /* [B], with parent                                             */
    const int32_t *token;             /* [B,N,K]; may be NULL for K = 0                               */
    float temperature;                /* in [1e-30, 1e30]                                             */
    float *logprob;                   /* [B,N,K]                                                      */
    float *entropy;                   /* [B,N]                                                        */
    int32_t *top_tokens;              /* [B,N,top]                                                    */
    float *top_logprobs;              /* [B,N,top]                                                    */
    int32_t *status;                  /* [B,N]                                                        */
} SpecLogprobs;
int32_t spec_token_logprobs(const SpecLogprobs *a, void *stream);

/*
 * Attention weight that entries of the cache get, added up: for every entry j of a request (committed tokens, then the tree's nodes)
 *   weights[slot of j] += sum over nodes i that see j, and query heads h, of exp(scale q[b,i,h] . k_j - lse[b,i,h]),
 * with lse from spec_tree_attention (or spec_prefix_attention) without a window.  Entries below protected[b] (tokens that are never evicted: a shared
 * prefix, the first few) are left out: neither their keys nor their weights are touched.  fresh != 0: the tree's entries count from 0,
 * whatever their slots held (the first layer of a step).  A row whose lse is not finite adds nothing, and nothing of its query matters.
 * Sums in fp32 in a fixed order: the same inputs give the same bits.  A key on a bad block is left out (SPEC_DEV_PAGE); a bad tree leaves
 * the request's weights as they were (SPEC_DEV_TOPOLOGY).  The blocks behind protected[b] must be the request's own.
 * What is no number (a score of NaN) adds nothing.  SPEC_DEV_TIMEOUT (a wait ran out, in any request's part of the work): the weights
 * of the call's requests are undefined.  `ws`: spec_cache_weights_workspace_bytes() bytes (contents do not matter).
 * D: 64, 128 or 256; q and cache SPEC_BF16 or SPEC_F16; strides in elements, multiples of 8, bases on 16 bytes.
 */
typedef struct {
    int32_t B, N, Hq, Hkv, D, dtype;
    int32_t num_blocks, block_size, table_width;
    int32_t fresh;
    float scale;                      /* >= 0, finite                                                 */
    const void *q;
    int64_t q_stride[3];              /* request, node, head                                          */
    const void *k_cache;
    int64_t k_cache_stride[3];        /* block, slot, head                                            */
    const float *lse;                 /* [B,N,Hq]                                                     */
    const int32_t *block_table;
    int64_t table_stride;
    const int32_t *lengths;           /* [B]                                                          */
    const int32_t *n_nodes;           /* optional [B]                                                 */
    const int32_t *parent;            /* [N], or [B,N] with topo_seq_stride = N                       */
    int64_t topo_seq_stride;
    const int32_t *protected_len;     /* optional [B]                                                 */
    float *weights;                   /* [num_blocks, block_size]                                     */
    int32_t *status;                  /* [B]                                                          */
} SpecWeights;
int32_t spec_cache_weights_workspace_bytes(const SpecWeights *a, int64_t *bytes);
int32_t spec_cache_weights(const SpecWeights *a, void *ws, int64_t ws_bytes, void *stream);

/*
 * Eviction: a request with more than `budget` committed tokens keeps `budget` entries: its first p = protected[b], its last
 * min(recent, budget - p), and of those between the ones with the largest weights (NaN below everything; of equal ones the lower entry).
 * They move together in order, in every cache and in weights; entries from `budget` on keep what they held.  lengths_out[b] = budget.
 * Blocks behind the shortened request go back to the ring behind the free ones, request by request: owned_out[b] = ceil(budget / block_size).
 * block_table stays as it is (its columns from owned_out[b] on are no longer the request's); owned and free_range are inputs and stay too.
 * Requests of at most `budget` tokens stay as they are, blocks included.
 * protected[b] > budget, or a negative one: SPEC_DEV_TOPOLOGY; a bad block id in the owned columns, or fewer of them than
 * the tokens need, or more tokens than the cache has slots or than 2^31 - 65537: SPEC_DEV_PAGE; then nothing of the request moves.  A ring without room for a request's blocks (or a free_range
 * outside it): SPEC_DEV_BLOCKS, the request is shortened but keeps its blocks.  Blocks that hold entries behind protected[b] must be the request's own.
 * No tree is under way: entries behind the committed tokens are not kept.
 * What lies behind the first entry that goes moves, in all caches, however few go: 16 requests of 4096 entries and 1, 4 or 16 more, 16 caches of 1 KB a row, take
 * 290, 420 and 490 us, of 8192 entries 500.  A loop that cuts now and then, to a budget so much lower, moves them less often.
 * `ws`: spec_cache_evict_workspace_bytes() bytes.
 */
typedef struct {
    int32_t B, caches, budget, recent;
    int32_t num_blocks, block_size, table_width;
    void *cache;                      /* row of slot e of block k of cache c: c * stride[0] + k * stride[1] + e * stride[2] bytes */
    int64_t stride[3];
    int64_t row_bytes;                /* below 2^31                                                   */
    float *weights;                   /* [num_blocks, block_size]                                     */
    const int32_t *block_table;
    int64_t table_stride;
    const int32_t *lengths;           /* [B]                                                          */
    const int32_t *owned;             /* [B]                                                          */
    const int32_t *protected_len;     /* optional [B]                                                 */
    int32_t *free_blocks;             /* [free_size]; entries behind the free ones are written        */
    int32_t free_size;
    const int32_t *free_range;        /* [2]                                                          */
    int32_t *lengths_out;             /* [B]                                                          */
    int32_t *owned_out;               /* [B]                                                          */
    int32_t *free_range_out;          /* [2]                                                          */
    int32_t *status;                  /* [B]                                                          */
} SpecEvict;
int32_t spec_cache_evict_workspace_bytes(const SpecEvict *a, int64_t *bytes);
int32_t spec_cache_evict(const SpecEvict *a, void *ws, int64_t ws_bytes, void *stream);

/* Launch plan of SpecInfer's walk for a vocabulary size and dtype, of a batch under top-k that fills the
 * device several times over (host-only query, for benchmarks and tests; smaller batches and batches
 * without top-k run the walk with one CTA per SM more often): CTAs per cluster, tokens per CTA slice,
 * dynamic shared memory bytes per CTA, threads per CTA. */
int32_t spec_query_plan(int32_t V, int32_t logits_dtype, int32_t *cluster_size, int32_t *slice_len,
                        int32_t *smem_bytes, int32_t *threads);

/* Number of kernels this library has enqueued in the calling process so far (host-only counter, for
 * benchmarks that report how many launches a timed region made).  Never fails. */
int64_t spec_kernel_launches(void);

/*
 * Test hooks (no counterpart in the paper; not for production callers).  Every wait inside the kernels
 * is bounded (Section "General rules": a wait that runs out is reported as SPEC_DEV_TIMEOUT, nothing
 * hangs); these two settings let a test watch that happen.  wait_cycles: the limit of every on-device
 * wait in clock cycles (<= 0: the default, about 2 s).  hold_slot: index b * N + node of one node whose
 * Traversal weight the node kernels then never publish, so that the node's own wait runs out, and whose
 * sequence's queries the tree attention and spec_cache_weights then never fetch, so that their waits for them do
 * (-1: none).  Synchronous (copies to constant memory of the current device); call it between
 * verification calls, never while one is in flight.
 */
int32_t spec_test_hooks(int64_t wait_cycles, int32_t hold_slot);

#ifdef __cplusplus
}
#endif
#endif /* SPECVERIFY_H */
