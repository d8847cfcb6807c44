/*
 * ltd_verify: the tree-verification step of Learning-to-Draft speculative
 * decoding (arXiv 2603.01639, section 3.2) on AMD Instinct MI355X (gfx950).
 *
 * One verification step of a draft-and-verify cycle is three calls on one
 * stream, with no host synchronisation between them:
 *
 *   ltd_tree_verify_attn  the target model's attention over its KV-cache prefix
 *                         plus the N flattened draft-tree candidates, each
 *                         candidate seeing only the prefix and its own ancestors
 *                         (the tree attention mask of section 3.2, "Candidate
 *                         Token Selection" / "Draft Tree Verification");
 *   ltd_tree_accept       the target's prediction at every node (vocabulary
 *                         argmax of its logits) and greedy acceptance: the
 *                         longest root path whose draft tokens all equal the
 *                         prediction at their parent, plus the target's token at
 *                         the first mismatch (section 3.2, "Draft Tree
 *                         Verification");
 *   ltd_kv_compact        the accepted path's K/V rows move next to the prefix
 *                         and the rest of the candidates are discarded (same
 *                         paragraph: the remainder after the first error is
 *                         dropped).
 *
 * The steps before it have calls of their own:
 *
 *   ltd_draft_expand      one round of the draft tree's beam expansion
 *                         (section 3.2, "Draft Tree Generation");
 *   ltd_policy_forward    the size and depth policies' decisions (section 4,
 *                         appendix A.2);
 *   ltd_select_candidates the V most probable candidates of the draft tree's
 *                         pool, flattened into the tree the three calls above
 *                         verify (section 3.2, "Candidate Token Selection").
 *
 * A KV cache held in 8 bits has the same cycle with calls of its own
 * (ltd_kv_append_q8, ltd_tree_verify_attn_q8, ltd_kv_compact_q8), and a
 * request's sampling rules (penalties, biases, a grammar's mask) stand between
 * the target's logits and acceptance (ltd_token_counts,
 * ltd_tree_process_logits, ltd_tree_accept_processed).
 *
 * Queries and keys get their rotary positions from ltd_tree_rope.  A model with
 * latent attention keeps one vector a token, which all heads share, and has the
 * cycle's calls for that cache (ltd_latent_append, ltd_tree_verify_attn_latent,
 * ltd_latent_compact).
 *
 * Conventions for every call
 * --------------------------
 * - All array pointers are DEVICE pointers, owned by the caller.  The library
 *   never allocates, frees or synchronises; every call is asynchronous on
 *   `stream` (a hipStream_t passed as void*, NULL = the default stream).
 * - Return value: LTD_OK, or a negative LTD_E* code when the call itself is
 *   malformed (nothing is launched then).  These checks use only the scalar
 *   arguments and the pointers themselves (null, aligned, apart where a call says so).
 * - Data-dependent checks (tree shape, prefix bounds, block ids, paths) run on
 *   the device only when `validate != 0`: a validation kernel writes an
 *   LTD_STATUS_* code to `*status` (0 when the data is well formed) and, when
 *   it is nonzero, the step's kernels write nothing.  The code reported is the
 *   one of the lowest failing sequence index, with checks in the order the
 *   codes are numbered.  With `validate == 0`, malformed data is undefined
 *   behaviour and `status` may be NULL.
 * - Trees: N counts the root.  parents[b][0] = -1 and 0 <= parents[b][i] < i
 *   (a topological order); node 0 is the root (the previous cycle's bonus
 *   token).  Tree node i of sequence b sits at logical cache row P_b + i.
 * - Calls on different streams that touch the same buffers race; calls that
 *   share a workspace must be stream-ordered.
 */
#ifndef LTD_VERIFY_H
#define LTD_VERIFY_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define LTD_OK 0
#define LTD_EINVAL (-1)       /* null pointer or out-of-range scalar argument */
#define LTD_EUNSUPPORTED (-2) /* dtype or head_dim the kernels do not implement */
#define LTD_EWORKSPACE (-3)   /* workspace missing or smaller than the query says */
#define LTD_EHIP (-4)         /* a HIP runtime call or kernel launch failed */

#define LTD_DTYPE_F32 0  /* IEEE binary32 */
#define LTD_DTYPE_BF16 1 /* bfloat16 */

#define LTD_STATUS_OK 0
#define LTD_STATUS_BAD_NNODES 1 /* n_nodes[b] outside [1, Nmax] */
#define LTD_STATUS_BAD_PARENT 2 /* parents[b][0] != -1 or parents[b][i] outside [0, i) */
#define LTD_STATUS_BAD_PREFIX 3 /* prefix_len[b] < 0, > max_prefix, or rows past capacity */
#define LTD_STATUS_BAD_BLOCK 4  /* a block id the sequence uses is outside [0, num_blocks) */
#define LTD_STATUS_BAD_PATH 5   /* accepted path not 0 = p_0 < p_1 < ..., or n_accepted out of range */
#define LTD_STATUS_BAD_SCORE 6  /* a pool score is NaN or above its parent's */
#define LTD_STATUS_BAD_RULE 7   /* a penalty is not finite, a repetition penalty <= 0, or n_bias out of range */

#define LTD_MAX_NODES 256 /* largest Nmax (the paper's size policy spans V in [20, 240]) */
#define LTD_MAX_POOL 1024 /* largest draft pool (1 + W + (D-2) W^2 = 1011 at W = 10, D = 12) */

#define LTD_SAMPLING_MAX_CHUNKS 64  /* sampling vocabulary up to 64 * 4096 = 262144 entries */

#define LTD_EXPAND_MAX_W 16          /* children per frontier node (the paper's W is 10) */
#define LTD_EXPAND_MAX_CHUNKS 64     /* vocabulary up to 64 * 4096 = 262144 entries */
#define LTD_EXPAND_MAX_CHILDREN 256  /* F * W per round */

#define LTD_MAX_BIAS 1024            /* biased tokens per sequence */
#define LTD_MAX_LENGTH (1 << 30)     /* rows, tokens and vocabulary of the 8-bit cache's and the rules' calls, positions */

#define LTD_ROPE_MAX_DIM 4096 /* head size of ltd_tree_rope */
#define LTD_LATENT_ROPE 64    /* rotated dims of a latent cache's rows */
#define LTD_LATENT_MAX_HEADS 65536

#define LTD_POLICY_SIZE 0          /* state [D, L, score of every pool candidate, pad ...] */
#define LTD_POLICY_DEPTH 1         /* state [scores of the newest in_dim-2 candidates, D, L] */
#define LTD_POLICY_MAX_IN 1024     /* state width (the size policy's is 2 + 1011) */
#define LTD_POLICY_MAX_HIDDEN 1024 /* hidden width (the paper's widest layer) */
#define LTD_POLICY_MAX_OUT 64      /* output logits (12 size actions, 2 depth actions) */

/*
 * Tree attention (section 3.2: candidates flattened with a tree attention
 * mask, verified in one target pass).
 *
 * For every sequence b, node i < n_nodes[b] and query head h (kv head
 * g = h / (Hq / Hkv)):
 *     out[b][i][h] = softmax_t(scale * <q[b][i][h], K[b][g][t]>) . V[b][g][t]
 * over the visible rows t = {0, ..., P_b - 1} u {P_b + j : j on the root path of
 * node i, i included}.  Accumulation is fp32; out has the input dtype.  On
 * the bf16 path the exponent of each weight is formed in fp32 as
 * s*c - m*c (c = scale * log2(e), m a running row maximum), exact to about
 * |m*c| * 2^-24: scaled scores up to ~1e5 in magnitude keep the bf16 output
 * accuracy (max-abs error ~1e-2 against exact arithmetic).
 *
 *   q           [B][Nmax][Hq][d] (dtype): the tree nodes' queries (position
 *               encoding already applied by the caller).
 *   k_cache,    contiguous (block_table == NULL): [B][Hkv][kv_rows][d], kv_rows
 *   v_cache     = capacity per sequence;
 *               paged: [num_blocks][Hkv][kv_rows][d], kv_rows = block size,
 *               logical row r of sequence b in block block_table[b][r / kv_rows].
 *               The tree's own K/V rows must already be written at P_b .. P_b+n-1.
 *   block_table [B][max_blocks] int32 or NULL.
 *   prefix_len  [B] int32, P_b >= 0.  max_prefix >= every P_b (host bound used
 *               to size the launch; checked on the device when validate != 0).
 *   parents     [B][Nmax] int32, n_nodes [B] int32 in [1, Nmax].
 *   out         [B][Nmax][Hq][d] (dtype); rows i >= n_nodes[b] are not written.
 *   Hq % Hkv == 0, d in {64, 128}, 1 <= Nmax <= LTD_MAX_NODES.
 *   scale       softmax scale, finite and > 0 (1/sqrt(d) for standard
 *               attention); anything else is LTD_EINVAL.
 *   workspace   device scratch of at least ltd_tree_verify_attn_workspace_size()
 *               bytes for the same (B, Nmax, Hq, Hkv, d, max_prefix, dtype) (that
 *               size covers every cache layout; it is 0 on the fp32 path,
 *               and workspace may then be NULL); it holds the partial results
 *               of units cut between workgroups, needs no initialisation and
 *               is garbage afterwards.
 */
size_t ltd_tree_verify_attn_workspace_size(int B, int Nmax, int Hq, int Hkv, int d, int max_prefix,
                                           int dtype);

int ltd_tree_verify_attn(const void* q, const void* k_cache, const void* v_cache,
                         const int32_t* block_table, const int32_t* prefix_len,
                         const int32_t* parents, const int32_t* n_nodes, void* out, int B, int Nmax,
                         int Hq, int Hkv, int d, int max_prefix, int kv_rows, int max_blocks,
                         int num_blocks, float scale, int dtype, void* workspace,
                         size_t workspace_bytes, int validate, int32_t* status, void* stream);

/*
 * Greedy acceptance (section 3.2, "Draft Tree Verification").
 *
 *   logits        [B][Nmax][Voc] fp32: the target's logits at every node.
 *   draft_tokens  [B][Nmax] int32; draft_tokens[b][0] is the root token.
 *   parents, n_nodes as for attention.
 * Outputs (entries past n_nodes[b] / n_accepted[b] are not written):
 *   pred           [B][Nmax] int32: argmax_v logits[b][i][v]; ties go to the
 *                  lowest v and -0.0 equals +0.0 (NaN logits are undefined).
 *   accepted_nodes [B][Nmax] int32: the accepted root path, root first
 *                  (accepted_nodes[b][0] = 0).  Node c is accepted when its
 *                  parent is and draft_tokens[b][c] == pred[b][parent(c)]; the
 *                  path ends at the deepest accepted node, the smallest index
 *                  among equally deep ones.
 *   out_tokens     [B][Nmax] int32: draft tokens of the accepted non-root path
 *                  nodes, then the bonus token pred[b][leaf].
 *   n_accepted     [B] int32: path length = number of emitted tokens (L_A).
 *   workspace      at least ltd_tree_accept_workspace_size(B, Nmax, Voc) bytes.
 */
size_t ltd_tree_accept_workspace_size(int B, int Nmax, int Voc);

int ltd_tree_accept(const float* logits, const int32_t* draft_tokens, const int32_t* parents,
                    const int32_t* n_nodes, int B, int Nmax, int Voc, int32_t* pred,
                    int32_t* accepted_nodes, int32_t* out_tokens, int32_t* n_accepted,
                    void* workspace, size_t workspace_bytes, int validate, int32_t* status,
                    void* stream);

/*
 * Greedy acceptance without a workspace, for callers that cannot allocate
 * device memory (code under HIP graph capture, tight serving loops, harnesses
 * that forbid hipMalloc).  Same arguments, results and validation as
 * ltd_tree_accept, minus the workspace: the argmax partials go to a scratch
 * array that the library holds on each GPU for the life of the process
 * (ltd_tree_accept_noalloc_max_bytes() bytes, 4 MiB).  The call allocates
 * nothing and frees nothing.
 *
 * Limits: ltd_tree_accept_workspace_size(B, Nmax, Voc) must not exceed
 * ltd_tree_accept_noalloc_max_bytes() (B * Nmax * ceil(Voc / 16384) * 8 bytes;
 * e.g. B = 16, Nmax = 256 and Voc = 262144 use 1 MiB), else LTD_EWORKSPACE and
 * nothing is launched.  LTD_EHIP if the scratch's device address cannot be
 * looked up on the current GPU.
 * Every call on one GPU shares that GPU's scratch and keeps the last call's
 * contents there (no call depends on them): calls that overlap on one GPU
 * (different streams without ordering between them) race and give undefined
 * results.
 */
size_t ltd_tree_accept_noalloc_max_bytes(void);

int ltd_tree_accept_noalloc(const float* logits, const int32_t* draft_tokens,
                            const int32_t* parents, const int32_t* n_nodes, int B, int Nmax,
                            int Voc, int32_t* pred, int32_t* accepted_nodes, int32_t* out_tokens,
                            int32_t* n_accepted, int validate, int32_t* status, void* stream);

/*
 * Acceptance at temperature T > 0 (the paper's T = 1 setting; its rule is
 * the baseline's, not printed in the paper): recursive rejection sampling
 * over each node's children, which must have been drawn without replacement
 * from the node's draft distribution, in ascending node order.
 *
 * At node u, with target P = softmax(logits[u] / T) and draft distribution
 * Q = draft_probs[u] / sum(draft_probs[u]), child c (token x) is accepted
 * when uniforms[c][0] * Q(x) < P(x), i.e. with probability min(1, P/Q), and
 * the walk moves to c.  On rejection P becomes max(P - Q, 0) renormalised and
 * Q drops x.  When no child is accepted (or u is a leaf) the bonus token is
 * the inverse-CDF sample of P at uniforms[u][1].  The emitted tokens are then
 * distributed exactly as the target's own sampling.
 *
 *   logits       [B][Nmax][Voc] float32, target logits at every node.
 *   draft_probs  [B][Nmax][Voc] float32, read only for nodes with children
 *                (non-negative, positive sum).
 *   draft_tokens [B][Nmax] int32 in [0, Voc); siblings distinct.
 *   uniforms     [B][Nmax][2] float32 in [0, 1).
 *   temperature  finite and > 0, else LTD_EINVAL.
 *   Outputs as ltd_tree_accept: accepted_nodes, out_tokens (the accepted
 *   drafts, then the bonus), n_accepted.  Entries past n_accepted untouched.
 *   Voc <= 4096 * LTD_SAMPLING_MAX_CHUNKS.
 *   workspace: ltd_tree_accept_sampling_workspace_size(B, Nmax, Voc) bytes.
 * Decisions are taken on float32 element arithmetic with double sums, so they
 * can differ from an exact evaluation only where a uniform lies within about
 * 1e-6 (relative) of its threshold.  The draft mass left after each rejection
 * is summed over the tokens not rejected, so it stays exact to double
 * rounding however little of it is left.
 */
size_t ltd_tree_accept_sampling_workspace_size(int B, int Nmax, int Voc);

int ltd_tree_accept_sampling(const float* logits, const float* draft_probs,
                             const int32_t* draft_tokens, const int32_t* parents,
                             const int32_t* n_nodes, const float* uniforms, int B, int Nmax,
                             int Voc, float temperature, int32_t* accepted_nodes,
                             int32_t* out_tokens, int32_t* n_accepted, void* workspace,
                             size_t workspace_bytes, int validate, int32_t* status, void* stream);

/*
 * KV compaction (the candidates after the first mismatch are discarded,
 * section 3.2, "Draft Tree Verification").
 *
 * For every sequence b, layer l < num_layers and kv head: logical row
 * P_b + accepted_nodes[b][j] moves to row P_b + j for j < n_accepted[b], all
 * reads before the writes they could overlap; then
 * new_prefix_len[b] = P_b + n_accepted[b].  Rows >= P_b + n_accepted[b] keep
 * whatever they held.  K and V of layer l start layer_stride_elems elements
 * after layer l-1; each layer has the attention call's layout.
 *
 *   k_cache, v_cache  device caches (modified in place).
 *   prefix_len        [B] int32 (read); new_prefix_len [B] int32 (written;
 *                     must not alias prefix_len).
 *   accepted_nodes    [B][Nmax], n_accepted [B]: as written by ltd_tree_accept.
 *   d * element size must be a multiple of 16 bytes.
 */
int ltd_kv_compact(void* k_cache, void* v_cache, const int32_t* block_table,
                   const int32_t* prefix_len, int32_t* new_prefix_len,
                   const int32_t* accepted_nodes, const int32_t* n_accepted, int B, int Nmax,
                   int Hkv, int d, int kv_rows, int max_blocks, int num_blocks, int num_layers,
                   int64_t layer_stride_elems, int dtype, int validate, int32_t* status,
                   void* stream);

/* Workgroups of the attention launch for a shape and cache layout
 * (kv_rows = capacity or block size, paged != 0 for a block table).  A bf16
 * call (head_dim 128 or 64) runs on the matrix-core kernels: a batch lays all
 * its (sequence, kv head, row tile) units' key tiles end to end and gives each
 * of that many workgroups (a power of two) an equal share; a single sequence
 * cuts each unit into KV splits.  Units cut between workgroups are merged by a
 * second kernel.  0 when the call runs on the fp32 vector kernel instead,
 * -1 on bad args.
 * Introspection for tests and benchmarks. */
int ltd_tree_verify_attn_grid(int B, int Nmax, int Hq, int Hkv, int d, int max_prefix, int dtype,
                              int kv_rows, int paged);

/*
 * Candidate token selection (section 3.2, "Candidate Token Selection"): of a
 * draft tree's candidate pool, keep the V = min(n_select[b], pool_size[b])
 * candidates with the highest cumulative path score and flatten them into a
 * tree in the form the verification calls take.
 *
 * Ranking: score descending; equal scores (-0.0 equals +0.0) rank the lower
 * pool index first.  Since the pool lists a parent before its children and a
 * child never scores above its parent, the kept candidates form a rooted
 * subtree.  They are flattened in pool order, so every parent precedes its
 * children (and a pool listed level by level comes out depth-major).
 *
 *   scores        [B][Vpool] float32: cumulative log-probability of each
 *                 candidate (any order-preserving image of its path
 *                 probability); never above its parent's, never NaN.
 *   pool_parents  [B][Vpool] int32: pool_parents[b][0] = -1 (the root) and
 *                 0 <= pool_parents[b][i] < i.
 *   pool_tokens   [B][Vpool] int32: the candidate tokens (copied, not read).
 *   pool_size     [B] int32 in [1, Vpool]; columns past it are never read.
 *   n_select      [B] int32 in [1, Nmax]: the verification size asked for
 *                 (the size policy's action).
 *   Vpool         1 <= Vpool <= LTD_MAX_POOL; 1 <= Nmax <= LTD_MAX_NODES.
 *   Outputs [B][Nmax] int32, rows k < V written, the rest untouched:
 *   selected      pool index of flattened node k (may be NULL);
 *   parents       parent of node k in the flattened order (-1 for the root);
 *                 the tree the verification calls take;
 *   tokens        token of node k (the verification's draft tokens);
 *   depth         depth of node k (the root is 0; may be NULL, which saves
 *                 the pass that computes it);
 *   n_nodes       [B] int32: V.
 * With validate != 0, malformed data is reported as LTD_STATUS_BAD_NNODES
 * (pool_size or n_select out of range), LTD_STATUS_BAD_PARENT or
 * LTD_STATUS_BAD_SCORE, and then nothing is written.  No workspace.
 */
int ltd_select_candidates(const float* scores, const int32_t* pool_parents,
                          const int32_t* pool_tokens, const int32_t* pool_size,
                          const int32_t* n_select, int B, int Vpool, int Nmax, int32_t* selected,
                          int32_t* parents, int32_t* tokens, int32_t* depth, int32_t* n_nodes,
                          int validate, int32_t* status, void* stream);

/*
 * One round of draft tree expansion (section 3.2, "Draft Tree Generation":
 * each leaf gets the W most probable tokens of its draft distribution as
 * children; the W children of highest cumulative path probability become the
 * next leaves).  The draft model's logits at the F frontier nodes are the
 * input; the children are appended to the candidate pool that
 * ltd_select_candidates and the policies read.
 *
 *   logits        [B][F][Voc] float32: draft logits at frontier node f.
 *   frontier      [B][F] int32: the frontier nodes' pool indices.
 *   scores, pool_parents, pool_tokens  [B][Vpool]: the pool, appended to.
 *   pool_size     [B] int32: read, then advanced by F*W.
 *   new_frontier  [B][W_next] int32: the next frontier (pool indices).
 * For frontier node f, in order, its children are the W tokens of largest
 * logit (equal logits: lower token index first), stored at pool_size + f*W
 * + r with parent frontier[f] and score = parent's score + log-softmax of the
 * logit (float32; the log-sum-exp is accumulated in double).  new_frontier
 * is the W_next new children of highest score, best first (equal scores:
 * lower pool index first).  A first round from the root has F = 1; after
 * D - 1 rounds of width W the pool holds 1 + W + (D-2) W^2 candidates.
 * Limits: 1 <= W <= LTD_EXPAND_MAX_W, W <= Voc <= 4096 * LTD_EXPAND_MAX_CHUNKS,
 * 1 <= F*W <= LTD_EXPAND_MAX_CHILDREN, 1 <= W_next <= F*W.
 * workspace: ltd_draft_expand_workspace_size(B, F, Voc, W) bytes.
 * With validate != 0: LTD_STATUS_BAD_NNODES if pool_size[b] < 1 or the
 * children would pass Vpool, LTD_STATUS_BAD_PARENT if a frontier index is
 * not in the pool; then nothing is written.
 */
size_t ltd_draft_expand_workspace_size(int B, int F, int Voc, int W);

int ltd_draft_expand(const float* logits, const int32_t* frontier, int B, int F, int Voc, int W,
                     int W_next, float* scores, int32_t* pool_parents, int32_t* pool_tokens,
                     int32_t* pool_size, int Vpool, int32_t* new_frontier, void* workspace,
                     size_t workspace_bytes, int validate, int32_t* status, void* stream);

/*
 * Draft-policy inference (section 4: the state vector of draft depth D,
 * context length L and candidate scores; appendix A.2: the size and depth
 * policies are fully connected ReLU networks with hidden widths [1024, 256]
 * and [1024], 12 and 2 actions, the action being the most likely one).
 *
 * The state of sequence b is built from its draft pool (no separate pass):
 *   LTD_POLICY_SIZE   [D_b, L_b, scores[b][0 .. min(n_b, F)), pad ...]
 *   LTD_POLICY_DEPTH  [pad ..., scores[b][n_b - F .. n_b), D_b, L_b]
 * with n_b = pool_size[b] and F = in_dim - 2 (the depth layout takes the last
 * F candidates, i.e. the newest expansion once the pool holds W^2 of them).
 * Then h1 = relu(w1 s + b1), optionally h2 = relu(w2 h1 + b2) (h2 > 0), and
 * logits = wo h + bo; action[b] = action_offset + action_scale * argmax
 * (lowest index on ties), so the size policy's V = 20 + 20 a can be written
 * straight into ltd_select_candidates' n_select.
 *
 *   scores [B][Vpool] float32, pool_size/depth/ctx_len [B] int32 (read).
 *   w1 [h1][in_dim], b1 [h1]; w2 [h2][h1], b2 [h2] (NULL when h2 = 0);
 *   wo [n_out][h2 or h1], bo [n_out]: float32, row-major (a row per unit).
 *   logits [B][n_out] float32, action [B] int32 (written).
 *   workspace: ltd_policy_workspace_size(B, h1, h2) bytes (hidden activations).
 * Limits: 3 <= in_dim <= LTD_POLICY_MAX_IN, 1 <= h1 <= LTD_POLICY_MAX_HIDDEN,
 * 0 <= h2 <= LTD_POLICY_MAX_HIDDEN, 1 <= n_out <= LTD_POLICY_MAX_OUT;
 * anything else, or a bad layout, is LTD_EINVAL.  Accumulation is float32 in
 * a fixed order (deterministic).
 */
size_t ltd_policy_workspace_size(int B, int h1, int h2);

int ltd_policy_forward(int layout, const float* scores, const int32_t* pool_size, int Vpool,
                       const int32_t* depth, const int32_t* ctx_len, float pad, int B, int in_dim,
                       const float* w1, const float* b1, int h1, const float* w2, const float* b2,
                       int h2, const float* wo, const float* bo, int n_out, int action_offset,
                       int action_scale, float* logits, int32_t* action, void* workspace,
                       size_t workspace_bytes, void* stream);

/*
 * The 8-bit KV cache.
 *
 * K and V rows are stored as OCP e4m3 codes (4 exponent and 3 fraction bits,
 * largest value 448, no infinity, one NaN code), one byte per element, in the
 * layouts of the attention call:
 *   codes   contiguous [B][Hkv][kv_rows][d], paged [num_blocks][Hkv][kv_rows][d];
 *   scales  [B or num_blocks][Hkv][ceil(kv_rows / scale_rows)] bytes, for K and
 *           V apart: row r of a cache (row r of its block when paged) and head g
 *           shares byte r / scale_rows with its neighbours.  A byte E stands for
 *           the power of two 2^(E - 127), and a code c for c * 2^(E - 127).
 * Powers of two keep all of a code's fraction bits: a value is exact in
 * bfloat16 and float32, and a block whose scale grows loses bits only where a
 * code falls below the format's normal range.
 *   scale_rows  16, 32, 64 or 128; a paged cache's kv_rows is a multiple of it.
 *   d           64 or 128.
 * Anything else is LTD_EUNSUPPORTED, as are more than LTD_MAX_LENGTH rows to
 * append or max_prefix; logical rows end at LTD_MAX_LENGTH too, whatever the
 * capacity.  Codes and rows passed to these calls are 16-byte aligned
 * (LTD_EINVAL otherwise).  Scale bytes of rows in use lie in
 * [27, 214], as ltd_kv_append_q8 writes them: values of up to 2^96, so that
 * float32 sums of them under softmax weights stay finite.
 */

/*
 * Appends rows to an 8-bit KV cache: a prompt's, or a draft tree's before its
 * verification.
 *
 * For every sequence b, kv head g and K and V apart, rows i < n_rows[b] of the
 * input become logical rows P_b + i of the cache (P_b = prefix_len[b]).  A
 * block of scale_rows rows that receives rows takes the smallest scale byte in
 * [27, 214] under which the block's new values are at most 448 in magnitude; if
 * it also holds rows below P_b, its scale is not lowered, and when it grows
 * those rows are encoded again.  Codes are rounded to nearest even.  NaN is
 * stored as NaN and has no part in the scale; infinities, and values above
 * 448 * 2^87, are stored as the largest code.  Other rows keep their bytes,
 * but rows past P_b + n_rows[b] in a block that receives rows stand for
 * undefined values afterwards (their scale may have changed).
 *
 *   k_new, v_new  [B][Nmax][Hkv][d] (dtype), with new_row_stride elements from
 *                 one row to the next (at least Hkv * d; rows may be views into
 *                 a fused projection's output); row i of sequence b starts at
 *                 (b * Nmax + i) * new_row_stride.  Each row is 16-byte aligned.
 *   n_rows        [B] int32 in [0, Nmax]; Nmax may exceed LTD_MAX_NODES here.
 *   prefix_len    [B] int32 (read only).
 * No two sequences may append to the same block.  With validate != 0:
 * LTD_STATUS_BAD_NNODES (n_rows), LTD_STATUS_BAD_PREFIX (P_b < 0, or rows past
 * the capacity or LTD_MAX_LENGTH) and LTD_STATUS_BAD_BLOCK (ids of the blocks that are written).
 */
int ltd_kv_append_q8(const void* k_new, const void* v_new, int64_t new_row_stride, void* k_cache,
                     void* v_cache, uint8_t* k_scale, uint8_t* v_scale, const int32_t* block_table,
                     const int32_t* prefix_len, const int32_t* n_rows, int B, int Nmax, int Hkv,
                     int d, int kv_rows, int max_blocks, int num_blocks, int scale_rows, int dtype,
                     int validate, int32_t* status, void* stream);

/*
 * Tree attention over an 8-bit KV cache: ltd_tree_verify_attn with K and V the
 * values their codes and scales stand for.  dtype is that of q and out.  The
 * other arguments, limits and results are that call's; the workspace is sized by
 * ltd_tree_verify_attn_q8_workspace_size().  A NaN code in a tree row reaches
 * the outputs of the nodes that see the row, and no others: a NaN in a visible
 * row's V may make every dimension of those outputs NaN.
 * With bfloat16, values below 2^-29 of the largest of an output row's dimensions
 * may be off by 2^-39 of that largest.
 */
size_t ltd_tree_verify_attn_q8_workspace_size(int B, int Nmax, int Hq, int Hkv, int d,
                                              int max_prefix, int dtype);

int ltd_tree_verify_attn_q8(const void* q, const void* k_cache, const void* v_cache,
                            const uint8_t* k_scale, const uint8_t* v_scale,
                            const int32_t* block_table, const int32_t* prefix_len,
                            const int32_t* parents, const int32_t* n_nodes, void* out, int B,
                            int Nmax, int Hq, int Hkv, int d, int max_prefix, int kv_rows,
                            int max_blocks, int num_blocks, int scale_rows, float scale, int dtype,
                            void* workspace, size_t workspace_bytes, int validate, int32_t* status,
                            void* stream);

/*
 * Compaction of an 8-bit KV cache: ltd_kv_compact on codes and scales.
 *
 * Rows move as there.  A block that receives rows (or keeps accepted ones)
 * takes the largest of their scale bytes, and its own if it holds rows below
 * P_b; every row of it below P_b + n_accepted[b] whose scale byte was smaller is
 * encoded again (rounded to nearest even), others keep their codes.  Rows >=
 * P_b + n_accepted[b] stand for undefined values afterwards.  No two sequences
 * may have the same block in rows >= P_b.
 *   layer_stride_elems  codes from one layer to the next (K and V);
 *   scale_stride_elems  scale bytes from one layer to the next; both > 0 with
 *                       more than one layer.
 */
int ltd_kv_compact_q8(void* k_cache, void* v_cache, uint8_t* k_scale, uint8_t* v_scale,
                      const int32_t* block_table, const int32_t* prefix_len,
                      int32_t* new_prefix_len, const int32_t* accepted_nodes,
                      const int32_t* n_accepted, int B, int Nmax, int Hkv, int d, int kv_rows,
                      int max_blocks, int num_blocks, int scale_rows, int num_layers,
                      int64_t layer_stride_elems, int64_t scale_stride_elems, int validate,
                      int32_t* status, void* stream);

/*
 * The table of token occurrences that penalties read, kept by the caller from
 * one cycle to the next.
 *
 *   counts    [B][Voc] int32: bits 0 .. 30 count how often the token was
 *             emitted, bit 31 is set when it occurs in the prompt.
 *   tokens    [B][T] int32, the first n_tokens[b] of row b are taken
 *             (n_tokens[b] is clamped into [0, T]; tokens outside [0, Voc) are
 *             skipped).  prompt == 0: each occurrence adds one to its count (the
 *             out_tokens and n_accepted of an acceptance call); prompt != 0: sets
 *             bit 31.
 *   reset     != 0: the table is zeroed first (a new request).
 * T and Voc are at most LTD_MAX_LENGTH (LTD_EUNSUPPORTED).
 */
int ltd_token_counts(const int32_t* tokens, const int32_t* n_tokens, int B, int T, int Voc,
                     int prompt, int reset, int32_t* counts, void* stream);

/*
 * A request's sampling rules on the target's logits, at every tree node.
 *
 * For node i < n_nodes[b] and token v let c be v's emitted count (counts) plus
 * its occurrences among the draft tokens of node i's root path, node i included
 * and the root left out (the root was emitted: counts has it).  With
 * (r, f, p) = penalties[b], x = logits[b][i][v] becomes, in float32 with every
 * step rounded,
 *     x > 0 ? x / r : x * r     if c > 0 or v occurs in the prompt,
 *     x - f * c, then x - p     if c > 0,
 *     x + bias                  if v is in the bias list (entries of one token
 *                               are added to each other in list order first),
 *     -infinity                 if v's bit of the node's mask is 0.
 * Tokens that no rule touches keep their bits.  A node whose mask allows
 * nothing gets -infinity everywhere; acceptance by sampling that ends at such a
 * node has no distribution to draw its bonus token from, and emits any token.
 *
 *   logits, out  [B][Nmax][Voc] float32; out may be logits (in place); any
 *                other overlap is LTD_EINVAL, a Voc above
 *                LTD_MAX_LENGTH LTD_EUNSUPPORTED.  Rows i >= n_nodes[b] are not written.
 *   draft_tokens [B][Nmax]; tokens outside [0, Voc) occur nowhere.
 *   counts       [B][Voc] as kept by ltd_token_counts, or NULL (all zero).
 *   penalties    [B][3] float32: repetition (> 0; 1 = none), frequency and
 *                presence (0 = none), all finite; NULL = none, and counts is then not read.
 *   bias_tokens, bias_values [B][max_bias], n_bias [B] int32 in [0, max_bias]:
 *                the lists; NULL with max_bias == 0 (max_bias <=
 *                LTD_MAX_BIAS).  Tokens outside [0, Voc) are skipped.
 *   mask         [B][Nmax][ceil(Voc / 32)] uint32: bit v % 32 of word v / 32
 *                allows token v; NULL = everything is allowed.
 * With validate != 0: LTD_STATUS_BAD_NNODES, LTD_STATUS_BAD_PARENT and
 * LTD_STATUS_BAD_RULE.
 */
int ltd_tree_process_logits(const float* logits, const int32_t* draft_tokens,
                            const int32_t* parents, const int32_t* n_nodes, const int32_t* counts,
                            const float* penalties, const int32_t* bias_tokens,
                            const float* bias_values, const int32_t* n_bias, const uint32_t* mask,
                            int B, int Nmax, int Voc, int max_bias, float* out, int validate,
                            int32_t* status, void* stream);

/*
 * Greedy acceptance (ltd_tree_accept) on the logits that
 * ltd_tree_process_logits would write, without writing them.  The rules are that
 * call's arguments, the outputs and the workspace
 * (ltd_tree_accept_workspace_size()) ltd_tree_accept's.  A node whose mask
 * allows nothing predicts token 0.
 */
int ltd_tree_accept_processed(const float* logits, const int32_t* draft_tokens,
                              const int32_t* parents, const int32_t* n_nodes,
                              const int32_t* counts, const float* penalties,
                              const int32_t* bias_tokens, const float* bias_values,
                              const int32_t* n_bias, const uint32_t* mask, int B, int Nmax,
                              int Voc, int max_bias, int32_t* pred, int32_t* accepted_nodes,
                              int32_t* out_tokens, int32_t* n_accepted, void* workspace,
                              size_t workspace_bytes, int validate, int32_t* status, void* stream);

/*
 * Rotary positions of queries and keys: a draft tree's, or consecutive tokens'.
 *
 * Row i of sequence b stands at position p = P_b + depth[b][i] (P_b =
 * prefix_len[b]).  In every head the dims [rot_offset, rot_offset + rot_dim) turn:
 * pair j < rot_dim / 2, with values (x0, x1) at dims (rot_offset + j, rot_offset +
 * rot_dim / 2 + j), or (rot_offset + 2j, rot_offset + 2j + 1) when interleaved != 0,
 * becomes
 *     (mscale (x0 cos t - x1 sin t), mscale (x1 cos t + x0 sin t)),  t = p * inv_freq[j].
 * The angle is formed and reduced in float64, so that a position a million tokens
 * out is as exact as the first; the rest is float32, rounded once.  Other dims
 * are copied: a factor that scores as a whole are to have (YaRN's, squared) goes into
 * mscale only where all dims turn, and into the attention's scale otherwise.
 *
 *   q, q_out     [B][Nmax] rows of Hq heads of d elements (dtype): row (b, i) starts
 *                at (b * Nmax + i) * q_row_stride, its head h q_head_stride elements
 *                after head h - 1; a head's elements follow one another.  q_out has
 *                strides of its own, with whole rows, or all rows of a head, one after
 *                another (LTD_EINVAL otherwise: no two heads may share memory).
 *                q_out may be q, with the same strides (in place).  Otherwise neither
 *                output shares memory with an input, or with the other output
 *                (LTD_EINVAL).  Interleaved heads of one buffer are apart where the
 *                two have the same strides, or their rows lie in different parts of the
 *                same row stride; ranges of other strides may not meet.
 *   k, k_out     the same with Hk heads, or Hk = 0 and NULL.
 *   inv_freq     [rot_dim / 2] float64: radians a position.
 *   depth        [B][Nmax] int32 >= 0 (as ltd_select_candidates writes it), or NULL
 *                for consecutive tokens (depth[b][i] = i).
 *   n_rows       [B] int32 in [0, Nmax]; rows i >= n_rows[b] are not written.
 *   rot_dim even, 2 <= rot_dim, rot_offset >= 0, rot_offset + rot_dim <= d <=
 *   LTD_ROPE_MAX_DIM, (Hq + Hk) * d <= 2^24, B * Nmax < 2^31 - 1, Nmax and positions
 *   up to LTD_MAX_LENGTH; Nmax may exceed LTD_MAX_NODES.  mscale is finite.
 * Any alignment is taken; 16-byte aligned rows and heads are faster.
 * With validate != 0: LTD_STATUS_BAD_NNODES (n_rows) and LTD_STATUS_BAD_PREFIX
 * (a position outside [0, LTD_MAX_LENGTH)).
 */
int ltd_tree_rope(const void* q, int64_t q_row_stride, int64_t q_head_stride, void* q_out,
                  int64_t q_out_row_stride, int64_t q_out_head_stride, const void* k,
                  int64_t k_row_stride, int64_t k_head_stride, void* k_out,
                  int64_t k_out_row_stride, int64_t k_out_head_stride, const double* inv_freq,
                  const int32_t* prefix_len, const int32_t* depth, const int32_t* n_rows, int B,
                  int Nmax, int Hq, int Hk, int d, int rot_offset, int rot_dim, int interleaved,
                  float mscale, int dtype, int validate, int32_t* status, void* stream);

/*
 * The latent cache.
 *
 * A model with latent attention keeps, for every token and layer, one row that all
 * heads share: d_latent dims (the compressed key and value) followed by d_rope dims
 * (the rotated key), in
 *   contiguous [B][kv_rows][d_latent + d_rope], paged [num_blocks][kv_rows][d_latent
 *   + d_rope] (dtype), logical row r of sequence b in block
 *   block_table[b][r / kv_rows].
 * d_latent is 256 or 512, d_rope is LTD_LATENT_ROPE; anything else is
 * LTD_EUNSUPPORTED, as are more than LTD_MAX_LENGTH rows to append or max_prefix,
 * and B * Nmax >= 2^31 - 1 rows to append.  Caches are 16-byte aligned (LTD_EINVAL otherwise).
 */

/*
 * Appends rows to a latent cache: a prompt's, or a draft tree's before its
 * verification.
 *
 * For every sequence b and i < n_rows[b], with (c, k) the first d_latent and the
 * last d_rope elements of row i, logical row P_b + i of the cache becomes
 *     [ c / sqrt(mean(c^2) + norm_eps) * norm_weight | k turned as in ltd_tree_rope ]
 * at position P_b + depth[b][i] (float32 statistics, each element rounded once); with
 * norm_weight NULL the latent part is copied.
 *
 *   kv_new       [B][Nmax][d_latent + d_rope] (dtype), row (b, i) at (b * Nmax + i) *
 *                new_row_stride (at least d_latent + d_rope: rows may be views into
 *                a fused projection's output); rows are 16-byte aligned and lie
 *                outside the cache (LTD_EINVAL).
 *   norm_weight  [d_latent] (dtype), 16-byte aligned, or NULL; norm_eps finite, >= 0.
 *   inv_freq     [d_rope / 2] float64; interleaved, mscale, depth and n_rows as for
 *                ltd_tree_rope (a factor for whole scores goes into the attention's
 *                scale: mscale would multiply the rotated part alone).
 * Other rows keep their bytes.  No two sequences may append to the same row.  With
 * validate != 0: LTD_STATUS_BAD_NNODES, LTD_STATUS_BAD_PREFIX (P_b < 0, rows past the
 * capacity or LTD_MAX_LENGTH) and LTD_STATUS_BAD_BLOCK (ids of the blocks that are
 * written); depth is not checked.
 */
int ltd_latent_append(const void* kv_new, int64_t new_row_stride, const void* norm_weight,
                      float norm_eps, const double* inv_freq, int interleaved, float mscale,
                      void* cache, const int32_t* block_table, const int32_t* prefix_len,
                      const int32_t* depth, const int32_t* n_rows, int B, int Nmax, int d_latent,
                      int d_rope, int kv_rows, int max_blocks, int num_blocks, int dtype,
                      int validate, int32_t* status, void* stream);

/*
 * Tree attention over a latent cache, in the absorbed form: the queries have been
 * multiplied into the latent space, and the output is in it.
 *
 * For every sequence b, node i < n_nodes[b] and head h, with x_t = [c_t | k_t] row t
 * of the cache:
 *     out[b][i][h] = softmax_t(scale * (<q_latent[b][i][h], c_t> + <q_rope[b][i][h], k_t>)) . c_t
 * over the visible rows t = {0, ..., P_b - 1} u {P_b + j : j on the root path of
 * node i, i included}.  Statistics and accumulation are float32, and so are partial
 * results of a row that the call splits over its keys; with bfloat16 the weights are
 * rounded to bfloat16 before they multiply the values (to 16 bits where Nmax * Hq <= 16),
 * and the sum that normalises them is that of the rounded ones.  Latent values may be
 * as large as 2^80: weights of up to 2^16 multiply them before the sum divides.
 *
 *   q_latent     rows of Hq heads of d_latent elements, q_rope of d_rope elements
 *                (dtype): row (b, i) at (b * Nmax + i) * row stride, head h at h * head
 *                stride (any layout whose heads' elements follow one another, such as
 *                [Hq][B][Nmax][d_latent], as a product per head leaves it).
 *                With bfloat16 rows and heads are 16-byte aligned (LTD_EINVAL).
 *   out          [B][Nmax][Hq][d_latent] (dtype), 16-byte aligned; rows i >=
 *                n_nodes[b] are not written.  It overlaps neither queries nor the cache
 *                (LTD_EINVAL where the two ranges of bytes meet).
 *   scale        finite and > 0 (that of the expanded heads, which the latent size
 *                does not tell, times the square of a context scaling's factor).
 *   prefix_len, max_prefix, parents, n_nodes, block_table as for
 *   ltd_tree_verify_attn; a single token a sequence is a tree of one node.
 *   workspace    at least ltd_tree_verify_attn_latent_workspace_size() bytes for the
 *                same (B, Nmax, Hq, d_latent, d_rope, max_prefix, dtype), 16-byte
 *                aligned; needs no initialisation.  The bytes that the query tells lie
 *                outside queries, cache and out (LTD_EINVAL).
 * A NaN or an infinity in a row's latent part, or a NaN score, reaches the outputs
 * of the nodes that see the row (where it may make every dimension NaN), and no
 * others.  Hq <= LTD_LATENT_MAX_HEADS; B <= 65535 with float32.
 */
size_t ltd_tree_verify_attn_latent_workspace_size(int B, int Nmax, int Hq, int d_latent,
                                                  int d_rope, int max_prefix, int dtype);

int ltd_tree_verify_attn_latent(const void* q_latent, int64_t ql_row_stride,
                                int64_t ql_head_stride, const void* q_rope, int64_t qr_row_stride,
                                int64_t qr_head_stride, const void* cache,
                                const int32_t* block_table, const int32_t* prefix_len,
                                const int32_t* parents, const int32_t* n_nodes, void* out, int B,
                                int Nmax, int Hq, int d_latent, int d_rope, int max_prefix,
                                int kv_rows, int max_blocks, int num_blocks, float scale,
                                int dtype, void* workspace, size_t workspace_bytes, int validate,
                                int32_t* status, void* stream);

/*
 * Compaction of a latent cache: ltd_kv_compact for its one row a token.  Layer l
 * starts layer_stride_elems elements after layer l - 1 (a multiple of 16 bytes).
 * num_layers <= 65535.
 */
int ltd_latent_compact(void* cache, const int32_t* block_table, const int32_t* prefix_len,
                       int32_t* new_prefix_len, const int32_t* accepted_nodes,
                       const int32_t* n_accepted, int B, int Nmax, int d_latent, int d_rope,
                       int kv_rows, int max_blocks, int num_blocks, int num_layers,
                       int64_t layer_stride_elems, int dtype, int validate, int32_t* status,
                       void* stream);

/* Library version string. */
const char* ltd_version(void);

#ifdef __cplusplus
}
#endif
#endif /* LTD_VERIFY_H */
