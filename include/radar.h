/*
 * radar.h -- C ABI of the MI355X (gfx950) hot path of RADAR's speculative-
 * sampling loop (arXiv 2512.14069).
 *
 * One decode cycle of the paper's pipeline (Sec. 4.1, App. A.1) runs, on the
 * device, three data-parallel pieces of work that this library provides:
 *
 *   radar_draft_expand   after every draft-model call: vocabulary-wide top-k,
 *                        cumulative log-probability ("confidence") scoring and
 *                        choice of the next frontier (App. A.1; Sec. 4.2 Eq. 3)
 *   radar_draft_rerank   when drafting stops: keep the best N candidates and
 *                        emit the serialized draft tree (Sec. 1, Sec. 2.3)
 *   radar_tree_attention inside every target layer: each tree node attends to
 *                        the prefix KV cache plus its own ancestors (Sec. 1,
 *                        Sec. 3: one parallel target pass over the tree)
 *   radar_verify_accept  after the target pass: greedy or rejection-sampling
 *                        walk down the tree (Sec. 3, Eq. 1-2; Sec. 4.3 Eq. 13)
 * and, around them, radar_policy_step (the prediction model's continue / stop
 * decision after each draft call, Sec. 4.2) and
 * radar_accept_length_distribution (Sec. 4.3, Eq. 11-13).
 *
 * Conventions for every call
 *   - Tensor arguments are DEVICE pointers owned by the caller; descriptors
 *     are HOST structs read during the call; scalars are passed by value.
 *   - A call validates what the host can see, enqueues its kernels on `stream`
 *     (a hipStream_t passed as void*; NULL = the default stream) and returns
 *     without synchronising.  Outputs are valid once the stream has reached
 *     the end of the enqueued work.  A call consists of kernel launches
 *     only, so it may be made on a stream that is being captured into a HIP
 *     graph (radar_workspace_init stays outside the capture; make each entry
 *     point's first call on a device outside a capture as well: it sets the
 *     kernels' launch attributes).
 *   - No call allocates or frees memory.  Scratch memory is a caller-owned
 *     device workspace whose size the matching *_workspace_bytes query gives.
 *     All of a workspace must be passed once through radar_workspace_init before
 *     its first use (it holds arrival counters, which the kernels leave zeroed
 *     again, and words from workgroup to workgroup that carry a mark when they are
 *     there, of which the kernels leave none); it may then be reused by any number of calls of the SAME entry
 *     point with the SAME descriptor on ONE stream.  Where the counters sit
 *     depends on the entry point and on the shape, so a workspace that goes
 *     over to another entry point or another descriptor is passed through
 *     radar_workspace_init again first.  Calls that share a workspace on
 *     different streams race.
 *   - Return value: RADAR_OK or a negative radar_status.  Nothing is printed,
 *     thrown or aborted.  On an error no kernel has been launched.
 *   - Device data is not validated (that would need a synchronisation).  The
 *     kernels stay in bounds and terminate for any content: a parent index
 *     that is not smaller than its child simply ends that node's ancestor
 *     chain; token ids outside [0,V) are not dereferenced.
 *     radar_debug_validate_tree checks a parent array on request.
 *
 * Tree convention (the paper leaves it open): a serialized tree has T_max row
 * slots per sequence of which the first n_nodes[b] are used; node 0 is the
 * root, i.e. the token the target produced last ("can" in App. A.1), with
 * parents[0] = -1; for i > 0, 0 <= parents[i] < i.
 */
#ifndef RADAR_H
#define RADAR_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef int32_t radar_status;
#define RADAR_OK                    0
#define RADAR_INVALID_ARG          -1   /* null pointer, non-positive size, inconsistent sizes   */
#define RADAR_UNSUPPORTED_SHAPE    -2   /* outside the compiled limits listed at each call      */
#define RADAR_WORKSPACE_TOO_SMALL  -3
#define RADAR_HIP_ERROR            -4   /* a HIP runtime call failed (launch, attribute query)  */

#define RADAR_T_MAX        64    /* most tree rows per sequence (one 64-bit ancestor word)  */
#define RADAR_K_MAX        16    /* largest branching factor k                              */
#define RADAR_F_MAX        64    /* most frontier rows per expand call                      */
#define RADAR_POOL_MAX   4096    /* most pooled candidates radar_draft_rerank accepts       */

/* Text for a status code; never NULL; static storage. */
const char *radar_status_string(radar_status status);

/* Library version: major * 10000 + minor * 100 + patch. */
int radar_version(void);

/* Zero a workspace before its first use.  `bytes` is the full size that was
 * allocated (what the *_workspace_bytes query returned, or more; at least 4096).
 * Enqueues one kernel. */
radar_status radar_workspace_init(void *workspace, size_t bytes, void *stream);

/* --------------------------------------------------------------------------
 * Tree-verify attention (Sec. 1 and Sec. 3: the target model checks the whole
 * serialized draft tree in one pass whose attention is masked by the tree).
 *
 * For sequence b, node i < n_nodes[b] and query head h:
 *     out[b,i,h,:] = softmax_j( scale * <q[b,i,h,:], k[b,h/G,j,:]> ) . v[b,h/G,j,:]
 * over cache rows j in [0, ctx_lens[b])  (the prefix)  and  j = ctx_lens[b] + a
 * for a = i and every ancestor a of i (cache row ctx_lens[b]+a holds the key /
 * value of tree node a: the verify pass appends the tree to the cache before
 * attention).  G = Hq / Hkv.  Rotary positions, if any, are already applied (radar_rope).
 * Inputs and output are bf16, scores / softmax / accumulation fp32.
 * Rows i >= n_nodes[b] of out (and lse) are written as zero.
 *
 * Limits: D in {64, 128}; Hq % Hkv == 0; 1 <= T_max <= RADAR_T_MAX;
 *         ctx_lens[b] + n_nodes[b] <= S_max (caller's contract).
 * Strides are in elements; the innermost (D) axis is contiguous; a stride of
 * 0 means "dense" ([B,T_max,Hq,D] for q / out, [B,Hkv,S_max,D] for caches).
 * All bf16 base pointers and strides must keep rows 16-byte aligned.
 * S_max is what the call is planned for: how many rows it is split into ranges for, or
 * whether it is one launch.  Where the cache is allocated for longer sequences, pass the rows in
 * use (the longest ctx_lens[b] + T_max) as S_max and the allocation's strides.
 */
typedef struct radar_attn_desc {
    int32_t B, T_max, Hq, Hkv, D, S_max;
    int64_t q_stride_b, q_stride_t, q_stride_h;
    int64_t kv_stride_b, kv_stride_h, kv_stride_s;
    int64_t out_stride_b, out_stride_t, out_stride_h;
    float   softmax_scale;      /* 0 => 1/sqrt(D); must not be negative */
    int32_t keys_per_split;     /* 0 => chosen by the library; else a multiple of 64: cache rows one
                                   workgroup streams before partial results are merged */
} radar_attn_desc;

size_t radar_tree_attention_workspace_bytes(const radar_attn_desc *desc);

/* q, out: bf16 [B,T_max,Hq,D]; k_cache, v_cache: bf16 [B,Hkv,S_max,D];
 * parents: i32 [B,T_max]; ctx_lens: i32 [B]; n_nodes: i32 [B] or NULL (= T_max
 * everywhere); lse_out: f32 [B,T_max,Hq] or NULL (natural-log sum of exp of the
 * scaled scores over the allowed set). */
radar_status radar_tree_attention(const void *q, const void *k_cache, const void *v_cache,
                                  const int32_t *parents, const int32_t *ctx_lens, const int32_t *n_nodes,
                                  void *out, float *lse_out, const radar_attn_desc *desc,
                                  void *workspace, size_t workspace_bytes, void *stream);

/* --------------------------------------------------------------------------
 * Draft expansion, one call per draft-model call (App. A.1; Sec. 2.3).
 *
 * Row f of `logits` is the draft model's output for frontier node f.  For each
 * row the k best tokens under the order (logit descending, token id ascending)
 * become candidate children c = f*k + r with
 *     cand_scores[c] = parent_scores[f] + (logit - logsumexp(row f))
 * i.e. the log of the path's cumulative draft probability.  The k best of the
 * F*k candidates under (score descending, c ascending) are the next frontier;
 * frontier_conf = exp(score) are the k confidences in [0,1] that the paper's
 * prediction model reads (Sec. 4.2, Eq. 3).  Every candidate is appended to
 * the pool at index pool_count + c with its parent's pool index, for the final
 * rerank.  Requires F*k >= k, i.e. always k frontier outputs.
 *
 * Limits: 1 <= F <= RADAR_F_MAX; 1 <= k <= min(RADAR_K_MAX, V);
 *         pool_count + F*k <= pool_capacity.  -inf logits are legal; NaN
 *         logits and rows that are entirely -inf give unspecified results
 *         (every output is written, tokens are tokens of the vocabulary).
 */
typedef struct radar_expand_desc {
    int32_t F, V, k;
    int32_t pool_count;      /* candidates already in the pool (host-tracked: grows by F*k per call) */
    int32_t pool_capacity;   /* length of the three pool arrays */
} radar_expand_desc;

/* One workspace serves every draft call of a cycle: the expansion family
 * (radar_draft_expand, _policy, _cycle, _batch) keeps its arrival counters at
 * fixed places at the head of the workspace and leaves them zero, and leaves
 * nothing that a later call could take for its own results, so calls with different descriptors (F = 1
 * for the root, then F = k; a growing pool_count) and different members of the
 * family may follow each other on one stream without radar_workspace_init in
 * between, provided the workspace has the size the largest of them asks for
 * and, for radar_draft_expand_batch, B stays the same (sequence b's counters
 * sit where another B keeps other data). */
size_t radar_draft_expand_workspace_bytes(const radar_expand_desc *desc);

/* logits f32 [F,V]; parent_scores f32 [F]; parent_pool_idx i32 [F] (-1 = root);
 * cand_tokens i32 [F*k]; cand_scores f32 [F*k];
 * frontier_pool_idx i32 [k]; frontier_tokens i32 [k]; frontier_scores f32 [k];
 * frontier_conf f32 [k];  pool_tokens i32, pool_scores f32, pool_parents i32
 * [pool_capacity] (entries [pool_count, pool_count+F*k) are written).
 * frontier_scores / frontier_pool_idx may be passed as the next call's
 * parent_scores / parent_pool_idx. */
radar_status radar_draft_expand(const float *logits, const float *parent_scores, const int32_t *parent_pool_idx,
                                int32_t *cand_tokens, float *cand_scores,
                                int32_t *frontier_pool_idx, int32_t *frontier_tokens,
                                float *frontier_scores, float *frontier_conf,
                                int32_t *pool_tokens, float *pool_scores, int32_t *pool_parents,
                                const radar_expand_desc *desc,
                                void *workspace, size_t workspace_bytes, void *stream);

/* radar_draft_expand for callers that cannot allocate or hand over a workspace (code under HIP
 * graph capture, tight serving loops, harnesses that forbid hipMalloc): the same kernels with
 * their scratch memory in a device array that this library holds itself,
 * RADAR_NOALLOC_SCRATCH_BYTES on every GPU it runs on, until the process ends.  Inputs and
 * outputs are the caller's, exactly as for radar_draft_expand; there is no workspace argument
 * and nothing is allocated or freed, by this call or by anything it calls.
 * Limits: those of radar_draft_expand, and radar_draft_expand_workspace_bytes(desc) <=
 * RADAR_NOALLOC_SCRATCH_BYTES (F = 10, V = 128256 needs 0.06 MB; about F * V <= 25 M logits
 * fit), else RADAR_UNSUPPORTED_SHAPE and nothing is launched.
 * All calls on one GPU share that GPU's array: calls that overlap in time on one GPU (two
 * streams, two threads) race and give unspecified results; calls that follow each other on one
 * stream, or are ordered by events, are fine, whatever their shapes.  The stream must belong to
 * the current device.  The first call on a device looks the array up and enqueues one extra
 * fill kernel that clears it; make that call outside a graph capture. */
#define RADAR_NOALLOC_SCRATCH_BYTES (1u << 20)
radar_status radar_draft_expand_noalloc(const float *logits, const float *parent_scores, const int32_t *parent_pool_idx,
                                        int32_t *cand_tokens, float *cand_scores,
                                        int32_t *frontier_pool_idx, int32_t *frontier_tokens,
                                        float *frontier_scores, float *frontier_conf,
                                        int32_t *pool_tokens, float *pool_scores, int32_t *pool_parents,
                                        const radar_expand_desc *desc, void *stream);

/* --------------------------------------------------------------------------
 * Rerank, once per cycle (Sec. 1 / Sec. 2.3: the dynamic tree is reordered
 * and pruned by confidence).
 *
 * Orders the pool by (score descending, pool index ascending), keeps the first
 * min(N, pool_count) and emits the tree to verify: node 0 is the root
 * (root_token, score 0, depth 0, parent -1), the candidate of rank r is node
 * 1+r, parents are re-indexed to node numbers (pool parent -1 => node 0),
 * depth = depth(parent) + 1.  Scores never grow from parent to child, so a kept
 * node's parent is kept and has a smaller node number; should the input break
 * that, the node's parent is written as -2 and its depth as 0.
 * Outputs are N+1 long; slots past n_nodes hold token -1, parent -1, score 0,
 * depth 0, pool_idx -1.  *n_nodes_out (device) = 1 + min(N, pool_count).
 *
 * Limits: 0 <= pool_count <= RADAR_POOL_MAX; 0 <= N < RADAR_T_MAX.
 */
size_t radar_draft_rerank_workspace_bytes(int32_t pool_count, int32_t N);

radar_status radar_draft_rerank(const int32_t *pool_tokens, const float *pool_scores, const int32_t *pool_parents,
                                int32_t pool_count, int32_t N, int32_t root_token,
                                int32_t *tree_tokens, int32_t *tree_parents, float *tree_scores,
                                int32_t *tree_depth, int32_t *tree_pool_idx, int32_t *n_nodes_out,
                                void *workspace, size_t workspace_bytes, void *stream);

/* --------------------------------------------------------------------------
 * Verification walk (Sec. 3, Eq. 1-2; tree form per Sec. 4.3, Eq. 11-13).
 *
 * Row r of target_logits is the target's next-token distribution after the
 * path ending in node r.  Starting at the root:
 *   mode RADAR_ACCEPT_GREEDY   descend to the child whose token is the argmax of
 *       the current row (lowest token id among equal logits, lowest node index
 *       among equal tokens); stop when none matches; bonus = that argmax.
 *   mode RADAR_ACCEPT_SAMPLE   p = softmax(row / temperature).  The children
 *       are fixed tokens (point-mass proposals), so Eq. 1 accepts child c with
 *       the residual probability of its token: visiting children in ascending
 *       node index with R = mass of those already rejected, accept iff
 *       uniforms[b,c] * (1 - R) < p(tok_c), else R += p(tok_c).  If none is
 *       accepted the bonus token is the inverse CDF, at uniforms[b,T_max] *
 *       (1 - R), of p with the rejected tokens removed (Eq. 2), scanning token
 *       ids upwards.  A leaf has R = 0.
 * accept_len[b] = number of accepted draft nodes (root excluded, <= depth);
 * accept_path[b,:] = node indices from the root, padded with -1, D_max+1 long;
 * a walk that would exceed D_max stops there.  bonus_token[b] = the extra token
 * every cycle emits (Sec. 3: between 1 and t+1 tokens per cycle).
 *
 * Limits: 1 <= T_max <= RADAR_T_MAX; 0 <= D_max < RADAR_T_MAX; V >= 1;
 *         temperature > 0 and uniforms != NULL in sampling mode.
 */
#define RADAR_ACCEPT_GREEDY 0
#define RADAR_ACCEPT_SAMPLE 1

typedef struct radar_accept_desc {
    int32_t B, T_max, V, D_max;
    int32_t mode;
    float   temperature;
} radar_accept_desc;

size_t radar_verify_accept_workspace_bytes(const radar_accept_desc *desc);

/* target_logits f32 [B,T_max,V]; draft_tokens, parents i32 [B,T_max];
 * n_nodes i32 [B] or NULL; uniforms f32 [B,T_max+1] or NULL (greedy);
 * accept_len i32 [B]; accept_path i32 [B,D_max+1]; bonus_token i32 [B]. */
radar_status radar_verify_accept(const float *target_logits, const int32_t *draft_tokens, const int32_t *parents,
                                 const int32_t *n_nodes, const float *uniforms,
                                 int32_t *accept_len, int32_t *accept_path, int32_t *bonus_token,
                                 const radar_accept_desc *desc,
                                 void *workspace, size_t workspace_bytes, void *stream);

/* --------------------------------------------------------------------------
 * Acceptance-length distribution of a draft tree (Sec. 4.3, Eq. 11-13): what
 * the walk above would return as accept_len, as a distribution over the
 * uniforms, computed without drawing.  With P_acc(child | parent) =
 * p_parent(token of child), p = softmax(row / temperature):
 *   reach(root) = 1, reach(v) = reach(parent) * p_parent(tok_v);
 *   P_stop(v) = reach(v) * (1 - sum over children c of p_v(tok_c))  (Eq. 12-13);
 *   dist[b,i] = sum of P_stop(v) over nodes of depth i              (Eq. 11).
 * A child that repeats an earlier sibling's token is never reached; nodes at
 * depth D_max keep all the mass that reaches them and deeper nodes get none
 * (the cut radar_verify_accept makes).  Every row of dist sums to 1.
 *
 * dist f64 [B,D_max+1] (device); the other tensors as for radar_verify_accept;
 * desc->mode is ignored, desc->temperature must be > 0.  Workspace: what
 * radar_verify_accept_workspace_bytes(desc) gives; one kernel is enqueued. */
radar_status radar_accept_length_distribution(const float *target_logits, const int32_t *draft_tokens,
                                              const int32_t *parents, const int32_t *n_nodes, double *dist,
                                              const radar_accept_desc *desc,
                                              void *workspace, size_t workspace_bytes, void *stream);

/* --------------------------------------------------------------------------
 * Verification with draft distributions (Sec. 3, Eq. 1-2 as printed): for
 * trees whose tokens were DRAWN from the draft model's distributions rather
 * than picked as its top-k.  With p_v = softmax(target row v / temperature),
 * q_c = softmax(draft row q_rows[c] / draft_temperature) the distribution node
 * c's token was drawn from, and r the running residual at node v (r = p_v at
 * first):
 *   for each child c of v in ascending node index, x = its token:
 *     accept c  iff  uniforms[b,c] * q_c(x) < r(x)          (probability min(1, r(x)/q_c(x)), Eq. 1)
 *     otherwise     r <- max(0, r - q_c), renormalised       (Eq. 2)
 *   when no child is accepted (or v is a leaf, or the walk is D_max deep) the
 *   bonus token is the inverse CDF of r at uniforms[b,T_max], scanning token ids
 *   upwards.  Should the residual vanish (p_v <= the rejected proposals
 *   everywhere, possible only through rounding) the bonus is drawn from p_v.
 * On a chain this is exactly the paper's procedure; for several children it is
 * the recursive form that keeps the emitted tokens distributed as the target's.
 * Children may repeat a token.  Outputs as for radar_verify_accept.
 *
 * target_logits f32 [B,T_max,V]; draft_logits f32 [B,Tq,V]; q_rows i32 [B,T_max]
 * (row of draft_logits per node, entry 0 unused; siblings drawn from one
 * distribution may share a row) or NULL (Tq == T_max, node c uses row c);
 * draft_tokens, parents i32 [B,T_max]; n_nodes i32 [B] or NULL; uniforms f32
 * [B,T_max+1].  Nodes whose token or draft row is out of range are skipped.
 * Limits: T_max <= RADAR_T_MAX; V <= 1048576; B * (T_max + Tq) <= 65535;
 *         both temperatures > 0.  One kernel is enqueued, which reads the rows that
 *         the walk visits and no others (a single-workgroup walk over few rows of a large vocabulary:
 *         two kernels, the first of which reads every row once).  The shared walk needs its
 *         B * G workgroups resident together; the library sizes G from the occupancy the runtime
 *         reports for the device (CUs x workgroups per CU) and bounds every wait (about 100 us by
 *         default, up to 0.7 ms where rows are too long for the workgroups' registers): where other work keeps some of them from running, the wait ends and the
 *         fall-back described at walk_spin_limit redoes the sequence.  On a GPU that is shared as a
 *         rule, pass walk_spin_limit < 0 (single-workgroup walk, no waiting at all). */
typedef struct radar_accept_q_desc {
    int32_t B, T_max, Tq, V, D_max;
    float   temperature, draft_temperature;
    int32_t walk_spin_limit;    /* 0: the library's choice.  The walk of one sequence is shared by several
                                   workgroups that meet at every node and after every rejection; the wait there
                                   is bounded, and a sequence whose workgroups gave up is redone by a single one
                                   (same results).  > 0: polls (about 0.5 us each) before giving up (tests
                                   pass 1 to force that path; the default is 256,
                                   more for rows too long for registers); < 0: single-workgroup
                                   walk only */
} radar_accept_q_desc;

size_t radar_verify_accept_q_workspace_bytes(const radar_accept_q_desc *desc);

radar_status radar_verify_accept_q(const float *target_logits, const float *draft_logits, const int32_t *q_rows,
                                   const int32_t *draft_tokens, const int32_t *parents, const int32_t *n_nodes,
                                   const float *uniforms,
                                   int32_t *accept_len, int32_t *accept_path, int32_t *bonus_token,
                                   const radar_accept_q_desc *desc,
                                   void *workspace, size_t workspace_bytes, void *stream);

/* --------------------------------------------------------------------------
 * Prediction-model step (Sec. 4.2, Eq. 3-5; architecture per App. A.3): after a
 * draft-model call, decide from the k frontier confidences whether to call the
 * draft model again.
 *
 * A single-layer LSTM cell reads x = the k confidences (frontier_conf of
 * radar_draft_expand) and the state (h, c); the new hidden vector is joined
 * with x and passed through a two-layer perceptron with ReLU to two logits:
 *     [i f g o] = w_ih x + b_ih + w_hh h + b_hh      (four blocks of H rows, this order)
 *     c' = sigm(f) * c + sigm(i) * tanh(g);   h' = sigm(o) * tanh(c')
 *     logits = w2 relu(w1 [h'; x] + b1) + b2;   probs = softmax(logits)
 * Index 0 is "stop drafting", index 1 "call the draft model again" (Eq. 5).
 * action[b] = 1 iff logits[b,1] > logits[b,0] (a tie stops), or, when uniforms
 * is given, 1 iff uniforms[b] < probs[b,1] (a draw from the policy).
 * The state starts at zero at the first draft step of a cycle (h_in = c_in =
 * NULL) and is handed from call to call; h_out / c_out may be h_in / c_in.
 * Training-time dropout has no counterpart here.  All arithmetic is fp32.
 *
 * Parameters are DEVICE arrays of fp32 in row-major [out, in] order (the
 * layout in which the common deep-learning toolkits keep an LSTM layer and a
 * linear layer, so trained weights can be handed over unchanged):
 *   w_ih [4H,k]  w_hh [4H,H]  b_ih, b_hh [4H]  w1 [M,H+k]  b1 [M]  w2 [2,M]  b2 [2]
 * Limits: H == 128; 1 <= k <= RADAR_K_MAX; 1 <= M <= 128; w_hh, h_in 16-byte aligned.
 * conf f32 [B,k]; h_in, c_in, h_out, c_out f32 [B,H]; logits, probs f32 [B,2];
 * action i32 [B]; uniforms f32 [B] or NULL.  One kernel, no workspace. */
typedef struct radar_policy_params {
    const float *w_ih, *w_hh, *b_ih, *b_hh;   /* LSTM cell   */
    const float *w1, *b1, *w2, *b2;           /* perceptron  */
    int32_t k, H, M;
} radar_policy_params;

radar_status radar_policy_step(const float *conf, const float *h_in, const float *c_in,
                               const radar_policy_params *params, const float *uniforms,
                               float *h_out, float *c_out, float *logits, float *probs, int32_t *action,
                               int32_t B, void *stream);

/* radar_draft_expand followed, in the same launch, by radar_policy_step on the
 * frontier_conf it has just written (batch of one: a drafting loop has one
 * frontier and one policy state).  Results are those of the two calls made one
 * after the other, bit for bit; the second launch and its latency are saved
 * (the paper's T_p, Sec. 4.2 Eq. 8-9, is mostly that).  params->k must equal
 * desc->k.  io is a HOST struct of DEVICE pointers: h_in, c_in f32 [H] or both
 * NULL (zero state); uniform f32 [1] or NULL (argmax action); h_out, c_out f32
 * [H] (may be h_in, c_in); logits, probs f32 [2]; action i32 [1].  Workspace and
 * all other arguments as for radar_draft_expand. */
typedef struct radar_policy_io {
    const float *h_in, *c_in, *uniform;
    float *h_out, *c_out, *logits, *probs;
    int32_t *action;
} radar_policy_io;

radar_status radar_draft_expand_policy(const float *logits, const float *parent_scores, const int32_t *parent_pool_idx,
                                       int32_t *cand_tokens, float *cand_scores,
                                       int32_t *frontier_pool_idx, int32_t *frontier_tokens,
                                       float *frontier_scores, float *frontier_conf,
                                       int32_t *pool_tokens, float *pool_scores, int32_t *pool_parents,
                                       const radar_expand_desc *desc,
                                       const radar_policy_params *params, const radar_policy_io *io,
                                       void *workspace, size_t workspace_bytes, void *stream);

/* --------------------------------------------------------------------------
 * A whole drafting cycle without the host in the loop (Sec. 4.1-4.2: after
 * every draft call the prediction model decides whether another one follows;
 * App. latency table: the decision and its round trip are what T_p pays for).
 *
 * The decision stays on the device: a radar_cycle_state in DEVICE memory holds
 * "stopped", the number of pooled candidates and the number of draft calls
 * made.  The host enqueues the longest cycle it allows (t_max draft calls,
 * Sec. 4.2) once -- directly or captured in a HIP graph -- and never reads a
 * result in between:
 *   radar_cycle_begin          resets the state (one small kernel, no memset);
 *       not needed before a cycle whose first draft call is made through
 *       radar_draft_expand_cycle with desc->pool_count == 0: that call starts
 *       the cycle itself (it ignores what the state holds and writes all of it)
 *   radar_draft_expand_cycle   one draft call's expansion; does NOTHING (every
 *       workgroup leaves at once, no output is touched) when the state says
 *       stopped; otherwise radar_draft_expand with the pool count taken from
 *       the state, followed, when params != NULL, by radar_policy_step on the
 *       new confidences as in radar_draft_expand_policy; then the state's pool
 *       count grows by F*k, steps_done by one, and action 0 sets stopped.
 *       Pass params = io = NULL for the last allowed draft call (no decision
 *       is needed after it).  desc->pool_count is the LARGEST count the state
 *       can hold when this call runs (what it would be had every earlier call
 *       run): the capacity check uses it, and a state outside [0, that] makes
 *       the call a no-op.  With desc->pool_count == 0 the call is the first
 *       of a cycle and always runs.
 *   radar_draft_rerank_cycle   radar_draft_rerank over the candidates the state
 *       counts (at most pool_count_max).
 * Because a skipped call leaves its outputs alone, the frontier arrays chained
 * from call to call still hold the last executed call's values.  All other
 * arguments, limits and the workspace are those of the plain calls. */
typedef struct radar_cycle_state {
    int32_t stopped;        /* 1 once a decision said "stop" */
    int32_t pool_count;     /* candidates pooled so far */
    int32_t steps_done;     /* draft calls whose expansion ran */
    int32_t last_action;    /* last decision (0 stop, 1 continue), -1 before the first */
} radar_cycle_state;

radar_status radar_cycle_begin(radar_cycle_state *state, void *stream);

radar_status radar_draft_expand_cycle(const float *logits, const float *parent_scores, const int32_t *parent_pool_idx,
                                      int32_t *cand_tokens, float *cand_scores,
                                      int32_t *frontier_pool_idx, int32_t *frontier_tokens,
                                      float *frontier_scores, float *frontier_conf,
                                      int32_t *pool_tokens, float *pool_scores, int32_t *pool_parents,
                                      const radar_expand_desc *desc,
                                      const radar_policy_params *params, const radar_policy_io *io,
                                      radar_cycle_state *state,
                                      void *workspace, size_t workspace_bytes, void *stream);

radar_status radar_draft_rerank_cycle(const int32_t *pool_tokens, const float *pool_scores, const int32_t *pool_parents,
                                      const radar_cycle_state *state, int32_t pool_count_max, int32_t N,
                                      int32_t root_token,
                                      int32_t *tree_tokens, int32_t *tree_parents, float *tree_scores,
                                      int32_t *tree_depth, int32_t *tree_pool_idx, int32_t *n_nodes_out,
                                      void *workspace, size_t workspace_bytes, void *stream);

/* --------------------------------------------------------------------------
 * One draft call for B sequences in ONE launch (the batch the other two steps
 * already take; Sec. 4.1-4.2: every sequence runs its own cycle and stops at
 * its own draft call, which is what makes the batch's trees ragged).
 *
 * Sequence b is an independent radar_draft_expand_cycle (states != NULL),
 * radar_draft_expand_policy (states == NULL, params != NULL) or
 * radar_draft_expand (both NULL): same results, same limits.  Every array of
 * those calls gains a leading dimension B, densely packed:
 * logits [B,F,V]; parent_scores, parent_pool_idx [B,F]; cand_* [B,F*k];
 * frontier_* [B,k]; pool_* [B,pool_capacity]; states [B]; and in io: h_in,
 * c_in, h_out, c_out [B,H], uniform [B], logits, probs [B,2], action [B].
 * desc (F, V, k, pool_count, pool_capacity) is shared by all sequences:
 * without states every sequence's pool holds desc->pool_count candidates; with
 * states each holds its own state's count, desc->pool_count being the largest
 * any may have, and a sequence whose state says stopped is skipped (its
 * workgroups leave at once) while the others run.  The model's weights
 * (params) are shared.
 * Batches whose workgroups all run at once (up to some 4 Mi logits, B*F*V) are
 * one launch, larger ones two: a streaming kernel over all sequences, then one workgroup per sequence
 * (which also runs the prediction model's step when params != NULL).  Integer results are the same
 * either way; scores may differ in the last bit (the sums are grouped differently).
 * Limits: 1 <= B <= 65535.  The workspace is sized by
 * radar_draft_expand_batch_workspace_bytes(desc, B) (equal to
 * radar_draft_expand_workspace_bytes(desc) for B = 1).
 */
size_t radar_draft_expand_batch_workspace_bytes(const radar_expand_desc *desc, int32_t B);

radar_status radar_draft_expand_batch(const float *logits, const float *parent_scores, const int32_t *parent_pool_idx,
                                      int32_t *cand_tokens, float *cand_scores,
                                      int32_t *frontier_pool_idx, int32_t *frontier_tokens,
                                      float *frontier_scores, float *frontier_conf,
                                      int32_t *pool_tokens, float *pool_scores, int32_t *pool_parents,
                                      const radar_expand_desc *desc, int32_t B,
                                      const radar_policy_params *params, const radar_policy_io *io,
                                      radar_cycle_state *states,
                                      void *workspace, size_t workspace_bytes, void *stream);

/* radar_draft_rerank for B sequences in one launch: pool_* [B,pool_capacity];
 * root_tokens i32 [B]; tree_* [B,N+1]; n_nodes_out i32 [B], i.e. the parents,
 * tokens and n_nodes arrays that radar_tree_attention and radar_verify_accept
 * take for a batch with T_max = N+1.  states == NULL: every pool holds
 * pool_count candidates; states [B]: each holds its own state's count, at most
 * pool_count.  Limits: those of radar_draft_rerank; pool_count <= pool_capacity;
 * 1 <= B <= 65535.  Workspace as for radar_draft_rerank. */
radar_status radar_draft_rerank_batch(const int32_t *pool_tokens, const float *pool_scores, const int32_t *pool_parents,
                                      const radar_cycle_state *states, int32_t pool_count, int32_t pool_capacity,
                                      int32_t B, int32_t N, const int32_t *root_tokens,
                                      int32_t *tree_tokens, int32_t *tree_parents, float *tree_scores,
                                      int32_t *tree_depth, int32_t *tree_pool_idx, int32_t *n_nodes_out,
                                      void *workspace, size_t workspace_bytes, void *stream);

/* --------------------------------------------------------------------------
 * Paged key/value cache in 4 bits: the memory that the target's layers keep
 * their keys and values in, in place of the dense bf16 caches above, for many
 * sequences and long contexts (a quarter of the bytes and nothing reserved for
 * rows that are not there).  A verification pass makes, in this order,
 *   radar_kvq_blocks              room for the batch's trees, and where each row goes
 *   radar_kvq_append              per layer: the trees' keys and values into the cache
 *   radar_tree_attention_kvq      per layer: every node over its prefix and ancestors
 *   radar_kvq_commit              after the walk: the accepted path's rows into place
 * and radar_kvq_read gives rows back as bf16, e.g. to hand a prefix on.
 * A sequence that radar_kvq_blocks refuses has no part in the pass: its rows are
 * not written, and the later calls reach no block that is not its own.  What they
 * give for it (outputs, an accepted path, new_ctx_lens) stands for nothing, and its
 * ctx_lens stays what it was.  (Given a negative length in its place they leave it
 * out; to radar_kvq_blocks that would mean that it has ended.)
 *
 * Format.  32 consecutive values x of a row of a head share a scale 2^e and are
 * 4-bit codes (sign; 0, 0.5, 1, 1.5, 2, 3, 4, 6).  With amax the largest |x|, e is
 * the smallest whole number for which amax < 7 * 2^e, kept within [-126, 125];
 * x * 2^-e is rounded to the nearest code, ties to the even one, larger ones to
 * +-6 (only where e was limited to 125).  No value is off by more than 2^e then.
 * The scale is kept as the byte e + 127.  A block that holds an infinity or NaN
 * has byte 255 and stands for 32 NaNs.  What codes stand for is exact in bf16
 * (bytes 253 and 254, which are never written, reach past its largest number;
 * radar_kvq_read gives infinity there, attention may take all of the block for NaN).
 *
 * Layout.  The cache is n_blocks blocks of block_rows rows per layer, every block
 * [Hkv] chunks of radar_kvq_block_bytes(block_rows, D) = block_rows * (D + D/16)
 * bytes.  With R = block_rows a chunk is
 *     K codes [R][D/2]  V codes [R/8][D/8][8][4]  K scales [R/8][D/32][8]  V scales [R/8][D/32][8]
 * (V codes: 8 rows next to each other for every 8 values of the head; an even
 * value is the low half of its byte).  A row's SLOT is block * R + row in block.
 * Row j of sequence b is row j % R of block block_tables[b][j / R].
 *
 * Limits for all of them: D in {64, 128}; block_rows in {16, 32, 64, 128};
 * n_blocks * block_rows < 2^31; Hkv <= 65535; layers <= 65535 and layers * Hkv
 * < 2^24; rows of a call times Hkv < 2^27; cache and layer_stride multiples of 16
 * bytes.  Block numbers and slots that are out of range are not
 * dereferenced: such a row is not there. */
typedef struct radar_kvq_desc {
    int32_t n_blocks, block_rows, Hkv, D;
    int32_t layers;          /* radar_kvq_commit and radar_kvq_read: how many layers the call covers */
    int64_t layer_stride;    /* bytes from one layer's cache to the next, a layer's at least; 0 => dense */
} radar_kvq_desc;

/* Bytes of one KV head's rows of one block; 0 where the limits are not met. */
size_t radar_kvq_block_bytes(int32_t block_rows, int32_t D);

/* Block tables and slot maps from the sequences' lengths.  Sequence b asks for
 * w = ceil((ctx_lens[b] + n_new[b]) / block_rows) blocks, none if ctx_lens[b] < 0
 * (a sequence that has ended), and has owned[b].  First every sequence with
 * owned[b] > w gives entries [w, owned[b]) of its table back: they are put onto the
 * free stack free_blocks[0 .. *n_free) in order of b and then of the entry.  Then
 * sequences that ask for more take theirs off the top of the stack, in order of b
 * and then of the entry, as long as what all of them up to and including b ask for
 * is there: granted[b] = 1, owned_out[b] = w.  Where it is not, granted[b] = 0 and
 * the sequence keeps what it has (so do all later ones that ask for more); a
 * sequence that asks for more than max_blocks is refused without counting.
 * slots[b,i] is the slot of row ctx_lens[b] + i for i < n_new[b] (clamped to
 * [0, T_max]), -1 for other i and for sequences that were not granted.
 * block_tables i32 [B,max_blocks] and free_blocks i32 [n_blocks] are updated in
 * place; entries behind the owned ones and the stack's height are left as they
 * were, but for a sequence that is not granted, whose entries [owned[b], max_blocks)
 * become -1 (later calls, which take rows behind ctx_lens[b] from the table, would
 * find what it gave back and others hold).  owned_out and n_free_out may be owned
 * and n_free, or other arrays: as long as they are, the call may be repeated with
 * the same result.
 * ctx_lens, owned, granted, owned_out i32 [B]; n_new i32 [B] or NULL (= T_max);
 * n_free, n_free_out i32 [1]; slots i32 [B,T_max].  No workspace; one kernel, or
 * two where B * T_max is large. */
typedef struct radar_kvq_blocks_desc {
    int32_t B, T_max, max_blocks, n_blocks, block_rows;
} radar_kvq_blocks_desc;

radar_status radar_kvq_blocks(const int32_t *ctx_lens, const int32_t *n_new, int32_t *block_tables,
                              const int32_t *owned, int32_t *free_blocks, const int32_t *n_free,
                              int32_t *owned_out, int32_t *n_free_out, int32_t *slots, int32_t *granted,
                              const radar_kvq_blocks_desc *desc, void *stream);

/* N rows of keys and values into one layer's cache, row n at slots[n] (rows whose
 * slot is out of range are dropped; of two rows with the same slot either may
 * leave any of its parts there).  k, v bf16 [N,Hkv,D], D contiguous, strides in
 * elements, the same for both, 0 => dense, rows 16-byte aligned; slots i32 [N];
 * cache: the layer's first block.  N >= 0.  One kernel. */
radar_status radar_kvq_append(const void *k, const void *v, const int32_t *slots, void *cache, int64_t N,
                              int64_t stride_n, int64_t stride_h, const radar_kvq_desc *desc, void *stream);

/* The rows at slots[N] of desc->layers layers as the values they stand for; rows
 * that are not there as zeros.  k, v bf16 [layers,N,Hkv,D], dense.  One kernel. */
radar_status radar_kvq_read(const void *cache, const int32_t *slots, void *k, void *v, int64_t N,
                            const radar_kvq_desc *desc, void *stream);

/* After radar_verify_accept: in each of desc->layers layers, row ctx_lens[b] + s of
 * sequence b becomes what row ctx_lens[b] + accept_path[b,s] was, for
 * 1 <= s <= accept_len[b] (any path: all rows are read before any is written),
 * codes and scales unchanged; other rows are left as they were.
 * new_ctx_lens[b] = ctx_lens[b] + accept_len[b] + 1 (the root is kept too), or
 * ctx_lens[b] if that is negative.  accept_path i32 [B,path_len] as
 * radar_verify_accept writes it (path_len = D_max + 1); accept_len is clamped to
 * [0, path_len - 1]; entries outside [0, RADAR_T_MAX) and rows that are not there
 * are skipped.  new_ctx_lens i32 [B] or NULL; not ctx_lens itself.  Sequences
 * must not share the blocks that hold their rows from ctx_lens[b] on.
 * Limits: 1 <= path_len <= RADAR_T_MAX; B <= 65535.  One kernel. */
radar_status radar_kvq_commit(void *cache, const int32_t *block_tables, int32_t max_blocks, const int32_t *ctx_lens,
                              const int32_t *accept_len, const int32_t *accept_path, int32_t path_len, int32_t B,
                              int32_t *new_ctx_lens, const radar_kvq_desc *desc, void *stream);

/* radar_tree_attention over the paged cache in 4 bits: the same formula, with the
 * values that the codes stand for.  Rows j < ctx_lens[b] and the rows of node i's
 * ancestors and its own, ctx_lens[b] + a, that are among the first S_max and in
 * blocks that are there.  A sequence with ctx_lens[b] < 0 is not there: its rows
 * of out and lse are written as zero, as are rows i >= n_nodes[b].  Where no row is
 * allowed, out is zero and lse -inf.  A row that is not allowed has no influence,
 * whatever it holds (NaN blocks included).
 * T_max = 1 takes single tokens (so does radar_chunk_attention_kvq, which is the
 * quicker call where they see hundreds of thousands of rows between them); parents
 * == NULL: node i hangs under node i - 1 (a chain: causal attention of up to
 * RADAR_T_MAX rows).
 * cache: the layer's first block; block_tables i32 [B,max_blocks]; S_max: the rows
 * that the call is planned for, at most max_blocks * block_rows (the longest
 * ctx_lens[b] + T_max where it is known).  Other arguments and limits as for
 * radar_tree_attention; B * Hkv * ceil(Hq / Hkv * T_max / 16) < 2^23 - 7; q and out
 * 16-byte aligned rows.  One kernel, or two where units of work are divided.  The
 * workspace's counters are at its head for all shapes: one that is large enough
 * serves calls of any shape that follow each other, initialised once.  The size
 * asked for goes by B, T_max and the heads: what a program's largest B and T_max
 * ask for serves all smaller ones and any S_max. */
typedef struct radar_kvq_attn_desc {
    radar_kvq_desc cache;    /* layers and layer_stride are ignored */
    int32_t B, T_max, Hq, max_blocks, S_max;
    int32_t rows_per_split;  /* 0 => chosen by the library; else a multiple of 64: the least rows that one
                                workgroup takes before partial results are merged */
    int64_t q_stride_b, q_stride_t, q_stride_h;
    int64_t out_stride_b, out_stride_t, out_stride_h;
    float   softmax_scale;   /* 0 => 1/sqrt(D); must not be negative */
} radar_kvq_attn_desc;

size_t radar_tree_attention_kvq_workspace_bytes(const radar_kvq_attn_desc *desc);

radar_status radar_tree_attention_kvq(const void *q, const void *cache, const int32_t *block_tables,
                                      const int32_t *parents, const int32_t *ctx_lens, const int32_t *n_nodes,
                                      void *out, float *lse_out, const radar_kvq_attn_desc *desc,
                                      void *workspace, size_t workspace_bytes, void *stream);

/* --------------------------------------------------------------------------
 * Rotary positions and chunks of new tokens.  Before a sequence's first tree, and between trees where sequences come and go,
 * the target takes prompts, pieces of prompts and single tokens: a serving step over a batch makes, per layer,
 *   radar_kvq_blocks             (once) room for the new rows, and where each goes
 *   radar_kvq_append_rope        q and k turned by their positions, k and v into the cache
 *   radar_chunk_attention_kvq    every new row over its sequence's cached rows and the new ones up to itself
 * and radar_rope turns q and k for caches of any other kind.
 *
 * Rows.  A batch's new tokens are either [B,T_max] (row_starts == NULL; N = B * T_max; n_new[b] of them are there, clamped to
 * [0, T_max], all if n_new == NULL) or one sequence's behind the other's: sequence b has rows row_starts[b] ... row_starts[b+1] - 1
 * of N, at most T_max of them (row_starts i32 [B+1] on the device, never falling; n_new must be NULL then).  T_max is what the call is planned for: the longest
 * sequence's number of rows, or more.  Rows behind the last sequence, and rows of a sequence behind its T_max-th, are not there.
 *
 * radar_rope.  Row i of sequence b, row n of the tensors, has the positions p_a = positions[a][n] + ctx_lens[b] (positions == NULL: i + ctx_lens[b];
 * ctx_lens == NULL: 0 in its place) on axes a < axes: one for text, three for time, height and width of images and video.  Tree
 * nodes are rows with positions = tree_depth and ctx_lens.  With P = rotary_dim / 2, pair j < P is values (j, j + P) of a head's row, or
 * (2 j, 2 j + 1) where interleaved, and is turned by t = p * inv_freq[j], p on the axis pair_axis[j]:
 *     (x, y) -> scale * (x cos t - y sin t, x sin t + y cos t)
 * Values from rotary_dim on are copied.  Angles and turns are computed in fp64 and rounded to fp32 and then to bf16 (angles are
 * good to |t| 2^-53; beyond 2^31 radians no further promise is made).  Rows that are not there, and rows of a sequence with
 * ctx_lens[b] < 0, are left as they were.  q_out may be q, and k_out k, with the same strides; other overlaps of an output are not allowed.
 * q, q_out bf16 [N,Hq,D], k, k_out bf16 [N,Hkv,D], D contiguous, strides in elements, 0 => dense, rows 16-byte aligned; q or k may be NULL
 * with its output; positions i32 [axes,N]; inv_freq f32 [P]; n_new, ctx_lens i32 [B].  No workspace; one kernel.
 * Limits: D and rotary_dim multiples of 16, D <= 256; 1 <= axes <= 4; B <= 2^30; N / 8 * (3 + (Hq + 2 Hkv) / 8) < 2^24. */
typedef struct radar_rope_desc {
    int32_t B, T_max;
    int32_t Hq, Hkv, D;
    int32_t rotary_dim;      /* 0 => D */
    int32_t axes;
    int32_t interleaved;     /* 0: pairs (j, j + P); 1: pairs (2 j, 2 j + 1) */
    float   scale;           /* of cosines and sines; 0 => 1 */
    int64_t N;
    int64_t q_stride_n, q_stride_h, kv_stride_n, kv_stride_h;      /* kv: of k, and of v, which has the same */
    int64_t q_out_stride_n, q_out_stride_h, k_out_stride_n, k_out_stride_h;
    uint8_t pair_axis[128];  /* of pair j < P */
} radar_rope_desc;

radar_status radar_rope(const void *q, const void *k, void *q_out, void *k_out, const float *inv_freq, const int32_t *positions,
                        const int32_t *ctx_lens, const int32_t *row_starts, const int32_t *n_new, const radar_rope_desc *desc, void *stream);

/* radar_rope of q and k, and k and v into one layer's cache, as radar_rope followed by radar_kvq_append would, bit for bit:
 * row i of sequence b goes to slots[b,i] (i32 [B,T_max], as radar_kvq_blocks writes them, also where the rows are one behind the other); a
 * row whose slot is out of range, or that is not there, is not written (of two rows with the same slot either may leave any of its parts there); q is
 * turned all the same, where its row is there.  v bf16 [N,Hkv,D] with k's strides;
 * q and q_out may both be NULL; k_out's strides are ignored.  cache: the layer's first block.  desc->D and desc->Hkv are the cache's.
 * Limits: those of both calls.  No workspace; one kernel. */
radar_status radar_kvq_append_rope(const void *q, const void *k, const void *v, void *q_out, const float *inv_freq, const int32_t *positions,
                                   const int32_t *ctx_lens, const int32_t *row_starts, const int32_t *n_new, const int32_t *slots, void *cache,
                                   const radar_rope_desc *desc, const radar_kvq_desc *cache_desc, void *stream);

/* Attention of chunks of new tokens over the paged 4-bit cache, for chunks of any length (radar_tree_attention_kvq takes up to
 * RADAR_T_MAX rows of a tree).  Row i of sequence b, whose key and value are cache row ctx_lens[b] + i already, sees rows j <= ctx_lens[b] + i
 * that are among the first S_max and in blocks that are there:
 *     out[n,h,:] = softmax_j( scale * <q[n,h,:], k[j,h/G,:]> ) . v[j,h/G,:]          lse[n,h] = log sum_j exp(...)
 * Where no row is there to be seen, out is zero and lse -inf.  A row that is not seen has no influence, whatever it holds (NaN blocks
 * included).  Rows of a sequence with ctx_lens[b] < 0 are zero in out and lse, and so are rows i >= n_new[b] of [B,T_max]; rows behind the last
 * sequence of row_starts, and of a sequence behind its T_max-th, are left as they were.
 * q, out bf16 [N,Hq,D] (or [B,T_max,Hq,D]: a stride_b of its own), strides as for radar_tree_attention, stride_b ignored with row_starts; out
 * must not overlap q (the same address is refused); lse_out f32 [N,Hq] dense or NULL; block_tables i32 [B,max_blocks]; S_max: the rows
 * that the call is planned for, at most max_blocks * block_rows (the longest ctx_lens[b] + rows where it is known).
 * Limits: those of the cache; B <= 65535; N < 2^31; Hq <= 65535; the blocks of 64 of a KV head's queries, about (N * Hq / Hkv / 64 + B) * Hkv, < 2^22.
 * One kernel.  The workspace's size depends on D only, and its counters are at its head: one, initialised once, serves calls of any shape that
 * follow each other on one stream.  (row_starts that fall are not a batch: nothing outside the tensors is read or written, but the rows'
 * results are undefined, and the workspace has to be initialised again.) */
typedef struct radar_kvq_chunk_desc {
    radar_kvq_desc cache;    /* layers and layer_stride are ignored */
    int32_t B, T_max, Hq, max_blocks, S_max;
    int32_t rows_per_split;  /* 0 => chosen by the library; else a multiple of 64: cache rows that one workgroup takes, and no fewer, before
                                partial results are joined (as many as the workspace has room for; rows of fewer than four times as many
                                are not divided, nor is anything in a call of more than 512 sequences) */
    int64_t N;
    int64_t q_stride_b, q_stride_t, q_stride_h;
    int64_t out_stride_b, out_stride_t, out_stride_h;
    float   softmax_scale;   /* 0 => 1/sqrt(D); must not be negative */
} radar_kvq_chunk_desc;

size_t radar_chunk_attention_kvq_workspace_bytes(const radar_kvq_chunk_desc *desc);

radar_status radar_chunk_attention_kvq(const void *q, const void *cache, const int32_t *block_tables, const int32_t *ctx_lens,
                                       const int32_t *row_starts, const int32_t *n_new, void *out, float *lse_out, const radar_kvq_chunk_desc *desc,
                                       void *workspace, size_t workspace_bytes, void *stream);

/* Counts, per call, the nodes i < n_nodes[b] whose parent breaks the tree
 * convention; *bad_count_out (device i32) is overwritten.  parents i32
 * [B,T_max]; n_nodes i32 [B] or NULL. */
radar_status radar_debug_validate_tree(const int32_t *parents, const int32_t *n_nodes, int32_t B, int32_t T_max,
                                       int32_t *bad_count_out, void *stream);

/* --------------------------------------------------------------------------
 * Measurement support (not part of the method; for benchmarks that report
 * achieved bandwidth per kernel as the paper's Table 5 reports time per
 * stage).  Between radar_profile_begin and radar_profile_end every kernel the
 * library launches, from any thread, carries a pair of HIP events stamped
 * with the dispatch's own begin and end on the device, i.e. the duration a
 * kernel trace shows, without launch gaps or event overhead.
 *
 * radar_profile_begin(max_launches) creates max_launches event pairs (host
 * objects; 1 <= max_launches <= 2^20) and starts recording; launches beyond
 * that number run unrecorded.  radar_profile_end stops recording, waits for
 * the recorded kernels, writes one entry per kernel name into out[0..capacity)
 * (HOST memory; names beyond capacity are dropped), stores the number of
 * entries in *n_out and destroys the events.  These two calls are the only
 * ones that create or destroy anything and that synchronise.  Neither may
 * run while another thread is inside a call of this library: a launch that
 * has taken its event pair must have been issued before radar_profile_end
 * destroys the events. */
typedef struct radar_kernel_time {
    char name[48];      /* "expand", "expand_stream", "expand_finish", "rerank", "accept",
                           "accept_length_distribution", "tree_attn_group_share",
                           "tree_attn_merge", "rope", "kvq_append_rope", "kvq_chunk_64x4" (blocks of 64
                           columns, four wavefronts a workgroup), ... */
    int64_t calls;
    double total_us;
    double min_us;
    double max_us;
} radar_kernel_time;

radar_status radar_profile_begin(int32_t max_launches);
radar_status radar_profile_end(radar_kernel_time *out, int32_t capacity, int32_t *n_out);

/* Measurement support: reads `bytes` (a multiple of 16 is read; src 16-byte aligned, DEVICE
 * memory) once with 16-byte loads from every CU and keeps nothing -- the time a pure streaming
 * read of that size takes on this chip, against which the streaming kernels above (logits
 * passes, KV passes) are priced besides the nominal peak.  sink: DEVICE u32 or NULL, written
 * practically never (it only keeps the loads alive).  One kernel ("hbm_read_probe" in the
 * timing table); enqueues and returns. */
radar_status radar_probe_hbm_read(const void *src, size_t bytes, uint32_t *sink, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* RADAR_H */
