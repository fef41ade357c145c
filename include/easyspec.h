/*
 * easyspec.h — C ABI of the MI355X (gfx950) EasySpec draft-model hot path.
 *
 * What the library computes (EasySpec, arXiv 2502.02493):
 *   - easyspec_draft_step     one layer-parallel "fuzzy" forward of the draft model
 *                             (paper Alg. 2; the layer-parallel strategy of Sec. 3.1.1)
 *   - easyspec_draft_tree_step  the same fuzzy forward over one level of a token tree (App. C)
 *   - easyspec_calibrate      bonus calibration: drop the fuzzy KV entries, refill the cache
 *                             with precise values by one token-parallel, layer-sequential
 *                             forward (paper Sec. 3.2, Alg. 1)
 *   - easyspec_greedy_accept  acceptance of drafted tokens at temperature 0 (paper Alg. 3)
 *   - easyspec_accept         acceptance by speculative sampling at a temperature > 0
 *                             (paper Alg. 3, bonus distribution of Sec. 2.1)
 *   - easyspec_beam_select, easyspec_kv_reorder   the best continuations of a group of beams, and the
 *                             beams' caches in the order of their parents
 *   - easyspec_attn_weights, easyspec_kv_evict    the attention weight that cached slots receive, and a
 *                             cache thinned by it
 *   - easyspec_kvq_store, _load, _select, _attention   a cache held in 4 bits, and attention over all of it or over the
 *                             blocks of it that matter to a token
 *   - easyspec_sample         tokens drawn from logits under top-k, top-p and min-p, and the logits that stay
 *
 * Model function: pre-norm decoder with RMSNorm, rotary embedding (pairs i, i + head_dim/2),
 * grouped-query attention (query head j reads KV head j / (n_q_heads/n_kv_heads)), SwiGLU MLP,
 * untied LM head.  Storage dtype (weights and KV cache) is fp32 or bf16; the residual stream,
 * queries, softmax and all accumulators are fp32.
 *
 * Conventions
 *   - Every function returns EASYSPEC_OK (0) or a negative error code.  Arguments are checked
 *     on the host before anything is launched: a failed call leaves lengths and device memory
 *     unchanged.  easyspec_last_error() returns a message for the last failure.
 *   - "dev" pointers are device memory owned by the caller; they must stay valid until the
 *     context's stream has passed the call.  "host" pointers are ordinary host memory.
 *     "host|dev" pointers may be either.  The library never frees caller memory.
 *   - Calls are asynchronous on the stream given at creation unless stated otherwise.
 *   - A context is not thread-safe; use one thread per context.
 *   - Passes of small models run as one launch whose workgroups wait for each other's values.  Every
 *     wait is bounded; a pass that waited some seconds in vain (a device that stopped advancing it)
 *     ends, but its results and cache entries are wrong, and the call that enqueued it has long
 *     returned.  Once such a pass has ended, draft steps, calibrations, easyspec_get_lens, _truncate,
 *     _kv_import, _kv_export, _get_hidden, _beam_fork, _beam_reorder, _track_attention, _evict and
 *     _get_attn_weights return EASYSPEC_EHIP on that context and keep doing so:
 *     destroy it.  The import and export look again after their synchronisation; a program that wants
 *     to know earlier, or replays captured passes without calling the library, synchronises its
 *     stream and calls easyspec_get_lens before it uses results.
 *   - The library has no CPU fallback: without a usable HIP device easyspec_create fails.
 *   - Measurement and test hooks (per-kernel timing, the bandwidth probe, host models of the
 *     kernels' index arithmetic, workspace poisoning) are declared apart, in easyspec_instrument.h:
 *     no caller of the method needs them.
 */
#ifndef EASYSPEC_H
#define EASYSPEC_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define EASYSPEC_OK 0
#define EASYSPEC_EINVAL (-1)    /* bad argument or unsupported shape */
#define EASYSPEC_ECAPACITY (-2) /* a sequence would exceed max_ctx, or too many tokens */
#define EASYSPEC_ESTATE (-3)    /* call not valid in the current state (no weights, no live sequence, ...) */
#define EASYSPEC_EHIP (-4)      /* a HIP runtime call or an earlier pass failed; message in easyspec_last_error */

#define EASYSPEC_DTYPE_F32 0
#define EASYSPEC_DTYPE_BF16 1

#define EASYSPEC_POLICY_ALIGNED 0 /* the rule in the text of Sec. 3.1.1 */
#define EASYSPEC_POLICY_PACKED 1  /* the 16-layer row of the strategy table of Sec. 3.1.1 */

#define EASYSPEC_MAX_BATCH 16        /* sequences per context */
#define EASYSPEC_MAX_CALIB_TOKENS 16 /* tokens of one sequence per calibration call */
#define EASYSPEC_MAX_SET 8           /* layers per layer-parallel set */
#define EASYSPEC_MAX_TREE_WIDTH 16   /* nodes one easyspec_draft_tree_step call may add (all sequences together) */
#define EASYSPEC_MAX_TREE_NODES 64   /* nodes of one sequence's token tree */

typedef struct easyspec_config {
  int32_t n_layers, d_model, n_q_heads, n_kv_heads, head_dim, d_ffn, vocab;
  float rms_eps, rope_theta;
  int32_t qkv_bias;         /* 0/1: q, k, v projections carry a bias */
  int32_t dtype;            /* EASYSPEC_DTYPE_*: storage type of matrices, embedding and KV cache */
  int32_t max_batch;        /* 1..EASYSPEC_MAX_BATCH sequences */
  int32_t max_ctx;          /* KV slots per sequence (precise + fuzzy) */
  int32_t max_calib_tokens; /* 1..EASYSPEC_MAX_CALIB_TOKENS */
} easyspec_config;
/* Shape limits: head_dim is 64 or 128; d_model, n_q_heads*head_dim and d_ffn are multiples
 * of 32; n_q_heads/n_kv_heads is 1, 2, 4, 7 or 8. */

typedef struct easyspec_layer_weights {
  /* row-major [out][in] matrices in the storage dtype (bf16 = raw 16-bit patterns) */
  const void *wq; /* [n_q_heads*head_dim][d_model]  */
  const void *wk; /* [n_kv_heads*head_dim][d_model] */
  const void *wv; /* [n_kv_heads*head_dim][d_model] */
  const void *wo; /* [d_model][n_q_heads*head_dim]  */
  const void *wg; /* [d_ffn][d_model]  gate */
  const void *wu; /* [d_ffn][d_model]  up   */
  const void *wd; /* [d_model][d_ffn]  down */
  /* fp32 vectors */
  const float *bq, *bk, *bv; /* biases, NULL unless qkv_bias */
  const float *g_attn;       /* [d_model] gain of the norm before attention */
  const float *g_mlp;        /* [d_model] gain of the norm before the MLP */
} easyspec_layer_weights;

typedef struct easyspec_weights {
  const easyspec_layer_weights *layers; /* host array of n_layers entries */
  const void *embed;                    /* [vocab][d_model] storage dtype */
  const void *lm_head;                  /* [vocab][d_model] storage dtype */
  const float *g_final;                 /* [d_model] fp32 */
} easyspec_weights;

typedef struct easyspec_ctx easyspec_ctx; /* opaque: owns its weight copy, KV cache and workspaces */

/* Create a context on the current HIP device.  hip_stream: a hipStream_t (NULL = the default
 * stream) on which every later call is ordered.  Allocates the packed weight arrays, the KV
 * cache ([layer][sequence][kv_head][slot][head_dim], K and V apart) and the workspaces; the
 * rotary table is computed on the host in double precision.  Starts with every layer in a set
 * of its own (plain sequential order, paper Alg. 1).  *out is NULL on failure. */
int easyspec_create(const easyspec_config *cfg, void *hip_stream, easyspec_ctx **out);

/* Frees everything the context owns (synchronises its stream first).  NULL is allowed. */
void easyspec_destroy(easyspec_ctx *ctx);

/* Copy the parameters into the context, repacked into the library's streaming layout: per
 * operation one layer-major array, so that the layers of any set are one contiguous range.
 * Every pointer inside src is host|dev; the caller keeps src.  Synchronous. */
int easyspec_load_weights(easyspec_ctx *ctx, const easyspec_weights *src);

/* Layer-parallel strategy (Sec. 3.1.1: the strategy is a configuration choice, no retraining).
 * bounds (host): bounds[0] = 0 < bounds[1] < ... < bounds[n_sets] = n_layers; set j is the
 * layers [bounds[j], bounds[j+1]), at most EASYSPEC_MAX_SET of them.  Only fuzzy steps use it. */
int easyspec_set_groups(easyspec_ctx *ctx, const int32_t *bounds, int32_t n_sets);

/* Boundaries of the paper's strategy for layer-parallel size N: first and last layer alone,
 * the layers between cut into N-sets (policy: see EASYSPEC_POLICY_*).  bounds (host) must hold
 * n_layers + 1 entries; *n_sets receives the number of sets.  Pure host function. */
int easyspec_default_groups(int32_t n_layers, int32_t N, int32_t policy, int32_t *bounds, int32_t *n_sets);

/* What the layers of a set share in fuzzy steps (easyspec_draft_step, easyspec_draft_tree_step).
 *   EASYSPEC_PARALLEL_ATTENTION (default)  Alg. 2: the attention layers of a set read the set's
 *       input; the MLPs run in layer order on the running residual.
 *   EASYSPEC_PARALLEL_FULL_LAYER  the ablation of App. B: attention AND MLP of every layer of the
 *       set work from the set's input h_1: a_i = Attn_i(h_1), m_i = MLP_i(h_1 + a_i),
 *       output = h_1 + sum_i (a_i + m_i).  The paper reports this variant as worse and does not
 *       define it; this is the reading "each layer of the set runs whole from the same input".
 * Sets of one layer are Alg. 1 in both modes.  Calibration is unaffected.  EASYSPEC_EINVAL for
 * an unknown mode. */
#define EASYSPEC_PARALLEL_ATTENTION 0
#define EASYSPEC_PARALLEL_FULL_LAYER 1
int easyspec_set_parallel_mode(easyspec_ctx *ctx, int32_t mode);

/* One fuzzy forward (Alg. 2) for every live sequence (precise length > 0), one token each.
 *   tokens_in  dev [max_batch]  token fed to sequence b (ignored for idle sequences)
 *   tokens_out dev [max_batch]  argmax of the logits, lowest index on ties (idle: untouched)
 *   logits_out dev [max_batch][vocab] fp32, or NULL
 * For each set, every attention layer of the set reads the hidden state entering the set and
 * stores the k, v it computes from it in slot precise+fuzzy; the MLPs run in layer order.
 * Afterwards fuzzy[b] += 1.  EASYSPEC_ESTATE if no sequence is live, EASYSPEC_ECAPACITY if a
 * live sequence is full. */
int easyspec_draft_step(easyspec_ctx *ctx, const int32_t *tokens_in, int32_t *tokens_out, float *logits_out);

/* One fuzzy forward (Alg. 2) over one level of a token tree (Sec. 3.1 last paragraph, App. C):
 * the drafted tokens of a sequence form a tree, every root-to-node path being one candidate
 * sequence; common prefixes share their KV entries and a node attends to the precise context,
 * its ancestors and itself (its row of the 2-D tree mask).  How the tree is grown (which tokens
 * become children of which node) is the caller's policy; the paper fixes none.
 *   tokens_in   dev  [max_batch][EASYSPEC_MAX_TREE_WIDTH]  tokens of the new nodes of sequence b
 *   n_nodes     host [max_batch]  number of new nodes of b, 0 = none; at most
 *                    EASYSPEC_MAX_TREE_WIDTH over all sequences
 *   parents     host [max_batch][EASYSPEC_MAX_TREE_WIDTH]  parent of new node j: a node index of b's
 *                    tree as it stood before the call (nodes are numbered in the order they were
 *                    added, 0 .. fuzzy[b]-1), or -1 = child of the last precise token
 *   tokens_out  dev  [max_batch][EASYSPEC_MAX_TREE_WIDTH]  argmax after each new node
 *   logits_out  dev  fp32 [max_batch][EASYSPEC_MAX_TREE_WIDTH][vocab] or NULL (for top-k children)
 * New node j of b takes slot precise[b] + fuzzy[b] + j in every layer (its k, v are those of the
 * fuzzy forward) and rotary position precise[b] + depth, depth = 0 for children of the last precise
 * token.  Afterwards fuzzy[b] += n_nodes[b].  A tree whose every node is the child of the previous
 * one is chain drafting.  Trees and easyspec_draft_step do not mix between two calibrations:
 * EASYSPEC_ESTATE if b holds chain-drafted slots (and easyspec_draft_step refuses a sequence that
 * holds a tree).  EASYSPEC_ECAPACITY beyond EASYSPEC_MAX_TREE_NODES nodes, max_ctx slots or the
 * per-call width; EASYSPEC_EINVAL for a parent that is not an earlier node.  Calibration drops
 * the whole tree like any fuzzy slots. */
int easyspec_draft_tree_step(easyspec_ctx *ctx, const int32_t *tokens_in, const int32_t *n_nodes, const int32_t *parents,
                             int32_t *tokens_out, float *logits_out);

/* Bonus calibration (Sec. 3.2) of the sequences with n_tokens[b] > 0; also the prompt prefill
 * (repeat in chunks of max_calib_tokens).
 *   tokens         dev  [max_batch][max_calib_tokens]  accepted tokens followed by the bonus token
 *   n_tokens       host [max_batch]  0 = leave sequence b alone, else 1..max_calib_tokens
 *   next_token_out dev  [max_batch]  argmax after the last token of b (untouched if n_tokens[b]=0)
 *   logits_out     dev  fp32 or NULL: logits_rows = 0 -> [max_batch][vocab] (last token of each);
 *                  logits_rows = 1 -> [max_batch][max_calib_tokens][vocab] (every token)
 * For each such sequence: fuzzy[b] = 0 (all fuzzy slots dropped, accepted or not); layers run
 * in order over the n tokens at positions precise[b] .. precise[b]+n-1, causal among themselves;
 * their k, v overwrite those slots; precise[b] += n.
 * Up to 16 tokens in all are one forward pass of 16 token columns.  More tokens: a bf16 model runs them as one wide
 * pass, every weight matrix read once; an fp32 model packs the sequences in index order into passes of 16 columns, a
 * sequence's tokens staying together, and two consecutive passes of equal column counts run together, each weight
 * matrix being read once for both.  The results depend on the packing by the order of fp32 sums only: the last bits in
 * an fp32 model.  In a bf16 model a last bit can round a cache entry to the neighbouring bf16 value, which the layers
 * that follow carry on, so a sequence's logits and cache can differ by such roundings with how many tokens the other
 * sequences bring (8B shape: a few 1e-4 in relative 2-norm, as far as either is from a 64-bit evaluation). */
int easyspec_calibrate(easyspec_ctx *ctx, const int32_t *tokens, const int32_t *n_tokens,
                       int32_t *next_token_out, float *logits_out, int32_t logits_rows);

/* Greedy acceptance (Alg. 3 with one-hot distributions): accept_len[b] = number of leading
 * positions where draft equals target_argmax; bonus[b] = target_argmax[b][accept_len[b]].
 *   draft [batch][gamma], target_argmax [batch][gamma+1], accept_len [batch], bonus [batch]
 * easyspec_greedy_accept: all four are dev arrays; one small kernel is launched on hip_stream (a
 * hipStream_t, NULL = the null stream, as everywhere in this header) and nothing is synchronised,
 * so the call is ordered with the draft steps that wrote `draft` on the same stream.
 * EASYSPEC_EINVAL for NULL pointers, batch < 1, gamma < 0, or an accept_len that is not device
 * memory (host arrays belong to the _host variant); EASYSPEC_EHIP without a HIP device.
 * easyspec_greedy_accept_host: all four are host arrays; a plain host loop, no device needed. */
int easyspec_greedy_accept(const int32_t *draft, const int32_t *target_argmax, int32_t batch, int32_t gamma,
                           int32_t *accept_len, int32_t *bonus, void *hip_stream);
int easyspec_greedy_accept_host(const int32_t *draft, const int32_t *target_argmax, int32_t batch, int32_t gamma,
                                int32_t *accept_len, int32_t *bonus);

/* Acceptance by speculative sampling (Alg. 3; Sec. 2.1) of `batch` sequences, in double
 * precision on the device, with the random numbers supplied by the caller.
 *   draft          dev [batch][gamma]            drafted tokens x'_i
 *   draft_logits   dev [batch][gamma][vocab]     fp32; p'_i = softmax(draft_logits[i] / temperature)
 *   target_logits  dev [batch][gamma+1][vocab]   fp32; p_i  = softmax(target_logits[i] / temperature)
 *   r              dev [batch][gamma]            uniforms in [0,1): position i is rejected when
 *                                                r_i > p_i(x'_i) / p'_i(x'_i)
 *   u              dev [batch]                   uniform in [0,1) for the bonus draw
 *   accept_len     dev [batch]  m = index of the first rejected position, or gamma
 *   bonus          dev [batch]  drawn from max(0, p_m - p'_m) normalised if m < gamma (the distributions
 *                               at the first rejected position), from p_gamma otherwise: the lowest token v
 *                               whose running sum over tokens 0..v exceeds u times the total
 *   workspace      dev, easyspec_accept_workspace_bytes(batch, gamma, vocab) bytes, 8-byte aligned
 *                  (about 8 bytes per vocabulary entry and sequence; statistics, sums and counters
 *                  take the smaller part of them); contents need not be kept between calls.  One call
 *                  at a time: the kernels hand values to each other through it, and of calls that overlap
 *                  on it (different streams or threads) some results are wrong, -1, or not written
 *   hip_stream     the hipStream_t to launch on (NULL = the null stream); nothing is synchronised
 * gamma may be 0 (plain sampling from p_0).  A drafted token outside 0..vocab-1 at or before
 * the first rejected position gives accept_len = bonus = -1 for that sequence; so does a value of
 * another workgroup that has not come after a quarter of a second, which only calls that overlap
 * on the workspace bring about (no call waits without end).  EASYSPEC_EINVAL for NULL pointers, batch < 1 or
 * > 65535, gamma outside 0..64, vocab < 1, or a temperature that is not positive and finite
 * (temperature 0 is easyspec_greedy_accept).  All arrays are the caller's and only read,
 * except accept_len, bonus and workspace. */
int easyspec_accept(const int32_t *draft, const float *draft_logits, const float *target_logits, const float *r,
                    const float *u, int32_t batch, int32_t gamma, int32_t vocab, float temperature,
                    int32_t *accept_len, int32_t *bonus, void *workspace, void *hip_stream);
int64_t easyspec_accept_workspace_bytes(int32_t batch, int32_t gamma, int32_t vocab); /* -1 for bad arguments */

/* easyspec_accept for callers that cannot allocate device memory and have no workspace to hand in
 * (code under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc): same
 * arguments, same kernels and same results, but the workspace is the library's own fixed device
 * array of easyspec_accept_static_max_bytes() bytes (8 MiB; every GPU the library runs on holds one
 * until the process ends).  The call allocates and frees nothing.  EASYSPEC_ECAPACITY, with nothing
 * launched, when easyspec_accept_workspace_bytes(batch, gamma, vocab) exceeds that size (about 8
 * bytes per vocabulary entry and sequence: 6 sequences at a vocabulary of 152 064); other errors as
 * easyspec_accept.  All calls on one GPU share the array, so two calls whose kernels can overlap
 * (different streams, different threads) race, with the results easyspec_accept's workspace names: keep
 * them on one stream, or order them yourself. */
int easyspec_accept_static(const int32_t *draft, const float *draft_logits, const float *target_logits, const float *r,
                           const float *u, int32_t batch, int32_t gamma, int32_t vocab, float temperature,
                           int32_t *accept_len, int32_t *bonus, void *hip_stream);
int64_t easyspec_accept_static_max_bytes(void);

/* ---- Drafting with beams ------------------------------------------------------------------------------------ */

#define EASYSPEC_MAX_BEAMS 64        /* beams of one group */
#define EASYSPEC_MAX_SELECT 64       /* continuations one easyspec_beam_select call picks per group */
#define EASYSPEC_MAX_BEAM_VOCAB 1048576

/* The n_select best continuations of every group of beams, over all its beams and the whole vocabulary:
 *   score(w, v) = scores[w] + logits[w][v] / temperature - log sum_u exp(logits[w][u] / temperature)
 * in descending order; of equal scores the lowest beam comes first, of one beam's candidates the highest logit, of equal
 * logits the lowest token.  Scores are compared in double precision.
 *   logits      dev [groups][beams][vocab]  fp32, as easyspec_draft_step and easyspec_draft_tree_step write them
 *   scores      dev [groups][beams]         fp32, cumulative log-probability of the beam; a beam of minus infinity (or NaN) offers
 *                                           no continuation and its logits are not read
 *   ended       dev [groups][beams] or NULL nonzero: the beam has ended; it offers one continuation, end_token, at its own
 *                                           score, and its logits are not read
 *   tokens_out  dev [groups][n_select]      the token; -1 where a group has fewer continuations than n_select
 *   parents_out dev [groups][n_select]      the beam it continues, 0..beams-1, or -1
 *   scores_out  dev [groups][n_select]      fp32, or minus infinity; may be `scores` if n_select == beams
 *   workspace   dev, easyspec_beam_select_workspace_bytes() bytes, 16-byte aligned; one call at a time; contents need not be kept.  A call of
 *               other sizes, smaller ones among them, may need more
 *   hip_stream  the hipStream_t to launch on (NULL = the null stream); nothing is synchronised
 * Logits of minus infinity and NaN are no continuations and add nothing to the sum; a beam with a logit of plus infinity, or
 * with none that is finite, offers nothing.  A beam selection over sequences 0..beams-1 of a context takes the logits of a
 * draft step as they are; over the nodes of a tree level, beams is EASYSPEC_MAX_TREE_WIDTH and the scores of unused rows are
 * minus infinity.  EASYSPEC_EINVAL for NULL pointers, groups or vocab < 1, groups * beams > 65535, beams, n_select or vocab
 * beyond the limits above, an end_token outside the vocabulary if `ended` is given, a temperature that is not positive and
 * finite, scores and scores_out that overlap otherwise, outputs or a workspace that overlap an input or each other, or arrays that
 * are not memory of the current device. */
int easyspec_beam_select(const float *logits, const float *scores, const int32_t *ended, int32_t groups, int32_t beams, int32_t vocab,
                         int32_t n_select, float temperature, int32_t end_token, int32_t *tokens_out, int32_t *parents_out,
                         float *scores_out, void *workspace, void *hip_stream);
int64_t easyspec_beam_select_workspace_bytes(int32_t groups, int32_t beams, int32_t vocab, int32_t n_select); /* -1 for bad arguments */

/* Caches of the caller, as a context holds them: K and V apart, [n_layers][n_seqs][n_kv_heads][max_slots][head_dim] in dtype,
 * contiguous, 16-byte aligned; n_layers * n_seqs * n_kv_heads < EASYSPEC_MAX_CACHE_ROWS. */
#define EASYSPEC_MAX_CACHE_ROWS 4194304
typedef struct easyspec_kv_layout {
  int32_t n_layers;
  int32_t n_seqs;     /* 1..EASYSPEC_MAX_BATCH */
  int32_t n_kv_heads;
  int32_t max_slots;  /* 1..65536 */
  int32_t head_dim;   /* 64 or 128 */
  int32_t dtype;      /* EASYSPEC_DTYPE_* */
} easyspec_kv_layout;

/* Beams' caches in the order of their parents.  The sequences are groups of `beams` (which divides n_seqs); in every layer and
 * KV head, sequence i of k_out, v_out receives the slots [from_slot, to_slot) of sequence
 * i - i % beams + parents[i] of k, v.  A parent outside 0..beams-1 (easyspec_beam_select's -1) stands for the sequence itself.
 *   k, v, k_out, v_out  dev  k_out == k and v_out == v (in place) or arrays apart from both
 *   parents             dev [n_seqs]
 * Other slots of k_out, v_out are left as they were.  Launched on hip_stream, nothing is synchronised.  EASYSPEC_EINVAL for
 * NULL pointers, a bad layout or slot range, beams that do not divide n_seqs, caches that overlap in part or are not 16-byte
 * aligned, parents inside k_out or v_out, or arrays that are not memory of the current device. */
int easyspec_kv_reorder(const void *k, const void *v, const easyspec_kv_layout *layout, const int32_t *parents, int32_t beams,
                        int32_t from_slot, int32_t to_slot, void *k_out, void *v_out, void *hip_stream);

/* The same on a context whose sequences are beams.
 * easyspec_beam_fork: sequences first .. first + count - 1 become copies of sequence `source` (which may be one of them): cache,
 * lengths, token tree, tracked weights.  One prompt is calibrated once and forked into its beams.  EASYSPEC_ESTATE if `source` is idle.
 * easyspec_beam_reorder: sequence first + i takes the slots from from_slot on of sequence first + parents[i]; parents: dev
 * [count], as easyspec_beam_select writes them for one group, -1 (or anything outside 0..count-1) = its own.  The slots below
 * from_slot are taken to be common to the beams: their precise length, as a rule, after which only drafted slots move.  The
 * sequences have to be of one length, precise and fuzzy, and without token trees: EASYSPEC_ESTATE otherwise.  Works in place.
 * Neither synchronises: draft step, selection and reordering of one beam search need no look at the host in between. */
int easyspec_beam_fork(easyspec_ctx *ctx, int32_t source, int32_t first, int32_t count);
int easyspec_beam_reorder(easyspec_ctx *ctx, int32_t first, int32_t count, const int32_t *parents, int32_t from_slot);

/* ---- Bounded caches ----------------------------------------------------------------------------------------- */

/* The attention weight that cached slots receive from new tokens: in every layer and KV head,
 *   weights_out[s] = weights_in[s] + sum over the sequence's new tokens and the query heads of the KV head of
 *                    softmax_s(q . k_s / sqrt(head_dim))
 * The new tokens of sequence b, n_tokens[b] of them, are its last: token t sits in slot lens[b] - n_tokens[b] + t and attends
 * to the slots up to its own (causal, as a calibration).
 *   q            dev fp32 [n_layers][sum of n_tokens][n_q_heads][head_dim]  rotated queries, sequences in index order
 *   k            dev      layout (keys with the new tokens' among them)
 *   n_tokens     host [n_seqs]  0..EASYSPEC_MAX_CALIB_TOKENS; 0: the sequence is left alone
 *   lens         host [n_seqs]  slots with the new tokens', n_tokens..max_slots
 *   n_q_heads    n_kv_heads times 1, 2, 4, 7 or 8
 *   weights_in   dev fp32 [n_layers][n_seqs][n_kv_heads][max_slots], read up to the new tokens' slots, which start from zero;
 *                NULL: zeros
 *   weights_out  dev, the same shape; slots from lens[b] on are left as they were; may be weights_in
 *   workspace    dev, easyspec_attn_weights_workspace_bytes() bytes, 16-byte aligned; one call at a time.  That is what this call needs: a
 *                call with other n_tokens or lens, shorter ones among them, may need more
 * The same call gives the same bits.  How the contexts are cut goes by the longest of the call and by its most query rows, so in the
 * last bits a sequence's weights may differ with the other sequences of the call.
 * Launched on hip_stream, nothing is synchronised.  EASYSPEC_EINVAL for NULL pointers (q and workspace may be NULL if no sequence
 * has new tokens), a bad layout, counts or lengths, weights_in and weights_out that overlap in part, weights_out or a workspace that
 * overlaps q, k or each other, a workspace that overlaps weights_in, arrays that are not 16-byte aligned (weights: 4) or not memory
 * of the current device. */
int easyspec_attn_weights(const float *q, const void *k, const easyspec_kv_layout *layout, const int32_t *n_tokens, const int32_t *lens,
                          int32_t n_q_heads, const float *weights_in, float *weights_out, void *workspace, void *hip_stream);
int64_t easyspec_attn_weights_workspace_bytes(const easyspec_kv_layout *layout, const int32_t *n_tokens, const int32_t *lens,
                                              int32_t n_q_heads); /* -1 for bad arguments */

/* A cache thinned: of sequence b min(keep[b], lens[b]) slots stay, in every layer and KV head its own: the last
 * min(recent, keep[b]) and, of the slots before them, the heaviest (of equal weights the lowest slot; a NaN is lighter than any
 * number).  They keep their order: slot j of the result is the j-th of the slots that stayed.
 *   k, v         dev layout
 *   weights      dev fp32 [n_layers][n_seqs][n_kv_heads][max_slots]
 *   lens, keep   host [n_seqs], 0..max_slots and >= 0; nothing is done for a sequence of which nothing stays
 *   out_slots    max_slots of the results, 1..65536
 *   k_out, v_out dev, the layout with out_slots; k_out == k, v_out == v and weights_out == weights with
 *                out_slots == max_slots (in place), or arrays apart from all inputs
 *   weights_out  dev fp32 [n_layers][n_seqs][n_kv_heads][out_slots]  the weights of the slots that stayed
 *   slots_out    dev [n_layers][n_seqs][n_kv_heads][out_slots]       which they were
 * Results from a sequence's last slot on are left as they were.  Keys keep the rotary positions that they were written with.
 * Launched on hip_stream, nothing is synchronised.  EASYSPEC_EINVAL for NULL pointers, a bad layout or lengths, more slots to
 * stay than out_slots, arrays that overlap in part or are not 16-byte aligned (weights, slots: 4), or not memory of the
 * current device. */
int easyspec_kv_evict(const void *k, const void *v, const float *weights, const easyspec_kv_layout *layout, const int32_t *lens,
                      const int32_t *keep, int32_t recent, int32_t out_slots, void *k_out, void *v_out, float *weights_out,
                      int32_t *slots_out, void *hip_stream);

/* The same on a context: drafting with a cache of bounded length.
 * easyspec_track_attention: from now on every calibration adds the attention weights of its tokens (easyspec_attn_weights; fuzzy
 * forwards add none) to the context's, one per layer, sequence, KV head and precise slot; slots filled before, by
 * easyspec_kv_import or by a calibration, start from zero.  Passes of such calibrations are separate launches also where a
 * small model's would be one.  max_positions: how far sequences may get, evicted slots counted (max_ctx ..
 * EASYSPEC_MAX_POSITIONS; max_ctx without this call).  Synchronous; EASYSPEC_ESTATE the second time.  A call that fails leaves the
 * context as it was.
 * easyspec_evict: of every sequence with 0 < keep[b] < precise[b] (keep: host [max_batch]; -1 leaves a sequence alone) keep[b]
 * precise slots stay, chosen as easyspec_kv_evict does in every layer and KV head, and move together; its fuzzy slots are dropped.
 * Afterwards precise[b] = keep[b].  Later tokens take the next free slots and go on at the next positions.  In place, on the
 * context's stream, not synchronised.  EASYSPEC_ESTATE if attention is not tracked.
 * easyspec_truncate refuses (EASYSPEC_ESTATE) to cut into the slots below the run of most recent ones that an eviction kept.
 * What stays after a cut keeps its weights as they are: those that the tokens cut off gave to earlier slots are in them, and the
 * tokens calibrated in their place add theirs.  (A calibration of tokens that are known to be accepted leaves nothing to cut off.)
 * easyspec_get_evicted: host [max_batch], the slots of each sequence evicted so far (precise + fuzzy + evicted = its position).
 * easyspec_get_attn_weights: the weights of the first n_slots precise slots of sequence b, host|dev fp32
 * [n_layers][n_kv_heads][n_slots].  Synchronous. */
#define EASYSPEC_MAX_POSITIONS 1048576
int easyspec_track_attention(easyspec_ctx *ctx, int32_t max_positions);
int easyspec_evict(easyspec_ctx *ctx, const int32_t *keep, int32_t recent);
int easyspec_get_evicted(const easyspec_ctx *ctx, int32_t *evicted);
int easyspec_get_attn_weights(easyspec_ctx *ctx, int32_t b, float *out, int32_t n_slots);

/* ---- Caches held in 4 bits ---------------------------------------------------------------------------------- */

/* K and V of a long context at 4.25 bits a value.  32 neighbouring channels of a slot share a scale, a power of two:
 *   E = max(floor(log2(largest magnitude of the 32)) - 2, -120), scale byte E + 127;
 *   code of x: the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 to |x| / 2^E (half-way: the even code; 6 above), with x's sign in bit 3
 * (E2M1 elements and E8M0 scales of the OCP microscaling formats).  A scale byte of 255 stands for 32 values of NaN: it is
 * what 32 channels with one that is not finite become.  Values of 4 bits are bf16 and fp32 numbers: nothing is rounded on the way back.
 * Slots are counted in blocks of EASYSPEC_KVQ_BLOCK; bounds hold every channel's lowest and highest key of a block. */
#define EASYSPEC_KVQ_BLOCK 64
#define EASYSPEC_MAX_KVQ_SELECT 1024 /* blocks of one list */
typedef struct easyspec_kvq { /* a host struct of dev arrays, contiguous, for an easyspec_kv_layout */
  void *k_codes, *v_codes;   /* [n_layers][n_seqs][n_kv_heads][max_slots][head_dim / 2] bytes, channel 2 i in the low half of byte i; 16-byte aligned */
  void *k_scales, *v_scales; /* [n_layers][n_seqs][n_kv_heads][max_slots][head_dim / 32] bytes */
  void *k_bounds;            /* bf16 [n_layers][n_seqs][n_kv_heads][ceil(max_slots / 64)][2][head_dim], 16-byte aligned; or NULL: none are kept */
} easyspec_kvq;

/* Slots brought into such a cache: of sequence b, slots src_from[b] .. src_from[b] + n_slots[b] - 1 of k, v become its slots from to[b] on.
 *   k, v      dev  [n_layers][n_seqs][n_kv_heads][src_slots][head_dim] in layout->dtype, 16-byte aligned: a cache, one that
 *                  easyspec_kv_export filled (n_seqs = 1, src_slots its n_slots), or the new tokens' keys and values
 *   src_from, n_slots, to   host [n_seqs]; n_slots[b] = 0: the sequence is left alone, its entries of the other arrays
 *                  (lens too) are not looked at
 *   lens      host [n_seqs]  slots that the sequence holds after the call, to[b] + n_slots[b] .. max_slots
 * k_bounds: those of every block that receives a slot become the bounds of its slots below lens[b], those that were there among
 * them (NaN is passed over; plus and minus infinity where nothing else is).  A sequence that is cut back keeps, in the block that the cut is in, bounds that cover the slots
 * cut off too, until a slot is stored in that block.  Launched on hip_stream, nothing is synchronised.  EASYSPEC_EINVAL for NULL pointers,
 * a bad layout, src_slots outside 1..65536, slots outside 0..src_slots or 0..lens[b] or lens outside 0..max_slots, arrays that overlap,
 * are not aligned or not memory of the current device. */
int easyspec_kvq_store(const void *k, const void *v, const easyspec_kv_layout *layout, int32_t src_slots, const int32_t *src_from,
                       const int32_t *n_slots, const int32_t *to, const int32_t *lens, const easyspec_kvq *cache, void *hip_stream);

/* The values that slots of such a cache stand for: slots from[b] .. from[b] + n_slots[b] - 1 of sequence b become the slots from to[b] on of
 * k_out, v_out: dev [n_layers][n_seqs][n_kv_heads][out_slots][head_dim] in layout->dtype.  Other slots are left as they were.  Host arrays,
 * launch and refusals as above. */
int easyspec_kvq_load(const easyspec_kvq *cache, const easyspec_kv_layout *layout, const int32_t *from, const int32_t *n_slots, int32_t out_slots,
                      const int32_t *to, void *k_out, void *v_out, void *hip_stream);

/* Attention of new tokens over a cache held in 4 bits: in every layer and query head
 *   out = sum over slots s of softmax_s(q . k_s / sqrt(head_dim)) v_s
 * The new tokens of sequence b, n_tokens[b] of them, are its last (their slots stored): token t sits in slot lens[b] - n_tokens[b] + t and
 * attends to the slots up to its own.  What a slot holds that a token does not see has no effect on it, values that are not finite among them.
 * Everything is as exact as fp32 arithmetic (queries to 2^-24 of the largest magnitude of their 32 neighbouring channels) while the largest magnitude of V
 * times the slots that a token sees is below 2^119 (V below 2^103: whatever the length); beyond that a result may be infinite or NaN.  Weights below 2^-126 of the highest
 * may count as 0.  A query with a channel that is not finite has NaN as its results.
 *   q            dev fp32 [n_layers][sum of n_tokens][n_q_heads][head_dim]  rotated queries, sequences in index order
 *   n_tokens     host [n_seqs]  0..EASYSPEC_MAX_CALIB_TOKENS
 *   lens         host [n_seqs]  slots with the new tokens', n_tokens..max_slots; not looked at where n_tokens is 0
 *   n_q_heads    n_kv_heads times 1, 2, 4, 7 or 8, 65535 at most
 *   blocks       dev [n_layers][sum of n_tokens][n_kv_heads][n_blocks], or NULL: every slot.  The blocks of EASYSPEC_KVQ_BLOCK slots that
 *                a token reads, ascending: an entry that is not above the entry in front of it (the first: above -1), or that names a
 *                block without a slot that the token sees, is passed over.  As easyspec_kvq_select writes them.
 *   n_blocks     1..EASYSPEC_MAX_KVQ_SELECT; 0 without blocks
 *   out          dev fp32, the shape of q; zeros where a token sees no slot of its blocks, or none whose score is above minus infinity
 *   workspace    dev, easyspec_kvq_attention_workspace_bytes() bytes, 16-byte aligned; one call at a time; contents need not be kept; what a
 *                call does not need of it is not looked at
 * The same call gives the same bits; how contexts are cut goes by all sequences of the call, so that in the last bits a sequence's results
 * may differ with the others.  k_bounds is not read.  Launched on hip_stream, nothing is synchronised.  EASYSPEC_EINVAL for NULL pointers (q, out and workspace may be NULL if no
 * sequence has new tokens), a bad layout, counts or lengths, out or a workspace that overlaps another array, arrays that are not 16-byte aligned (scales: 1,
 * blocks: 4) or not memory of the current device. */
int easyspec_kvq_attention(const float *q, const easyspec_kvq *cache, const easyspec_kv_layout *layout, const int32_t *n_tokens, const int32_t *lens,
                           int32_t n_q_heads, const int32_t *blocks, int32_t n_blocks, float *out, void *workspace, void *hip_stream);
int64_t easyspec_kvq_attention_workspace_bytes(const easyspec_kv_layout *layout, const int32_t *n_tokens, const int32_t *lens, int32_t n_q_heads,
                                               int32_t n_blocks); /* -1 for bad arguments */
/* A workspace of _workspace_bytes() for some lens and n_blocks holds every call with the same layout, n_tokens and n_q_heads whose lens are no
 * longer, and n_blocks (if not 0) no more.  Across n_tokens, and between calls with and without lists, it may rise or fall: _workspace_limit() holds every
 * call on the layout with up to max_tokens (1..EASYSPEC_MAX_CALIB_TOKENS) new tokens of a sequence, without lists or with lists of up to max_blocks (0: without only). */
int64_t easyspec_kvq_attention_workspace_limit(const easyspec_kv_layout *layout, int32_t max_tokens, int32_t n_q_heads, int32_t max_blocks); /* -1 for bad arguments */

/* The blocks that matter to a new token, for every layer and KV head: of the blocks that hold a slot it sees, the first keep_first, the last
 * keep_last and, of the others, those with the highest
 *   score(j) = max over the query heads of the KV head of  sum over channels d of  q_d hi_jd where q_d > 0, q_d lo_jd elsewhere,
 * which no q . k_s of the block exceeds: n_select in all, or all there are.  A block without a number in some channel (lo plus, hi minus infinity: every
 * q . k_s is NaN) thus has a score of minus infinity or NaN and goes behind all others.  Of equal scores the lowest block goes first, a score of NaN (passed
 * over where another query head has a number) last; scores are compared in double precision.  If n_select < keep_first + keep_last the
 * lowest of those stay.
 *   k_bounds     dev       as easyspec_kvq_store keeps them
 *   q, n_tokens, lens, n_q_heads   as above
 *   keep_first, keep_last  >= 0; with keep_last >= 1 the token's own block is read
 *   n_select     1..EASYSPEC_MAX_KVQ_SELECT
 *   blocks_out   dev [n_layers][sum of n_tokens][n_kv_heads][n_select]  ascending, then -1
 *   workspace    dev, easyspec_kvq_select_workspace_bytes() bytes, 16-byte aligned; one call at a time; contents need not be kept
 * Launched on hip_stream, nothing is synchronised; refusals as above. */
int easyspec_kvq_select(const float *q, const void *k_bounds, const easyspec_kv_layout *layout, const int32_t *n_tokens, const int32_t *lens,
                        int32_t n_q_heads, int32_t keep_first, int32_t keep_last, int32_t n_select, int32_t *blocks_out, void *workspace,
                        void *hip_stream);
int64_t easyspec_kvq_select_workspace_bytes(const easyspec_kv_layout *layout, const int32_t *n_tokens, const int32_t *lens, int32_t n_q_heads,
                                            int32_t n_select); /* -1 for bad arguments */

/* ---- Drafting by sampling ----------------------------------------------------------------------------------- */

#define EASYSPEC_MAX_SAMPLE_VOCAB 1048576

/* Tokens drawn from logits, and the logits that stay.  The words of a row stand in the order of their logits, the highest first, of equal
 * ones the lowest token; logits of minus infinity and NaN are no words.  With weights w_v = exp((logits[v] - highest) / temperature), those stay that are
 *   among the first top_k                                        (0: all)
 *   and have in front of them less than top_p of the weight of the first top_k   (1: all)
 *   and weigh at least min_p                                     (0: all; the first word weighs 1)
 * so that the first always does.  The token drawn is the first in that order whose running weight exceeds u times the weight of all that stay.
 *   logits      dev [rows][vocab]  fp32, as easyspec_draft_step writes them
 *   u           dev [rows]         uniform in [0,1) (1 or more, or NaN: the last word with a weight); not read without tokens_out
 *   tokens_out  dev [rows] or NULL: none is drawn; -1 for a row that holds plus infinity or no word
 *   logits_out  dev [rows][vocab] or NULL: the logits that stay, minus infinity for the others (all of them in a row without a token); may be
 *               logits.  softmax(logits_out / temperature) is what the token was drawn from: what easyspec_accept takes as draft_logits
 *               and, of the target's logits filtered alike, as target_logits
 *   workspace   dev, easyspec_sample_workspace_bytes() bytes, 16-byte aligned; one call at a time; contents need not be kept.  Fewer rows or words
 *               never need more
 *   hip_stream  the hipStream_t to launch on (NULL = the null stream); nothing is synchronised
 * Weights are worked out in double precision (to 2.2e-13) and kept as whole multiples of 2^-s, s = 62 - ceil(log2(vocab)) and 51 at most (45 at
 * 128 256 words), below 2^-48 as 0: sums of them are exact, so results do not depend on their order, and a decision can differ from that of the real numbers only
 * within about vocab 2^-s of its border.  EASYSPEC_EINVAL for NULL logits or
 * workspace, neither output, tokens_out without u, rows outside 1..65535, vocab outside 1..EASYSPEC_MAX_SAMPLE_VOCAB, a temperature that is
 * not positive and finite (temperature 0 is the argmax that the draft step writes), top_k < 0, top_p outside (0, 1], min_p outside [0, 1],
 * arrays that overlap otherwise or are not memory of the current device. */
int easyspec_sample(const float *logits, const float *u, int32_t rows, int32_t vocab, float temperature, int32_t top_k, float top_p, float min_p,
                    int32_t *tokens_out, float *logits_out, void *workspace, void *hip_stream);
int64_t easyspec_sample_workspace_bytes(int32_t rows, int32_t vocab); /* -1 for bad arguments */

/* Host copies of the per-sequence lengths; each of precise, fuzzy: host [max_batch] or NULL. */
int easyspec_get_lens(const easyspec_ctx *ctx, int32_t *precise, int32_t *fuzzy);

/* Shorten sequence b to new_precise_len precise slots and no fuzzy ones (base-model rollback
 * after verification; 0 makes the sequence idle).  Host state only: tracked weights that the tokens cut off gave to the slots
 * that stay remain in them.  EASYSPEC_ESTATE if that cuts into what an eviction left of the sequence's older slots
 * (easyspec_evict). */
int easyspec_truncate(easyspec_ctx *ctx, int32_t b, int32_t new_precise_len);

/* Replace the cache of sequence b by n_slots precise entries.  k, v: host|dev
 * [n_layers][n_kv_heads][n_slots][head_dim] in the storage dtype.  Synchronous.  The sequence goes on at position n_slots; its
 * slots have no tracked weights and count as never evicted from (a thinned cache that was exported goes on nearer to its slots). */
int easyspec_kv_import(easyspec_ctx *ctx, int32_t b, const void *k, const void *v, int32_t n_slots);

/* Copy slots [0, n_slots) of sequence b out (same layout as import; fuzzy slots included if
 * n_slots reaches them).  Synchronous. */
int easyspec_kv_export(easyspec_ctx *ctx, int32_t b, void *k, void *v, int32_t n_slots);

/* Final residual-stream rows (before the last norm) of the most recent forward, in the order
 * the forward processed them (draft step: live sequences by index; calibration: sequences by
 * index, tokens in order).  out: dev fp32 [n_rows][d_model]; *n_rows (host) receives the count.
 * For parity checks of hidden states. */
int easyspec_get_hidden(easyspec_ctx *ctx, float *out, int32_t max_rows, int32_t *n_rows);

/* Algorithmic HBM bytes of one draft step in the current state: layer weights + LM head + the
 * KV slots each live sequence reads.  Pure host arithmetic, for roofline reports. */
int64_t easyspec_step_bytes(const easyspec_ctx *ctx);

/* Message of the last failed call on ctx (ctx == NULL: of the last failed easyspec_create or
 * context-free call on this thread).  Never NULL. */
const char *easyspec_last_error(const easyspec_ctx *ctx);

#ifdef __cplusplus
}
#endif
#endif /* EASYSPEC_H */
