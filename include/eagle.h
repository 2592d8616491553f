/*
 * libeagle -- one EAGLE speculative-decoding step on one AMD MI355X (gfx950), C ABI.
 *
 * The library implements the method of arXiv 2401.15077:
 *   drafting     (Sec. 3.1, App. A.1): the Autoregression Head -- concat(feature, embedding of the token one
 *                step ahead) -> FC 2d->d -> one decoder layer -> the target's LM head -- run once per tree
 *                level to expand a static draft tree; greedy children are the top-k tokens, non-greedy
 *                children are k tokens sampled without replacement;
 *   verification (Sec. 3.3): ONE target forward over all tree nodes with tree attention;
 *   acceptance   (Sec. 2 "Speculative sampling", App. A.2 Alg. 1): greedy walk, or multi-round speculative
 *                sampling applied recursively at every node; the accepted tokens' KV rows and features are
 *                kept for the next drafting phase (Sec. 3.3, last sentence).
 *
 * Conventions
 *   - Every call returns 0 (EAGLE_OK) or a negative error code; eagle_last_error() gives the text.
 *     Nothing throws or aborts across the boundary.
 *   - "dev" pointers are device (HIP) addresses, "host" pointers are ordinary host memory.
 *   - The library NEVER allocates device memory.  The caller hands in one workspace of
 *     eagle_workspace_bytes() bytes (256-byte aligned) that must stay valid until eagle_free();
 *     weights are copied (re-tiled) into that workspace by eagle_load_weight(), after which the caller may
 *     release its own copy.
 *   - All work is enqueued on the hipStream_t given to eagle_init().  Calls that return host data
 *     synchronise that stream; the others are asynchronous.
 *   - Sequences are slots 0..max_batch-1.  eagle_prefill() activates a slot; the step calls
 *     (draft / verify / accept / step / vanilla) act on ALL active slots at once, which must be slots
 *     0..n_active-1.  Calls on one context must not overlap in time.
 *   - Static draft tree: n_nodes nodes in BFS order, node 0 is the root (the last committed token, whose
 *     target forward has not run yet), parent[0] = -1, parent[v] < v, rank[v] = v's index among its
 *     siblings (0 = most probable).  At most 64 nodes.
 */
#ifndef EAGLE_H
#define EAGLE_H
#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct eagle_ctx eagle_ctx;

enum { EAGLE_OK = 0, EAGLE_EINVAL = -1, EAGLE_ENOMEM = -2, EAGLE_ESEQ_FULL = -3, EAGLE_ESTATE = -4, EAGLE_EHIP = -5 };
enum { EAGLE_F32 = 0, EAGLE_BF16 = 1, EAGLE_E4M3 = 2, EAGLE_INT8 = 3 };   /* the last two: codes of a cache (eagle_coded_kv) only */

typedef struct {
  int32_t dtype;                      /* EAGLE_F32 | EAGLE_BF16: type of the weight matrices (and of the embedding) */
  int32_t kv_dtype;                   /* EAGLE_F32 | EAGLE_BF16: storage type of the KV cache entries */
  int32_t n_layers, d_model, n_heads, n_kv_heads, head_dim, d_ffn, vocab;
  int32_t n_experts, experts_per_tok; /* 0,0 = dense MLP; else top-k routed SwiGLU experts */
  int32_t draft_moe;                  /* the head's decoder layer is a MoE layer too */
  float rms_eps, rope_theta;
  int32_t max_batch, max_seq, page_tokens; /* KV paging: page_tokens slots per page (power of two) */
  int32_t n_nodes;                    /* draft tree (host arrays, copied) */
  const int32_t *parent, *rank;
  float temperature;                  /* 0 = greedy */
  uint64_t seed;                      /* counter-based generator for the non-greedy draws */
  int32_t weight_bits;                /* 0 or 16: weight matrices stay in `dtype`.  4: eagle_load_weight quantises every
                                         weight matrix of the layers, the head's FC and the LM head (not the embedding)
                                         to 4 bits as it copies it (Sec. 4.2: the int4 case study) -- weight-only,
                                         symmetric, per output row and group of 128 input columns: scale = bf16(max|w| / 7),
                                         code = clip(rint(w / scale), -8, 7), value scale * code.  Needs a dense bf16
                                         model whose widths are multiples of 128, and at most 32 rows per pass
                                         (max_batch * n_nodes <= 32); prompts may be longer. */
  int32_t head_loss_rows;             /* 0: off.  > 0: the workspace also holds what eagle_head_loss needs -- a second
                                         copy of the LM head re-tiled for the product with its transpose, and one
                                         pass's gradient of the logits -- (about 2 * vocab * d_model + 4 * vocab * pass
                                         rows bytes); needs a bf16 model with weight_bits 0 / 16 and vocab % 64 == 0.
                                         The value sizes those passes (up to 1024 rows): give the usual row count.  Any
                                         row count is processed, in as many passes as it takes. */
} eagle_config;

/* Which tensor eagle_load_weight() is given.  Matrices are row-major [out_features, in_features] in the
 * model dtype; norm gains and the FC bias are fp32 vectors.  MoE expert matrices are [n_experts, out, in]; the
 * router is an [n_experts, d_model] matrix in the model dtype (the library keeps and applies it in fp32). */
enum {
  EAGLE_W_EMBED = 0, EAGLE_W_LM_HEAD, EAGLE_W_FINAL_NORM, EAGLE_W_FC, EAGLE_W_FC_BIAS,
  EAGLE_W_ATTN_NORM, EAGLE_W_Q, EAGLE_W_K, EAGLE_W_V, EAGLE_W_O, EAGLE_W_MLP_NORM, EAGLE_W_ROUTER,
  EAGLE_W_GATE, EAGLE_W_UP, EAGLE_W_DOWN, EAGLE_W_COUNT
};
#define EAGLE_HEAD_LAYER (-1)         /* `layer` argument naming the Autoregression Head's decoder layer */

/* Device bytes the context needs for this config (weights in library layout, KV pages, activations). */
size_t eagle_workspace_bytes(const eagle_config *cfg);

/* Create a context inside `workspace_dev` (size >= eagle_workspace_bytes(cfg)).  `hip_stream` is a hipStream_t
 * (NULL = default stream).  EAGLE_EINVAL on a bad config / tree, EAGLE_ENOMEM if the workspace is too small. */
int eagle_init(const eagle_config *cfg, void *workspace_dev, size_t workspace_bytes, void *hip_stream, eagle_ctx **out);
void eagle_free(eagle_ctx *ctx);      /* releases host state only; the workspace belongs to the caller */

/* Copy one tensor (see enum) into the library's tiled layout.  `layer` is 0..n_layers-1, EAGLE_HEAD_LAYER, or
 * ignored for the global tensors.  `src_dev` is a device pointer holding the whole tensor; it may be released
 * as soon as the stream has passed this call.  All tensors must be loaded before eagle_prefill(). */
int eagle_load_weight(eagle_ctx *ctx, int32_t which, int32_t layer, const void *src_dev);

/* Forget all sequences (KV pages are returned, weights stay). */
int eagle_reset(eagle_ctx *ctx);

/* Target forward over the prompt (host int32[n], n >= 1) for slot `seq`, first token chosen from the target
 * distribution (argmax when greedy), and the head's forward over the pairs (f_i, x_{i+1}) -- Sec. 3.1's
 * "feature sequence and token sequence advanced by one time step".  *first_token (host) may be NULL. */
int eagle_prefill(eagle_ctx *ctx, int32_t seq, const int32_t *prompt_host, int32_t n, int32_t *first_token);

/* Drafting phase: D forward passes of the head expand the tree of every active slot.
 * tree_tokens_host: NULL or int32[n_active * n_nodes] receiving the tree's tokens (root first). */
int eagle_draft_tree(eagle_ctx *ctx, int32_t *tree_tokens_host);

/* Verification phase: one tree-masked target forward; logits [n_nodes, vocab] and features [n_nodes, d_model]
 * per slot stay in the context (read them with eagle_get_buffer). */
int eagle_verify(eagle_ctx *ctx);

/* Acceptance + commit: walks each slot's tree (greedy or Alg. 1), then moves the accepted path's KV rows and
 * features to consecutive slots in ONE kernel launch.  Host outputs, each may be NULL:
 *   out_tokens int32[n_active * (depth+1)]  accepted draft tokens followed by the bonus token
 *   out_len    int32[n_active]              number of tokens emitted, 1..depth+1
 *   path       int32[n_active * (depth+1)]  accepted node indices (= KV compaction sources), path[0] = 0 */
int eagle_accept(eagle_ctx *ctx, int32_t *out_tokens, int32_t *out_len, int32_t *path);

/* eagle_accept for callers that cannot allocate or hand over scratch memory (code that must not call hipMalloc: tight
 * serving loops, harnesses that forbid it): the same kernels, but their scratch -- the two fp32 [n_active, vocab]
 * probability vectors of Alg. 1 (vocabularies of at most 32768 entries keep them in registers), and the nodes'
 * outcomes -- lives in a 4 MiB array that is part of the library's device code instead of in the context's
 * workspace.  Inputs (the verified logits, the tree) and outputs are those of eagle_accept.  Limit, whatever the
 * vocabulary: non-greedy, n_active * vocab <= 524288 (16 slots at vocab 32000); greedy always fits.  EAGLE_EINVAL beyond
 * that, before anything is launched.  The call allocates nothing.  Every context on one GPU shares that GPU's array (it
 * keeps the last call's contents; the kernels write every element they read): calls that overlap in time on one GPU race,
 * also across contexts and streams. */
int eagle_accept_static(eagle_ctx *ctx, int32_t *out_tokens, int32_t *out_len, int32_t *path);

/* draft + verify + accept back to back with no host synchronisation in between; outputs as eagle_accept. */
int eagle_step(eagle_ctx *ctx, int32_t *out_tokens, int32_t *out_len, int32_t *path);

/* Plain autoregression with the same kernels: the target on the root token only; one token per slot
 * (host int32[n_active], may be NULL). */
int eagle_vanilla_step(eagle_ctx *ctx, int32_t *tokens_host);

/* Convenience loop for one sequence in slot `seq` (all other slots must be inactive): reset, prefill, then
 * speculative steps until max_new tokens exist.  out: host int32[max_new]; *n_out tokens written;
 * *mean_accept_len = tokens emitted per target forward (the paper's tau). */
int eagle_generate(eagle_ctx *ctx, int32_t seq, const int32_t *prompt_host, int32_t n_prompt, int32_t max_new,
                   int32_t *out, int32_t *n_out, float *mean_accept_len);

/* Acceptance knob of the synthetic workload: future[i] is the token the target will emit at absolute index i
 * of slot `seq`'s token sequence.  While a draft node's path follows `future`, the draft logit of the next
 * future token gets +bias when hash(seed, index) < alpha and -bias otherwise.  n = 0 switches it off. */
int eagle_set_hint(eagle_ctx *ctx, int32_t seq, const int32_t *future_host, int32_t n, float alpha, float bias, uint64_t seed);

/* ---- Injection: lock-step tests and callers that bring their own decisions -------------------------------------
 * These calls let the CPU side of a lock-step comparison drive the engine along ITS choices (Sec. 3.1 / App. A.1
 * tree, Sec. 3.3 / App. A.2 acceptance), and let the child-selection and acceptance kernels be run on logits the
 * caller supplies.  All of them synchronise the stream. */

/* KV paging: physical page of every (slot, logical page), host int32[max_batch * pages_per_slot] with
 * pages_per_slot = ceil(max_seq / page_tokens); must be a permutation of 0..max_batch*pages_per_slot-1.  Allowed only
 * while no slot is active (EAGLE_ESTATE otherwise).  The default is the interleaved map page*max_batch + slot. */
int eagle_set_page_table(eagle_ctx *ctx, const int32_t *table_host);

/* Overwrite a context-owned buffer of slot `seq` from host memory: EAGLE_BUF_LOGITS, _FEATURES, _DRAFT_LOGITS,
 * _DRAFT_FEATURES or _TREE_TOKENS; `bytes` must be the buffer's full size (see the enum below). */
int eagle_set_buffer(eagle_ctx *ctx, int32_t which, int32_t seq, const void *host_src, size_t bytes);

/* Replace the tokens of slot `seq`'s drafted tree (host int32[n_nodes], node 0 = the root token) between
 * eagle_draft_tree and eagle_verify.  The knob's on-path flags are not recomputed. */
int eagle_force_tree(eagle_ctx *ctx, int32_t seq, const int32_t *tokens_host);

/* Child selection alone (App. A.1): the children of the nodes of tree level `level` (-1 = the root, else
 * 1..depth-1: the level's nodes that have children) are chosen from whatever EAGLE_BUF_DRAFT_LOGITS holds --
 * top-k when greedy, Gumbel top-k with the context's seed and draw counter otherwise -- for every active slot. */
int eagle_expand_level(eagle_ctx *ctx, int32_t level);

/* Commit given paths instead of running the acceptance rule, then compact as eagle_accept does.  Host arrays:
 * path int32[n_active * (depth+1)] (node indices, path[0] = 0, each node a child of its predecessor),
 * len int32[n_active] (1..depth+1 tokens emitted: len-1 accepted drafts + the bonus), bonus int32[n_active]. */
int eagle_force_accept(eagle_ctx *ctx, const int32_t *path_host, const int32_t *len_host, const int32_t *bonus_host);

/* Test / bench access to context-owned buffers (synchronises). `which`: */
enum {
  EAGLE_BUF_LOGITS = 0,        /* fp32 [n_nodes, vocab]     verify logits of slot seq                      */
  EAGLE_BUF_FEATURES,          /* fp32 [n_nodes, d_model]   verify features                               */
  EAGLE_BUF_DRAFT_LOGITS,      /* fp32 [n_nodes, vocab]     head logits per node (rows of leaves are unset) */
  EAGLE_BUF_DRAFT_FEATURES,    /* fp32 [n_nodes, d_model]   head output feature per node                   */
  EAGLE_BUF_TREE_TOKENS,       /* int32 [n_nodes]                                                          */
  EAGLE_BUF_TOKENS,            /* int32 [n committed tokens] the slot's whole token sequence               */
  EAGLE_BUF_VANILLA_LOGITS,    /* fp32 [vocab]              logits of the last eagle_vanilla_step / prefill */
  EAGLE_BUF_STATE,             /* int32 [4]: committed tokens, cached target positions, pending features, steps */
  EAGLE_BUF_KV_ROW,            /* see eagle_get_kv_row                                                      */
  EAGLE_BUF_GEMM_TRACE,        /* profiling builds of the library (-DEAGLE_TRACE) only, all zero otherwise:
                                  uint64 [1024 work-groups][8 events], 100 MHz time stamps of ONE launch of the
                                  weight-streaming GEMM kernel, selected with the environment variable
                                  EAGLE_GEMM_TRACE=<index of the launch within the verify phase> (read by eagle_init);
                                  events: 0 entered, 1 activations staged, 2 weight stream done, 3 partial sums
                                  published, 4 epilogue done (the work-groups that ran one). */
  EAGLE_BUF_PREFILL_FEATURES   /* fp32 [rows, d_model]: target features of the last rows of the most recent prompt of
                                  eagle_prefill: its last window of 512 rows for bf16 models (128 where a width is no
                                  multiple of 64 and for fp32 models, 32 for 4-bit weights), the whole prompt when it
                                  fits one -- Sec. 3.1: what the head's prompt pass consumes */
};
int eagle_get_buffer(eagle_ctx *ctx, int32_t which, int32_t seq, void *host_dst, size_t cap_bytes);
/* K and V (fp32, [n_kv_heads*head_dim] each) of target layer `layer` (or EAGLE_HEAD_LAYER) at cache position pos. */
int eagle_get_kv_row(eagle_ctx *ctx, int32_t seq, int32_t layer, int32_t pos, float *k_host, float *v_host);

/* Timing (HIP events on the context's stream).  mode 0 = off, 1 = phases (draft / verify / accept per eagle_step),
 * 2 = additionally every launch of the weight-streaming GEMM kernels and of the attention kernel inside eagle_step,
 * each with a start and a stop event attached to the dispatch itself (the kernel's own begin and end time stamps:
 * the figure a kernel trace shows for the launch). */
int eagle_set_profiling(eagle_ctx *ctx, int32_t mode);
typedef struct {
  double draft_ms, verify_ms, accept_ms;   /* sums over the steps since the last reset of the counters */
  int64_t steps;
  double gemm_ms; int64_t gemm_launches; double gemm_weight_bytes;  /* mode 2 only */
  double verify_weight_bytes, verify_kv_bytes;                    /* algorithmic bytes of the verify phases */
} eagle_profile;
int eagle_get_profile(eagle_ctx *ctx, eagle_profile *out, int32_t reset);
/* Mode 2, per class of launch and per phase (0 = drafting, 1 = verification): summed kernel durations, launches and
 * algorithmic HBM bytes (a weight matrix once in its stored type; for attention the keys and values of the context
 * and the pass's rows once).  name: qkv | attention | o_proj | gate_up | down | lm_head | fc; kernel: the template
 * that ran.  Up to `cap` entries are written, *n of them. */
typedef struct { char name[16]; char kernel[48]; double ms; int64_t launches; double bytes; } eagle_kernel_stat;
int eagle_get_kernel_stats(eagle_ctx *ctx, int32_t phase, eagle_kernel_stat *out, int32_t cap, int32_t *n, int32_t reset);

/* Training loss of the Autoregression Head and its gradient (Sec. 3.2 "Training of the draft models"):
 *   L_reg = mean over rows and columns of SmoothL1(fhat - f)      (threshold 1: 0.5 x^2 if |x| < 1, else |x| - 0.5)
 *   L_cls = mean over rows of -sum_v p_v log phat_v,  p = softmax(LM_Head(f)), phat = softmax(LM_Head(fhat))
 *   L     = L_reg + w_cls * L_cls                                  (the paper sets w_cls = 0.1)
 *   grad  = dL/dfhat = clip(fhat - f, -1, 1) / (rows * d_model) + w_cls / rows * (phat - p) W_lm_head
 * f (the target's feature of the next position: the label) and fhat (the head's prediction) are DEVICE pointers to
 * fp32 [rows, d_model], row-major, only read; the LM head is the one loaded into the context (frozen: it gets no
 * gradient).  grad_fhat: DEVICE pointer, fp32 [rows, d_model], written (may be null: loss only).  loss_out: HOST
 * pointer to 3 floats: L, L_reg, L_cls.  Any rows >= 1; the rows are processed in passes of head_loss_rows rows,
 * at most 1024, and at least half of the context's largest pass.  Leaves the decoding state of the context untouched
 * (it uses only buffers that live within one pass).  Needs cfg.head_loss_rows > 0 and the LM head loaded
 * (EAGLE_ESTATE otherwise).  Synchronises the stream (the loss is returned by value). */
int eagle_head_loss(eagle_ctx *ctx, const float *f_dev, const float *fhat_dev, int32_t rows, float w_cls,
                    float *grad_fhat_dev, float *loss_out);

/* Data augmentation of Sec. 3.2: out[r][k] = in[r][k] + amplitude * n(r, k), n uniform on (-1, 1): the odd multiples of
 * 2^-24 drawn by the library's counter-based generator from (seed, step, r, k) -- reproducible, and a different
 * stream for every step.  fp32 [rows, d_model] DEVICE pointers; in == out is allowed.  The paper's amplitude is 0.1.
 * Needs no head_loss_rows.  Asynchronous on the context's stream. */
int eagle_feature_noise(eagle_ctx *ctx, const float *in_dev, float *out_dev, int32_t rows, float amplitude,
                        uint64_t seed, uint64_t step);

/* Measurement reference, independent of any context: a bare streaming read of `bytes` bytes of device memory
 * (16-byte loads, nothing computed), run `iters` times on `hip_stream`, each launch timed by its own start/stop
 * events; *gb_per_s = bytes read / summed kernel time.  The buffer is only read.  Synchronises the stream. */
int eagle_probe_stream_read(const void *buf_dev, size_t bytes, int32_t iters, void *hip_stream, double *gb_per_s);

/* ---- Operators on the caller's own tensors ----------------------------------------------------------------------
 * Rotary positions with the append to a paged cache, attention of a chunk of new tokens over it, the rules logits pass before a token is
 * chosen, and the choice: what a step does inside a context, for tensors of the caller (another head, a model of another layout, a scheduler of its own).  The cache holds fp32 or bf16, or
 * 8-bit codes with scales.
 *   - They need no context.  Every tensor lies on the device that `hip_stream` belongs to, which must be the calling thread's current device; work
 *     is enqueued on that stream only, nothing is allocated and nothing synchronises, so the calls may be captured into graphs.
 *   - Calls on different streams or threads may overlap as long as they share no output and no workspace (two captured graphs that share a
 *     workspace must not run at the same time).
 *   - Arguments the host holds are checked: EAGLE_EINVAL, nothing launched.  What lies in device memory (lengths, page numbers, token ids) cannot
 *     be; the kernels bound every access instead, as said at each field.
 *   - Types are EAGLE_F32 and EAGLE_BF16; sums and statistics are kept in 32 bits.  Attention of EAGLE_BF16 queries rounds each softmax weight to bf16 (by 2^-8 of it at most) before it is
 *     multiplied with its value, as the result is rounded; with EAGLE_F32 queries nothing is, and a product is off by 2^-22 of itself at most. */

/* New tokens of a batch of sequences: sequence s has the rows row_start[s] .. row_start[s+1]-1 of the row tensors, and with them key_len[s] tokens in
 * the cache (row i of n is token key_len[s] - n + i).  A draft tree instead of consecutive tokens: tree_base[s] tokens are in front of the tree, node u lies
 * at token tree_base[s] + u, and bit u of tree_mask[row] says that node u is the row's own node or an ancestor (parents before children, so the
 * highest bit is the row's own); a node's position is tree_base[s] + its number of ancestors.  key_len[s] counts all nodes in the cache, also those that
 * have no row in this call.
 * max_rows and max_keys bound the rows of a sequence and key_len: rows and tokens beyond are not processed. */
typedef struct {
  int32_t n_seqs, n_rows, max_rows, max_keys;
  const int32_t *row_start;           /* dev int32 [n_seqs + 1] */
  const int32_t *key_len;             /* dev int32 [n_seqs] */
  const int32_t *tree_base;           /* dev int32 [n_seqs], with tree_mask; or both null */
  const uint64_t *tree_mask;          /* dev uint64 [n_rows] */
} eagle_chunk;

/* Paged keys and values: element (page, kv head, token in page, i) of k and v at page * page_stride + head * head_stride + token * token_stride + i
 * (strides in elements, the same for both).  page_table[s * table_stride + t / page_tokens] is the page of token t of sequence s; a number outside
 * 0..n_pages-1 (-1, say) is a page that is not there: its tokens are invisible and rows are not stored to it. */
typedef struct {
  void *k, *v;
  int32_t dtype, n_kv_heads, head_dim, page_tokens /* power of two */, n_pages, pages_per_seq;
  int64_t page_stride, head_stride, token_stride, table_stride;
  const int32_t *page_table;          /* dev int32 [n_seqs][table_stride >= pages_per_seq] */
} eagle_paged_kv;

/* How positions turn a head: pair p (p < rot_dim / 2) of the first rot_dim elements by the angle position * f_p, f_p = theta^(-2p/rot_dim), scaled:
 *   EAGLE_ROPE_LINEAR  f / factor
 *   EAGLE_ROPE_BASE    theta * factor^(rot_dim / (rot_dim - 2)) in place of theta
 *   EAGLE_ROPE_BANDS   by wavelength w = 2 pi / f against L = trained_len: f where w < L / high, f / factor where w > L / low, between them
 *                      f * (s + (1 - s) / factor) with s = (L / w - low) / (high - low)
 *   EAGLE_ROPE_RAMP    by pair: f up to pair a, f / factor from pair b, linear between, with a = max(0, floor(P(high))), b = min(rot_dim - 1, ceil(P(low))),
 *                      P(n) = rot_dim * ln(L / (2 pi n)) / (2 ln theta): the pair that turns n times over L positions
 * Cosines and sines are multiplied by mscale.  Pair p is (p, p + rot_dim / 2), or (2p, 2p + 1) if interleaved.  rot_dim is even, at most head_dim <= 256. */
enum { EAGLE_ROPE_NONE = 0, EAGLE_ROPE_LINEAR, EAGLE_ROPE_BASE, EAGLE_ROPE_BANDS, EAGLE_ROPE_RAMP };
typedef struct {
  int32_t head_dim, rot_dim, interleaved, scaling;
  double theta, factor, low, high;    /* low < high: BANDS and RAMP only; factor >= 1: unread with NONE */
  int32_t trained_len;                /* BANDS and RAMP */
  float mscale;
} eagle_rope_config;
/* The same, worked out: turn[p] = f_p / (2 pi) as a fraction of 2^64.  Host memory; made once, passed to every call. */
typedef struct {
  int32_t head_dim, rot_dim, interleaved;
  float mscale;
  uint64_t turn[128];
} eagle_rope_plan;
int eagle_rope_plan_init(const eagle_rope_config *cfg, eagle_rope_plan *out);

/* Rotates q [n_rows][n_heads][head_dim] into q_out and k [n_rows][n_kv_heads][head_dim] into the cache, together with v -- or, without a cache (kv null), k into
 * k_out.  Row and head strides in elements, elements of a head consecutive; an output may be its input (the same strides), else outputs lie apart from
 * all other tensors of the call.  With a cache `chunk` is needed; v null leaves the
 * cache's values alone.  positions (dev int32 [n_rows]) overrides the positions that `chunk` gives; without a chunk (null: n_rows is the field here) it
 * is needed.  q (with q_out) or k may be null.  Rows that no sequence owns, and those from a sequence's max_rows on, are left as they are, in the outputs too (without a chunk there are none), and
 * a token at or behind max_keys, or on a page that is not there, is not stored.
 * inverse: the transposed map (angles negated, the same mscale): the gradient of the rotation with respect to its input; without a cache only.
 * Two rows of one call must not be the same token of the cache. */
typedef struct {
  int32_t n_rows, n_heads, n_kv_heads, dtype, inverse;
  const void *q, *k, *v;
  void *q_out, *k_out;
  int64_t q_row, q_head, k_row, k_head, v_row, v_head, q_out_row, q_out_head, k_out_row, k_out_head;
  const int32_t *positions;
} eagle_rope_args;
int eagle_rope(const eagle_rope_plan *plan, const eagle_rope_args *args, const eagle_chunk *chunk, const eagle_paged_kv *kv, void *hip_stream);

/* out = softmax(score) v over the visible tokens of the cache, for every row and head (query head h uses kv head h / (n_heads / n_kv_heads)):
 *   score(row, j) = scale * q . k_j;  softcap > 0: softcap * tanh(score / softcap);  slopes: minus slopes[h] * |distance|
 * distance = the row's position - token j's (a token in front of the chunk lies at its index).  Token j is visible to a row if j < key_len[s], its page is there, and
 *   - j comes before the row or is the row itself (tree: is in front of the tree, or the row's node or an ancestor), and distance < window if window > 0, or
 *   - j < prefix[s] (tree: at most the tokens in front of the tree): a prefix every row of the sequence sees, in front of the window and ahead of the row.
 * A row that sees nothing gets zeros.  q, out: EAGLE_F32 over a cache of either type, or EAGLE_BF16 over EAGLE_BF16; out is of q's type and is q
 * (the same strides) or lies apart from it.
 * head_dim: a multiple of 8, 8..128.  q's rows and the cache's tokens start on multiples of 16 bytes, out's of 8 elements.  NaN and infinities in a token stay with
 * the rows that see it: a key that is not finite may make NaN of a score; a value that is infinite makes its element of the row's result infinite or NaN, never finite.  Rows that no sequence owns are left as they are.
 * workspace (dev, 256-byte aligned): eagle_chunk_attention_workspace() bytes, for the same arguments; its contents need not be kept or cleared. */
typedef struct {
  int32_t n_heads, dtype, window;
  const void *q;
  void *out;
  int64_t q_row, q_head, out_row, out_head;   /* elements */
  float scale, softcap;
  const float *slopes;                /* dev [n_heads] or null */
  const int32_t *prefix;              /* dev [n_seqs] or null */
} eagle_attention_args;
size_t eagle_chunk_attention_workspace(const eagle_attention_args *args, const eagle_chunk *chunk, const eagle_paged_kv *kv);
int eagle_chunk_attention(const eagle_attention_args *args, const eagle_chunk *chunk, const eagle_paged_kv *kv, void *workspace_dev, size_t workspace_bytes,
                          void *hip_stream);

/* Paged keys and values in 8 bits: codes, a byte each, at the places that eagle_paged_kv's fields say (strides in codes), and a scale (fp32) for every block of block_tokens tokens
 * of a page's kv head: that of the block that holds token t of a page at page * scale_page + head * scale_head + t / block_tokens (strides in floats).  An element is code * scale.
 * EAGLE_E4M3: a sign, four bits of exponent, three of mantissa, up to 448, NaN and no infinity; EAGLE_INT8: -127..127 (-128 is read as itself).  A scale's sign is not looked at. */
typedef struct {
  void *k, *v;
  float *k_scale, *v_scale;
  int32_t dtype, n_kv_heads, head_dim, page_tokens /* power of two */, block_tokens /* 16, 32, 64 or 128, at most page_tokens */, n_pages, pages_per_seq;
  int64_t page_stride, head_stride, token_stride, table_stride, scale_page, scale_head;
  const int32_t *page_table;          /* dev int32 [n_seqs][table_stride >= pages_per_seq] */
} eagle_coded_kv;

/* eagle_rope with the append to a cache of codes (chunk, kv and k are needed, k_out is null).  With M the largest code (448 or 127), for every block that new tokens go to, keys and values
 * each for themselves, a = the largest absolute value of the new tokens' finite elements (keys as they are after the rotation):
 *   - the block holds no other token of the sequence (one below key_len that this call does not write), or its scale is not positive and finite: scale = 2^e, e the least whole number in
 *     -100..100 with a <= M 2^e; codes of other tokens become 0
 *   - else scale = its scale times 2^n, n the least whole number >= 0 with a <= M scale 2^n, which stays within 2^100; codes of other tokens are rounded again where n > 0
 *   - code = element / scale, to nearest, ties to even, within -M..M (an infinity is M); NaN stays NaN in EAGLE_E4M3 and becomes 0 in EAGLE_INT8
 * with everything from the position to the code worked out in 64 bits.  Codes at or behind key_len, of pages that are not there and of blocks without new tokens stay as they are:
 * a tree's node that lies there is not stored and counts for no scale.
 * Two sequences of one call must not append to the same block. */
int eagle_rope_coded(const eagle_rope_plan *plan, const eagle_rope_args *args, const eagle_chunk *chunk, const eagle_coded_kv *kv, void *hip_stream);

/* eagle_chunk_attention over a cache of codes: k_j and v_j are code * scale, q and out EAGLE_F32 or EAGLE_BF16; codes and their products with the queries are exact as those of a bf16 cache are.
 * head_dim: a multiple of 16, 16..128; the cache's tokens start on multiples of 16 bytes.  With EAGLE_BF16 queries a value scale below 2^-96 counts as 2^-96 (one below
 * 2^-64 may count as 2^-64 where the sequence has one above 2^96), and the weight that is rounded to bf16 is the one times the scale.  Value scales may be as large as fp32 has them: where codes times
 * scales are finite, so are sums of them times weights.  What a scale that is not finite makes of scores and results stays with the rows that see a
 * token of its block: a value scale makes all of their result NaN, a key scale their scores infinite or NaN. */
size_t eagle_chunk_attention_coded_workspace(const eagle_attention_args *args, const eagle_chunk *chunk, const eagle_coded_kv *kv);
int eagle_chunk_attention_coded(const eagle_attention_args *args, const eagle_chunk *chunk, const eagle_coded_kv *kv, void *workspace_dev, size_t workspace_bytes, void *hip_stream);

/* What logits pass before a token is chosen.  The text of row r is its sequence's tokens and, along a draft tree, the tokens of the nodes on its path; with
 * c = how often token t occurs in it behind the sequence's first n_prompt tokens:
 *   x = logit;  t anywhere in the text: x / repetition if x > 0, else x * repetition;  c > 0: x - presence - frequency * c;  x + bias[t];
 *   t not allowed: -inf
 * Every array may be null (no such rule).  Token ids outside the vocabulary count for nothing.  A token may stand in a bias list more than once: the last entry
 * counts.  A repetition that is not above 0 counts as 1, one below 2^-126 as 2^-126.  A mask may leave a row empty: all of it is -inf. */
typedef struct {
  int32_t n_seqs;
  const int32_t *tokens;              /* dev, sequence s at s * token_stride; stride 0: one text for all */
  int64_t token_stride;
  int32_t max_tokens;                 /* of a sequence, at most 2^29; where n_tokens says more, the rest is not read */
  const int32_t *n_tokens, *n_prompt; /* dev [n_seqs]; n_prompt null: 0 */
  const float *repetition, *presence, *frequency;   /* dev [n_seqs] */
  const int32_t *bias_start, *bias_token;           /* dev [n_seqs + 1], [bias_start[n_seqs]]; entries beyond n_bias are not read */
  const float *bias_value;
  int32_t n_bias;
} eagle_logit_rules;
/* in, out: [n_rows][vocab] of `dtype`, row strides in elements; out is in (the same stride) or lies apart from it.  Sequence s has the rows row_start[s] .. row_start[s+1]-1 (null: row r is
 * sequence r's, and n_rows = n_seqs); rows that no sequence owns are left as they are.  path_token (dev [n_rows]) and path_mask (dev uint64 [n_rows]), or both
 * null: bit u of a row's mask adds the token of its sequence's row u to its text (u < 64).  allowed: bit t % 32 of word t / 32 of row allowed_row[r] of
 * [n_masks][mask_stride] words (allowed_row null: row r); a row number outside 0..n_masks-1 (-1, say): no mask. */
typedef struct {
  int32_t n_rows, vocab, dtype, n_masks;
  const void *in;
  void *out;
  int64_t in_stride, out_stride, mask_stride;
  const int32_t *row_start;
  const int32_t *path_token;
  const uint64_t *path_mask;
  const uint32_t *allowed;
  const int32_t *allowed_row;
} eagle_logits;
int eagle_apply_logit_rules(const eagle_logits *logits, const eagle_logit_rules *rules, void *hip_stream);

/* The choice of one token a row of logits [n_rows][vocab] of `dtype` (row stride in elements), from a given random number.  With the row's tokens in order of their logits, descending, equal ones
 * by index, NaN as -inf, and w = exp((logit - largest) / temperature):
 *   top_k > 0: the first top_k;  top_p < 1: of those the shortest run from the front that holds top_p of their mass;  min_p > 0: of those, w >= min_p;  the first in any case
 *   token = the first in order whose running mass exceeds uniform * (mass of those kept), uniform in [0, 1);  logprob = ln(w / mass of those kept)
 * A temperature that is not above 0 takes the first (logprob 0).  Logits of +inf, where there are any, count 1 each and all others 0.  A row of nothing but -inf: token -1, logprob -inf.
 * Weights are worked out in 64 bits, to 2^-33 of themselves for up to 131072 tokens (a bit less for each doubling beyond), and rounded to whole numbers that are added up exactly: a call's result is
 * the same every time.  What weighs less than 2^-64 of the largest counts as nothing in sums.
 * Parameters are arrays with an entry a row; null: 1, no top_k, no top_p, no min_p.  A parameter that is NaN is no filter.  Outputs lie apart from all inputs.
 * logits start on a multiple of an element, rows from 1 to 2^24, vocab to 2^30.  Row stride: at least vocab, where there is more than one row.
 * workspace (dev, 256-byte aligned): eagle_sample_workspace() bytes, for the same arguments; its contents need not be kept or cleared (reserved: nothing uses it today). */
typedef struct {
  int32_t n_rows, vocab, dtype;
  const void *logits;
  int64_t stride;
  const float *uniform, *temperature; /* dev [n_rows] */
  const int32_t *top_k;
  const float *top_p, *min_p;
  int32_t *token;                     /* dev [n_rows] */
  float *logprob;                     /* dev [n_rows] or null */
} eagle_sample_args;
size_t eagle_sample_workspace(const eagle_sample_args *args);
int eagle_sample(const eagle_sample_args *args, void *workspace_dev, size_t workspace_bytes, void *hip_stream);

/* ---- Positions, attention and logit rules inside a context -------------------------------------------------
 * Positions: how the target's and the head's layers turn queries and keys (null: the default again, pairs (i, i + head_dim / 2) of the whole head by cfg.rope_theta).
 * theta of the given configuration counts, not cfg's.  Before the first EAGLE_W_Q / _K is loaded (they are laid out by pairs), EAGLE_ESTATE after that.  Keys are read
 * back (eagle_get_kv_row) in the model's own order of elements. */
int eagle_set_rope(eagle_ctx *ctx, const eagle_rope_config *rope_host);

/* Scores of every layer of the target and the head: cap, window and slopes as in eagle_attention_args (all of them 0 / null, or rules null: plain again).  slopes is the caller's device
 * memory and stays theirs: [n_heads], read by every pass.  Only while no slot is active (EAGLE_ESTATE otherwise).  The passes take eagle_chunk_attention's kernels then, which
 * eagle_get_kernel_stats does not list. */
typedef struct { float softcap; int32_t window; const float *slopes_dev; } eagle_attention_rules;
int eagle_set_attention(eagle_ctx *ctx, const eagle_attention_rules *rules_host);

/* Rules that the TARGET's logits pass before a token is chosen or a draft is accepted: the first token of a prompt, eagle_vanilla_step, and every node of eagle_verify
 * (along the node's path); a slot's prompt counts as n_prompt.  EAGLE_BUF_LOGITS and EAGLE_BUF_VANILLA_LOGITS hold what came out.  The head's own logits are as they were: it drafts
 * without the rules, acceptance (greedy or Alg. 1) is exact for the ruled target.  Arrays are the caller's device memory, read whenever logits are made, so they may be rewritten between
 * calls (masks between eagle_draft_tree, which says the tree's tokens, and eagle_verify).  By slot: repetition, presence, frequency [max_batch], bias_start [max_batch + 1].
 * allowed_row [max_batch][n_nodes]: a node's mask; node 0's serves prompts and vanilla steps too.  Any array may be null.  A mask that leaves a node nothing leaves the token
 * that follows it unspecified.  rules null: none.  Survives eagle_reset. */
typedef struct {
  const float *repetition, *presence, *frequency;
  const int32_t *bias_start, *bias_token;
  const float *bias_value;
  int32_t n_bias, n_masks;
  const uint32_t *allowed;
  int64_t mask_stride;
  const int32_t *allowed_row;
} eagle_context_rules;
int eagle_set_logit_rules(eagle_ctx *ctx, const eagle_context_rules *rules_host);

const char *eagle_last_error(void);   /* thread-local text of the last failure */
const char *eagle_version(void);

#ifdef __cplusplus
}
#endif
#endif
