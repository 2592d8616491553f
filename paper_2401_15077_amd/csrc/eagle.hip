// libeagle: host side -- context, workspace layout, weight loading, and the orchestration of one EAGLE
// speculative step (drafting: Sec. 3.1 / App. A.1; verification: Sec. 3.3; acceptance: Sec. 2 / App. A.2).
#include "host.h"
#include "operators.h"
#include "kernels.h"
#include "kernels2.h"
#include "plans.h"
#include <hip/hip_ext.h>

#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <cstdlib>
#include <vector>
#include <algorithm>
#include <mutex>

static thread_local char g_err[512] = "";
int fail(int code, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_err, sizeof(g_err), fmt, ap);
  va_end(ap);
  return code;
}

// ---------------------------------------------------------------------------- static device scratch
// Scratch of eagle_accept_static(): a fixed array in the code object instead of caller-provided memory, for callers
// that cannot allocate.  Every GPU the library runs on holds its own copy at its own address until the process ends.
// In host code the array's name is only a handle for hipGetSymbolAddress: the address that kernels, copies and fills
// are given is the one that call returned for the device at hand (g_scratch_dev), never the name.
#define EAGLE_STATIC_SCRATCH_BYTES (4u << 20)
#define EAGLE_MAX_DEVICES 64
static __device__ __align__(256) unsigned char scratch[EAGLE_STATIC_SCRATCH_BYTES];
static void* g_scratch_dev[EAGLE_MAX_DEVICES];
static std::mutex g_scratch_mutex;

// ---------------------------------------------------------------------------- descriptors
struct PackedW {            // a weight matrix in tiled layout
  bf16_t* w = nullptr;
  size_t plane_stride = 0;  // elements between planes
  int N = 0, Npad = 0, NRB = 0, K = 0, KS = 0;
  bool q4 = false;          // 4-bit codes (w) + bf16 group scales (sc), see k_pack_weight_q4
  bf16_t* sc = nullptr;
  int NG = 0;
  double bytes(int elt) const { return q4 ? (double)N * K * 0.5 + (double)N * NG * 2.0 : (double)N * K * elt; }   // as stored
};
struct LayerW {
  PackedW qkv, o, gu, dn;
  std::vector<PackedW> e_gu, e_dn;   // MoE experts
  float* router = nullptr;           // fp32 [E][d]
  float *attn_norm = nullptr, *mlp_norm = nullptr;
  bool moe = false;
};

// Kernel classes of the per-launch timing (profiling mode 2): what the launch computes, not which template ran
// (the template's name is recorded beside it).
enum { KC_QKV = 0, KC_ATTN, KC_O, KC_GATEUP, KC_DOWN, KC_LMHEAD, KC_FC, KC_COUNT };
static const char* const kKernelClassName[KC_COUNT] = {"qkv", "attention", "o_proj", "gate_up", "down", "lm_head", "fc"};
struct KStat { double ms = 0, bytes = 0; long launches = 0; char kernel[48] = ""; };
struct TimedLaunch { int phase, kclass; double bytes; };

struct Arena {
  char* base; size_t off = 0;
  explicit Arena(char* b) : base(b) {}
  template <typename T> T* take(size_t n) {
    off = (off + 255) & ~(size_t)255;
    T* p = (T*)(base + off);
    off += n * sizeof(T);
    return p;
  }
};

struct eagle_ctx {
  eagle_config cfg;
  hipStream_t stream;
  char* ws; size_t ws_bytes, zero_end;
  bool f32, kv_f32, q4 = false;      // q4: weight matrices stored in 4 bits
  bool q4_staged = true;
  int NWP, NXP, elt, kv_elt;         // weight planes, activation planes, bytes per weight / per KV element
  TreeDev tree_h; TreeDev* tree_d;
  int M, D, Mmax, max_level_rows;
  int last_rows = 0, last_off = 0;     // the last window of the most recent prompt (EAGLE_BUF_PREFILL_FEATURES): rows, first row in chunk_f
  // most rows of one prompt pass: where the large-M GEMM exists (bf16, every K a multiple of 64) a pass is as long as keeps the
  // activations a small part of the card's memory, since every pass streams all weights, needs K slices (and their partial
  // sums) to fill the chip with its narrow matrices, and rounds its tiles up once per matrix
  int pf_chunk = EAGLE_PREFILL_CHUNK, pf_window = EAGLE_PREFILL_CHUNK;
  bool big_gemm = false;
  // Dense models with a bf16 cache keep the order of sums that a pass of so many rows has always had.  The cache rounds K and V,
  // which turns a difference of 1e-7 between two orders of an fp32 sum into one of 2^-9 in about one entry of a thousand (1e-4
  // relative on the logits of a 32-layer model): neither order is the more accurate one, but results would move visibly from
  // release to release.  Kept: K slices by plan_slices, prompt passes of 512 rows (32 with 4-bit weights, whose codes then expand
  // around 128 in every pass), the norm's sums of k_resnorm_fixed, k_gemm up to 64 rows, the K slices of 4-bit LM heads,
  // the key splits of attention over few tokens.  (How many rows a pass has decides the order here as everywhere on the general path.)  Mixtures of experts are not held to it: grouping the rows by expert has
  // reordered their sums already, and a router near-tie moves their logits as much as the rounding of the cache does.
  bool fixed_sums = false;
  int q4_rot = Q4_ROT_LARGE_M;       // 4-bit codes: rotation of the packed words (3: they expand to 16 + code, 0: to 128 + code)
  // weights
  void* embed; PackedW lm_head, fc; float *final_norm, *fc_bias;
  std::vector<LayerW> layers;        // [n_layers] target + [1] head
  bool loaded[EAGLE_W_COUNT][2];
  std::vector<std::vector<char>> loaded_layer;  // [which][layer+1]
  // caches
  void *kc, *vc, *dkc, *dvc; size_t layer_stride; int* page_table; int pps, page_shift;
  float *rope_cos, *rope_sin;
  // state
  SeqState st; HintDev hint;
  int *hint_future, *hint_n; float *hint_alpha, *hint_bias; unsigned long long* hint_seed;
  float *pend_f, *node_f, *F, *chunk_f, *featbuf;
  float *draft_logits, *L, *vanilla_logits, *pbuf, *qbuf;
  unsigned long long* part_keys; int* cnt_expand;               // child selection: the best keys of a row's parts, arrivals
  int *tree_tok, *on_path, *path, *tok_out, *len_out; int2* outcome;
  void* res_host = nullptr;          // pinned host copy of [path | tok_out | len_out]
  ~eagle_ctx() { if (res_host) (void)hipHostFree(res_host); }
  // activations
  float *h, *Q, *PT, *part_o, *part_ml;
  size_t part_rows = 0;
  bf16_t *xf_d, *xf_2d, *xf_att, *xf_ffn;
  size_t pt_floats;
  // fast path (passes of <= 32 rows)
  float *h2, *PT2, *ssq1, *ssq2; int *cnt_gemm, *cnt_attn; size_t pt2_floats, pt2_all;   // of one launch's plan, of the buffer
  bf16_t *xf2_d, *xf2_dB, *xf2_2d, *xf2_att, *xf2_ffn;
  float* group_sums;                   // 4-bit weights: -24 * sum of x per (group of 128 columns, row) of the GEMM input at hand
  // grouped experts (general path of the bf16 models): which rows go to which expert, the gathered rows and their MLP inputs
  MoePlan* moe_plan; int *moe_slot, *moe_row; bf16_t *xf_moe;
  RowFact* facts;                      // [Mmax] rows of the pass in flight (written by its first kernel)
  float *moe_w, *xn; int* expert_used; int* experts_touched;   // (profiling) experts used, summed over the layers of a verify    // routing weights [E][largest pass], used flags [E], fp32 normalised rows (general path)
  int ssq1_groups = 0, ssq2_groups = 0;
  unsigned long long* trace = nullptr; int trace_sel = -1, gemm_no = 0, attn_trace_sel = -1, attn_no = 0;   // profiling builds only
  int n_cu = 256;                      // compute units of the device (queried by eagle_init; 256 assumed when no device is visible)
  int device = 0;
  void* static_scratch = nullptr;      // this device's address of the library's static scratch array
  // positions, scores and logit rules other than the default (eagle_set_rope, eagle_set_attention, eagle_set_logit_rules)
  int rope_mode = PACK_ROPE;           // how rows of q and k are paired
  bool attn_ruled = false; eagle_attention_rules attn_rules{};
  bool logits_ruled = false; eagle_context_rules logit_rules{};
  int *op_start, *op_len, *op_base, *op_prompt, *op_tokens, *op_mask_row, *op_verify_start; unsigned long long *op_mask, *op_path;
  std::vector<int> h_prompt;           // prompt length by slot
  // training loss of the head (cfg.head_loss_rows > 0): the LM head re-tiled as [d_model rows][vocab columns], the
  // gradient of one pass's logits as a GEMM input, per-row losses of a pass, the running sums of a call
  PackedW lm_head_T; bf16_t* hl_dz = nullptr; float* hl_row_loss = nullptr; double* hl_acc = nullptr; int hl_chunk = 0;
  // host mirror
  std::vector<int> h_ctx, h_ntok; std::vector<char> active, head_stale;
  int n_active = 0;
  int phase = 0;                      // 0 idle, 1 drafted, 2 verified
  // profiling
  int prof_mode = 0;
  hipEvent_t ev[4];
  std::vector<hipEvent_t> gemm_ev; size_t gemm_ev_used = 0; std::vector<TimedLaunch> timed;
  KStat kstat[2][KC_COUNT];           // [0 drafting phase | 1 verification phase][class]
  int cur_phase = -1, cur_class = KC_QKV;   // phase of the step that is being enqueued (-1: outside a step, not timed)
  eagle_profile prof;
};

static bool use_pf(const eagle_ctx* c, int MT) { return plan_is_large_m(MT, c->big_gemm, c->fixed_sums, c->q4); }

static int build_tree(const eagle_config* cfg, TreeDev* t) {
  int M = cfg->n_nodes;
  if (M < 1 || M > EAGLE_MAX_NODES) return fail(EAGLE_EINVAL, "n_nodes must be 1..%d", EAGLE_MAX_NODES);
  if (!cfg->parent || !cfg->rank) return fail(EAGLE_EINVAL, "parent/rank arrays missing");
  memset(t, 0, sizeof(*t));
  t->M = M;
  if (cfg->parent[0] != -1) return fail(EAGLE_EINVAL, "node 0 must be the root (parent -1)");
  t->parent[0] = -1; t->anc[0] = 1ull;
  for (int v = 1; v < M; ++v) {
    int p = cfg->parent[v];
    if (p < 0 || p >= v) return fail(EAGLE_EINVAL, "parent[%d]=%d must precede its child", v, p);
    t->parent[v] = p; t->depth[v] = t->depth[p] + 1;
    if (t->depth[v] < t->depth[v - 1]) return fail(EAGLE_EINVAL, "nodes must be in BFS order");
    if (t->depth[v] > EAGLE_MAX_DEPTH) return fail(EAGLE_EINVAL, "tree deeper than %d", EAGLE_MAX_DEPTH);
    t->anc[v] = t->anc[p] | (1ull << v);
    int r = cfg->rank[v];
    if (r < 0 || r >= EAGLE_MAX_CHILD) return fail(EAGLE_EINVAL, "rank[%d]=%d out of range", v, r);
    t->child[p][r] = v; t->nchild[p]++;
    if (t->depth[v] > t->D) t->D = t->depth[v];
  }
  for (int v = 0; v < M; ++v) {       // sibling ranks must be exactly 0..k-1
    unsigned seen = 0;
    for (int c = 1; c < M; ++c) if (t->parent[c] == v) {
      if (cfg->rank[c] >= t->nchild[v] || (seen >> cfg->rank[c]) & 1u) return fail(EAGLE_EINVAL, "sibling ranks of node %d are not 0..k-1", v);
      seen |= 1u << cfg->rank[c];
    }
    if (t->nchild[v] > 0 && t->depth[v] >= 1) t->level_rows[t->depth[v]][t->n_level_rows[t->depth[v]]++] = v;
  }
  return EAGLE_OK;
}

static int check_cfg(const eagle_config* c) {
  if (!c) return fail(EAGLE_EINVAL, "null config");
  if (c->dtype != EAGLE_F32 && c->dtype != EAGLE_BF16) return fail(EAGLE_EINVAL, "dtype must be EAGLE_F32 or EAGLE_BF16");
  if (c->kv_dtype != EAGLE_F32 && c->kv_dtype != EAGLE_BF16) return fail(EAGLE_EINVAL, "kv_dtype must be EAGLE_F32 or EAGLE_BF16");
  if (c->n_layers < 1 || c->d_model < 64 || c->d_model % 64) return fail(EAGLE_EINVAL, "d_model must be a positive multiple of 64");
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 32) return fail(EAGLE_EINVAL, "head_dim must be 32, 64 or 128");
  if (c->n_heads < 1 || c->n_kv_heads < 1 || c->n_heads % c->n_kv_heads) return fail(EAGLE_EINVAL, "n_heads must be a multiple of n_kv_heads");
  if ((c->n_heads * c->head_dim) % 32 || (c->n_kv_heads * c->head_dim) % 32) return fail(EAGLE_EINVAL, "attention widths must be multiples of 32");
  if (c->d_ffn < 16 || c->d_ffn % 16) return fail(EAGLE_EINVAL, "d_ffn must be a multiple of 16");
  if (c->vocab < 2) return fail(EAGLE_EINVAL, "vocab too small");
  if (c->n_experts < 0 || c->n_experts > 64 || (c->n_experts > 0 && (c->experts_per_tok < 1 || c->experts_per_tok > c->n_experts || c->experts_per_tok > 4)))
    return fail(EAGLE_EINVAL, "bad expert counts");
  if (c->max_batch < 1 || c->max_batch > 64) return fail(EAGLE_EINVAL, "max_batch must be 1..64");
  if (c->page_tokens < 32 || (c->page_tokens & (c->page_tokens - 1))) return fail(EAGLE_EINVAL, "page_tokens must be a power of two >= 32");
  if (c->max_seq < c->n_nodes + 2) return fail(EAGLE_EINVAL, "max_seq too small for the tree");
  if (!(c->temperature >= 0.f)) return fail(EAGLE_EINVAL, "temperature must be >= 0");
  if (!(c->rms_eps > 0.f) || !(c->rope_theta > 1.f)) return fail(EAGLE_EINVAL, "bad rms_eps / rope_theta");
  if (c->weight_bits != 0 && c->weight_bits != 16 && c->weight_bits != 4) return fail(EAGLE_EINVAL, "weight_bits must be 0 / 16 (weights as given) or 4");
  return EAGLE_OK;
}

static void take_packed(Arena& a, PackedW& w, int N, int K, int NWP, bool q4 = false) {
  w.N = N; w.K = K; w.Npad = (N + 31) / 32 * 32; w.NRB = w.Npad / 32; w.KS = K / 16;
  w.plane_stride = (size_t)w.Npad * K;
  w.q4 = q4;
  if (q4) {
    w.NG = K / EAGLE_Q4_GROUP;
    w.w = a.take<bf16_t>(w.plane_stride / 4);                 // half a byte per weight
    w.sc = a.take<bf16_t>((size_t)w.NRB * w.NG * 32);
  } else w.w = a.take<bf16_t>(w.plane_stride * NWP);
}

// Streamed split-K plan of a matrix on the fast path (S = 0: the LDS-staged kernel).
static PlanXK xk_plan(const eagle_ctx* c, const PackedW& w) { return plan_streamed(w.NRB, w.KS, c->NXP, c->NWP, c->n_cu, c->pt2_floats, w.q4); }
// Mixture of experts on the fast path: all experts' gate/up in one launch and all their downs in another.
static bool moe_in_two(const eagle_ctx* c, const PackedW& gu, const PackedW& dn) {
  return c->cfg.n_experts > 1 && c->big_gemm && plan_experts_in_two(gu.NRB, gu.KS, dn.NRB, dn.KS, c->NXP, c->NWP, c->n_cu, c->pt2_floats);
}

// Lays the context's buffers out in the workspace (or just measures when c->ws == nullptr).
static size_t layout(eagle_ctx* c) {
  const eagle_config& g = c->cfg;
  Arena a(c->ws);
  const int d = g.d_model, V = g.vocab, H = g.n_heads, KVH = g.n_kv_heads, dh = g.head_dim, F = g.d_ffn, B = g.max_batch;
  const int M = c->M, D1 = c->D + 1;
  c->tree_d = a.take<TreeDev>(1);
  c->rope_cos = a.take<float>((size_t)g.max_seq * dh / 2);
  c->rope_sin = a.take<float>((size_t)g.max_seq * dh / 2);
  // weights
  c->embed = a.take<char>((size_t)V * d * c->elt);
  take_packed(a, c->lm_head, V, d, c->NWP, c->q4);
  if (g.head_loss_rows > 0) {
    take_packed(a, c->lm_head_T, d, V, c->NWP);
    c->hl_dz = a.take<bf16_t>((size_t)c->NXP * c->hl_chunk * V);
    c->hl_row_loss = a.take<float>((size_t)2 * c->hl_chunk);
    c->hl_acc = a.take<double>(2);
  }
  take_packed(a, c->fc, d, 2 * d, c->NWP, c->q4);
  c->final_norm = a.take<float>(d);
  c->fc_bias = a.take<float>(d);
  c->layers.assign(g.n_layers + 1, LayerW());
  for (int l = 0; l <= g.n_layers; ++l) {
    LayerW& w = c->layers[l];
    take_packed(a, w.qkv, (H + 2 * KVH) * dh, d, c->NWP, c->q4);
    take_packed(a, w.o, d, H * dh, c->NWP, c->q4);
    w.moe = g.n_experts > 0 && (l < g.n_layers || g.draft_moe);
    if (w.moe) {
      w.e_gu.resize(g.n_experts); w.e_dn.resize(g.n_experts);
      for (int e = 0; e < g.n_experts; ++e) { take_packed(a, w.e_gu[e], 2 * F, d, c->NWP); take_packed(a, w.e_dn[e], d, F, c->NWP); }
      w.router = a.take<float>((size_t)g.n_experts * d);
    } else {
      take_packed(a, w.gu, 2 * F, d, c->NWP, c->q4);
      take_packed(a, w.dn, d, F, c->NWP, c->q4);
    }
    w.attn_norm = a.take<float>(d);
    w.mlp_norm = a.take<float>(d);
  }
  // KV pages
  c->pps = (g.max_seq + g.page_tokens - 1) / g.page_tokens;
  c->page_shift = 0;
  while ((1 << c->page_shift) < g.page_tokens) c->page_shift++;
  c->layer_stride = (size_t)B * c->pps * KVH * g.page_tokens * dh;
  c->kc = a.take<char>(c->layer_stride * g.n_layers * c->kv_elt);
  c->vc = a.take<char>(c->layer_stride * g.n_layers * c->kv_elt);
  c->dkc = a.take<char>(c->layer_stride * c->kv_elt);
  c->dvc = a.take<char>(c->layer_stride * c->kv_elt);
  c->page_table = a.take<int>((size_t)B * c->pps);
  // state
  c->st.ctx_len = a.take<int>(B); c->st.n_pend = a.take<int>(B); c->st.n_tok = a.take<int>(B);
  c->st.step_no = a.take<int>(B); c->st.commit_base = a.take<int>(B);
  c->st.tok_stride = g.max_seq + 8;
  c->st.tokens = a.take<int>((size_t)B * c->st.tok_stride);
  c->hint_future = a.take<int>((size_t)B * c->st.tok_stride);
  c->hint_n = a.take<int>(B); c->hint_alpha = a.take<float>(B); c->hint_bias = a.take<float>(B);
  c->hint_seed = a.take<unsigned long long>(B);
  c->pend_f = a.take<float>((size_t)B * D1 * d);
  c->node_f = a.take<float>((size_t)B * M * d);
  c->F = a.take<float>((size_t)B * M * d);
  c->chunk_f = a.take<float>((size_t)c->pf_chunk * d);
  c->featbuf = a.take<float>((size_t)c->Mmax * d);
  c->draft_logits = a.take<float>((size_t)B * M * V);
  c->L = a.take<float>((size_t)B * M * V);
  c->vanilla_logits = a.take<float>((size_t)B * V);
  c->pbuf = a.take<float>((size_t)B * V);
  c->qbuf = a.take<float>((size_t)B * V);
  c->part_keys = a.take<unsigned long long>((size_t)B * std::max(1, c->max_level_rows) * EXPAND_PARTS_MAX * EAGLE_MAX_CHILD);
  c->cnt_expand = a.take<int>((size_t)B * std::max(1, c->max_level_rows) * COUNTER_STRIDE);
  c->tree_tok = a.take<int>((size_t)B * M); c->on_path = a.take<int>((size_t)B * M); c->outcome = a.take<int2>((size_t)B * M);
  c->path = a.take<int>((size_t)B * D1); c->tok_out = a.take<int>((size_t)B * D1); c->len_out = a.take<int>(B);   // kept adjacent: fetched in one copy
  // activations
  const int Mm = c->Mmax, MTm = Mm / 32;
  c->h = a.take<float>((size_t)Mm * d);
  c->Q = a.take<float>((size_t)Mm * H * dh);
  c->xf_d = a.take<bf16_t>((size_t)c->NXP * std::max(Mm, 2 * c->hl_chunk) * d);
  c->xf_2d = a.take<bf16_t>((size_t)c->NXP * Mm * 2 * d);
  c->xf_att = a.take<bf16_t>((size_t)c->NXP * Mm * H * dh);
  const bool grouped = c->big_gemm && g.n_experts > 0;
  const int slots = grouped ? 32 * moe_tiles(Mm, g.experts_per_tok, g.n_experts) : 0;
  c->xf_ffn = a.take<bf16_t>((size_t)c->NXP * std::max(Mm, slots) * F);
  c->group_sums = a.take<float>(c->q4 ? (size_t)std::max(std::max(F, H * dh), 2 * d) / EAGLE_Q4_GROUP * Mm : 1);
  c->moe_plan = a.take<MoePlan>(1);
  c->moe_slot = a.take<int>(grouped ? (size_t)g.n_experts * Mm : 1);
  c->moe_row = a.take<int>(std::max(1, slots));
  c->xf_moe = a.take<bf16_t>(std::max((size_t)8, (size_t)c->NXP * slots * d));
  // fast path buffers
  size_t worst2 = 0;
  auto consider2 = [&](const PackedW& w) {
    worst2 = std::max(worst2, plan2(w.NRB, w.KS, c->NXP, c->NWP, c->n_cu, w.q4).S * (size_t)w.Npad * 32);
  };
  consider2(c->lm_head); consider2(c->fc);
  for (auto& w : c->layers) {
    consider2(w.qkv); consider2(w.o);
    if (w.moe) { consider2(w.e_gu[0]); consider2(w.e_dn[0]); } else { consider2(w.gu); consider2(w.dn); }
  }
  c->pt2_floats = worst2;
  bool two = false;                                             // all experts of a layer in one launch: an input of down each
  for (auto& w : c->layers) two = two || (w.moe && moe_in_two(c, w.e_gu[0], w.e_dn[0]));
  c->h2 = a.take<float>((size_t)32 * d);
  c->xf2_d = a.take<bf16_t>((size_t)c->NXP * 32 * d);
  c->xf2_dB = a.take<bf16_t>(g.n_experts > 0 ? (size_t)c->NXP * 32 * d : 8);
  c->moe_w = a.take<float>((size_t)std::max(1, g.n_experts) * c->Mmax);
  c->expert_used = a.take<int>(std::max(1, g.n_experts));
  c->experts_touched = a.take<int>(1);
  c->xn = a.take<float>(g.n_experts > 0 ? (size_t)Mm * d : 8);
  c->xf2_2d = a.take<bf16_t>((size_t)c->NXP * 32 * 2 * d);
  c->xf2_att = a.take<bf16_t>((size_t)c->NXP * 32 * H * dh);
  c->xf2_ffn = a.take<bf16_t>((size_t)c->NXP * 32 * F * (two ? g.n_experts : 1));
  c->facts = a.take<RowFact>(Mm);
  c->op_start = a.take<int>(B + 1); c->op_len = a.take<int>(B); c->op_base = a.take<int>(B); c->op_prompt = a.take<int>(B); c->op_tokens = a.take<int>(B);
  c->op_mask_row = a.take<int>(B); c->op_verify_start = a.take<int>(B + 1); c->op_mask = a.take<unsigned long long>(Mm); c->op_path = a.take<unsigned long long>((size_t)B * M);
  c->ssq1 = a.take<float>(PLAN_MAX_NORM_GROUPS * 32); c->ssq2 = a.take<float>(PLAN_MAX_NORM_GROUPS * 32);
  c->trace = a.take<unsigned long long>(1024 * 8);
  c->cnt_gemm = a.take<int>(1024 * COUNTER_STRIDE); c->cnt_attn = a.take<int>((size_t)128 * H * COUNTER_STRIDE);
  for (auto& w : c->layers)                                     // (and the slices of each)
    if (w.moe && moe_in_two(c, w.e_gu[0], w.e_dn[0])) { worst2 = std::max(worst2, (size_t)g.n_experts * xk_plan(c, w.e_dn[0]).S * w.e_dn[0].Npad * 32); break; }
  c->pt2_all = worst2;
  c->PT2 = a.take<float>(worst2);
  // scratch that every pass writes before it reads (not cleared by eagle_init)
  c->zero_end = a.off;
  // split-K partials of the general path: the largest S * Npad * rows over the GEMM shapes and the passes that run them
  size_t worst = c->pt_floats;                                  // (found by an earlier call for the same context)
  struct Seen { int NRB, KS, mt_max; bool fused; };
  std::vector<Seen> seen;                                       // (the layers repeat the same few shapes)
  auto consider = [&](const PackedW& w, int mt_max, bool fused) {
    if (c->pt_floats) return;
    for (const Seen& q : seen) if (q.NRB == w.NRB && q.KS == w.KS && q.mt_max == mt_max && q.fused == fused) return;
    seen.push_back(Seen{w.NRB, w.KS, mt_max, fused});
    for (int mt = mt_max; mt >= 1 && (size_t)PLAN_MAX_SLICES * w.Npad * (size_t)(mt * 32) > worst; --mt) {   // (shorter passes cannot need more)
      const GemmPlan p = use_pf(c, mt) ? plan_pf(w.NRB, w.KS, mt, c->n_cu, fused, c->q4, c->fixed_sums) : plan_gemm(w.NRB, w.KS, c->NXP, mt);
      if (fused && use_pf(c, mt) && p.S == 1) continue;          // SwiGLU inside the GEMM: nothing goes through memory
      worst = std::max(worst, (size_t)p.S * w.Npad * (size_t)(mt * 32));
    }
  };
  if (g.head_loss_rows > 0) { consider(c->lm_head, 2 * c->hl_chunk / 32, false); consider(c->lm_head_T, c->hl_chunk / 32, false); }
  consider(c->lm_head, 4, false);                               // tree and vanilla passes; a prompt needs its last row tile only
  consider(c->fc, MTm, false);
  bool moe_seen = false;
  for (auto& w : c->layers) {
    consider(w.qkv, MTm, false); consider(w.o, MTm, false);
    if (w.moe && grouped) {
      for (int mt = MTm; mt >= 1 && !moe_seen && !c->pt_floats; --mt) {           // (the layers are alike)
        if ((size_t)PLAN_MAX_SLICES * w.e_dn[0].Npad * 32 * moe_tiles(32 * mt, g.experts_per_tok, g.n_experts) <= worst) break;
        const PlanMoe p = plan_moe(w.e_gu[0].NRB, w.e_gu[0].KS, w.e_dn[0].NRB, w.e_dn[0].KS, 32 * mt, g.experts_per_tok, g.n_experts, c->n_cu);
        worst = std::max(worst, (size_t)p.dn.S * w.e_dn[0].Npad * 32 * moe_tiles(32 * mt, g.experts_per_tok, g.n_experts));
      }
      moe_seen = true;
    } else if (w.moe) { consider(w.e_gu[0], MTm, false); consider(w.e_dn[0], MTm, false); } else { consider(w.gu, MTm, true); consider(w.dn, MTm, false); }
  }
  c->pt_floats = worst;
  c->PT = a.take<float>(worst);
  // attention partials: rows x KV splits, which attn_splits bounds (a pass of many row blocks is not split)
  size_t part_rows = 32 * 16;
  for (int rb = 2; rb <= MTm + B; ++rb) {                       // (sequence, 32-row block) pairs of a pass
    const int s = std::min(16, c->n_cu / (H * rb));
    if (s > 1) part_rows = std::max(part_rows, (size_t)32 * rb * s);
  }
  c->part_rows = part_rows;
  c->part_o = a.take<float>(part_rows * H * dh);
  c->part_ml = a.take<float>(part_rows * H * 2);
  return (a.off + 255) & ~(size_t)255;
}

// Compute units of the current device.  The work splits are planned for at most 256 of them (the per-row-group
// buffers are sized for that); without a visible device (size queries on a build machine) 256 is assumed.
static int query_cus(int* device) {
  int dev = 0, n = 0;
  if (hipGetDevice(&dev) != hipSuccess || hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n < 1) {
    (void)hipGetLastError();
    *device = -1;
    return 256;
  }
  *device = dev;
  return std::min(n, 256);
}

static int prepare(const eagle_config* cfg, eagle_ctx* c) {
  int rc = check_cfg(cfg);
  if (rc) return rc;
  c->cfg = *cfg;
  c->n_cu = query_cus(&c->device);
  rc = build_tree(cfg, &c->tree_h);
  if (rc) return rc;
  c->f32 = cfg->dtype == EAGLE_F32;
  c->NWP = c->f32 ? 3 : 1; c->NXP = c->f32 ? 3 : 2; c->elt = c->f32 ? 4 : 2;
  c->kv_f32 = cfg->kv_dtype == EAGLE_F32; c->kv_elt = c->kv_f32 ? 4 : 2;
  c->q4 = cfg->weight_bits == 4;
  c->fixed_sums = !c->kv_f32 && cfg->n_experts == 0;
  c->M = c->tree_h.M; c->D = c->tree_h.D;
  c->max_level_rows = 1;
  for (int dlev = 1; dlev <= c->D; ++dlev) c->max_level_rows = std::max(c->max_level_rows, c->tree_h.n_level_rows[dlev]);
  if (cfg->max_batch * c->M > 128) return fail(EAGLE_EINVAL, "max_batch * n_nodes = %d rows exceeds the 128-row limit of one pass", cfg->max_batch * c->M);
  // (the large-M GEMM walks K in stages of 4 k-steps: every K of the model must be a multiple of 64)
  c->big_gemm = !c->f32 && cfg->weight_bits != 4 && cfg->d_ffn % 64 == 0 && (cfg->n_heads * cfg->head_dim) % 64 == 0;
  if (c->big_gemm) {
    c->pf_window = EAGLE_PREFILL_WINDOW;
    c->pf_chunk = c->fixed_sums ? EAGLE_PREFILL_WINDOW
                                : std::min(EAGLE_PREFILL_MAX, (cfg->max_seq + EAGLE_PREFILL_WINDOW - 1) / EAGLE_PREFILL_WINDOW * EAGLE_PREFILL_WINDOW);
  }
  if (c->q4) {
    // 4-bit weights: tree and vanilla passes exist in the fused kernels of the fast path only (at most 32 rows); prompt passes of
    // more rows take the large-M GEMM
    if (c->f32 || cfg->n_experts > 0) return fail(EAGLE_EINVAL, "weight_bits = 4 needs a dense bf16 model");
    if (cfg->d_model % EAGLE_Q4_GROUP || cfg->d_ffn % EAGLE_Q4_GROUP || (cfg->n_heads * cfg->head_dim) % EAGLE_Q4_GROUP)
      return fail(EAGLE_EINVAL, "weight_bits = 4 needs d_model, d_ffn and n_heads * head_dim to be multiples of %d", EAGLE_Q4_GROUP);
    if (cfg->max_batch * c->M > 32 || cfg->max_batch * (c->D + 1) > 32) return fail(EAGLE_EINVAL, "weight_bits = 4: max_batch * n_nodes and max_batch * (depth + 1) must not exceed 32 rows");
    c->pf_window = 32;
    c->pf_chunk = c->fixed_sums ? 32 : std::min(EAGLE_PREFILL_MAX, (cfg->max_seq + 31) / 32 * 32);
    c->q4_rot = c->fixed_sums ? 0 : Q4_ROT_LARGE_M;
  }
  int rows = std::max(c->pf_chunk, cfg->max_batch * c->M);
  c->Mmax = (rows + 31) / 32 * 32;
  if (cfg->head_loss_rows < 0) return fail(EAGLE_EINVAL, "head_loss_rows must be >= 0");
  if (cfg->head_loss_rows > 0) {
    if (c->f32 || c->q4) return fail(EAGLE_EINVAL, "head_loss_rows > 0 needs a bf16 model with its weights as given");
    if (cfg->vocab % 64) return fail(EAGLE_EINVAL, "head_loss_rows > 0 needs vocab to be a multiple of 64");
    // label rows and prediction rows share one pass of the LM head
    const int want = std::min(EAGLE_PREFILL_MAX, 2 * ((cfg->head_loss_rows + 31) / 32 * 32));
    c->hl_chunk = std::max(c->Mmax, want) / 2 / 32 * 32;
    if (c->hl_chunk < 32) return fail(EAGLE_EINVAL, "internal: no room for a loss pass");
  }
  return EAGLE_OK;
}

extern "C" size_t eagle_workspace_bytes(const eagle_config* cfg) {
  eagle_ctx tmp{};
  if (prepare(cfg, &tmp)) return 0;
  tmp.ws = nullptr;
  return layout(&tmp);
}

extern "C" const char* eagle_last_error(void) { return g_err; }
extern "C" const char* eagle_version(void) { return "libeagle 0.1 (gfx950)"; }

// Cosines and sines of every position: plan null: angle = pos * theta^(-2i/dh) formed in fp64, rounded once to fp32; else of the plan's pairs (pairs that
// do not turn: 1 and 0).  Synchronises.
static int upload_rope(eagle_ctx* c, const eagle_rope_plan* plan) {
  const eagle_config& g = c->cfg;
  const int half = g.head_dim / 2;
  std::vector<float> cs((size_t)g.max_seq * half), sn((size_t)g.max_seq * half);
  for (int p = 0; p < g.max_seq; ++p)
    for (int i = 0; i < half; ++i) {
      float &x = cs[(size_t)p * half + i], &y = sn[(size_t)p * half + i];
      if (plan && i >= plan->rot_dim / 2) { x = 1.f; y = 0.f; continue; }
      const double ang = plan ? (double)(int64_t)((uint64_t)p * plan->turn[i]) * (6.283185307179586477 / 18446744073709551616.0)   // (the product wraps at whole turns)
                              : (double)p * std::pow((double)g.rope_theta, -2.0 * i / g.head_dim);
      const double m = plan ? plan->mscale : 1.0;
      x = (float)(std::cos(ang) * m);
      y = (float)(std::sin(ang) * m);
    }
  if (hipMemcpyAsync(c->rope_cos, cs.data(), cs.size() * 4, hipMemcpyHostToDevice, c->stream) != hipSuccess ||
      hipMemcpyAsync(c->rope_sin, sn.data(), sn.size() * 4, hipMemcpyHostToDevice, c->stream) != hipSuccess ||
      hipStreamSynchronize(c->stream) != hipSuccess) return fail(EAGLE_EHIP, "rope table upload failed");
  return EAGLE_OK;
}

extern "C" int eagle_init(const eagle_config* cfg, void* workspace_dev, size_t workspace_bytes, void* hip_stream, eagle_ctx** out) {
  if (!out) return fail(EAGLE_EINVAL, "out is null");
  *out = nullptr;
  eagle_ctx* c = new eagle_ctx();
  int rc = prepare(cfg, c);
  if (rc) { delete c; return rc; }
  if (!workspace_dev || ((uintptr_t)workspace_dev & 255)) { delete c; return fail(EAGLE_EINVAL, "workspace must be a 256-byte aligned device pointer"); }
  c->ws = nullptr;
  size_t need = layout(c);
  if (workspace_bytes < need) { delete c; return fail(EAGLE_ENOMEM, "workspace of %zu bytes is smaller than the %zu needed", workspace_bytes, need); }
  c->ws = (char*)workspace_dev; c->ws_bytes = workspace_bytes;
  layout(c);
  c->stream = (hipStream_t)hip_stream;
  const eagle_config& g = c->cfg;
  {  // address of the static scratch array on the current device, looked up once per device
    if (c->device < 0 || c->device >= EAGLE_MAX_DEVICES) { delete c; return fail(EAGLE_EHIP, "no usable HIP device is current"); }
    std::lock_guard<std::mutex> lock(g_scratch_mutex);
    if (!g_scratch_dev[c->device]) {
      void* p = nullptr;
      hipError_t e = hipGetSymbolAddress(&p, HIP_SYMBOL(scratch));
      if (e != hipSuccess || !p) { delete c; return fail(EAGLE_EHIP, "hipGetSymbolAddress(scratch) failed: %s", hipGetErrorString(e)); }
      g_scratch_dev[c->device] = p;
    }
    c->static_scratch = g_scratch_dev[c->device];
  }
  // the tree arrays are copied: the caller's pointers need not outlive this call
  c->cfg.parent = nullptr; c->cfg.rank = nullptr;
  memset(c->loaded, 0, sizeof(c->loaded));
  c->loaded_layer.assign(EAGLE_W_COUNT, std::vector<char>(g.n_layers + 1, 0));
  c->h_prompt.assign(g.max_batch, 0);
  c->h_ctx.assign(g.max_batch, 0); c->h_ntok.assign(g.max_batch, 0); c->active.assign(g.max_batch, 0); c->head_stale.assign(g.max_batch, 0);
  // zero everything that is not a weight (finite garbage-free caches and padding rows)
  char* z0 = (char*)c->kc;
  size_t zbytes = (size_t)(c->ws + ((c->zero_end + 3) & ~(size_t)3) - z0);
  k_fill_u32<<<2048, 256, 0, c->stream>>>((uint32_t*)z0, 0u, zbytes / 4);
  if (hipGetLastError() != hipSuccess) { delete c; return fail(EAGLE_EHIP, "fill launch failed"); }
  if (hipMemcpyAsync(c->tree_d, &c->tree_h, sizeof(TreeDev), hipMemcpyHostToDevice, c->stream) != hipSuccess) { delete c; return fail(EAGLE_EHIP, "tree upload failed"); }
  {
    const size_t span = (size_t)((const char*)(c->len_out + c->cfg.max_batch) - (const char*)c->path);
    if (hipHostMalloc(&c->res_host, span, hipHostMallocDefault) != hipSuccess) { c->res_host = nullptr; delete c; return fail(EAGLE_ENOMEM, "pinned result buffer"); }
  }
  rc = upload_rope(c, nullptr);
  if (rc) { delete c; return rc; }
  {  // static paging: logical page lp of slot s lives in physical page lp*max_batch + s (interleaved on purpose)
    std::vector<int> pt((size_t)g.max_batch * c->pps);
    for (int s = 0; s < g.max_batch; ++s)
      for (int lp = 0; lp < c->pps; ++lp) pt[(size_t)s * c->pps + lp] = lp * g.max_batch + s;
    if (hipMemcpyAsync(c->page_table, pt.data(), pt.size() * 4, hipMemcpyHostToDevice, c->stream) != hipSuccess ||
        hipStreamSynchronize(c->stream) != hipSuccess) { delete c; return fail(EAGLE_EHIP, "page table upload failed"); }
  }
  if (g.temperature > 0.f && g.vocab <= 32768 &&
      (hipFuncSetAttribute((const void*)k_outcome<ACCEPT_SAMPLED>, hipFuncAttributeMaxDynamicSharedMemorySize, CDF_LDS) != hipSuccess ||
       hipFuncSetAttribute((const void*)k_choose<false>, hipFuncAttributeMaxDynamicSharedMemorySize, CDF_LDS) != hipSuccess)) { delete c; return fail(EAGLE_EHIP, "shared memory of the sampling kernels"); }
  c->hint.future = c->hint_future; c->hint.stride = c->st.tok_stride; c->hint.n = c->hint_n;
  c->hint.alpha = c->hint_alpha; c->hint.bias = c->hint_bias; c->hint.seed = c->hint_seed;
  for (int i = 0; i < 4; ++i)
    if (hipEventCreate(&c->ev[i]) != hipSuccess) { delete c; return fail(EAGLE_EHIP, "event creation failed"); }
  memset(&c->prof, 0, sizeof(c->prof));
#ifdef EAGLE_TRACE
  if (const char* t = getenv("EAGLE_Q4_STAGED")) c->q4_staged = atoi(t) != 0;
  if (const char* t = getenv("EAGLE_GEMM_TRACE")) c->trace_sel = atoi(t);
  if (const char* t = getenv("EAGLE_ATTN_TRACE")) c->attn_trace_sel = atoi(t);
#endif
  *out = c;
  return EAGLE_OK;
}

extern "C" void eagle_free(eagle_ctx* c) {
  if (!c) return;
  (void)hipStreamSynchronize(c->stream);
  for (int i = 0; i < 4; ++i) (void)hipEventDestroy(c->ev[i]);
  for (auto e : c->gemm_ev) (void)hipEventDestroy(e);
  delete c;
}

// ---------------------------------------------------------------------------- weights
static int pack_into(eagle_ctx* c, const void* src, PackedW& w, int N, int K, int row_offset, int mode = PACK_PLAIN) {
  if (K != w.K || row_offset % 32) return fail(EAGLE_EINVAL, "internal: pack shape mismatch");
  int last = mode == PACK_PLAIN ? row_offset + (N + 31) / 32 * 32 : row_offset + pack_row_map(mode, N - 1, c->cfg.head_dim) + 1;
  if ((mode & 15) == PACK_ROPE) last = row_offset + N;
  if (last > w.Npad) return fail(EAGLE_EINVAL, "internal: packed rows overflow");
  if ((mode & 15) == PACK_ROPE && N % c->cfg.head_dim) return fail(EAGLE_EINVAL, "internal: rope packing needs whole heads");
  if ((mode == PACK_GATE || mode == PACK_UP) && N % 16) return fail(EAGLE_EINVAL, "d_ffn must be a multiple of 16");
  if (w.q4) {
    const size_t items = (size_t)(mode == PACK_PLAIN ? (N + 31) / 32 * 32 : N) * w.NG;
    k_pack_weight_q4<bf16_t><<<(unsigned)((items + 255) / 256), 256, 0, c->stream>>>((const bf16_t*)src, (uint32_t*)w.w, w.sc, N, K, row_offset, mode, c->cfg.head_dim, c->q4_rot);
    LAUNCH_CHECK();
    return EAGLE_OK;
  }
  size_t total = (size_t)((N + 31) / 32) * w.KS * 64;
  int blocks = (int)((total + 255) / 256);
  if (c->f32) k_pack_weight<float><<<blocks, 256, 0, c->stream>>>((const float*)src, w.w, N, K, row_offset, w.KS, c->NWP, w.plane_stride, mode, c->cfg.head_dim);
  else k_pack_weight<bf16_t><<<blocks, 256, 0, c->stream>>>((const bf16_t*)src, w.w, N, K, row_offset, w.KS, c->NWP, w.plane_stride, mode, c->cfg.head_dim);
  LAUNCH_CHECK();
  return EAGLE_OK;
}

__global__ void k_to_f32(const bf16_t* src, float* dst, size_t n) {
  for (size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (size_t)gridDim.x * blockDim.x) dst[i] = bf16_to_f32(src[i]);
}

extern "C" int eagle_load_weight(eagle_ctx* c, int32_t which, int32_t layer, const void* src) {
  if (!c || !src) return fail(EAGLE_EINVAL, "null argument");
  if (which < 0 || which >= EAGLE_W_COUNT) return fail(EAGLE_EINVAL, "unknown tensor id %d", which);
  const eagle_config& g = c->cfg;
  const int d = g.d_model, H = g.n_heads, KVH = g.n_kv_heads, dh = g.head_dim, F = g.d_ffn;
  int rc = EAGLE_OK;
  if (which < EAGLE_W_ATTN_NORM) {
    switch (which) {
      case EAGLE_W_EMBED: HIPCHK(hipMemcpyAsync(c->embed, src, (size_t)g.vocab * d * c->elt, hipMemcpyDeviceToDevice, c->stream)); break;
      case EAGLE_W_LM_HEAD:
        rc = pack_into(c, src, c->lm_head, g.vocab, d, 0);
        if (!rc && g.head_loss_rows > 0) {        // W^T for the gradient: row n = column n of the LM head, K = vocab
          PackedW& t = c->lm_head_T;
          const size_t total = (size_t)t.NRB * t.KS * 64;
          k_pack_weight<bf16_t><<<(unsigned)((total + 255) / 256), 256, 0, c->stream>>>((const bf16_t*)src, t.w, d, g.vocab, 0, t.KS, c->NWP, t.plane_stride,
                                                                                      PACK_PLAIN, g.head_dim, (size_t)1, (size_t)d);
          if (hipGetLastError() != hipSuccess) rc = fail(EAGLE_EHIP, "LM head transpose launch failed");
        }
        break;
      case EAGLE_W_FINAL_NORM: HIPCHK(hipMemcpyAsync(c->final_norm, src, (size_t)d * 4, hipMemcpyDeviceToDevice, c->stream)); break;
      case EAGLE_W_FC: rc = pack_into(c, src, c->fc, d, 2 * d, 0); break;
      case EAGLE_W_FC_BIAS: HIPCHK(hipMemcpyAsync(c->fc_bias, src, (size_t)d * 4, hipMemcpyDeviceToDevice, c->stream)); break;
    }
    if (rc) return rc;
    c->loaded_layer[which][0] = 1;
    return EAGLE_OK;
  }
  int li = layer == EAGLE_HEAD_LAYER ? g.n_layers : layer;
  if (li < 0 || li > g.n_layers) return fail(EAGLE_EINVAL, "layer %d out of range", layer);
  LayerW& w = c->layers[li];
  const char* s = (const char*)src;
  switch (which) {
    case EAGLE_W_ATTN_NORM: HIPCHK(hipMemcpyAsync(w.attn_norm, src, (size_t)d * 4, hipMemcpyDeviceToDevice, c->stream)); break;
    case EAGLE_W_MLP_NORM: HIPCHK(hipMemcpyAsync(w.mlp_norm, src, (size_t)d * 4, hipMemcpyDeviceToDevice, c->stream)); break;
    case EAGLE_W_Q: rc = pack_into(c, src, w.qkv, H * dh, d, 0, c->rope_mode); break;
    case EAGLE_W_K: rc = pack_into(c, src, w.qkv, KVH * dh, d, H * dh, c->rope_mode); break;
    case EAGLE_W_V: rc = pack_into(c, src, w.qkv, KVH * dh, d, (H + KVH) * dh); break;
    case EAGLE_W_O: rc = pack_into(c, src, w.o, d, H * dh, 0); break;
    case EAGLE_W_ROUTER:
      if (!w.moe) return fail(EAGLE_EINVAL, "layer %d has no router", layer);
      if (c->f32) HIPCHK(hipMemcpyAsync(w.router, src, (size_t)g.n_experts * d * 4, hipMemcpyDeviceToDevice, c->stream));
      else { k_to_f32<<<64, 256, 0, c->stream>>>((const bf16_t*)src, w.router, (size_t)g.n_experts * d); LAUNCH_CHECK(); }
      break;
    case EAGLE_W_GATE:
    case EAGLE_W_UP:
      if (w.moe) for (int e = 0; e < g.n_experts && !rc; ++e) rc = pack_into(c, s + (size_t)e * F * d * c->elt, w.e_gu[e], F, d, 0, which == EAGLE_W_UP ? PACK_UP : PACK_GATE);
      else rc = pack_into(c, src, w.gu, F, d, 0, which == EAGLE_W_UP ? PACK_UP : PACK_GATE);
      break;
    case EAGLE_W_DOWN:
      if (w.moe) for (int e = 0; e < g.n_experts && !rc; ++e) rc = pack_into(c, s + (size_t)e * d * F * c->elt, w.e_dn[e], d, F, 0);
      else rc = pack_into(c, src, w.dn, d, F, 0);
      break;
  }
  if (rc) return rc;
  c->loaded_layer[which][li] = 1;
  return EAGLE_OK;
}

static int all_loaded(eagle_ctx* c) {
  const eagle_config& g = c->cfg;
  for (int w = 0; w < EAGLE_W_ATTN_NORM; ++w)
    if (w != EAGLE_W_FC_BIAS && !c->loaded_layer[w][0]) return fail(EAGLE_ESTATE, "tensor %d was never loaded", w);
  for (int li = 0; li <= g.n_layers; ++li)
    for (int w = EAGLE_W_ATTN_NORM; w < EAGLE_W_COUNT; ++w) {
      if (w == EAGLE_W_ROUTER && !c->layers[li].moe) continue;
      if (!c->loaded_layer[w][li]) return fail(EAGLE_ESTATE, "tensor %d of layer %d was never loaded", w, li == g.n_layers ? -1 : li);
    }
  return EAGLE_OK;
}

// ---------------------------------------------------------------------------- launches
// Launches a kernel; in profiling mode 2, inside a step, with a start and a stop event attached to the dispatch itself
// (hipExtLaunchKernelGGL): the pair reads the kernel's own begin and end time stamps, so no event-record overhead
// enters the measured duration.  `bytes` = the launch's algorithmic HBM bytes; `name` = the kernel template.
template <typename K, typename... A>
static hipError_t launch_k(eagle_ctx* c, int kclass, double bytes, const char* name, K kernel, dim3 grid, dim3 block, size_t lds, A... args) {
  if (c->prof_mode == 2 && c->cur_phase >= 0) {
    if (c->gemm_ev_used + 2 > c->gemm_ev.size())
      for (int i = 0; i < 512; ++i) {
        hipEvent_t e;
        hipError_t rc = hipEventCreate(&e);
        if (rc != hipSuccess) return rc;
        c->gemm_ev.push_back(e);
      }
    hipExtLaunchKernelGGL(kernel, grid, block, (uint32_t)lds, c->stream, c->gemm_ev[c->gemm_ev_used], c->gemm_ev[c->gemm_ev_used + 1], 0, args...);
    c->gemm_ev_used += 2;
    c->timed.push_back(TimedLaunch{c->cur_phase, kclass, bytes});
    KStat& ks = c->kstat[c->cur_phase][kclass];
    if (!ks.kernel[0]) snprintf(ks.kernel, sizeof(ks.kernel), "%s", name);
  } else {
    kernel<<<grid, block, lds, c->stream>>>(args...);
  }
  return hipGetLastError();
}
template <int NWP, int NXP>
static hipError_t launch_gemm_mt(eagle_ctx* c, const PackedW& w, const bf16_t* XF, float* PT, int MT, const GemmPlan& p) {
  dim3 grid((w.NRB + 3) / 4, p.S);
  size_t lds = (size_t)NXP * MT * GemmChunk<NXP>::CH * 1024;
  const double bytes = (double)w.N * w.K * c->elt;
  const int kc = c->cur_class;
  switch (MT) {
    case 1: return launch_k(c, kc, bytes, "k_gemm<MT=1>", k_gemm<NWP, NXP, 1>, grid, dim3(256), lds, (const bf16_t*)w.w, w.plane_stride, XF, PT, w.NRB, w.KS, p.ks_per_split, w.Npad);
    case 2: return launch_k(c, kc, bytes, "k_gemm<MT=2>", k_gemm<NWP, NXP, 2>, grid, dim3(256), lds, (const bf16_t*)w.w, w.plane_stride, XF, PT, w.NRB, w.KS, p.ks_per_split, w.Npad);
    case 3: return launch_k(c, kc, bytes, "k_gemm<MT=3>", k_gemm<NWP, NXP, 3>, grid, dim3(256), lds, (const bf16_t*)w.w, w.plane_stride, XF, PT, w.NRB, w.KS, p.ks_per_split, w.Npad);
    default: return launch_k(c, kc, bytes, "k_gemm<MT=4>", k_gemm<NWP, NXP, 4>, grid, dim3(256), lds, (const bf16_t*)w.w, w.plane_stride, XF, PT, w.NRB, w.KS, p.ks_per_split, w.Npad);
  }
}

// The work-group tile of the plan, with or without the SwiGLU epilogue.
template <int RBW, int MW, bool SWIGLU, bool PLAIN>
static hipError_t launch_pf(eagle_ctx* c, const PackedW& w, const bf16_t* XF, int MT, const GemmPlan& p, bf16_t* swiglu_out, int M) {
  return launch_k(c, c->cur_class, (double)w.N * w.K * c->elt, SWIGLU ? "k_gemm_pf<swiglu>" : "k_gemm_pf", k_gemm_pf<RBW, MW, SWIGLU, false, PLAIN>, dim3(pf_grid(w.NRB, pf_cols(MT, p), p)),
                  dim3(128 * MW), (size_t)0, (const bf16_t*)w.w, XF, c->PT, w.NRB, w.KS, p.ks_per_split, p.S, w.Npad, MT, swiglu_out, M, (const MoePlan*)nullptr, (size_t)0, 0);
}
template <int RBW, int MW>
static hipError_t launch_pf(eagle_ctx* c, const PackedW& w, const bf16_t* XF, int MT, const GemmPlan& p, bf16_t* swiglu_out, int M) {
  if constexpr (MW <= 2)
    if (plan_pf_plain_loads(w.NRB, MT, M, c->n_cu, p)) return swiglu_out ? launch_pf<RBW, MW, true, true>(c, w, XF, MT, p, swiglu_out, M) : launch_pf<RBW, MW, false, true>(c, w, XF, MT, p, nullptr, M);
  return swiglu_out ? launch_pf<RBW, MW, true, false>(c, w, XF, MT, p, swiglu_out, M) : launch_pf<RBW, MW, false, false>(c, w, XF, MT, p, nullptr, M);
}

template <int RBW, int MW, bool SWIGLU, bool PLAIN = false>
static hipError_t launch_pf_moe(eagle_ctx* c, const std::vector<PackedW>& w, const bf16_t* XF, int MT, const GemmPlan& p, int cols, bf16_t* act) {
  if constexpr (MW <= 2 && !PLAIN)
    if (plan_pf_one_round(w[0].NRB, cols, c->n_cu, p)) return launch_pf_moe<RBW, MW, SWIGLU, true>(c, w, XF, MT, p, cols, act);
  const size_t stride = w.size() > 1 ? (size_t)(w[1].w - w[0].w) : 0;
  return launch_k(c, c->cur_class, (double)w[0].N * w[0].K * c->elt * w.size(), "k_gemm_pf<experts>", k_gemm_pf<RBW, MW, SWIGLU, true, PLAIN>,
                  dim3(pf_grid(w[0].NRB, cols, p)), dim3(128 * MW), (size_t)0, (const bf16_t*)w[0].w, XF, c->PT, w[0].NRB, w[0].KS, p.ks_per_split, p.S,
                  w[0].Npad, MT, act, 0, (const MoePlan*)c->moe_plan, stride, cols);
}
template <bool SWIGLU>
static hipError_t launch_pf_moe(eagle_ctx* c, const std::vector<PackedW>& w, const bf16_t* XF, int MT, const GemmPlan& p, int cols, bf16_t* act) {
  if (p.mw == 4) return p.rbw == 4 ? launch_pf_moe<4, 4, SWIGLU>(c, w, XF, MT, p, cols, act) : p.rbw == 3 ? launch_pf_moe<3, 4, SWIGLU>(c, w, XF, MT, p, cols, act)
                                                                                                : launch_pf_moe<2, 4, SWIGLU>(c, w, XF, MT, p, cols, act);
  return p.rbw == 4 ? launch_pf_moe<4, 2, SWIGLU>(c, w, XF, MT, p, cols, act) : launch_pf_moe<3, 2, SWIGLU>(c, w, XF, MT, p, cols, act);
}

static hipError_t launch_pf_q4(eagle_ctx* c, const PackedW& w, const bf16_t* XF, int MT, const GemmPlan& p, bf16_t* swiglu_out, int M) {
  const int MQ = (MT + 3) / 4, G = ((w.NRB + 3) / 4) * p.S;
  return launch_k(c, c->cur_class, w.bytes(c->elt), "k_gemm_pf<4-bit weights>", swiglu_out ? k_gemm_pf_q4<true> : k_gemm_pf_q4<false>,
                  dim3((G + 7) / 8 * 8 * MQ), dim3(256), (size_t)0, (const u32x4*)w.w, (const bf16_t*)w.sc, XF, (const float*)c->group_sums, c->PT, w.NRB, w.KS,
                  p.ks_per_split / 8, p.S, w.Npad, MT, swiglu_out, M);
}

// PT <- X (XF layout, M rows in MT row tiles) times W^T.  Returns the split count through *S.
// swiglu_out (gate/up matrices only): where the plan has a single K slice in the large-M kernel, the SwiGLU epilogue runs
// inside the GEMM and its output goes to swiglu_out in GEMM-input layout; *S is then 0 (nothing left in PT).
static int gemm(eagle_ctx* c, const PackedW& w, const bf16_t* XF, int MT, int M, int* S, bf16_t* swiglu_out = nullptr) {
  const bool big = use_pf(c, MT);
  GemmPlan p = big ? plan_pf(w.NRB, w.KS, MT, c->n_cu, swiglu_out != nullptr, c->q4, c->fixed_sums) : plan_gemm(w.NRB, w.KS, c->NXP, MT);
  const bool fuse = big && swiglu_out && p.S == 1;
  if (!fuse && (size_t)p.S * w.Npad * MT * 32 > c->pt_floats) return fail(EAGLE_EINVAL, "internal: partial buffer too small");
  if (MT < 1 || MT * 32 > std::max(c->Mmax, 2 * c->hl_chunk) || M <= 32 * (MT - 1) || M > 32 * MT || (big && c->f32)) return fail(EAGLE_EINVAL, "internal: rows out of range");
  *S = fuse ? 0 : p.S;
  hipError_t e;
  if (w.q4) {
    if (c->q4_rot != Q4_ROT_LARGE_M) return fail(EAGLE_EINVAL, "internal: the large-M GEMM does not read 4-bit codes in this packing");
    bf16_t* out = fuse ? swiglu_out : nullptr;
    k_group_sums<<<dim3(MT, (w.NG + 3) / 4), 256, 0, c->stream>>>(XF, c->group_sums, MT, w.KS, c->NXP);
    LAUNCH_CHECK();
    e = launch_pf_q4(c, w, XF, MT, p, out, M);
  } else if (big) {
    bf16_t* out = fuse ? swiglu_out : nullptr;
    if (p.mw == 4) e = p.rbw == 4 ? launch_pf<4, 4>(c, w, XF, MT, p, out, M) : p.rbw == 3 ? launch_pf<3, 4>(c, w, XF, MT, p, out, M) : launch_pf<2, 4>(c, w, XF, MT, p, out, M);
    else if (p.mw == 2) e = p.rbw == 4 ? launch_pf<4, 2>(c, w, XF, MT, p, out, M) : launch_pf<3, 2>(c, w, XF, MT, p, out, M);
    else e = p.rbw == 4 ? launch_pf<4, 1>(c, w, XF, MT, p, out, M) : launch_pf<3, 1>(c, w, XF, MT, p, out, M);
  } else e = c->f32 ? launch_gemm_mt<3, 3>(c, w, XF, c->PT, MT, p) : launch_gemm_mt<1, 2>(c, w, XF, c->PT, MT, p);
  if (e != hipSuccess) return fail(EAGLE_EHIP, "gemm launch failed: %s", hipGetErrorString(e));
  return EAGLE_OK;
}

template <int NRMAX, int MT>
static hipError_t launch_wk(eagle_ctx* c, double bytes, const GemmWK& g) {
  static bool attr_set = false;
  if (!attr_set) {
    hipError_t e = hipFuncSetAttribute((const void*)k_gemm_wk<NRMAX, MT>, hipFuncAttributeMaxDynamicSharedMemorySize, 128 * 1024);
    if (e != hipSuccess) return e;
    attr_set = true;
  }
  return launch_k(c, c->cur_class, bytes, "k_gemm_wk", k_gemm_wk<NRMAX, MT>, dim3(c->n_cu), dim3(256), (size_t)128 * 1024, g);
}
// act <- SwiGLU of X (M rows in MT row tiles) times the gate/up matrix, all of K in a work-group (plan_is_wk).
static int gemm_wk(eagle_ctx* c, const PackedW& w, const bf16_t* XF, int MT, int M, bf16_t* act) {
  const GemmWK g{w.w, XF, w.NRB, w.KS, M, act};
  const double bytes = w.bytes(c->elt);
  const int nrmax = (w.NRB + c->n_cu - 1) / c->n_cu;
  if (nrmax < 3 || nrmax > 4 || (nrmax == 4 && MT != 2) || w.KS % 4 || M <= 32 * (MT - 1) || M > 32 * MT) return fail(EAGLE_EINVAL, "internal: no whole-K plan for %d row blocks and %d rows", w.NRB, M);
  hipError_t e = nrmax == 4 ? launch_wk<4, 2>(c, bytes, g) : MT == 2 ? launch_wk<3, 2>(c, bytes, g) : MT == 3 ? launch_wk<3, 3>(c, bytes, g) : launch_wk<3, 4>(c, bytes, g);
  if (e != hipSuccess) return fail(EAGLE_EHIP, "gemm launch failed: %s", hipGetErrorString(e));
  return EAGLE_OK;
}

// Reads the event pairs of the launches timed since the last call (the stream must have been synchronised).
static int collect_gemm_events(eagle_ctx* c) {
  for (size_t i = 0; i < c->timed.size(); ++i) {
    float ms = 0.f;
    HIPCHK(hipEventElapsedTime(&ms, c->gemm_ev[2 * i], c->gemm_ev[2 * i + 1]));
    const TimedLaunch& t = c->timed[i];
    KStat& ks = c->kstat[t.phase][t.kclass];
    ks.ms += ms; ks.launches += 1; ks.bytes += t.bytes;
    if (t.kclass != KC_ATTN) { c->prof.gemm_ms += ms; c->prof.gemm_launches += 1; c->prof.gemm_weight_bytes += t.bytes; }
  }
  c->gemm_ev_used = 0; c->timed.clear();
  return EAGLE_OK;
}

static int attn_splits(const eagle_ctx* c, int tokens, int units) { return plan_attn_splits(c->fixed_sums, tokens, units, c->n_cu); }

// Algorithmic HBM bytes of one attention launch: keys and values of every sequence's cached context plus the pass's
// own rows, once (host mirror of the cached lengths; prefill chunks: the chunk's causal prefix).
static double attn_bytes(const eagle_ctx* c, const Pass& p, int n_new) {
  const eagle_config& g = c->cfg;
  double toks = 0;
  if (p.kind == PASS_PREFILL_T || p.kind == PASS_PREFILL_D) toks = p.chunk_start + p.chunk_n;
  else for (int i = 0; i < p.n_seq; ++i) toks += c->h_ctx[p.seq0 + i] + n_new;
  return toks * 2.0 * g.n_kv_heads * g.head_dim * c->kv_elt;
}

static KVCache kv_for(eagle_ctx* c, int li) {
  KVCache kv;
  const eagle_config& g = c->cfg;
  bool head = li == g.n_layers;
  char* kb = (char*)(head ? c->dkc : c->kc);
  char* vb = (char*)(head ? c->dvc : c->vc);
  size_t off = head ? 0 : (size_t)li * c->layer_stride * c->kv_elt;
  kv.k = kb + off; kv.v = vb + off;
  kv.page_table = c->page_table; kv.pages_per_seq = c->pps; kv.page_shift = c->page_shift;
  kv.n_kv_heads = g.n_kv_heads; kv.head_dim = g.head_dim;
  return kv;
}

static AttnArgs attn_args(eagle_ctx* c, const Pass& pass, const KVCache& kv, int n_splits, int n_new, bf16_t* xf_out, int MT, int rblocks, unsigned long long* trace) {
  AttnArgs a;
  a.rows_per_seq = pass.rows_per_seq; a.causal = pass.kind >= PASS_PREFILL_T || pass.kind == PASS_DRAFT_PENDING;
  a.facts = c->facts; a.kv = kv; a.Q = c->Q; a.part_o = c->part_o; a.part_ml = c->part_ml;
  a.H = c->cfg.n_heads; a.n_splits = n_splits; a.n_new = n_new; a.scale = 1.0f / std::sqrt((float)c->cfg.head_dim);
  a.counters = c->cnt_attn; a.xf_out = xf_out; a.nplanes = c->NXP; a.MT = MT; a.rblocks = rblocks; a.trace = trace;
  const bool known = pass.ctx_known && (pass.kind == PASS_VERIFY || pass.kind == PASS_VANILLA || pass.kind == PASS_DRAFT_LEVEL);
  const int before = pass.kind == PASS_DRAFT_LEVEL ? 1 : 0;     // (row_info)
  a.slot0 = known ? pass.seq0 : -1;
  a.ctx[0] = pass.ctx0 - before; a.ctx[1] = pass.ctx1 - before; a.ctx[2] = pass.ctx2 - before; a.ctx[3] = pass.ctx3 - before;
  return a;
}

static int resnorm(eagle_ctx* c, int M, int MT, const float* h_in, const float* PT, int S, int Npad, const float* bias,
                   const float* gain, bf16_t* XF, float* xout, const float* row_w = nullptr) {
  if (c->fixed_sums) {
    k_resnorm_fixed<<<M, 256, 0, c->stream>>>(h_in, PT, S, Npad, MT * 32, bias, c->h, gain, c->cfg.rms_eps, XF, MT, c->NXP, xout, c->cfg.d_model);
    LAUNCH_CHECK();
    return EAGLE_OK;
  }
  k_resnorm<false><<<M, RESNORM_THREADS, 0, c->stream>>>(h_in, PT, S, Npad, MT * 32, bias, c->h, gain, c->cfg.rms_eps, XF, MT, c->NXP, xout, c->cfg.d_model, row_w,
                                                         nullptr, nullptr, 0, 0);
  LAUNCH_CHECK();
  return EAGLE_OK;
}

// Attention under eagle_set_attention: the pass as a chunk over the layer's cache (pass_chunk), in place over the queries, then re-laid as input of the output projection.
static int pass_chunk(eagle_ctx* c, const Pass& pass, int n_new) {
  if (!c->attn_ruled) return EAGLE_OK;
  k_pass_chunk<<<1, 256, 0, c->stream>>>(c->facts, pass.kind, pass.n_seq, pass.rows_per_seq, n_new, pass.chunk_start + pass.chunk_n, c->op_start, c->op_len, c->op_base, c->op_mask);
  LAUNCH_CHECK();
  return EAGLE_OK;
}
static int ruled_attention(eagle_ctx* c, const Pass& pass, int M, int MT, const KVCache& kv, int max_keys, bf16_t* xf) {
  const eagle_config& g = c->cfg;
  const int H = g.n_heads, dh = g.head_dim;
  const bool prompt = pass.kind >= PASS_PREFILL_T;
  eagle_chunk ch{};
  ch.n_seqs = pass.n_seq; ch.n_rows = M; ch.max_rows = pass.rows_per_seq; ch.max_keys = std::min(max_keys, c->pps << c->page_shift);
  ch.row_start = c->op_start; ch.key_len = c->op_len;
  if (!prompt) { ch.tree_base = c->op_base; ch.tree_mask = (const uint64_t*)c->op_mask; }
  eagle_paged_kv pk{};
  pk.k = kv.k; pk.v = kv.v; pk.dtype = c->kv_f32 ? EAGLE_F32 : EAGLE_BF16; pk.n_kv_heads = g.n_kv_heads; pk.head_dim = dh; pk.page_tokens = g.page_tokens;
  pk.n_pages = g.max_batch * c->pps; pk.pages_per_seq = c->pps; pk.token_stride = dh; pk.head_stride = (int64_t)g.page_tokens * dh; pk.page_stride = pk.head_stride * g.n_kv_heads;
  pk.table_stride = c->pps; pk.page_table = c->page_table + (size_t)pass.seq0 * c->pps;
  eagle_attention_args aa{};
  aa.n_heads = H; aa.dtype = EAGLE_F32; aa.window = c->attn_rules.window; aa.q = c->Q; aa.out = c->Q; aa.q_row = aa.out_row = (int64_t)H * dh; aa.q_head = aa.out_head = dh;
  aa.scale = 1.0f / std::sqrt((float)dh); aa.softcap = c->attn_rules.softcap; aa.slopes = c->attn_rules.slopes_dev;
  const int rc = chunk_attention(&aa, &ch, &pk, c->part_o, (size_t)((char*)(c->part_ml + c->part_rows * H * 2) - (char*)c->part_o), true, c->stream);
  if (rc) return rc;
  k_rows_to_xf<<<dim3(M, (H * dh + 2047) / 2048), 256, 0, c->stream>>>(c->Q, 0, xf, MT, c->NXP, H * dh);
  LAUNCH_CHECK();
  return EAGLE_OK;
}

// One decoder layer on the rows of `pass` (h and xf_d hold the residual stream and its normalised copy).
// next_gain: the RMSNorm gain applied to the layer's output for whoever consumes it next (nullptr = none).
static int layer_forward(eagle_ctx* c, const Pass& pass, int M, int MT, int li, int t_max, int n_new, const float* next_gain, float* xout) {
  const eagle_config& g = c->cfg;
  LayerW& w = c->layers[li];
  const int H = g.n_heads, dh = g.head_dim, F = g.d_ffn;
  int S = 1, rc;
  KVCache kv = kv_for(c, li);
  if ((rc = (c->cur_class = KC_QKV, gemm(c, w.qkv, c->xf_d, MT, M, &S)))) return rc;
  {
    dim3 grid(M, (w.qkv.N / 4 + 255) / 256);
    if (c->kv_f32) k_qkv_rope_store<float><<<grid, 256, 0, c->stream>>>(c->facts, c->PT, S, w.qkv.N, w.qkv.Npad, MT * 32, c->rope_cos, c->rope_sin, c->Q, kv, H);
    else k_qkv_rope_store<bf16_t><<<grid, 256, 0, c->stream>>>(c->facts, c->PT, S, w.qkv.N, w.qkv.Npad, MT * 32, c->rope_cos, c->rope_sin, c->Q, kv, H);
    LAUNCH_CHECK();
  }
  if (c->attn_ruled) { if ((rc = ruled_attention(c, pass, M, MT, kv, t_max, c->xf_att))) return rc; }
  else {
    // the MFMA attention kernel of the fast path, one work-group per (KV split, head, sequence x 32-row block)
    int rblocks = (pass.rows_per_seq + 31) / 32;
    int n_splits = attn_splits(c, t_max, H * pass.n_seq * rblocks);
    // (dense models with a bf16 cache keep k2_attn's order of sums, see fixed_sums)
    const bool prompt = !c->fixed_sums && pass.kind >= PASS_PREFILL_T && pass.n_seq == 1 && n_splits == 1 && plan_is_prompt_attn(M, H, c->n_cu);
    if (pass.n_seq * rblocks > 128) return fail(EAGLE_EINVAL, "internal: too many (sequence, row block) pairs in one pass");
    dim3 grid(n_splits, H, pass.n_seq * rblocks);
#define ATTNG(CT, DH)                                                                                                   \
  do {                                                                                                                  \
    static bool attr_done = false;                                                                                      \
    if (!attr_done) {                                                                                                   \
      HIPCHK(hipFuncSetAttribute((const void*)k2_attn<CT, DH>, hipFuncAttributeMaxDynamicSharedMemorySize, 80 * 1024)); \
      HIPCHK(hipFuncSetAttribute((const void*)k2_attn_prompt<CT, DH>, hipFuncAttributeMaxDynamicSharedMemorySize, 144 * 1024)); \
      attr_done = true;                                                                                                 \
    }                                                                                                                   \
    const AttnArgs aa = attn_args(c, pass, kv, n_splits, n_new, c->xf_att, MT, rblocks, nullptr);                       \
    hipError_t e_ = prompt                                                                                              \
        ? launch_k(c, KC_ATTN, attn_bytes(c, pass, n_new), "k2_attn_prompt", k2_attn_prompt<CT, DH>, dim3(H, (M + 127) / 128), dim3(ATTN_PROMPT_THREADS), std::max((size_t)DH / 16 * 8 * 2048, (size_t)4 * (DH / 2 + 2) * 256), aa) \
        : launch_k(c, KC_ATTN, attn_bytes(c, pass, n_new), "k2_attn", k2_attn<CT, DH>, grid, dim3(256), (size_t)(4 * 32 * (DH + 4) + 4 * 2 * 32) * 4, aa); \
    if (e_ != hipSuccess) return fail(EAGLE_EHIP, "attention launch failed: %s", hipGetErrorString(e_));                \
  } while (0)
    if (c->kv_f32) { if (dh == 128) ATTNG(float, 128); else if (dh == 64) ATTNG(float, 64); else ATTNG(float, 32); }
    else { if (dh == 128) ATTNG(bf16_t, 128); else if (dh == 64) ATTNG(bf16_t, 64); else ATTNG(bf16_t, 32); }
#undef ATTNG
    LAUNCH_CHECK();
  }
  if ((rc = (c->cur_class = KC_O, gemm(c, w.o, c->xf_att, MT, M, &S)))) return rc;
  if ((rc = resnorm(c, M, MT, c->h, c->PT, S, w.o.Npad, nullptr, w.mlp_norm, c->xf_d, w.moe ? c->xn : nullptr))) return rc;
  if (w.moe) {
    const int E = g.n_experts;
    k_fill_u32<<<1, 64, 0, c->stream>>>((uint32_t*)c->expert_used, 0u, (size_t)E);
    LAUNCH_CHECK();
    k_router<<<M, 256, 0, c->stream>>>(c->xn, nullptr, nullptr, 0, 0.f, 0.f, nullptr, w.router, E, g.experts_per_tok, g.d_model, M, c->moe_w, c->Mmax, c->expert_used);
    LAUNCH_CHECK();
    if (c->prof_mode) { k_count_used<<<1, 64, 0, c->stream>>>(c->expert_used, E, c->experts_touched); LAUNCH_CHECK(); }
    if (c->big_gemm) {
      // every row goes to its own experts only: the rows are gathered by expert, the MLP of all experts is two launches, and
      // the results are added per row in expert order.  (Every expert over all rows, row weights of 0 included, is E / topk
      // times the matrix work and 4 launches an expert: Mixtral widths, 1000 rows: 6.2 ms a layer, grouped 1.9.)
      const int k = g.experts_per_tok, tiles = moe_tiles(32 * MT, k, E);
      const PlanMoe p = plan_moe(w.e_gu[0].NRB, w.e_gu[0].KS, w.e_dn[0].NRB, w.e_dn[0].KS, 32 * MT, k, E, c->n_cu);
      if (p.cols > MOE_MAX_COLS || (size_t)p.dn.S * w.e_dn[0].Npad * 32 * tiles > c->pt_floats) return fail(EAGLE_EINVAL, "internal: expert plan out of range");
      k_moe_plan<<<1, 1024, 0, c->stream>>>(c->moe_w, c->Mmax, E, M, 2 * p.gu.mw, c->moe_plan, c->moe_slot, c->moe_row);
      LAUNCH_CHECK();
      k_moe_gather<<<dim3(tiles, (g.d_model / 16 + 15) / 16), 256, 0, c->stream>>>(c->moe_plan, c->moe_row, c->xf_d, MT, c->xf_moe, tiles, g.d_model / 16, c->NXP);
      LAUNCH_CHECK();
      const int cols = std::min(p.cols, M * k);                 // every column has a row
      hipError_t e = (c->cur_class = KC_GATEUP, launch_pf_moe<true>(c, w.e_gu, c->xf_moe, tiles, p.gu, cols, c->xf_ffn));
      if (e == hipSuccess) e = (c->cur_class = KC_DOWN, launch_pf_moe<false>(c, w.e_dn, c->xf_ffn, tiles, p.dn, cols, nullptr));
      if (e != hipSuccess) return fail(EAGLE_EHIP, "expert gemm launch failed: %s", hipGetErrorString(e));
      k_resnorm<true><<<M, RESNORM_THREADS, 0, c->stream>>>(c->h, c->PT, p.dn.S, w.e_dn[0].Npad, tiles * 32, nullptr, c->h, next_gain, g.rms_eps, c->xf_d, MT, c->NXP, xout,
                                          g.d_model, nullptr, c->moe_w, c->moe_slot, c->Mmax, E);
      LAUNCH_CHECK();
      return EAGLE_OK;
    }
    // (fp32 models: every expert over all rows; a row's result is scaled by its routing weight, 0 for experts it did not select)
    for (int e = 0; e < E; ++e) {
      if ((rc = (c->cur_class = KC_GATEUP, gemm(c, w.e_gu[e], c->xf_d, MT, M, &S)))) return rc;
      dim3 grid((F / 16 + 3) / 4, MT);
      k_swiglu<<<grid, 256, 0, c->stream>>>(c->PT, S, w.e_gu[e].Npad, MT * 32, F, M, c->xf_ffn, MT, c->NXP);
      LAUNCH_CHECK();
      if ((rc = (c->cur_class = KC_DOWN, gemm(c, w.e_dn[e], c->xf_ffn, MT, M, &S)))) return rc;
      const bool last = e + 1 == E;     // only the last expert's pass produces the normalised output
      if ((rc = resnorm(c, M, MT, c->h, c->PT, S, w.e_dn[e].Npad, nullptr, last ? next_gain : nullptr, last ? c->xf_d : nullptr,
                        last ? xout : nullptr, c->moe_w + (size_t)e * c->Mmax))) return rc;
    }
    return EAGLE_OK;
  }
  c->cur_class = KC_GATEUP;
  if (plan_is_wk(w.gu.NRB, w.gu.KS, MT, c->n_cu, c->big_gemm, c->fixed_sums, c->q4)) {
    if ((rc = gemm_wk(c, w.gu, c->xf_d, MT, M, c->xf_ffn))) return rc;
    S = 0;
  } else if ((rc = gemm(c, w.gu, c->xf_d, MT, M, &S, c->xf_ffn))) return rc;
  if (S > 0) {
    dim3 grid((F / 16 + 3) / 4, MT);
    k_swiglu<<<grid, 256, 0, c->stream>>>(c->PT, S, w.gu.Npad, MT * 32, F, M, c->xf_ffn, MT, c->NXP);
    LAUNCH_CHECK();
  }
  if ((rc = (c->cur_class = KC_DOWN, gemm(c, w.dn, c->xf_ffn, MT, M, &S)))) return rc;
  return resnorm(c, M, MT, c->h, c->PT, S, w.dn.Npad, nullptr, next_gain, c->xf_d, xout);
}

static int lm_head(eagle_ctx* c, const Pass& pass, int M, int MT, float* out, int out_kind, int only_last_row,
                   const bf16_t* XF = nullptr) {
  int S, rc;
  if ((rc = (c->cur_class = KC_LMHEAD, gemm(c, c->lm_head, XF ? XF : c->xf_d, MT, M, &S)))) return rc;
  dim3 grid((c->cfg.vocab + 255) / 256, M);
  k_logits<<<grid, 256, 0, c->stream>>>(pass, c->tree_d, c->st, c->PT, S, c->lm_head.Npad, MT * 32, out, out_kind, c->cfg.vocab, only_last_row);
  LAUNCH_CHECK();
  return EAGLE_OK;
}

static int lm_head2(eagle_ctx* c, int M, bool scaled, float* out, const bf16_t* XF = nullptr);

// Target model over the rows of `pass`: embedding -> layers -> final norm (= features) -> LM head.
static int target_forward(eagle_ctx* c, const Pass& pass, int t_max, int n_new, bool want_logits, float* logits_out, int out_kind, int only_last_row) {
  const eagle_config& g = c->cfg;
  const int M = pass.rows_per_seq * pass.n_seq, MT = (M + 31) / 32;
  int rc;
  if (c->f32) k_embed<float><<<M, 256, 0, c->stream>>>(pass, c->tree_d, c->st, c->tree_tok, (const float*)c->embed, c->h, g.d_model, g.vocab, kv_for(c, 0), c->facts);
  else k_embed<bf16_t><<<M, 256, 0, c->stream>>>(pass, c->tree_d, c->st, c->tree_tok, (const bf16_t*)c->embed, c->h, g.d_model, g.vocab, kv_for(c, 0), c->facts);
  LAUNCH_CHECK();
  if ((rc = pass_chunk(c, pass, n_new))) return rc;
  if ((rc = resnorm(c, M, MT, c->h, nullptr, 0, 0, nullptr, c->layers[0].attn_norm, c->xf_d, nullptr))) return rc;
  for (int l = 0; l < g.n_layers; ++l) {
    bool last = l + 1 == g.n_layers;
    if ((rc = layer_forward(c, pass, M, MT, l, t_max, n_new, last ? c->final_norm : c->layers[l + 1].attn_norm, last ? c->featbuf : nullptr))) return rc;
  }
  k_store_rows<<<M, 256, 0, c->stream>>>(pass, c->tree_d, c->st, c->featbuf, c->F, c->pend_f, c->chunk_f, g.d_model);
  LAUNCH_CHECK();
  if (want_logits && only_last_row && pass.kind == PASS_PREFILL_T && MT > 1) {
    // a prompt pass needs the distribution of its last position only: the LM head runs over the last 32-row tile,
    // whose features (already normalised) are re-laid as a one-tile GEMM input
    const int row0 = (MT - 1) * 32, nr = M - row0;
    if ((rc = resnorm(c, nr, 1, c->featbuf + (size_t)row0 * g.d_model, nullptr, 0, 0, nullptr, nullptr, c->xf_2d, nullptr))) return rc;
    Pass sub = pass;
    sub.rows_per_seq = nr; sub.chunk_start = pass.chunk_start + row0; sub.chunk_n = nr;
    if (c->q4) {
      k_row_facts<<<1, 64, 0, c->stream>>>(sub, c->tree_d, c->st, nr, kv_for(c, 0), c->facts);
      LAUNCH_CHECK();
      return lm_head2(c, nr, false, logits_out, c->xf_2d);
    }
    return lm_head(c, sub, nr, 1, logits_out, out_kind, only_last_row, c->xf_2d);
  }
  if (want_logits) return lm_head(c, pass, M, MT, logits_out, out_kind, only_last_row);
  return EAGLE_OK;
}

static LevelParents level_parents(const eagle_ctx* c, const Pass& p) {
  LevelParents l;
  memset(&l, 0, sizeof(l));
  l.M = c->M; l.D1 = c->D + 1;
  if (p.kind == PASS_DRAFT_LEVEL)
    for (int i = 0; i < p.rows_per_seq; ++i) { const int v = c->tree_h.level_rows[p.level][i]; l.node[i] = (uint8_t)v; l.parent[i] = (uint8_t)c->tree_h.parent[v]; }
  return l;
}
// Autoregression Head over the rows of `pass`: concat(feature, token embedding) -> FC -> decoder layer (-> LM head).
static int head_forward(eagle_ctx* c, const Pass& pass, int t_max, int n_new, bool want_logits) {
  const eagle_config& g = c->cfg;
  const int M = pass.rows_per_seq * pass.n_seq, MT = (M + 31) / 32;
  int rc, S;
  if (c->f32) k_fc_input<float><<<dim3(M, 4), 256, 0, c->stream>>>(pass, c->tree_d, c->st, c->tree_tok, c->pend_f, c->node_f, c->chunk_f, (const float*)c->embed, c->xf_2d, g.d_model, g.vocab, MT, c->NXP, kv_for(c, g.n_layers), c->facts, level_parents(c, pass));
  else k_fc_input<bf16_t><<<dim3(M, 4), 256, 0, c->stream>>>(pass, c->tree_d, c->st, c->tree_tok, c->pend_f, c->node_f, c->chunk_f, (const bf16_t*)c->embed, c->xf_2d, g.d_model, g.vocab, MT, c->NXP, kv_for(c, g.n_layers), c->facts, level_parents(c, pass));
  LAUNCH_CHECK();
  if ((rc = pass_chunk(c, pass, n_new))) return rc;
  if ((rc = (c->cur_class = KC_FC, gemm(c, c->fc, c->xf_2d, MT, M, &S)))) return rc;
  const float* bias = c->loaded_layer[EAGLE_W_FC_BIAS][0] ? c->fc_bias : nullptr;
  if ((rc = resnorm(c, M, MT, nullptr, c->PT, S, c->fc.Npad, bias, c->layers[g.n_layers].attn_norm, c->xf_d, nullptr))) return rc;
  if ((rc = layer_forward(c, pass, M, MT, g.n_layers, t_max, n_new, nullptr, c->featbuf))) return rc;
  if (!want_logits) return EAGLE_OK;
  k_store_rows<<<M, 256, 0, c->stream>>>(pass, c->tree_d, c->st, c->featbuf, c->node_f, c->pend_f, c->chunk_f, g.d_model);
  LAUNCH_CHECK();
  return lm_head(c, pass, M, MT, c->draft_logits, 0, 0);
}

// ---------------------------------------------------------------------------- fast path (<= 32 rows)
template <int NWP, int NXP, int RW, int DEPTH, bool Q4 = false>
static hipError_t launch_k2(eagle_ctx* c, double bytes, const Gemm2& g, size_t lds) {
  static bool attr_set = false;
  if (!attr_set) {
    hipError_t e = hipFuncSetAttribute((const void*)k2_gemm<NWP, NXP, RW, DEPTH, Q4>, hipFuncAttributeMaxDynamicSharedMemorySize, 144 * 1024);
    if (e != hipSuccess) return e;
    attr_set = true;
  }
  return launch_k(c, c->cur_class, bytes, Q4 ? "k2_gemm<4-bit weights>" : "k2_gemm", k2_gemm<NWP, NXP, RW, DEPTH, Q4>, dim3(g.groups * g.S), dim3(V2_THREADS), lds, g);
}

template <int EPI, int NRMAX, bool HALF, int NWP, int NXP, bool Q4, bool EXPERTS>
static hipError_t launch_fk_epi(eagle_ctx* c, double bytes, Gemm2& g, int grid, int experts) {
  static bool attr_set = false;
  const size_t lds = (size_t)8 * NRMAX * 4096;
  if (lds > 144 * 1024) return hipErrorInvalidValue;
  if (!attr_set) {
    hipError_t e = hipFuncSetAttribute((const void*)k2_gemm_fk<EPI, NWP, NXP, NRMAX, HALF, Q4, EXPERTS>, hipFuncAttributeMaxDynamicSharedMemorySize, 144 * 1024);
    if (e != hipSuccess) return e;
    attr_set = true;
  }
  const Share sh = share_of(HALF ? 2 * g.NRB : g.NRB, grid);
  g.groups = grid; g.share_a = sh.a; g.share_b = sh.b;
  return launch_k(c, c->cur_class, bytes, Q4 ? "k2_gemm_fk<4-bit weights>" : HALF ? "k2_gemm_fk<half blocks>" : "k2_gemm_fk", k2_gemm_fk<EPI, NWP, NXP, NRMAX, HALF, Q4, EXPERTS>,
                  dim3(grid, experts), dim3(V2_THREADS), lds, g);
}
template <int NRMAX, bool HALF = false, int NWP = 1, int NXP = 2, bool EXPERTS = false, bool Q4 = false>
static hipError_t launch_fk(eagle_ctx* c, double bytes, Gemm2& g, int grid, int experts = 1) {
  if constexpr (HALF) return launch_fk_epi<EPI_QKV, NRMAX, HALF, NWP, NXP, Q4, EXPERTS>(c, bytes, g, grid, experts);
  else if constexpr (EXPERTS) return launch_fk_epi<EPI_SWIGLU, NRMAX, HALF, NWP, NXP, Q4, EXPERTS>(c, bytes, g, grid, experts);
  else {
    if constexpr (NRMAX <= 2)
      if (g.epi == EPI_RESID) return launch_fk_epi<EPI_RESID, NRMAX, HALF, NWP, NXP, Q4, EXPERTS>(c, bytes, g, grid, experts);
    switch (g.epi) {
      case EPI_QKV: return launch_fk_epi<EPI_QKV, NRMAX, HALF, NWP, NXP, Q4, EXPERTS>(c, bytes, g, grid, experts);
      case EPI_SWIGLU: return launch_fk_epi<EPI_SWIGLU, NRMAX, HALF, NWP, NXP, Q4, EXPERTS>(c, bytes, g, grid, experts);
      case EPI_LOGITS: return launch_fk_epi<EPI_LOGITS, NRMAX, HALF, NWP, NXP, Q4, EXPERTS>(c, bytes, g, grid, experts);
      default: return hipErrorInvalidValue;
    }
  }
}

template <bool RESID, int NRMAX, bool Q4, bool EXPERTS>
static hipError_t launch_xk_epi(eagle_ctx* c, double bytes, Gemm2& g, int experts) {
  static bool attr_set = false;
  const size_t lds = (size_t)8 * NRMAX * 4096;
  if (!attr_set) {
    hipError_t e = hipFuncSetAttribute((const void*)k2_gemm_xk<RESID, 2, NRMAX, Q4, EXPERTS>, hipFuncAttributeMaxDynamicSharedMemorySize, 144 * 1024);
    if (e != hipSuccess) return e;
    attr_set = true;
  }
  g.share_a = magic_of(g.groups); g.S_magic = magic_of(g.S);
  if (!magic_holds((uint64_t)g.groups * g.NRB, g.groups) || !magic_holds((uint64_t)g.S * (Q4 ? g.NG : g.KS), g.S)) return hipErrorInvalidValue;   // (at most 256 groups of 4 row blocks, 16 slices)
  return launch_k(c, c->cur_class, bytes, Q4 ? "k2_gemm_xk<4-bit weights>" : "k2_gemm_xk", k2_gemm_xk<RESID, 2, NRMAX, Q4, EXPERTS>, dim3(g.S, g.groups, experts), dim3(V2_THREADS), lds, g);
}
template <int NRMAX, bool EXPERTS = false, bool Q4 = false>
static hipError_t launch_xk(eagle_ctx* c, double bytes, Gemm2& g, int experts = 1) {
  if constexpr (!EXPERTS && !Q4)
    if (g.epi != EPI_RESID) return launch_xk_epi<false, NRMAX, Q4, EXPERTS>(c, bytes, g, experts);
  return launch_xk_epi<true, NRMAX, Q4, EXPERTS>(c, bytes, g, experts);
}

// Work split of the streamed split-K kernel for 4-bit weights: slices of whole groups, at least one group per wave, at
// most 3 row blocks per work-group (registers); same cost form as plan_xk with the weights at a quarter of the bytes.
static PlanXK plan_xk_q4(int NRB, int NG, int NXP, int n_cu, size_t pt_floats_per_slice, size_t pt_floats) {
  PlanXK best; best.S = 0; best.groups = 0; best.nrmax = 0; best.cost = -1;
  for (int S = 1; S <= 16; ++S) {
    const int groups = std::min(NRB, n_cu / S);
    if (groups < 1 || NG / S < 8) break;
    const int nrm = (NRB + groups - 1) / groups, kt = 8 * ((NG + S - 1) / S);
    if (nrm > 3 || (size_t)S * pt_floats_per_slice > pt_floats) continue;
    const long cost = (long)nrm * kt / 4 + (long)NXP * kt * 4 / 5 + 2L * S * nrm * 4;
    if (best.cost < 0 || cost < best.cost) { best.S = S; best.groups = groups; best.nrmax = nrm; best.cost = cost; }
  }
  return best;
}

// Runs one fused GEMM: g carries the epilogue description; the matrix, the input and the work split are filled here.
static int gemm2(eagle_ctx* c, const PackedW& w, const bf16_t* XF, Gemm2& g, int* groups_out, int experts = 1) {
  Plan2 p = plan2(w.NRB, w.KS, c->NXP, c->NWP, c->n_cu, w.q4);
  const int R = (w.NRB + p.groups - 1) / p.groups;
  if ((R + p.lanes - 1) / p.lanes > p.RW) return fail(EAGLE_EINVAL, "internal: %d row blocks per wave exceed the kernel's %d", (R + p.lanes - 1) / p.lanes, p.RW);
  if ((size_t)p.S * w.Npad * 32 > c->pt2_floats) return fail(EAGLE_EINVAL, "internal: fast-path partial buffer too small");
  if (p.groups > 1024 || p.lds > 144 * 1024 || p.lanes * p.kparts != 8) return fail(EAGLE_EINVAL, "internal: bad work split");
  g.W = w.w; g.wps = w.plane_stride; g.NRB = w.NRB; g.KS = w.KS; g.Npad = w.Npad; g.N = w.N;
  g.XF = XF; g.S = p.S; g.groups = p.groups; g.lanes = p.lanes; g.kparts = p.kparts;
  g.PT = c->PT2; g.counters = c->cnt_gemm;
  g.trace = (c->gemm_no++ == c->trace_sel && p.groups * p.S <= 1024) ? c->trace : nullptr;
  if (g.ssq_out && p.groups > PLAN_MAX_NORM_GROUPS) return fail(EAGLE_EINVAL, "internal: more than 256 row groups feed a norm");
  if (groups_out) *groups_out = p.groups;
  const double bytes = w.bytes(c->elt) * experts;
  hipError_t e;
  if (w.q4 && g.epi == EPI_RESID) {
    // the streamed split-K kernel.  d = 4096, 26 rows, us: streamed split-K / split-K in LDS, whose 128 KB slice limit forces 11 slices at
    // K = 11008 / whole-K: O 10.5 / 12.0 / 14.6, down 16.4 / 24.5 / 29.0, FC (4 rows) 12.9 / 17.3 / 18.5; but QKV 20.6 streamed, 18.5 whole-K.
    const PlanXK px = plan_xk_q4(w.NRB, w.NG, c->NXP, c->n_cu, (size_t)w.Npad * 32, c->pt2_floats);
    if (px.S > 0) {
      g.S = px.S; g.groups = px.groups; g.SC = w.sc; g.NG = w.NG; g.q4 = q4_format(c->q4_rot);
      g.trace = nullptr;
      if (groups_out) *groups_out = px.groups;
      if (g.ssq_out && px.groups > PLAN_MAX_NORM_GROUPS) return fail(EAGLE_EINVAL, "internal: more than 256 row groups feed a norm");
      e = px.nrmax <= 1 ? launch_xk<1, false, true>(c, bytes, g) : px.nrmax == 2 ? launch_xk<2, false, true>(c, bytes, g) : launch_xk<3, false, true>(c, bytes, g);
      if (e != hipSuccess) return fail(EAGLE_EHIP, "4-bit gemm launch failed: %s", hipGetErrorString(e));
      return EAGLE_OK;
    }
  }
  if (w.q4 && g.epi == EPI_LOGITS && plan_is_logits_q4(w.NRB, c->n_cu, p, c->fixed_sums)) {   // the LM head: one round of whole-K work-groups of four row blocks
    constexpr size_t lds = (size_t)LQ4_PARTS * LQ4_BLOCKS * 4096;
    g.SC = w.sc; g.NG = w.NG; g.q4 = q4_format(c->q4_rot);
    g.trace = nullptr;
    const Share sh = share_of(w.NRB, c->n_cu);
    g.groups = c->n_cu; g.share_a = sh.a; g.share_b = sh.b;
    static bool attr_set = false;
    if (!attr_set) {
      HIPCHK(hipFuncSetAttribute((const void*)k2_logits_q4, hipFuncAttributeMaxDynamicSharedMemorySize, lds));
      attr_set = true;
    }
    e = launch_k(c, c->cur_class, bytes, "k2_logits_q4", k2_logits_q4, dim3(c->n_cu), dim3(V2_THREADS), lds, g);
    if (e != hipSuccess) return fail(EAGLE_EHIP, "4-bit gemm launch failed: %s", hipGetErrorString(e));
    return EAGLE_OK;
  }
  if (w.q4 && c->q4_staged && (g.epi == EPI_RESID || (w.NRB + 2) / 3 > c->n_cu)) {   // (or too many row blocks for one round of whole-K work-groups: larger LM heads)
    // 4-bit weights, LM heads that k2_logits_q4 does not take (and narrow matrices the streamed split-K plan cannot take): split-K with the activation
    // slice staged in LDS.  With a quarter of the weight bytes the activation fragments are most of what a CU fetches;
    // staged, a work-group fetches its K slice of them once.  (The wide matrices are faster whole-K, us at d = 4096: QKV 20.2
    // against 27.3, since their epilogues would run on 64 CUs only.)
    g.SC = w.sc; g.NG = w.NG; g.q4 = q4_format(c->q4_rot);
    g.trace = nullptr;
    switch (p.RW) {
      case 1: e = launch_k2<1, 2, 1, 1, true>(c, bytes, g, p.lds); break;
      case 2: e = launch_k2<1, 2, 2, 1, true>(c, bytes, g, p.lds); break;
      default: e = launch_k2<1, 2, 3, 1, true>(c, bytes, g, p.lds); break;
    }
    if (e != hipSuccess) return fail(EAGLE_EHIP, "4-bit gemm launch failed: %s", hipGetErrorString(e));
    return EAGLE_OK;
  }
  if (w.q4) {
    // wide matrices: whole-K work-groups of up to three row blocks, epilogue in place
    const int grid = std::max(c->n_cu, (w.NRB + 2) / 3);
    const int nrmax = (w.NRB + grid - 1) / grid;
    if (g.epi == EPI_RESID && (grid > 256 || nrmax > 2)) return fail(EAGLE_EINVAL, "internal: residual epilogue on a matrix with %d row blocks", w.NRB);
    g.SC = w.sc; g.NG = w.NG; g.q4 = q4_format(c->q4_rot);
    g.trace = nullptr;
    if (groups_out) *groups_out = grid;
    e = nrmax <= 1 ? launch_fk<1, false, 1, 2, false, true>(c, bytes, g, grid) : nrmax == 2 ? launch_fk<2, false, 1, 2, false, true>(c, bytes, g, grid) : launch_fk<3, false, 1, 2, false, true>(c, bytes, g, grid);
    if (e != hipSuccess) return fail(EAGLE_EHIP, "4-bit gemm launch failed: %s", hipGetErrorString(e));
    return EAGLE_OK;
  }
  // wide matrices of the bf16 configuration: whole-K work-groups with the epilogue in place (no partials) ...
  const int fk_grid = std::max(c->n_cu, (w.NRB + 3) / 4);
  // (not for the residual epilogue: O and down at d = 8192 have exactly one row block per CU, and a work-group that owns
  // one row block over all of K fetches twice as many activation bytes as weight bytes -- measured there: down 109.7 us
  // whole-K against 85.8 us split-K, O 37.5 against 34.8; short K is another matter, see `small`)
  const bool fullk = !c->f32 && w.NRB >= c->n_cu && g.epi != EPI_RESID;
  // (dense models with a bf16 cache keep their K slices, see fixed_sums)
  const bool small = !c->fixed_sums && plan_is_whole_k(w.NRB, w.KS, c->NWP + c->NXP, c->n_cu);
  // other matrices of the bf16 configuration: split-K, with the activations either staged in LDS (plan2) or streamed
  // (plan_xk), whichever the fetch model prices lower
  PlanXK px; px.S = 0;
  if (!fullk && !c->f32) px = xk_plan(c, w);
  if (experts > 1 && (small || !(g.epi == EPI_RESID ? px.S > 0 : fullk && g.epi == EPI_SWIGLU))) return fail(EAGLE_EINVAL, "internal: this plan takes one expert a launch");
  if (experts > 1) g.trace = nullptr;
  if (small) {
    if (groups_out) *groups_out = w.NRB;
    g.trace = nullptr;
    e = c->f32 ? launch_fk<1, false, 3, 3>(c, bytes, g, w.NRB) : launch_fk<1>(c, bytes, g, w.NRB);
  } else if (px.S > 0) {
    g.S = px.S; g.groups = px.groups;
    if (groups_out) *groups_out = px.groups;
    g.trace = (g.trace && px.groups * px.S <= 1024) ? g.trace : nullptr;
    if ((size_t)experts * px.S * w.Npad * 32 > c->pt2_all) return fail(EAGLE_EINVAL, "internal: fast-path partial buffer too small");
    if (experts > 1) e = px.nrmax <= 2 ? launch_xk<2, true>(c, bytes, g, experts) : px.nrmax == 3 ? launch_xk<3, true>(c, bytes, g, experts) : launch_xk<4, true>(c, bytes, g, experts);
    else e = px.nrmax <= 2 ? launch_xk<2>(c, bytes, g) : px.nrmax == 3 ? launch_xk<3>(c, bytes, g) : launch_xk<4>(c, bytes, g);
  } else if (fullk) {
    const int grid = fk_grid;
    if (groups_out) *groups_out = grid;
    const int nrmax = (w.NRB + grid - 1) / grid;
    g.trace = (g.trace && grid <= 1024) ? g.trace : nullptr;
    // QKV: split by half row blocks where that lowers the largest share (3 halves instead of 2 blocks at d = 4096);
    // a run of u halves touches at most u/2 + 1 blocks
    const int umax = (2 * w.NRB + grid - 1) / grid;
    const bool half = g.epi == EPI_QKV && umax < 2 * nrmax && umax / 2 + 1 <= 2;
    if (half) e = launch_fk<2, true>(c, bytes, g, grid);
    else if (experts > 1) e = nrmax <= 2 ? launch_fk<2, false, 1, 2, true>(c, bytes, g, grid, experts) : nrmax == 3 ? launch_fk<3, false, 1, 2, true>(c, bytes, g, grid, experts) : launch_fk<4, false, 1, 2, true>(c, bytes, g, grid, experts);
    else e = nrmax <= 2 ? launch_fk<2>(c, bytes, g, grid) : nrmax == 3 ? launch_fk<3>(c, bytes, g, grid) : launch_fk<4>(c, bytes, g, grid);
  } else if (c->f32) {
    switch (p.RW) {
      case 1: e = launch_k2<3, 3, 1, 4>(c, bytes, g, p.lds); break;
      case 2: e = launch_k2<3, 3, 2, 2>(c, bytes, g, p.lds); break;
      default: e = launch_k2<3, 3, 3, 2>(c, bytes, g, p.lds); break;
    }
  } else {
    switch (p.RW) {
      case 1: e = launch_k2<1, 2, 1, 16>(c, bytes, g, p.lds); break;
      case 2: e = launch_k2<1, 2, 2, 8>(c, bytes, g, p.lds); break;
      default: e = launch_k2<1, 2, 3, 5>(c, bytes, g, p.lds); break;
    }
  }
  if (e != hipSuccess) return fail(EAGLE_EHIP, "fused gemm launch failed: %s", hipGetErrorString(e));
  return EAGLE_OK;
}

static Gemm2 gemm2_base(eagle_ctx* c, int M) {
  Gemm2 g;
  memset(&g, 0, sizeof(g));
  g.M = M; g.facts = c->facts; g.d = c->cfg.d_model; g.in_scale.ssq = c->ssq1;   // (no row scale: groups stays 0)
  g.rope_cos = c->rope_cos; g.rope_sin = c->rope_sin; g.H = c->cfg.n_heads; g.kv_f32 = c->kv_f32; g.Q = c->Q;
  return g;
}
static RowScale scale_of(eagle_ctx* c, const float* ssq, int groups) {
  RowScale rs; rs.ssq = ssq; rs.groups = groups; rs.inv_d = 1.0f / (float)c->cfg.d_model; rs.eps = c->cfg.rms_eps;
  return rs;
}

// One decoder layer on <= 32 rows.  In: h2 (residual), xf2_d = h2 * (this layer's attn gain), ssq2 (row sums of squares).
// Out: the same three for the consumer named by next_gain (nullptr: xf2_d = h2 itself).
static int layer2(eagle_ctx* c, const Pass& pass, int M, int li, int ctx_max, int n_new, const float* next_gain) {
  const eagle_config& cf = c->cfg;
  LayerW& w = c->layers[li];
  const int H = cf.n_heads, dh = cf.head_dim, d = cf.d_model, F = cf.d_ffn;
  int rc;
  Gemm2 g = gemm2_base(c, M);
  g.epi = EPI_QKV; g.in_scale = scale_of(c, c->ssq2, c->ssq2_groups); g.kv = kv_for(c, li);
  if ((rc = (c->cur_class = KC_QKV, gemm2(c, w.qkv, c->xf2_d, g, nullptr)))) return rc;
  if (c->attn_ruled) { if ((rc = ruled_attention(c, pass, M, 1, kv_for(c, li), ctx_max + n_new, c->xf2_att))) return rc; }
  else {
    int n_splits = attn_splits(c, ctx_max + 64, H * pass.n_seq);
    unsigned long long* atrace = (c->attn_no++ == c->attn_trace_sel && n_splits * H <= 1024) ? c->trace : nullptr;
    dim3 grid(n_splits, H, pass.n_seq);
    KVCache kv = kv_for(c, li);
#define ATTN2(CT, DH)                                                                                                   \
  do {                                                                                                                  \
    static bool attr_done = false;                                                                                      \
    if (!attr_done) {                                                                                                   \
      HIPCHK(hipFuncSetAttribute((const void*)k2_attn<CT, DH>, hipFuncAttributeMaxDynamicSharedMemorySize, 80 * 1024)); \
      attr_done = true;                                                                                                 \
    }                                                                                                                   \
    hipError_t e_ = launch_k(c, KC_ATTN, attn_bytes(c, pass, n_new), "k2_attn", k2_attn<CT, DH>, grid, dim3(256), (size_t)(4 * 32 * (DH + 4) + 4 * 2 * 32) * 4, \
        attn_args(c, pass, kv, n_splits, n_new, c->xf2_att, 1, 1, atrace)); \
    if (e_ != hipSuccess) return fail(EAGLE_EHIP, "attention launch failed: %s", hipGetErrorString(e_));                \
  } while (0)
    if (c->kv_f32) { if (dh == 128) ATTN2(float, 128); else if (dh == 64) ATTN2(float, 64); else ATTN2(float, 32); }
    else { if (dh == 128) ATTN2(bf16_t, 128); else if (dh == 64) ATTN2(bf16_t, 64); else ATTN2(bf16_t, 32); }
#undef ATTN2
    LAUNCH_CHECK();
  }
  g = gemm2_base(c, M);
  g.epi = EPI_RESID; g.h_in = c->h2; g.h_out = c->h2; g.gain_next = w.mlp_norm; g.xf_out = c->xf2_d; g.xf_KS = d / 16; g.ssq_out = c->ssq1;
  if ((rc = (c->cur_class = KC_O, gemm2(c, w.o, c->xf2_att, g, &c->ssq1_groups)))) return rc;
  if (w.moe) {
    // routed experts (see the general path): experts no row selected are skipped on the device (skip_flag)
    const int E = cf.n_experts;
    k_fill_u32<<<1, 64, 0, c->stream>>>((uint32_t*)c->expert_used, 0u, (size_t)E);
    LAUNCH_CHECK();
    k_router<<<M, 256, 0, c->stream>>>(nullptr, c->h2, c->ssq1, c->ssq1_groups, 1.0f / (float)d, cf.rms_eps, w.mlp_norm, w.router, E,
                                       cf.experts_per_tok, d, M, c->moe_w, c->Mmax, c->expert_used);
    LAUNCH_CHECK();
    if (c->prof_mode) { k_count_used<<<1, 64, 0, c->stream>>>(c->expert_used, E, c->experts_touched); LAUNCH_CHECK(); }
    // All experts in two launches where both matrices are large (moe_in_two); else two launches an expert.
    const bool two = moe_in_two(c, w.e_gu[0], w.e_dn[0]);
    const size_t act = (size_t)c->NXP * 32 * F;
    for (int e = 0; e < (two ? 1 : E); ++e) {
      g = gemm2_base(c, M);
      g.epi = EPI_SWIGLU; g.in_scale = scale_of(c, c->ssq1, c->ssq1_groups); g.xf_out = c->xf2_ffn; g.xf_KS = F / 16;
      g.skip_flag = c->expert_used + e;
      if (two) { g.w_stride = (size_t)(w.e_gu[1].w - w.e_gu[0].w); g.out_stride = act; g.row_w = c->moe_w; g.row_w_stride = c->Mmax; }
      if ((rc = (c->cur_class = KC_GATEUP, gemm2(c, w.e_gu[e], c->xf2_d, g, nullptr, two ? E : 1)))) return rc;
      g = gemm2_base(c, M);
      g.epi = EPI_RESID; g.h_in = c->h2; g.h_out = c->h2; g.gain_next = next_gain; g.xf_out = c->xf2_dB; g.xf_KS = d / 16; g.ssq_out = c->ssq2;
      g.row_w = c->moe_w + (size_t)e * c->Mmax; g.skip_flag = c->expert_used + e;
      if (two) { g.w_stride = (size_t)(w.e_dn[1].w - w.e_dn[0].w); g.x_stride = act; g.row_w_stride = c->Mmax; }
      if ((rc = (c->cur_class = KC_DOWN, gemm2(c, w.e_dn[e], c->xf2_ffn, g, &c->ssq2_groups, two ? E : 1)))) return rc;
    }
    std::swap(c->xf2_d, c->xf2_dB);     // the experts all read the old xf2_d; the new one was built beside it
    return EAGLE_OK;
  }
  g = gemm2_base(c, M);
  g.epi = EPI_SWIGLU; g.in_scale = scale_of(c, c->ssq1, c->ssq1_groups); g.xf_out = c->xf2_ffn; g.xf_KS = F / 16;
  if ((rc = (c->cur_class = KC_GATEUP, gemm2(c, w.gu, c->xf2_d, g, nullptr)))) return rc;
  g = gemm2_base(c, M);
  g.epi = EPI_RESID; g.h_in = c->h2; g.h_out = c->h2; g.gain_next = next_gain; g.xf_out = c->xf2_d; g.xf_KS = d / 16; g.ssq_out = c->ssq2;
  return (c->cur_class = KC_DOWN, gemm2(c, w.dn, c->xf2_ffn, g, &c->ssq2_groups));
}

static int lm_head2(eagle_ctx* c, int M, bool scaled, float* out, const bf16_t* XF) {
  Gemm2 g = gemm2_base(c, M);
  g.epi = EPI_LOGITS; g.logits = out; g.V = c->cfg.vocab;
  if (scaled) g.in_scale = scale_of(c, c->ssq2, c->ssq2_groups);
  return (c->cur_class = KC_LMHEAD, gemm2(c, c->lm_head, XF ? XF : c->xf2_d, g, nullptr));
}

static int target_forward2(eagle_ctx* c, const Pass& pass, int ctx_max, int n_new, float* logits_out, bool want_logits = true) {
  const eagle_config& cf = c->cfg;
  const int M = pass.rows_per_seq * pass.n_seq, d = cf.d_model;
  int rc;
  const int eg = std::max(1, std::min(64, d / 64));
  if (c->f32) k2_embed<float, 3><<<eg, 256, 0, c->stream>>>(pass, c->tree_d, c->st, c->tree_tok, (const float*)c->embed, cf.vocab, M, c->M, d, c->h2, c->layers[0].attn_norm, c->xf2_d, c->ssq2, kv_for(c, 0), c->facts);
  else k2_embed<bf16_t, 2><<<eg, 256, 0, c->stream>>>(pass, c->tree_d, c->st, c->tree_tok, (const bf16_t*)c->embed, cf.vocab, M, c->M, d, c->h2, c->layers[0].attn_norm, c->xf2_d, c->ssq2, kv_for(c, 0), c->facts);
  LAUNCH_CHECK();
  c->ssq2_groups = eg;
  if ((rc = pass_chunk(c, pass, n_new))) return rc;
  for (int l = 0; l < cf.n_layers; ++l)
    if ((rc = layer2(c, pass, M, l, ctx_max, n_new, l + 1 < cf.n_layers ? c->layers[l + 1].attn_norm : c->final_norm))) return rc;
  k2_features<<<M, 256, 0, c->stream>>>(pass, c->tree_d, c->st, c->h2, scale_of(c, c->ssq2, c->ssq2_groups), c->final_norm, d, c->F, c->pend_f, c->chunk_f);
  LAUNCH_CHECK();
  if (!want_logits) return EAGLE_OK;
  return lm_head2(c, M, true, logits_out);
}

static int head_forward2(eagle_ctx* c, const Pass& pass, int ctx_max, int n_new, bool store_rows = true, bool want_logits = true) {
  const eagle_config& cf = c->cfg;
  const int M = pass.rows_per_seq * pass.n_seq, d = cf.d_model;
  int rc;
  if (c->f32) k_fc_input<float><<<dim3(M, 4), 256, 0, c->stream>>>(pass, c->tree_d, c->st, c->tree_tok, c->pend_f, c->node_f, c->chunk_f, (const float*)c->embed, c->xf2_2d, d, cf.vocab, 1, c->NXP, kv_for(c, cf.n_layers), c->facts, level_parents(c, pass));
  else k_fc_input<bf16_t><<<dim3(M, 4), 256, 0, c->stream>>>(pass, c->tree_d, c->st, c->tree_tok, c->pend_f, c->node_f, c->chunk_f, (const bf16_t*)c->embed, c->xf2_2d, d, cf.vocab, 1, c->NXP, kv_for(c, cf.n_layers), c->facts, level_parents(c, pass));
  LAUNCH_CHECK();
  if ((rc = pass_chunk(c, pass, n_new))) return rc;
  Gemm2 g = gemm2_base(c, M);
  g.epi = EPI_RESID; g.h_in = nullptr; g.h_out = c->h2; g.bias = c->loaded_layer[EAGLE_W_FC_BIAS][0] ? c->fc_bias : nullptr;
  g.gain_next = c->layers[cf.n_layers].attn_norm; g.xf_out = c->xf2_d; g.xf_KS = d / 16; g.ssq_out = c->ssq2;
  if ((rc = (c->cur_class = KC_FC, gemm2(c, c->fc, c->xf2_2d, g, &c->ssq2_groups)))) return rc;
  if ((rc = layer2(c, pass, M, cf.n_layers, ctx_max, n_new, nullptr))) return rc;
  if (!want_logits) return EAGLE_OK;         // prompt rows of the head: only their cache entries are wanted
  if (store_rows) {                          // (the draft passes leave this copy to k_expand)
    k_store_rows<<<M, 256, 0, c->stream>>>(pass, c->tree_d, c->st, c->h2, c->node_f, c->pend_f, c->chunk_f, d);
    LAUNCH_CHECK();
  }
  return lm_head2(c, M, false, c->draft_logits);
}

// The rules of eagle_set_logit_rules on the logits of slots seq0 .. seq0 + n - 1: a row a slot (vanilla_logits), or a row a tree node (L).
static int rule_logits(eagle_ctx* c, int seq0, int n, bool nodes, const int* n_tokens) {
  if (!c->logits_ruled) return EAGLE_OK;
  const eagle_config& g = c->cfg;
  const eagle_context_rules& r = c->logit_rules;
  const int M = c->M;
  eagle_logits l{};
  l.n_rows = nodes ? n * M : n; l.vocab = g.vocab; l.dtype = EAGLE_F32; l.in_stride = l.out_stride = g.vocab;
  l.out = nodes ? c->L : c->vanilla_logits + (size_t)seq0 * g.vocab;
  l.in = l.out;
  if (nodes) { l.row_start = c->op_verify_start; l.path_token = c->tree_tok; l.path_mask = (const uint64_t*)c->op_path; }
  if (r.allowed) {
    l.allowed = r.allowed; l.n_masks = r.n_masks; l.mask_stride = r.mask_stride;
    l.allowed_row = r.allowed_row + (size_t)seq0 * M;
    if (!nodes && n > 1) {                                        // node 0's of every slot, side by side
      k_node0_rows<<<1, 64, 0, c->stream>>>(l.allowed_row, M, n, c->op_mask_row);
      LAUNCH_CHECK();
      l.allowed_row = c->op_mask_row;
    }
  }
  eagle_logit_rules lr{};
  lr.n_seqs = n; lr.tokens = c->st.tokens + (size_t)seq0 * c->st.tok_stride; lr.token_stride = c->st.tok_stride; lr.max_tokens = (int32_t)c->st.tok_stride; lr.n_tokens = n_tokens + seq0; lr.n_prompt = c->op_prompt + seq0;
  lr.repetition = r.repetition ? r.repetition + seq0 : nullptr; lr.presence = r.presence ? r.presence + seq0 : nullptr; lr.frequency = r.frequency ? r.frequency + seq0 : nullptr;
  if (r.bias_token) { lr.bias_start = r.bias_start + seq0; lr.bias_token = r.bias_token; lr.bias_value = r.bias_value; lr.n_bias = r.n_bias; }
  return eagle_apply_logit_rules(&l, &lr, c->stream);
}

// The next token of n sequences from seq0 on, from their rows of vanilla_logits.
static int choose(eagle_ctx* c, int n, int seq0, int is_prefill, int prefill_n) {
  const eagle_config& g = c->cfg;
  if (g.vocab > 32768) k_choose<true><<<n, 1024, 0, c->stream>>>(c->st, seq0, c->vanilla_logits, g.vocab, g.temperature, g.seed, c->pbuf, is_prefill, prefill_n, c->D);
  else k_choose<false><<<n, 1024, g.temperature > 0.f ? CDF_LDS : 0, c->stream>>>(c->st, seq0, c->vanilla_logits, g.vocab, g.temperature, g.seed, c->pbuf, is_prefill, prefill_n, c->D);
  LAUNCH_CHECK();
  return EAGLE_OK;
}

// ---------------------------------------------------------------------------- sequence life cycle
extern "C" int eagle_reset(eagle_ctx* c) {
  if (!c) return fail(EAGLE_EINVAL, "null context");
  const int B = c->cfg.max_batch;
  HIPCHK(hipMemsetAsync(c->st.ctx_len, 0, (size_t)B * 4, c->stream));
  HIPCHK(hipMemsetAsync(c->st.n_pend, 0, (size_t)B * 4, c->stream));
  HIPCHK(hipMemsetAsync(c->st.n_tok, 0, (size_t)B * 4, c->stream));
  HIPCHK(hipMemsetAsync(c->st.step_no, 0, (size_t)B * 4, c->stream));
  HIPCHK(hipMemsetAsync(c->hint_n, 0, (size_t)B * 4, c->stream));
  std::fill(c->h_ctx.begin(), c->h_ctx.end(), 0); std::fill(c->h_ntok.begin(), c->h_ntok.end(), 0);
  std::fill(c->active.begin(), c->active.end(), 0); std::fill(c->head_stale.begin(), c->head_stale.end(), 0);
  c->n_active = 0; c->phase = 0;
  return EAGLE_OK;
}

extern "C" int eagle_prefill(eagle_ctx* c, int32_t seq, const int32_t* prompt, int32_t n, int32_t* first_token) {
  if (!c || !prompt) return fail(EAGLE_EINVAL, "null argument");
  const eagle_config& g = c->cfg;
  int rc = all_loaded(c);
  if (rc) return rc;
  if (seq < 0 || seq >= g.max_batch) return fail(EAGLE_EINVAL, "slot %d out of range", seq);
  if (seq != c->n_active) return fail(EAGLE_ESTATE, "slots must be prefilled in order: next is %d", c->n_active);
  if (n < 1) return fail(EAGLE_EINVAL, "empty prompt");
  if (n + 1 + c->M > g.max_seq) return fail(EAGLE_ESEQ_FULL, "prompt of %d tokens leaves no room for a step (max_seq %d)", n, g.max_seq);
  for (int i = 0; i < n; ++i)
    if (prompt[i] < 0 || prompt[i] >= g.vocab) return fail(EAGLE_EINVAL, "prompt token %d at %d outside the vocabulary", prompt[i], i);
  HIPCHK(hipMemcpyAsync(c->st.tokens + (size_t)seq * c->st.tok_stride, prompt, (size_t)n * 4, hipMemcpyHostToDevice, c->stream));
  int zero = 0;
  HIPCHK(hipMemcpyAsync(c->st.ctx_len + seq, &zero, 4, hipMemcpyHostToDevice, c->stream));
  HIPCHK(hipStreamSynchronize(c->stream));   // `zero` and `prompt` are host memory of the caller
  // passes of about equal length, whole windows each (so the last window lies in the last pass)
  const int n_pass = (n + c->pf_chunk - 1) / c->pf_chunk;
  const int pass_rows = ((n + n_pass - 1) / n_pass + c->pf_window - 1) / c->pf_window * c->pf_window;
  for (int start = 0; start < n; start += pass_rows) {
    const int cn = std::min(pass_rows, n - start);
    const bool last = start + cn == n;
    c->last_off = (cn - 1) / c->pf_window * c->pf_window; c->last_rows = cn - c->last_off;
    Pass pt{PASS_PREFILL_T, cn, 1, seq, 0, start, cn};
    const bool fast = plan_is_short_prompt(cn, g.d_model, c->NWP + c->NXP, c->f32, c->q4, c->fixed_sums, g.n_experts);
    if ((rc = fast ? target_forward2(c, pt, start + cn, cn, c->vanilla_logits, last)
                   : target_forward(c, pt, start + cn, cn, last, c->vanilla_logits, 1, 1))) return rc;
    if (last) {
      if (c->logits_ruled) {
        k_fill_u32<<<1, 64, 0, c->stream>>>((uint32_t*)c->op_prompt + seq, (uint32_t)n, 1);
        k_fill_u32<<<1, 64, 0, c->stream>>>((uint32_t*)c->op_tokens + seq, (uint32_t)n, 1);
        LAUNCH_CHECK();
        if ((rc = rule_logits(c, seq, 1, false, c->op_tokens))) return rc;
      }
      if ((rc = choose(c, 1, seq, 1, n))) return rc;
      HIPCHK(hipMemcpyAsync(c->pend_f + (size_t)seq * (c->D + 1) * g.d_model, c->chunk_f + (size_t)(cn - 1) * g.d_model,
                            (size_t)g.d_model * 4, hipMemcpyDeviceToDevice, c->stream));
    }
    // the head's rows for this chunk: pairs (f_i, x_{i+1}); the prompt's last position stays pending
    const int dn = last ? cn - 1 : cn;
    if (dn > 0) {
      Pass pd{PASS_PREFILL_D, dn, 1, seq, 0, start, dn};
      if ((rc = fast ? head_forward2(c, pd, start + dn, dn, false, false) : head_forward(c, pd, start + dn, dn, false))) return rc;
    }
  }
  int tok = 0;
  HIPCHK(hipMemcpyAsync(&tok, c->st.tokens + (size_t)seq * c->st.tok_stride + n, 4, hipMemcpyDeviceToHost, c->stream));
  HIPCHK(hipStreamSynchronize(c->stream));
  if (first_token) *first_token = tok;
  c->h_prompt[seq] = n;
  c->h_ctx[seq] = n; c->h_ntok[seq] = n + 1; c->active[seq] = 1; c->head_stale[seq] = 0;
  c->n_active = seq + 1; c->phase = 0;
  return EAGLE_OK;
}

// ---------------------------------------------------------------------------- training loss of the head (Sec. 3.2)
extern "C" int eagle_head_loss(eagle_ctx* c, const float* f, const float* fhat, int32_t rows, float w_cls, float* grad, float* loss_out) {
  if (!c || !f || !fhat || !loss_out) return fail(EAGLE_EINVAL, "null argument");
  const eagle_config& g = c->cfg;
  if (g.head_loss_rows <= 0) return fail(EAGLE_ESTATE, "the context was created without head_loss_rows");
  if (!c->loaded_layer[EAGLE_W_LM_HEAD][0]) return fail(EAGLE_ESTATE, "the LM head was never loaded");
  if (rows < 1) return fail(EAGLE_EINVAL, "rows must be >= 1");
  if (!(w_cls >= 0.f)) return fail(EAGLE_EINVAL, "w_cls must be >= 0");
  const int d = g.d_model, V = g.vocab;
  k_fill_u32<<<1, 64, 0, c->stream>>>((uint32_t*)c->hl_acc, 0u, (size_t)4);
  LAUNCH_CHECK();
  const float cls_scale = w_cls / (float)rows, reg_scale = 1.0f / ((float)rows * (float)d);
  for (int r0 = 0; r0 < rows; r0 += c->hl_chunk) {
    const int rc_ = std::min(c->hl_chunk, rows - r0), rpad = (rc_ + 31) / 32 * 32;
    const int MTf = 2 * rpad / 32, MTb = rpad / 32;
    if (MTf * 32 > 2 * c->hl_chunk) return fail(EAGLE_EINVAL, "internal: loss pass of %d rows exceeds the pass limit", MTf * 32);
    // labels in rows [0, rc_), predictions in rows [rpad, rpad + rc_) of one LM-head pass
    k_rows_to_xf<<<dim3(rc_, 2), 256, 0, c->stream>>>(f + (size_t)r0 * d, 0, c->xf_d, MTf, c->NXP, d);
    LAUNCH_CHECK();
    k_rows_to_xf<<<dim3(rc_, 2), 256, 0, c->stream>>>(fhat + (size_t)r0 * d, rpad, c->xf_d, MTf, c->NXP, d);
    LAUNCH_CHECK();
    int S, rc;
    if ((rc = (c->cur_class = KC_LMHEAD, gemm(c, c->lm_head, c->xf_d, MTf, MTf * 32, &S)))) return rc;
    auto loss_row = V <= 4 * 8192 ? k_head_loss_row<4> : k_head_loss_row<0>;   // larger vocabularies would spill: they stream
    loss_row<<<rc_, 1024, 0, c->stream>>>(c->PT, S, MTf * 32, c->lm_head.Npad, rpad, V, f + (size_t)r0 * d, fhat + (size_t)r0 * d, d,
                                          cls_scale, reg_scale, c->hl_dz, MTb, c->NXP, grad ? grad + (size_t)r0 * d : nullptr, c->hl_row_loss);
    LAUNCH_CHECK();
    k_head_loss_accumulate<<<1, 64, 0, c->stream>>>(c->hl_row_loss, rc_, c->hl_acc);
    LAUNCH_CHECK();
    if (grad) {
      if ((rc = (c->cur_class = KC_LMHEAD, gemm(c, c->lm_head_T, c->hl_dz, MTb, rc_, &S)))) return rc;
      k_head_loss_grad_finish<<<dim3((d + 255) / 256, rc_), 256, 0, c->stream>>>(c->PT, S, MTb * 32, c->lm_head_T.Npad, grad + (size_t)r0 * d, d);
      LAUNCH_CHECK();
    }
  }
  double acc[2] = {0.0, 0.0};
  HIPCHK(hipMemcpyAsync(acc, c->hl_acc, sizeof(acc), hipMemcpyDeviceToHost, c->stream));
  HIPCHK(hipStreamSynchronize(c->stream));
  const double L_reg = acc[0] / ((double)rows * (double)d), L_cls = acc[1] / (double)rows;
  loss_out[0] = (float)(L_reg + (double)w_cls * L_cls); loss_out[1] = (float)L_reg; loss_out[2] = (float)L_cls;
  return EAGLE_OK;
}

extern "C" int eagle_feature_noise(eagle_ctx* c, const float* in, float* out, int32_t rows, float amplitude, uint64_t seed, uint64_t step) {
  if (!c || !in || !out) return fail(EAGLE_EINVAL, "null argument");
  if (rows < 1) return fail(EAGLE_EINVAL, "rows must be >= 1");
  if (!(amplitude >= 0.f)) return fail(EAGLE_EINVAL, "amplitude must be >= 0");
  const size_t n = (size_t)rows * c->cfg.d_model;
  const unsigned blocks = (unsigned)std::min<size_t>((n + 255) / 256, 4096);
  k_feature_noise<<<blocks, 256, 0, c->stream>>>(in, out, rows, c->cfg.d_model, amplitude, rng_prefix(seed, PURPOSE_NOISE, step));
  LAUNCH_CHECK();
  return EAGLE_OK;
}

extern "C" int eagle_set_hint(eagle_ctx* c, int32_t seq, const int32_t* future, int32_t n, float alpha, float bias, uint64_t seed) {
  if (!c) return fail(EAGLE_EINVAL, "null context");
  if (seq < 0 || seq >= c->cfg.max_batch) return fail(EAGLE_EINVAL, "slot %d out of range", seq);
  if (n < 0 || n > c->st.tok_stride) return fail(EAGLE_EINVAL, "hint length %d out of range", n);
  if (n > 0 && !future) return fail(EAGLE_EINVAL, "future is null");
  for (int i = 0; i < n; ++i)
    if (future[i] < 0 || future[i] >= c->cfg.vocab) return fail(EAGLE_EINVAL, "hint token outside the vocabulary");
  unsigned long long s64 = seed;
  if (n > 0) HIPCHK(hipMemcpyAsync(c->hint_future + (size_t)seq * c->st.tok_stride, future, (size_t)n * 4, hipMemcpyHostToDevice, c->stream));
  HIPCHK(hipMemcpyAsync(c->hint_n + seq, &n, 4, hipMemcpyHostToDevice, c->stream));
  HIPCHK(hipMemcpyAsync(c->hint_alpha + seq, &alpha, 4, hipMemcpyHostToDevice, c->stream));
  HIPCHK(hipMemcpyAsync(c->hint_bias + seq, &bias, 4, hipMemcpyHostToDevice, c->stream));
  HIPCHK(hipMemcpyAsync(c->hint_seed + seq, &s64, 8, hipMemcpyHostToDevice, c->stream));
  HIPCHK(hipStreamSynchronize(c->stream));
  return EAGLE_OK;
}

extern "C" int eagle_set_rope(eagle_ctx* c, const eagle_rope_config* rope) try {
  if (!c) return fail(EAGLE_EINVAL, "null context");
  for (int w : {(int)EAGLE_W_Q, (int)EAGLE_W_K})
    for (char loaded : c->loaded_layer[w])
      if (loaded) return fail(EAGLE_ESTATE, "eagle_set_rope must come before the query and key matrices are loaded (they are laid out by pairs)");
  if (!rope) {
    const int rc = upload_rope(c, nullptr);
    if (!rc) c->rope_mode = PACK_ROPE;
    return rc;
  }
  if (rope->head_dim != c->cfg.head_dim) return fail(EAGLE_EINVAL, "head_dim %d of the positions is not the model's %d", rope->head_dim, c->cfg.head_dim);
  eagle_rope_plan plan;
  int rc = eagle_rope_plan_init(rope, &plan);
  if (rc || (rc = upload_rope(c, &plan))) return rc;
  c->rope_mode = rope_pack(plan.rot_dim, plan.interleaved);
  return EAGLE_OK;
} catch (const std::exception&) {
  return fail(EAGLE_ENOMEM, "out of host memory");
}

extern "C" int eagle_set_attention(eagle_ctx* c, const eagle_attention_rules* r) {
  if (!c) return fail(EAGLE_EINVAL, "null context");
  if (c->n_active != 0) return fail(EAGLE_ESTATE, "the attention rules can only change while no sequence is active (after eagle_init / eagle_reset)");
  if (r && (!(r->softcap >= 0.f) || !std::isfinite(r->softcap) || (r->softcap > 0.f && r->softcap < 1e-30f) || r->window < 0)) return fail(EAGLE_EINVAL, "softcap must be 0 or 10^-30 and more and finite, window >= 0");
  c->attn_rules = r ? *r : eagle_attention_rules{};
  c->attn_ruled = r && (r->softcap > 0.f || r->window > 0 || r->slopes_dev);
  return EAGLE_OK;
}

extern "C" int eagle_set_logit_rules(eagle_ctx* c, const eagle_context_rules* r) try {
  if (!c) return fail(EAGLE_EINVAL, "null context");
  if (r) {
    if (r->bias_token && (!r->bias_start || !r->bias_value || r->n_bias < 0)) return fail(EAGLE_EINVAL, "biases need bias_start, bias_value and n_bias >= 0");
    if (r->allowed && (!r->allowed_row || r->n_masks < 1 || r->mask_stride < (c->cfg.vocab + 31) / 32)) return fail(EAGLE_EINVAL, "masks need allowed_row, n_masks >= 1 and %d words a row", (c->cfg.vocab + 31) / 32);
    const int B = c->cfg.max_batch;
    std::vector<int> start(B + 1);
    std::vector<unsigned long long> path((size_t)B * c->M);
    for (int s = 0; s <= B; ++s) start[s] = s * c->M;
    for (size_t i = 0; i < path.size(); ++i) path[i] = c->tree_h.anc[i % c->M] & ~1ull;   // (the root is the last committed token)
    HIPCHK(hipMemcpyAsync(c->op_verify_start, start.data(), start.size() * 4, hipMemcpyHostToDevice, c->stream));
    HIPCHK(hipMemcpyAsync(c->op_path, path.data(), path.size() * 8, hipMemcpyHostToDevice, c->stream));
    HIPCHK(hipMemcpyAsync(c->op_prompt, c->h_prompt.data(), (size_t)B * 4, hipMemcpyHostToDevice, c->stream));
    HIPCHK(hipStreamSynchronize(c->stream));
  }
  c->logit_rules = r ? *r : eagle_context_rules{};
  c->logits_ruled = r != nullptr;
  return EAGLE_OK;
} catch (const std::exception&) {
  return fail(EAGLE_ENOMEM, "out of host memory");
}

static int step_ready(eagle_ctx* c) {
  if (c->n_active < 1) return fail(EAGLE_ESTATE, "no active sequence: call eagle_prefill first");
  for (int s = 0; s < c->n_active; ++s) {
    if (c->h_ctx[s] + c->M + 1 > c->cfg.max_seq) return fail(EAGLE_ESEQ_FULL, "slot %d: %d cached positions + %d tree nodes exceed max_seq %d", s, c->h_ctx[s], c->M, c->cfg.max_seq);
  }
  return EAGLE_OK;
}
// Gives a decode-time pass the cached lengths the host mirrors (at most 4 sequences).
static void pass_ctx(eagle_ctx* c, Pass& p) {
  p.ctx_known = 0;
  if (p.n_seq > 4) return;
  int v[4] = {0, 0, 0, 0};
  for (int i = 0; i < p.n_seq; ++i) v[i] = c->h_ctx[p.seq0 + i];
  p.ctx_known = 1; p.ctx0 = v[0]; p.ctx1 = v[1]; p.ctx2 = v[2]; p.ctx3 = v[3];
}
static int max_ctx(eagle_ctx* c) {
  int m = 0;
  for (int s = 0; s < c->n_active; ++s) m = std::max(m, c->h_ctx[s]);
  return m;
}

static LevelNodes level_nodes(const eagle_ctx* c, int level) {
  LevelNodes l;
  memset(&l, 0, sizeof(l));                                      // (-1: the root)
  if (level >= 0) for (int i = 0; i < c->tree_h.n_level_rows[level]; ++i) l.node[i] = (uint8_t)c->tree_h.level_rows[level][i];
  return l;
}

// The children of a level's nr parent nodes (level -1: the root) of every sequence, from their rows of draft_logits.
static int expand(eagle_ctx* c, int level, int nr, const float* feat_src, int src_rows) {
  const eagle_config& g = c->cfg;
  const int parts = plan_expand_parts(g.vocab);
  if (nr > std::max(1, c->max_level_rows)) return fail(EAGLE_EINVAL, "internal: %d parent nodes in a level", nr);
  k_expand<<<dim3(parts, nr, c->n_active), EXPAND_THREADS, 0, c->stream>>>(level, level_nodes(c, level), c->tree_d, c->M, c->st, c->draft_logits, c->tree_tok, c->on_path, c->hint,
                                                                          g.vocab, parts, (g.vocab + parts - 1) / parts, nr, g.temperature, g.seed, c->part_keys, c->cnt_expand, feat_src, c->node_f, g.d_model, src_rows);
  LAUNCH_CHECK();
  return EAGLE_OK;
}

static int do_draft(eagle_ctx* c) {
  int rc = step_ready(c);
  if (rc) return rc;
  for (int s = 0; s < c->n_active; ++s)
    if (c->head_stale[s]) return fail(EAGLE_ESTATE, "slot %d was advanced by eagle_vanilla_step; the head's cache is stale (prefill again)", s);
  const int B = c->n_active, D1 = c->D + 1, ctx = max_ctx(c);
  const eagle_config& g = c->cfg;
  Pass p1{PASS_DRAFT_PENDING, D1, B, 0, 0, 0, 0};
  pass_ctx(c, p1);
  const bool fast1 = D1 * B <= 32;
  if ((rc = (fast1 ? head_forward2(c, p1, ctx, D1, false) : head_forward(c, p1, ctx + D1, D1, true)))) return rc;
  if ((rc = expand(c, -1, 1, fast1 ? c->h2 : nullptr, D1))) return rc;   // fast path: k_expand stores the root's head feature itself
  for (int lev = 1; lev < c->D; ++lev) {
    int nr = c->tree_h.n_level_rows[lev];
    if (nr == 0) break;
    Pass pl{PASS_DRAFT_LEVEL, nr, B, 0, lev, 0, 0};
    pass_ctx(c, pl);
    const bool fastl = nr * B <= 32;
    if ((rc = (fastl ? head_forward2(c, pl, ctx, c->M, false) : head_forward(c, pl, ctx + c->M, c->M, true)))) return rc;
    if ((rc = expand(c, lev, nr, fastl ? c->h2 : nullptr, nr))) return rc;
  }
  c->phase = 1;
  return EAGLE_OK;
}

static int do_verify(eagle_ctx* c) {
  if (c->phase != 1) return fail(EAGLE_ESTATE, "eagle_verify needs a drafted tree (call eagle_draft_tree first)");
  c->gemm_no = 0; c->attn_no = 0;
  int rc = EAGLE_OK;
  if (c->prof_mode && c->cfg.n_experts > 0) { k_fill_u32<<<1, 64, 0, c->stream>>>((uint32_t*)c->experts_touched, 0u, 1); LAUNCH_CHECK(); }
  if (c->M * c->n_active <= 32) {
    Pass pv{PASS_VERIFY, c->M, c->n_active, 0, 0, 0, 0};
    pass_ctx(c, pv);
    rc = target_forward2(c, pv, max_ctx(c), c->M, c->L);
  } else {
    Pass pv{PASS_VERIFY, c->M, c->n_active, 0, 0, 0, 0};
    pass_ctx(c, pv);
    rc = target_forward(c, pv, max_ctx(c) + c->M, c->M, true, c->L, 0, 0);
  }
  if (rc) return rc;
  if ((rc = rule_logits(c, 0, c->n_active, true, c->st.n_tok))) return rc;
  c->phase = 2;
  return EAGLE_OK;
}

// Path, tokens and lengths, KV rows, pending features and the sequences' state: from the nodes' outcomes, or (null) along a path that is there.
static int do_commit(eagle_ctx* c, const int2* outcome) {
  const eagle_config& g = c->cfg;
  const dim3 grid(1, g.n_layers + 1, c->n_active);
  const KVCache kv = kv_for(c, 0);
  Pass p{PASS_VERIFY, c->M, c->n_active, 0, 0, 0, 0};
  pass_ctx(c, p);                                              // (the lengths before this step: fetch_results adds to them)
#define COMMIT(CT, WALK) k_commit<CT, WALK><<<grid, 1024, 0, c->stream>>>(c->M, c->D + 1, p, c->st, outcome, c->tree_tok, c->path, c->len_out, c->tok_out, c->kc, c->vc, c->layer_stride, g.n_layers, kv, c->F, c->pend_f, g.d_model)
  if (c->kv_f32) { if (outcome) COMMIT(float, true); else COMMIT(float, false); }
  else { if (outcome) COMMIT(bf16_t, true); else COMMIT(bf16_t, false); }
#undef COMMIT
  LAUNCH_CHECK();
  c->phase = 0;
  return EAGLE_OK;
}

// Acceptance + commit.  pbuf / qbuf (fp32 [n_active][vocab] each, walks over large vocabularies only) and outcome ([n_active][M]) are the
// kernels' scratch: the caller's workspace, or the library's static device array.
static int do_accept(eagle_ctx* c, float* pbuf, float* qbuf, int2* outcome) {
  if (c->phase != 2) return fail(EAGLE_ESTATE, "eagle_accept needs verified logits (call eagle_verify first)");
  const eagle_config& g = c->cfg;
  const int B = c->n_active;
  const dim3 nodes(c->M, B);
  if (g.temperature <= 0.f)
    k_outcome<ACCEPT_GREEDY><<<nodes, 1024, 0, c->stream>>>(c->tree_d, c->M, c->st, c->L, c->draft_logits, c->tree_tok, g.vocab, g.temperature, g.seed, outcome);
  else if (g.vocab <= 32768)
    k_outcome<ACCEPT_SAMPLED><<<nodes, 1024, CDF_LDS, c->stream>>>(c->tree_d, c->M, c->st, c->L, c->draft_logits, c->tree_tok, g.vocab, g.temperature, g.seed, outcome);
  else {
    k_accept<<<B, 1024, 0, c->stream>>>(c->tree_d, c->st, c->L, c->draft_logits, c->tree_tok, g.vocab, g.temperature, g.seed, pbuf, qbuf, c->path, c->tok_out, c->len_out);
    outcome = nullptr;
  }
  LAUNCH_CHECK();
  return do_commit(c, outcome);
}
static int do_accept(eagle_ctx* c) { return do_accept(c, c->pbuf, c->qbuf, c->outcome); }

static int fetch_results(eagle_ctx* c, int32_t* out_tokens, int32_t* out_len, int32_t* path) {
  const int B = c->n_active, D1 = c->D + 1;
  // path, tokens and lengths lie next to each other in the workspace: one copy into pinned host memory brings all three
  const size_t span = (size_t)((const char*)(c->len_out + c->cfg.max_batch) - (const char*)c->path);
  HIPCHK(hipMemcpyAsync(c->res_host, c->path, span, hipMemcpyDeviceToHost, c->stream));
  HIPCHK(hipStreamSynchronize(c->stream));
  const char* rh = (const char*)c->res_host;
  const int* len = (const int*)(rh + ((const char*)c->len_out - (const char*)c->path));
  if (out_tokens) memcpy(out_tokens, rh + ((const char*)c->tok_out - (const char*)c->path), (size_t)B * D1 * 4);
  if (path) memcpy(path, rh, (size_t)B * D1 * 4);
  for (int s = 0; s < B; ++s) {
    if (len[s] < 1 || len[s] > D1) return fail(EAGLE_EHIP, "internal: accepted length %d out of range", len[s]);
    c->h_ctx[s] += len[s]; c->h_ntok[s] += len[s];
    if (out_len) out_len[s] = len[s];
  }
  return EAGLE_OK;
}

extern "C" int eagle_draft_tree(eagle_ctx* c, int32_t* tree_tokens) {
  if (!c) return fail(EAGLE_EINVAL, "null context");
  int rc = do_draft(c);
  if (rc) return rc;
  if (tree_tokens) {
    HIPCHK(hipMemcpyAsync(tree_tokens, c->tree_tok, (size_t)c->n_active * c->M * 4, hipMemcpyDeviceToHost, c->stream));
    HIPCHK(hipStreamSynchronize(c->stream));
  }
  return EAGLE_OK;
}
extern "C" int eagle_verify(eagle_ctx* c) {
  if (!c) return fail(EAGLE_EINVAL, "null context");
  return do_verify(c);
}
extern "C" int eagle_accept(eagle_ctx* c, int32_t* out_tokens, int32_t* out_len, int32_t* path) {
  if (!c) return fail(EAGLE_EINVAL, "null context");
  int rc = do_accept(c);
  if (rc) return rc;
  return fetch_results(c, out_tokens, out_len, path);
}

extern "C" int eagle_accept_static(eagle_ctx* c, int32_t* out_tokens, int32_t* out_len, int32_t* path) {
  if (!c) return fail(EAGLE_EINVAL, "null context");
  const eagle_config& g = c->cfg;
  const size_t B = (size_t)c->n_active;
  const size_t vec = (B * g.vocab * 4 + 255) & ~(size_t)255;                  // one fp32 [n_active][vocab] array
  // (one limit for every vocabulary, though those up to 32768 no longer use the vectors: what a call accepts does not hang on the kernel that serves it)
  const size_t need = std::max(B * c->M * sizeof(int2), g.temperature > 0.f ? 2 * vec : 0);
  if (need > EAGLE_STATIC_SCRATCH_BYTES)
    return fail(EAGLE_EINVAL, "eagle_accept_static: %zu active slots x vocab %d need %zu bytes of scratch, the static array holds %u", B, g.vocab, need, EAGLE_STATIC_SCRATCH_BYTES);
  char* sp = (char*)c->static_scratch;
  int rc = do_accept(c, (float*)sp, (float*)(sp + vec), (int2*)sp);
  if (rc) return rc;
  return fetch_results(c, out_tokens, out_len, path);
}

extern "C" int eagle_step(eagle_ctx* c, int32_t* out_tokens, int32_t* out_len, int32_t* path) {
  if (!c) return fail(EAGLE_EINVAL, "null context");
  int rc;
  const bool prof = c->prof_mode > 0;
  if (prof) HIPCHK(hipEventRecord(c->ev[0], c->stream));
  c->cur_phase = 0;
  rc = do_draft(c);
  c->cur_phase = -1;
  if (rc) return rc;
  if (prof) HIPCHK(hipEventRecord(c->ev[1], c->stream));
  c->cur_phase = 1;
  rc = do_verify(c);
  c->cur_phase = -1;
  if (rc) return rc;
  if (prof) HIPCHK(hipEventRecord(c->ev[2], c->stream));
  if ((rc = do_accept(c))) return rc;
  if (prof) HIPCHK(hipEventRecord(c->ev[3], c->stream));
  std::vector<int> ctx_before(c->h_ctx.begin(), c->h_ctx.begin() + c->n_active);
  if ((rc = fetch_results(c, out_tokens, out_len, path))) return rc;
  if (prof) {
    float a, b, d;
    HIPCHK(hipEventElapsedTime(&a, c->ev[0], c->ev[1]));
    HIPCHK(hipEventElapsedTime(&b, c->ev[1], c->ev[2]));
    HIPCHK(hipEventElapsedTime(&d, c->ev[2], c->ev[3]));
    c->prof.draft_ms += a; c->prof.verify_ms += b; c->prof.accept_ms += d; c->prof.steps += 1;
    // algorithmic bytes of this verify: every target weight once, KV read of the context, KV write + logits
    const eagle_config& g = c->cfg;
    double wbytes = c->lm_head.bytes(c->elt);
    for (int l = 0; l < g.n_layers; ++l) {
      const LayerW& w = c->layers[l];
      wbytes += w.qkv.bytes(c->elt) + w.o.bytes(c->elt);
      if (!w.moe) wbytes += w.gu.bytes(c->elt) + w.dn.bytes(c->elt);
    }
    if (g.n_experts > 0) {   // experts that at least one row selected, summed over the layers (counted on the device)
      int touched = 0;
      HIPCHK(hipMemcpy(&touched, c->experts_touched, 4, hipMemcpyDeviceToHost));
      const LayerW& w = c->layers[0];
      wbytes += (double)touched * ((double)w.e_gu[0].N * w.e_gu[0].K + (double)w.e_dn[0].N * w.e_dn[0].K) * c->elt
                + (double)g.n_layers * g.n_experts * g.d_model * 4.0;
    }
    double kvb = 0;
    for (int s = 0; s < c->n_active; ++s)   // context read once + the tree's own rows written
      kvb += 2.0 * g.n_layers * g.n_kv_heads * g.head_dim * c->kv_elt * (double)(ctx_before[s] + c->M);
    wbytes += (double)c->n_active * c->M * g.vocab * 4.0;   // logits written
    c->prof.verify_weight_bytes += wbytes; c->prof.verify_kv_bytes += kvb;
    if (c->prof_mode == 2 && (rc = collect_gemm_events(c))) return rc;
  }
  return EAGLE_OK;
}

extern "C" int eagle_vanilla_step(eagle_ctx* c, int32_t* tokens) {
  if (!c) return fail(EAGLE_EINVAL, "null context");
  int rc = step_ready(c);
  if (rc) return rc;
  const eagle_config& g = c->cfg;
  const int B = c->n_active;
  Pass pv{PASS_VANILLA, 1, B, 0, 0, 0, 0};
  pass_ctx(c, pv);
  if ((rc = (B <= 32 ? target_forward2(c, pv, max_ctx(c), 1, c->vanilla_logits)
                     : target_forward(c, pv, max_ctx(c) + 1, 1, true, c->vanilla_logits, 1, 0)))) return rc;
  if ((rc = rule_logits(c, 0, B, false, c->st.n_tok))) return rc;
  if ((rc = choose(c, B, 0, 0, 0))) return rc;
  std::vector<int> tk(B);
  for (int s = 0; s < B; ++s)
    HIPCHK(hipMemcpyAsync(&tk[s], c->st.tokens + (size_t)s * c->st.tok_stride + c->h_ntok[s], 4, hipMemcpyDeviceToHost, c->stream));
  HIPCHK(hipStreamSynchronize(c->stream));
  for (int s = 0; s < B; ++s) {
    c->h_ctx[s] += 1; c->h_ntok[s] += 1; c->head_stale[s] = 1;
    if (tokens) tokens[s] = tk[s];
  }
  c->phase = 0;
  return EAGLE_OK;
}

extern "C" int eagle_generate(eagle_ctx* c, int32_t seq, const int32_t* prompt, int32_t n_prompt, int32_t max_new,
                              int32_t* out, int32_t* n_out, float* mean_accept_len) {
  if (!c || !out || !n_out) return fail(EAGLE_EINVAL, "null argument");
  if (seq != 0) return fail(EAGLE_EINVAL, "eagle_generate runs a single sequence in slot 0");
  if (max_new < 1) return fail(EAGLE_EINVAL, "max_new must be >= 1");
  if (n_prompt + max_new + c->M + c->D + 2 > c->cfg.max_seq) return fail(EAGLE_ESEQ_FULL, "prompt + max_new + tree does not fit max_seq");
  int rc;
  if ((rc = eagle_reset(c))) return rc;
  int first;
  if ((rc = eagle_prefill(c, 0, prompt, n_prompt, &first))) return rc;
  int produced = 0, steps = 0, emitted = 0;
  out[produced++] = first;
  std::vector<int> toks(c->D + 1);
  while (produced < max_new) {
    int len;
    if ((rc = eagle_step(c, toks.data(), &len, nullptr))) return rc;
    ++steps; emitted += len;
    for (int i = 0; i < len && produced < max_new; ++i) out[produced++] = toks[i];
  }
  *n_out = produced;
  if (mean_accept_len) *mean_accept_len = steps ? (float)emitted / steps : 0.f;
  return EAGLE_OK;
}

// ---------------------------------------------------------------------------- injection (lock-step tests, external schedulers)
extern "C" int eagle_set_page_table(eagle_ctx* c, const int32_t* table) {
  if (!c || !table) return fail(EAGLE_EINVAL, "null argument");
  if (c->n_active != 0) return fail(EAGLE_ESTATE, "the page table can only change while no sequence is active (after eagle_init / eagle_reset)");
  const size_t n = (size_t)c->cfg.max_batch * c->pps;
  std::vector<char> seen(n, 0);
  for (size_t i = 0; i < n; ++i) {
    if (table[i] < 0 || (size_t)table[i] >= n || seen[table[i]]) return fail(EAGLE_EINVAL, "page table entry %zu = %d: entries must be a permutation of 0..%zu", i, table[i], n - 1);
    seen[table[i]] = 1;
  }
  HIPCHK(hipMemcpyAsync(c->page_table, table, n * 4, hipMemcpyHostToDevice, c->stream));
  HIPCHK(hipStreamSynchronize(c->stream));
  return EAGLE_OK;
}

extern "C" int eagle_set_buffer(eagle_ctx* c, int32_t which, int32_t seq, const void* src, size_t bytes) {
  if (!c || !src) return fail(EAGLE_EINVAL, "null argument");
  const eagle_config& g = c->cfg;
  if (seq < 0 || seq >= g.max_batch) return fail(EAGLE_EINVAL, "slot %d out of range", seq);
  void* dst = nullptr;
  size_t need = 0;
  switch (which) {
    case EAGLE_BUF_LOGITS: dst = c->L + (size_t)seq * c->M * g.vocab; need = (size_t)c->M * g.vocab * 4; break;
    case EAGLE_BUF_FEATURES: dst = c->F + (size_t)seq * c->M * g.d_model; need = (size_t)c->M * g.d_model * 4; break;
    case EAGLE_BUF_DRAFT_LOGITS: dst = c->draft_logits + (size_t)seq * c->M * g.vocab; need = (size_t)c->M * g.vocab * 4; break;
    case EAGLE_BUF_DRAFT_FEATURES: dst = c->node_f + (size_t)seq * c->M * g.d_model; need = (size_t)c->M * g.d_model * 4; break;
    case EAGLE_BUF_TREE_TOKENS: {
      const int32_t* t = (const int32_t*)src;
      if (bytes == (size_t)c->M * 4)
        for (int v = 0; v < c->M; ++v) if (t[v] < 0 || t[v] >= g.vocab) return fail(EAGLE_EINVAL, "token %d of node %d outside the vocabulary", t[v], v);
      dst = c->tree_tok + (size_t)seq * c->M; need = (size_t)c->M * 4; break;
    }
    default: return fail(EAGLE_EINVAL, "buffer %d cannot be written", which);
  }
  if (bytes != need) return fail(EAGLE_EINVAL, "source of %zu bytes, the buffer holds %zu", bytes, need);
  HIPCHK(hipMemcpyAsync(dst, src, need, hipMemcpyHostToDevice, c->stream));
  HIPCHK(hipStreamSynchronize(c->stream));
  return EAGLE_OK;
}

extern "C" int eagle_force_tree(eagle_ctx* c, int32_t seq, const int32_t* tokens) {
  if (!c || !tokens) return fail(EAGLE_EINVAL, "null argument");
  if (c->phase != 1) return fail(EAGLE_ESTATE, "eagle_force_tree replaces the tokens of a drafted tree (call eagle_draft_tree first)");
  if (seq < 0 || seq >= c->n_active) return fail(EAGLE_EINVAL, "slot %d is not active", seq);
  return eagle_set_buffer(c, EAGLE_BUF_TREE_TOKENS, seq, tokens, (size_t)c->M * 4);
}

extern "C" int eagle_expand_level(eagle_ctx* c, int32_t level) {
  if (!c) return fail(EAGLE_EINVAL, "null context");
  if (c->n_active < 1) return fail(EAGLE_ESTATE, "no active sequence");
  if (level != -1 && (level < 1 || level >= c->D)) return fail(EAGLE_EINVAL, "level must be -1 (the root) or 1..depth-1");
  const int nr = level < 0 ? 1 : c->tree_h.n_level_rows[level];
  if (nr == 0) return EAGLE_OK;
  return expand(c, level, nr, nullptr, nr);
}

extern "C" int eagle_force_accept(eagle_ctx* c, const int32_t* path, const int32_t* len, const int32_t* bonus) {
  if (!c || !path || !len || !bonus) return fail(EAGLE_EINVAL, "null argument");
  if (c->phase != 2) return fail(EAGLE_ESTATE, "eagle_force_accept needs a verified tree (call eagle_verify first)");
  const int B = c->n_active, D1 = c->D + 1;
  for (int s = 0; s < B; ++s) {
    if (len[s] < 1 || len[s] > D1) return fail(EAGLE_EINVAL, "slot %d: length %d outside 1..%d", s, len[s], D1);
    if (path[s * D1] != 0) return fail(EAGLE_EINVAL, "slot %d: a path starts at the root (node 0)", s);
    for (int i = 1; i < len[s]; ++i) {
      const int v = path[s * D1 + i];
      if (v < 1 || v >= c->M || c->tree_h.parent[v] != path[s * D1 + i - 1]) return fail(EAGLE_EINVAL, "slot %d: node %d at step %d is not a child of its predecessor", s, v, i);
    }
    if (bonus[s] < 0 || bonus[s] >= c->cfg.vocab) return fail(EAGLE_EINVAL, "slot %d: bonus token outside the vocabulary", s);
  }
  HIPCHK(hipMemcpyAsync(c->path, path, (size_t)B * D1 * 4, hipMemcpyHostToDevice, c->stream));
  HIPCHK(hipMemcpyAsync(c->len_out, len, (size_t)B * 4, hipMemcpyHostToDevice, c->stream));
  HIPCHK(hipMemcpyAsync(c->outcome, bonus, (size_t)B * 4, hipMemcpyHostToDevice, c->stream));   // (idle scratch: B ints)
  HIPCHK(hipStreamSynchronize(c->stream));
  k_force_commit<<<(B + 63) / 64, 64, 0, c->stream>>>(c->tree_d, c->st, c->path, c->len_out, (const int*)c->outcome, c->tree_tok, c->tok_out, B);
  LAUNCH_CHECK();
  int rc = do_commit(c, nullptr);
  if (rc) return rc;
  return fetch_results(c, nullptr, nullptr, nullptr);
}

// ---------------------------------------------------------------------------- test / bench access
extern "C" int eagle_get_buffer(eagle_ctx* c, int32_t which, int32_t seq, void* dst, size_t cap) {
  if (!c || !dst) return fail(EAGLE_EINVAL, "null argument");
  const eagle_config& g = c->cfg;
  if (seq < 0 || seq >= g.max_batch) return fail(EAGLE_EINVAL, "slot %d out of range", seq);
  const void* src = nullptr;
  size_t bytes = 0;
  int state[4];
  switch (which) {
    case EAGLE_BUF_LOGITS: src = c->L + (size_t)seq * c->M * g.vocab; bytes = (size_t)c->M * g.vocab * 4; break;
    case EAGLE_BUF_FEATURES: src = c->F + (size_t)seq * c->M * g.d_model; bytes = (size_t)c->M * g.d_model * 4; break;
    case EAGLE_BUF_DRAFT_LOGITS: src = c->draft_logits + (size_t)seq * c->M * g.vocab; bytes = (size_t)c->M * g.vocab * 4; break;
    case EAGLE_BUF_DRAFT_FEATURES: src = c->node_f + (size_t)seq * c->M * g.d_model; bytes = (size_t)c->M * g.d_model * 4; break;
    case EAGLE_BUF_TREE_TOKENS: src = c->tree_tok + (size_t)seq * c->M; bytes = (size_t)c->M * 4; break;
    case EAGLE_BUF_TOKENS: src = c->st.tokens + (size_t)seq * c->st.tok_stride; bytes = (size_t)c->h_ntok[seq] * 4; break;
    case EAGLE_BUF_VANILLA_LOGITS: src = c->vanilla_logits + (size_t)seq * g.vocab; bytes = (size_t)g.vocab * 4; break;
    case EAGLE_BUF_STATE: {
      HIPCHK(hipStreamSynchronize(c->stream));
      HIPCHK(hipMemcpy(&state[0], c->st.n_tok + seq, 4, hipMemcpyDeviceToHost));
      HIPCHK(hipMemcpy(&state[1], c->st.ctx_len + seq, 4, hipMemcpyDeviceToHost));
      HIPCHK(hipMemcpy(&state[2], c->st.n_pend + seq, 4, hipMemcpyDeviceToHost));
      HIPCHK(hipMemcpy(&state[3], c->st.step_no + seq, 4, hipMemcpyDeviceToHost));
      if (cap < sizeof(state)) return fail(EAGLE_EINVAL, "destination too small");
      memcpy(dst, state, sizeof(state));
      return EAGLE_OK;
    }
    case EAGLE_BUF_GEMM_TRACE: src = c->trace; bytes = (size_t)1024 * 8 * 8; break;
    case EAGLE_BUF_PREFILL_FEATURES: src = c->chunk_f + (size_t)c->last_off * g.d_model; bytes = (size_t)c->last_rows * g.d_model * 4; break;
    default: return fail(EAGLE_EINVAL, "unknown buffer id %d", which);
  }
  if (cap < bytes) return fail(EAGLE_EINVAL, "destination of %zu bytes is smaller than the %zu needed", cap, bytes);
  HIPCHK(hipMemcpyAsync(dst, src, bytes, hipMemcpyDeviceToHost, c->stream));
  HIPCHK(hipStreamSynchronize(c->stream));
  return EAGLE_OK;
}

extern "C" int eagle_get_kv_row(eagle_ctx* c, int32_t seq, int32_t layer, int32_t pos, float* k_host, float* v_host) {
  if (!c || !k_host || !v_host) return fail(EAGLE_EINVAL, "null argument");
  const eagle_config& g = c->cfg;
  int li = layer == EAGLE_HEAD_LAYER ? g.n_layers : layer;
  if (seq < 0 || seq >= g.max_batch || li < 0 || li > g.n_layers || pos < 0 || pos >= g.max_seq) return fail(EAGLE_EINVAL, "index out of range");
  const int n = g.n_kv_heads * g.head_dim;
  float* tmp = c->featbuf;   // scratch, idle between passes
  if ((size_t)2 * n > (size_t)c->Mmax * g.d_model) return fail(EAGLE_EINVAL, "internal: scratch too small");
  KVCache kv = kv_for(c, li);
  if (c->kv_f32) k_read_kv_row<float><<<4, 256, 0, c->stream>>>(kv, seq, pos, tmp, tmp + n);
  else k_read_kv_row<bf16_t><<<4, 256, 0, c->stream>>>(kv, seq, pos, tmp, tmp + n);
  LAUNCH_CHECK();
  HIPCHK(hipMemcpyAsync(k_host, tmp, (size_t)n * 4, hipMemcpyDeviceToHost, c->stream));
  HIPCHK(hipMemcpyAsync(v_host, tmp + n, (size_t)n * 4, hipMemcpyDeviceToHost, c->stream));
  HIPCHK(hipStreamSynchronize(c->stream));
  if (c->rope_mode != PACK_ROPE) {                                // the cache holds pair p's members at p and p + head_dim / 2
    const int dh = g.head_dim;
    float head[128];
    for (int h = 0; h < g.n_kv_heads; ++h) {
      memcpy(head, k_host + (size_t)h * dh, dh * 4);
      for (int r = 0; r < dh; ++r) {
        const int at = rope_pair(c->rope_mode, r, dh);
        k_host[(size_t)h * dh + r] = head[(at >> 1) + (at & 1) * (dh / 2)];
      }
    }
  }
  return EAGLE_OK;
}

// ---------------------------------------------------------------------------- measurement reference
// A bare streaming read: every lane loads 16 bytes per instruction, 8 instructions in flight, work-groups walk the
// buffer grid-strided in 32 KiB pieces; nothing is computed beyond an xor that keeps the loads alive.  What it
// sustains is the practical ceiling against which the weight-streaming kernels are read.
__global__ __launch_bounds__(256) void k_stream_read(const u32x4* __restrict__ src, size_t n16, uint32_t* sink) {
  uint32_t acc = 0;
  const size_t stride = (size_t)gridDim.x * 2048;
  for (size_t base = (size_t)blockIdx.x * 2048; base < n16; base += stride) {
    u32x4 v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const size_t i = base + (size_t)u * 256 + threadIdx.x;
      v[u] = __builtin_nontemporal_load(src + (i < n16 ? i : n16 - 1));
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) acc ^= v[u].x ^ v[u].y ^ v[u].z ^ v[u].w;
  }
  if (acc == 0x9E3779B9u) *sink = acc;
}

extern "C" int eagle_probe_stream_read(const void* buf_dev, size_t bytes, int32_t iters, void* hip_stream, double* gb_per_s) {
  if (!buf_dev || !gb_per_s || ((uintptr_t)buf_dev & 15)) return fail(EAGLE_EINVAL, "buffer must be a 16-byte aligned device pointer");
  if (bytes < (1u << 20) + 64 || iters < 1 || iters > 1000) return fail(EAGLE_EINVAL, "need at least 1 MiB + 64 bytes and 1..1000 iterations");
  hipStream_t st = (hipStream_t)hip_stream;
  // the last 64 bytes of the buffer serve as the (never written) sink
  const size_t n16 = (bytes - 64) / 16;
  uint32_t* sink = (uint32_t*)((char*)buf_dev + n16 * 16);
  hipEvent_t e0, e1;
  HIPCHK(hipEventCreate(&e0));
  HIPCHK(hipEventCreate(&e1));
  k_stream_read<<<2048, 256, 0, st>>>((const u32x4*)buf_dev, n16, sink);        // warm-up
  double ms_sum = 0;
  for (int i = 0; i < iters; ++i) {
    hipExtLaunchKernelGGL(k_stream_read, dim3(2048), dim3(256), 0, st, e0, e1, 0, (const u32x4*)buf_dev, n16, sink);
    if (hipGetLastError() != hipSuccess) return fail(EAGLE_EHIP, "probe launch failed");
    HIPCHK(hipEventSynchronize(e1));
    float ms = 0.f;
    HIPCHK(hipEventElapsedTime(&ms, e0, e1));
    ms_sum += ms;
  }
  (void)hipEventDestroy(e0); (void)hipEventDestroy(e1);
  *gb_per_s = (double)n16 * 16.0 * iters / (ms_sum * 1e-3) / 1e9;
  return EAGLE_OK;
}

extern "C" int eagle_set_profiling(eagle_ctx* c, int32_t mode) {
  if (!c || mode < 0 || mode > 2) return fail(EAGLE_EINVAL, "mode must be 0, 1 or 2");
  c->prof_mode = mode;
  return EAGLE_OK;
}
extern "C" int eagle_get_profile(eagle_ctx* c, eagle_profile* out, int32_t reset) {
  if (!c || !out) return fail(EAGLE_EINVAL, "null argument");
  *out = c->prof;
  if (reset) memset(&c->prof, 0, sizeof(c->prof));
  return EAGLE_OK;
}
extern "C" int eagle_get_kernel_stats(eagle_ctx* c, int32_t phase, eagle_kernel_stat* out, int32_t cap, int32_t* n_out, int32_t reset) {
  if (!c || !out || !n_out) return fail(EAGLE_EINVAL, "null argument");
  if (phase != 0 && phase != 1) return fail(EAGLE_EINVAL, "phase must be 0 (drafting) or 1 (verification)");
  int n = 0;
  for (int k = 0; k < KC_COUNT; ++k) {
    KStat& ks = c->kstat[phase][k];
    if (ks.launches == 0) continue;
    if (n >= cap) return fail(EAGLE_EINVAL, "room for %d entries is not enough", cap);
    eagle_kernel_stat& o = out[n++];
    memset(&o, 0, sizeof(o));
    snprintf(o.name, sizeof(o.name), "%s", kKernelClassName[k]);
    snprintf(o.kernel, sizeof(o.kernel), "%s", ks.kernel);
    o.ms = ks.ms; o.launches = ks.launches; o.bytes = ks.bytes;
    if (reset) ks = KStat();
  }
  *n_out = n;
  return EAGLE_OK;
}
