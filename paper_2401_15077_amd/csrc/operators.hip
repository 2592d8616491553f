// libeagle: operators on the caller's own tensors (host side): argument checks, launch shapes.
#include "checks.h"
#include "rope.h"
#include "rope_coded.h"
#include "attention.h"
#include "logit_rules.h"

#include <cstring>

// ---------------------------------------------------------------------------- rotary positions
extern "C" int eagle_rope_plan_init(const eagle_rope_config* c, eagle_rope_plan* out) {
  if (!c || !out) return fail(EAGLE_EINVAL, "null argument");
  if (c->head_dim < 2 || c->head_dim > 256) return fail(EAGLE_EINVAL, "rope: head_dim must be 2..256");
  if (c->rot_dim < 2 || c->rot_dim > c->head_dim || c->rot_dim % 2) return fail(EAGLE_EINVAL, "rope: rot_dim must be even, 2..head_dim");
  if (c->scaling < EAGLE_ROPE_NONE || c->scaling > EAGLE_ROPE_RAMP) return fail(EAGLE_EINVAL, "rope: unknown scaling %d", c->scaling);
  if (!(c->theta > 1.0) || !std::isfinite(c->theta)) return fail(EAGLE_EINVAL, "rope: theta must be above 1");
  if (!std::isfinite(c->mscale)) return fail(EAGLE_EINVAL, "rope: mscale must be finite");
  if (c->scaling != EAGLE_ROPE_NONE && (!(c->factor >= 1.0) || !std::isfinite(c->factor))) return fail(EAGLE_EINVAL, "rope: factor must be >= 1");
  if (c->scaling == EAGLE_ROPE_BASE && c->rot_dim < 4) return fail(EAGLE_EINVAL, "rope: a scaled base needs rot_dim >= 4");
  const bool bands = c->scaling == EAGLE_ROPE_BANDS || c->scaling == EAGLE_ROPE_RAMP;
  if (bands && (c->trained_len < 1 || !(c->low > 0.0) || !(c->high > c->low) || !std::isfinite(c->high))) return fail(EAGLE_EINVAL, "rope: this scaling needs trained_len >= 1 and 0 < low < high");
  const long double pi = 3.14159265358979323846264338327950288L;
  const int rot = c->rot_dim;
  long double theta = c->theta;
  const long double factor = c->scaling == EAGLE_ROPE_NONE ? 1.0L : (long double)c->factor, L = c->trained_len;
  if (c->scaling == EAGLE_ROPE_BASE) theta *= powl(factor, (long double)rot / (rot - 2));
  long double a = 0, b = 0;
  if (c->scaling == EAGLE_ROPE_RAMP) {
    a = std::max(0.0L, floorl(rot * logl(L / (2 * pi * c->high)) / (2 * logl(theta))));
    b = std::min((long double)(rot - 1), ceill(rot * logl(L / (2 * pi * c->low)) / (2 * logl(theta))));
  }
  memset(out, 0, sizeof(*out));
  for (int p = 0; p < rot / 2; ++p) {
    long double f = powl(theta, -2.0L * p / rot);
    if (c->scaling == EAGLE_ROPE_LINEAR) f /= factor;
    if (c->scaling == EAGLE_ROPE_BANDS) {
      const long double s = std::min(1.0L, std::max(0.0L, (L * f / (2 * pi) - c->low) / ((long double)c->high - c->low)));
      f *= s + (1 - s) / factor;
    }
    if (c->scaling == EAGLE_ROPE_RAMP) {
      const long double t = std::min(1.0L, std::max(0.0L, (p - a) / std::max(b - a, 0.001L)));
      f = f * (1 - t) + f / factor * t;
    }
    out->turn[p] = (uint64_t)(f / (2 * pi) * 18446744073709551616.0L + 0.5L);     // f <= 1
  }
  out->head_dim = c->head_dim; out->rot_dim = rot; out->interleaved = c->interleaved != 0; out->mscale = c->mscale;
  return EAGLE_OK;
}

template <typename T, typename CT>
static void launch_rope(const RopeDev& d, bool runs, dim3 grid, hipStream_t stream) {
  if (runs) k_rope<T, CT, 16 / sizeof(T)><<<grid, 256, 0, stream>>>(d);
  else k_rope<T, CT, 1><<<grid, 256, 0, stream>>>(d);
}

// Checks of a rotation, with `cache`: keys and values go to a cache of cache_heads heads of cache_dim; what the kernels have to know; whether 16-byte runs may be moved.
static int check_rope(const eagle_rope_plan* plan, const eagle_rope_args* a, const eagle_chunk* chunk, bool cache, int cache_heads, int cache_dim, RopeDev* d, bool* runs) {
  int rc;
  if (chunk) {
    if ((rc = check_chunk(chunk, &d->chunk))) return rc;
    if (chunk->n_rows != a->n_rows) return fail(EAGLE_EINVAL, "rope: the chunk has %d rows, the tensors %d", chunk->n_rows, a->n_rows);
  }
  const int elt = elt_of(a->dtype);
  *runs = plan->rot_dim / 2 * elt % 16 == 0 && plan->head_dim * elt % 16 == 0;
  if (cache) {
    if (!chunk) return fail(EAGLE_EINVAL, "rope: a cache needs a chunk");
    if (!a->k || a->k_out) return fail(EAGLE_EINVAL, "rope: with a cache k is needed, and goes there: k_out must be null");
    if (a->inverse) return fail(EAGLE_EINVAL, "rope: the transposed map goes without a cache");
    if (cache_heads != a->n_kv_heads || cache_dim != plan->head_dim) return fail(EAGLE_EINVAL, "rope: the cache has %d heads of %d, k %d of %d", cache_heads, cache_dim, a->n_kv_heads, plan->head_dim);
  } else {
    if (a->k && !a->k_out) return fail(EAGLE_EINVAL, "rope: without a cache k needs k_out");
    if (a->v) return fail(EAGLE_EINVAL, "rope: v goes to a cache only");
  }
  if ((a->q && ((a->n_rows > 1 && a->q_out_row == 0) || (a->n_heads > 1 && a->q_out_head == 0))) ||
      (a->k && !cache && ((a->n_rows > 1 && a->k_out_row == 0) || (a->n_kv_heads > 1 && a->k_out_head == 0)))) return fail(EAGLE_EINVAL, "rope: rows or heads of an output lie on each other");
  if (a->q) *runs = *runs && runs_ok(a->q, a->q_row, a->q_head, elt) && runs_ok(a->q_out, a->q_out_row, a->q_out_head, elt);
  if (a->k) *runs = *runs && runs_ok(a->k, a->k_row, a->k_head, elt);
  if (a->k && !cache) *runs = *runs && runs_ok(a->k_out, a->k_out_row, a->k_out_head, elt);
  if (a->v) *runs = *runs && runs_ok(a->v, a->v_row, a->v_head, elt);
  memcpy(d->turn, plan->turn, sizeof(d->turn));
  d->mscale = plan->mscale; d->sign = a->inverse ? -1.f : 1.f;
  d->rot_dim = plan->rot_dim; d->interleaved = plan->interleaved; d->head_dim = plan->head_dim;
  d->n_rows = a->n_rows; d->H = a->q ? a->n_heads : 0; d->KVH = a->k ? a->n_kv_heads : 0;
  const long long heads = (long long)d->H + d->KVH + (a->v ? d->KVH : 0);
  if (heads > 65535) return fail(EAGLE_EINVAL, "rope: too many heads");
  {
    const Heads q{a->q, a->n_rows, a->q_row, a->n_heads, a->q_head, plan->head_dim, elt}, k{a->k, a->n_rows, a->k_row, a->n_kv_heads, a->k_head, plan->head_dim, elt};
    const Heads v{a->v, a->n_rows, a->v_row, a->n_kv_heads, a->v_head, plan->head_dim, elt}, q_out{a->q ? a->q_out : nullptr, a->n_rows, a->q_out_row, a->n_heads, a->q_out_head, plan->head_dim, elt};
    const Heads k_out{a->k && !cache ? a->k_out : nullptr, a->n_rows, a->k_out_row, a->n_kv_heads, a->k_out_head, plan->head_dim, elt};
    if (torn(q_out, q) || torn(k_out, k)) return fail(EAGLE_EINVAL, "rope: an output lies on part of its input: it must be the input or apart from it");
    if (share_elements(q_out, k) || share_elements(q_out, v) || share_elements(k_out, q) || share_elements(q_out, k_out)) return fail(EAGLE_EINVAL, "rope: an output lies on another tensor of the call");
  }
  d->n_heads_all = (int)heads;
  d->q = a->q; d->k = a->k; d->v = a->v; d->q_out = a->q_out; d->k_out = a->k_out;
  d->q_row = a->q_row; d->q_head = a->q_head; d->k_row = a->k_row; d->k_head = a->k_head; d->v_row = a->v_row; d->v_head = a->v_head;
  d->q_out_row = a->q_out_row; d->q_out_head = a->q_out_head; d->k_out_row = a->k_out_row; d->k_out_head = a->k_out_head;
  d->positions = a->positions; d->has_chunk = chunk != nullptr; d->has_kv = cache;
  return EAGLE_OK;
}
// The arguments that need no chunk and no cache to be judged.
static int check_rope_args(const eagle_rope_plan* plan, const eagle_rope_args* a) {
  if (!plan || !a) return fail(EAGLE_EINVAL, "null argument");
  if (plan->head_dim < 2 || plan->head_dim > 256 || plan->rot_dim < 2 || plan->rot_dim > plan->head_dim || plan->rot_dim % 2) return fail(EAGLE_EINVAL, "rope: the plan was not made by eagle_rope_plan_init");
  if (!is_type(a->dtype)) return fail(EAGLE_EINVAL, "rope: dtype must be EAGLE_F32 or EAGLE_BF16");
  if (a->n_rows < 0) return fail(EAGLE_EINVAL, "rope: n_rows must be >= 0");
  if (a->n_rows == 0) return EAGLE_OK;
  if (!a->q && !a->k) return fail(EAGLE_EINVAL, "rope: neither q nor k is given");
  if (a->q && (!a->q_out || a->n_heads < 1)) return fail(EAGLE_EINVAL, "rope: q needs q_out and n_heads >= 1");
  if (a->k && a->n_kv_heads < 1) return fail(EAGLE_EINVAL, "rope: k needs n_kv_heads >= 1");
  return EAGLE_OK;
}
// Work-groups a row of d->n_heads_all heads is taken by.
static int rope_parts(RopeDev* d, int dtype, bool runs) {
  const int VE = runs ? 16 / elt_of(dtype) : 1;
  const int units = (d->head_dim + 2 * VE - 1) / (2 * VE), least = std::max(1, 256 / units);
  const int parts = std::max(1, std::min(1024 / d->n_rows, (d->n_heads_all + least - 1) / least));   // (few rows: their heads in parts, of at least a unit a thread)
  d->heads_per_wg = (d->n_heads_all + parts - 1) / parts;
  return (d->n_heads_all + d->heads_per_wg - 1) / d->heads_per_wg;
}

extern "C" int eagle_rope(const eagle_rope_plan* plan, const eagle_rope_args* a, const eagle_chunk* chunk, const eagle_paged_kv* kv, void* hip_stream) {
  RopeDev d;
  memset(&d, 0, sizeof(d));
  int rc = check_rope_args(plan, a);
  if (rc || a->n_rows == 0) return rc;
  if (!chunk && !a->positions) return fail(EAGLE_EINVAL, "rope: without a chunk the rows need positions");
  bool runs;
  if (kv && (rc = check_kv(kv, &d.kv))) return rc;
  if ((rc = check_rope(plan, a, chunk, kv != nullptr, kv ? kv->n_kv_heads : 0, kv ? kv->head_dim : 0, &d, &runs))) return rc;
  if (kv) runs = runs && aligned(kv->k, 16) && aligned(kv->v, 16) && kv->page_stride % 8 == 0 && kv->head_stride % 8 == 0 && kv->token_stride % 8 == 0;
  const dim3 grid(a->n_rows, rope_parts(&d, a->dtype, runs));
  const hipStream_t stream = (hipStream_t)hip_stream;
  const bool cf = kv && kv->dtype == EAGLE_F32;
  if (a->dtype == EAGLE_F32) { if (cf) launch_rope<float, float>(d, runs, grid, stream); else launch_rope<float, bf16_t>(d, runs, grid, stream); }
  else { if (cf) launch_rope<bf16_t, float>(d, runs, grid, stream); else launch_rope<bf16_t, bf16_t>(d, runs, grid, stream); }
  LAUNCH_CHECK();
  return EAGLE_OK;
}

// Up to as many work-groups those that append come first: theirs is the longer way, and what is left of the chip takes the queries.  Beyond, they are spread evenly among the queries', since they
// keep the vector unit busy and the others the memory (8 kv heads of 128, bf16, 64 query heads: 1024 rows first 13.2, spread 17.1, 2048 22.0 / 23.8, 4096 39.3 / 38.3, 8191 in five sequences 88.7 / 82.4;
// 32 heads of both, fp32: 512 rows 18.2 / 18.8, 2048 56.0 / 50.7).
constexpr int APPEND_FRONT = 4096;

template <typename T, bool E4M3>
static void launch_append(const AppendDev& d, bool runs, int groups, hipStream_t stream) {
  if (runs) k_rope_coded<T, E4M3, 16 / sizeof(T)><<<groups, 256, 0, stream>>>(d);
  else k_rope_coded<T, E4M3, 1><<<groups, 256, 0, stream>>>(d);
}

extern "C" int eagle_rope_coded(const eagle_rope_plan* plan, const eagle_rope_args* a, const eagle_chunk* chunk, const eagle_coded_kv* kv, void* hip_stream) {
  AppendDev d;
  memset(&d, 0, sizeof(d));
  int rc = check_rope_args(plan, a);
  if (rc || a->n_rows == 0) return rc;
  bool runs;
  if ((rc = check_coded(kv, &d.kv)) || (rc = check_rope(plan, a, chunk, true, kv->n_kv_heads, kv->head_dim, &d.rope, &runs))) return rc;
  runs = runs && aligned(kv->k, 8) && aligned(kv->v, 8) && kv->page_stride % 8 == 0 && kv->head_stride % 8 == 0 && kv->token_stride % 8 == 0;
  d.k = a->k; d.v = a->v; d.k_row = a->k_row; d.k_head = a->k_head; d.v_row = a->v_row; d.v_head = a->v_head;
  d.KVH = a->n_kv_heads;
  // blocks that the rows may reach: of n consecutive tokens at most (n - 1) / B + 2 and n, of a tree's 64 nodes 62 / B + 2 a sequence
  const long long R = a->n_rows, S = std::min<long long>(chunk->n_seqs, R), B = kv->block_tokens;
  d.seq_blocks = 62 / kv->block_tokens + 2;
  const long long blocks = chunk->tree_mask ? (long long)chunk->n_seqs * d.seq_blocks : std::min(R, (R - S) / B + 2 * S), kv_groups = blocks * d.KVH * (a->v ? 2 : 1);
  // the queries' work-groups find no keys and values in `rope`
  d.rope.KVH = 0; d.rope.k = d.rope.v = nullptr; d.rope.has_kv = 0; d.rope.n_heads_all = d.rope.H;
  const long long q_groups = a->q ? (long long)R * rope_parts(&d.rope, a->dtype, runs) : 0;
  if (kv_groups + q_groups > 0x7FFFFFFF) return fail(EAGLE_EINVAL, "rope: too many rows");
  const int groups = (int)(kv_groups + q_groups);
  d.kv_groups = (int)kv_groups;
  d.kv_share = groups <= APPEND_FRONT ? 1ull << 32 : (((unsigned long long)kv_groups << 32) + groups - 1) / groups;
  const hipStream_t stream = (hipStream_t)hip_stream;
  const bool e4m3 = kv->dtype == EAGLE_E4M3;
  if (a->dtype == EAGLE_F32) { if (e4m3) launch_append<float, true>(d, runs, groups, stream); else launch_append<float, false>(d, runs, groups, stream); }
  else { if (e4m3) launch_append<bf16_t, true>(d, runs, groups, stream); else launch_append<bf16_t, false>(d, runs, groups, stream); }
  LAUNCH_CHECK();
  return EAGLE_OK;
}

// ---------------------------------------------------------------------------- attention over a paged cache
static int check_attention(const eagle_attention_args* a, const eagle_chunk* chunk, const eagle_paged_kv* kv, ChunkAttnDev* d) {
  if (!a) return fail(EAGLE_EINVAL, "null argument");
  int rc;
  memset(d, 0, sizeof(*d));
  if ((rc = check_kv(kv, &d->kv))) return rc;
  if (a->dtype == EAGLE_BF16 && kv->dtype != EAGLE_BF16) return fail(EAGLE_EINVAL, "attention: bf16 queries need a bf16 cache");
  return check_attention(a, chunk, elt_of(kv->dtype), d);
}

extern "C" size_t eagle_chunk_attention_workspace(const eagle_attention_args* a, const eagle_chunk* chunk, const eagle_paged_kv* kv) {
  ChunkAttnDev d;
  bool wide;
  if (check_attention(a, chunk, kv, &d)) return 0;
  return plan_attention(&d, a->dtype, elt_of(kv->dtype), SIZE_MAX, &wide);
}

int chunk_attention(const eagle_attention_args* a, const eagle_chunk* chunk, const eagle_paged_kv* kv, void* workspace, size_t workspace_bytes, bool fit, hipStream_t stream) {
  ChunkAttnDev d;
  int rc = check_attention(a, chunk, kv, &d);
  if (rc) return rc;
  bool wide, mods;
  if ((rc = place_attention(&d, a, elt_of(kv->dtype), workspace, workspace_bytes, fit, &wide, &mods)) || chunk->n_rows == 0) return rc;
  if (a->dtype == EAGLE_BF16) return launch_attention<bf16_t, bf16_t>(d, wide, mods, stream);
  if (kv->dtype == EAGLE_BF16) return launch_attention<float, bf16_t>(d, wide, mods, stream);
  return launch_attention<float, float>(d, wide, mods, stream);
}

extern "C" int eagle_chunk_attention(const eagle_attention_args* a, const eagle_chunk* chunk, const eagle_paged_kv* kv, void* workspace, size_t workspace_bytes,
                                     void* hip_stream) {
  return chunk_attention(a, chunk, kv, workspace, workspace_bytes, false, (hipStream_t)hip_stream);
}

// ---------------------------------------------------------------------------- logit rules
template <typename T>
static int launch_rules(RulesDev d, bool runs, hipStream_t stream) {
  // A slice costs its work-group a walk over the row's text and a word of LDS a token, so a row is cut into no more slices than 512 threads need, or than make 1024 work-groups, four a CU;
  // and into slices of one length, so that no short one walks the text for little.  160 rows of 100003 bf16 logits: 26.2 us with 512 threads, 27.7 with 256, 31.0 with 1024 (two work-groups a CU,
  // a third round nearly empty); 104 rows of 32000 fp32 logits: 10.5 us at 1024 work-groups, 11.0 at 512.  Runs a thread: bf16 26.0 with two, 27.4 with three; fp32 10.5 with two, 9.9 with three.
  constexpr int VE = 16 / sizeof(T), PIECES = sizeof(T) == 4 ? 3 : 2;
  auto pieces = [&](int t) { return (d.vocab + t * VE * PIECES - 1) / (t * VE * PIECES); };
  const int parts = std::max(pieces(512), std::min((1024 + d.n_rows - 1) / d.n_rows, pieces(128)));
  const int threads = (pieces(64) + parts - 1) / parts * 64;
  const int slice = threads * VE * PIECES;
  const int reach = d.vocab + (runs ? VE - 1 : 0);              // (the first piece of a row may begin up to VE - 1 elements in front of it)
  const dim3 grid((reach + slice - 1) / slice, d.n_rows);
  auto kernel = runs ? k_logit_rules<T, VE, PIECES> : k_logit_rules<T, 1, VE * PIECES>;
  kernel<<<grid, threads, (size_t)slice * 4 + 16, stream>>>(d);      // (at most 32 KB)
  LAUNCH_CHECK();
  return EAGLE_OK;
}

extern "C" int eagle_apply_logit_rules(const eagle_logits* l, const eagle_logit_rules* rules, void* hip_stream) {
  if (!l || !rules) return fail(EAGLE_EINVAL, "null argument");
  if (!is_type(l->dtype)) return fail(EAGLE_EINVAL, "logits: dtype must be EAGLE_F32 or EAGLE_BF16");
  if (l->n_rows < 0 || l->n_rows > 65535 || l->vocab < 1 || l->vocab > 1 << 30 || rules->n_seqs < 1) return fail(EAGLE_EINVAL, "logits: n_rows must be 0..65535, vocab 1..2^30, n_seqs >= 1");
  if (l->n_rows == 0) return EAGLE_OK;
  if (!l->in || !l->out) return fail(EAGLE_EINVAL, "logits: in or out is null");
  if (l->in_stride < l->vocab || l->out_stride < l->vocab) return fail(EAGLE_EINVAL, "logits: rows of %d entries need strides of at least that", l->vocab);
  if (!l->row_start && l->n_rows != rules->n_seqs) return fail(EAGLE_EINVAL, "logits: without row_start there is one row a sequence (%d rows, %d sequences)", l->n_rows, rules->n_seqs);
  if (!l->path_token != !l->path_mask) return fail(EAGLE_EINVAL, "logits: path_token and path_mask belong together");
  if (l->allowed && (l->n_masks < 1 || l->mask_stride < (l->vocab + 31) / 32)) return fail(EAGLE_EINVAL, "logits: masks need n_masks >= 1 and %d words a row", (l->vocab + 31) / 32);
  if (rules->tokens && (!rules->n_tokens || rules->token_stride < 0 || rules->max_tokens < 0 || rules->max_tokens > 1 << 29))
    return fail(EAGLE_EINVAL, "logits: tokens need n_tokens, token_stride >= 0 and max_tokens 0..2^29");
  if (rules->bias_token && (!rules->bias_start || !rules->bias_value || rules->n_bias < 0)) return fail(EAGLE_EINVAL, "logits: biases need bias_start, bias_value and n_bias >= 0");
  RulesDev d{l->n_rows, l->vocab, l->n_masks, rules->n_seqs, rules->n_bias, rules->max_tokens, l->in, l->out, l->in_stride, l->out_stride, l->mask_stride, rules->token_stride,
             l->row_start, l->path_token, l->allowed_row, rules->tokens, rules->n_tokens, rules->n_prompt, rules->bias_start, rules->n_bias > 0 ? rules->bias_token : nullptr,
             (const unsigned long long*)l->path_mask, l->allowed, rules->repetition, rules->presence, rules->frequency, rules->bias_value};
  const int elt = elt_of(l->dtype);
  if (torn(Heads{l->out, l->n_rows, l->out_stride, 1, 0, l->vocab, elt}, Heads{l->in, l->n_rows, l->in_stride, 1, 0, l->vocab, elt}))
    return fail(EAGLE_EINVAL, "logits: out lies on part of in: it must be in or apart from it");
  const bool runs = aligned(l->in, elt) && ((uintptr_t)l->in - (uintptr_t)l->out) % 16 == 0 && (l->in_stride - l->out_stride) * elt % 16 == 0;
  return l->dtype == EAGLE_F32 ? launch_rules<float>(d, runs, (hipStream_t)hip_stream) : launch_rules<bf16_t>(d, runs, (hipStream_t)hip_stream);
}
