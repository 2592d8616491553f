// libeagle: operators on the caller's own tensors (host side): argument checks, launch shapes.
#include "operators.h"
#include "rope.h"
#include "chunk_attn.h"
#include "logit_rules.h"

#include <cfloat>
#include <cmath>
#include <cstring>
#include <algorithm>

// ---------------------------------------------------------------------------- shared checks
static bool is_type(int t) { return t == EAGLE_F32 || t == EAGLE_BF16; }
static int elt_of(int t) { return t == EAGLE_F32 ? 4 : 2; }
static bool aligned(const void* p, size_t n) { return (uintptr_t)p % n == 0; }

static int check_chunk(const eagle_chunk* c, ChunkDev* d) {
  if (!c) return fail(EAGLE_EINVAL, "chunk is null");
  if (c->n_seqs < 1 || c->n_rows < 0 || c->max_rows < 1 || c->max_keys < 1) return fail(EAGLE_EINVAL, "chunk: n_seqs, max_rows and max_keys must be >= 1, n_rows >= 0");
  if (c->n_rows > 1 << 30 || c->max_rows > 1 << 30 || c->max_keys > 1 << 30) return fail(EAGLE_EINVAL, "chunk: n_rows, max_rows and max_keys must be at most 2^30");
  if (!c->row_start || !c->key_len) return fail(EAGLE_EINVAL, "chunk: row_start or key_len is null");
  if (c->n_rows > 0 && !c->tree_base != !c->tree_mask) return fail(EAGLE_EINVAL, "chunk: tree_base and tree_mask belong together");
  *d = ChunkDev{c->n_seqs, c->n_rows, c->max_rows, c->max_keys, c->row_start, c->key_len, c->tree_base, (const unsigned long long*)c->tree_mask};
  return EAGLE_OK;
}
static int check_kv(const eagle_paged_kv* k, PagedDev* d) {
  if (!k) return fail(EAGLE_EINVAL, "kv is null");
  if (!k->k || !k->v || !k->page_table) return fail(EAGLE_EINVAL, "kv: k, v or page_table is null");
  if (!is_type(k->dtype)) return fail(EAGLE_EINVAL, "kv: dtype must be EAGLE_F32 or EAGLE_BF16");
  if (k->n_kv_heads < 1 || k->head_dim < 1 || k->n_pages < 1 || k->pages_per_seq < 1) return fail(EAGLE_EINVAL, "kv: n_kv_heads, head_dim, n_pages and pages_per_seq must be >= 1");
  if (k->page_tokens < 1 || (k->page_tokens & (k->page_tokens - 1))) return fail(EAGLE_EINVAL, "kv: page_tokens must be a power of two");
  if (k->page_stride < 1 || k->head_stride < 1 || k->token_stride < 1) return fail(EAGLE_EINVAL, "kv: strides must be positive");
  if (k->table_stride < k->pages_per_seq) return fail(EAGLE_EINVAL, "kv: table_stride %lld is smaller than pages_per_seq %d", (long long)k->table_stride, k->pages_per_seq);
  int shift = 0;
  while ((1 << shift) < k->page_tokens) ++shift;
  *d = PagedDev{k->k, k->v, k->n_kv_heads, k->head_dim, shift, k->n_pages, k->pages_per_seq, k->page_stride, k->head_stride, k->token_stride, k->table_stride, k->page_table};
  return EAGLE_OK;
}
// Whether runs of 16 bytes (of an element of `elt` bytes) may be moved at every (row, head).
static bool runs_ok(const void* p, int64_t row, int64_t head, int elt) { return aligned(p, 16) && row * elt % 16 == 0 && head * elt % 16 == 0; }

// Rows of heads of consecutive elements: (row, head) begins at p + (row * row_stride + head * head_stride) * elt.
struct Heads { const void* p; int64_t rows, row, heads, head; int dim, elt; };
static bool same_place(const Heads& a, const Heads& b) { return a.p == b.p && (a.rows == 1 || a.row == b.row) && (a.heads == 1 || a.head == b.head); }
// Whether a and b share an element, as far as that is easily seen: strides that differ say nothing (callers keep such tensors apart).  At most two divisions a head, where the ranges overlap.
static bool share_elements(Heads a, Heads b) {
  if (!a.p || !b.p) return false;
  auto range = [](const Heads& x, int64_t* lo, int64_t* hi) {
    const int64_t r = (x.rows - 1) * x.row, h = (x.heads - 1) * x.head;
    *lo = (int64_t)(uintptr_t)x.p + (std::min<int64_t>(r, 0) + std::min<int64_t>(h, 0)) * x.elt;
    *hi = (int64_t)(uintptr_t)x.p + (std::max<int64_t>(r, 0) + std::max<int64_t>(h, 0) + x.dim) * x.elt;
  };
  int64_t alo, ahi, blo, bhi;
  range(a, &alo, &ahi);
  range(b, &blo, &bhi);
  if (ahi <= blo || bhi <= alo) return false;
  if (a.heads == 1) a.head = b.head;
  if (b.heads == 1) b.head = a.head;
  if (a.rows == 1) a.row = b.rows == 1 ? 0 : b.row;
  if (b.rows == 1) b.row = a.row;
  if (a.row != b.row || a.head != b.head || a.elt != b.elt) return false;
  // a's (i, h) and b's (i', h') lie (i' - i) * row + (h' - h) * head + (b - a) elements apart: closer than a head's length?
  const int64_t apart = (int64_t)(uintptr_t)b.p - (int64_t)(uintptr_t)a.p, row = a.row * a.elt, len = (int64_t)a.dim * a.elt;
  for (int64_t h = 1 - a.heads; h < b.heads; ++h) {
    const int64_t d = apart + h * a.head * a.elt, near = row ? -d / row : 0;
    for (int64_t i = near - 1; i <= near + 1; ++i)
      if (std::abs(d + std::max(1 - a.rows, std::min(i, b.rows - 1)) * row) < len) return true;
  }
  return false;
}
// An output and what is read: the same tensor, or apart.
static bool torn(const Heads& out, const Heads& in) { return !same_place(out, in) && share_elements(out, in); }

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

extern "C" int eagle_rope(const eagle_rope_plan* plan, const eagle_rope_args* a, const eagle_chunk* chunk, const eagle_paged_kv* kv, void* hip_stream) {
  if (!plan || !a) return fail(EAGLE_EINVAL, "null argument");
  RopeDev d;
  memset(&d, 0, sizeof(d));
  int rc;
  if (plan->head_dim < 2 || plan->head_dim > 256 || plan->rot_dim < 2 || plan->rot_dim > plan->head_dim || plan->rot_dim % 2) return fail(EAGLE_EINVAL, "rope: the plan was not made by eagle_rope_plan_init");
  if (!is_type(a->dtype)) return fail(EAGLE_EINVAL, "rope: dtype must be EAGLE_F32 or EAGLE_BF16");
  if (a->n_rows < 0) return fail(EAGLE_EINVAL, "rope: n_rows must be >= 0");
  if (a->n_rows == 0) return EAGLE_OK;
  if (!a->q && !a->k) return fail(EAGLE_EINVAL, "rope: neither q nor k is given");
  if (a->q && (!a->q_out || a->n_heads < 1)) return fail(EAGLE_EINVAL, "rope: q needs q_out and n_heads >= 1");
  if (a->k && a->n_kv_heads < 1) return fail(EAGLE_EINVAL, "rope: k needs n_kv_heads >= 1");
  if (!chunk && !a->positions) return fail(EAGLE_EINVAL, "rope: without a chunk the rows need positions");
  if (chunk) {
    if ((rc = check_chunk(chunk, &d.chunk))) return rc;
    if (chunk->n_rows != a->n_rows) return fail(EAGLE_EINVAL, "rope: the chunk has %d rows, the tensors %d", chunk->n_rows, a->n_rows);
  }
  bool runs = plan->rot_dim / 2 * elt_of(a->dtype) % 16 == 0 && plan->head_dim * elt_of(a->dtype) % 16 == 0;
  if (kv) {
    if (!chunk) return fail(EAGLE_EINVAL, "rope: a cache needs a chunk");
    if (!a->k || a->k_out) return fail(EAGLE_EINVAL, "rope: with a cache k is needed, and goes there: k_out must be null");
    if (a->inverse) return fail(EAGLE_EINVAL, "rope: the transposed map goes without a cache");
    if ((rc = check_kv(kv, &d.kv))) return rc;
    if (kv->n_kv_heads != a->n_kv_heads || kv->head_dim != plan->head_dim) return fail(EAGLE_EINVAL, "rope: the cache has %d heads of %d, k %d of %d", kv->n_kv_heads, kv->head_dim, a->n_kv_heads, plan->head_dim);
    runs = runs && aligned(kv->k, 16) && aligned(kv->v, 16) && kv->page_stride % 8 == 0 && kv->head_stride % 8 == 0 && kv->token_stride % 8 == 0;
  } else {
    if (a->k && !a->k_out) return fail(EAGLE_EINVAL, "rope: without a cache k needs k_out");
    if (a->v) return fail(EAGLE_EINVAL, "rope: v goes to a cache only");
  }
  if ((a->q && ((a->n_rows > 1 && a->q_out_row == 0) || (a->n_heads > 1 && a->q_out_head == 0))) ||
      (a->k && !kv && ((a->n_rows > 1 && a->k_out_row == 0) || (a->n_kv_heads > 1 && a->k_out_head == 0)))) return fail(EAGLE_EINVAL, "rope: rows or heads of an output lie on each other");
  const int elt = elt_of(a->dtype);
  if (a->q) runs = runs && runs_ok(a->q, a->q_row, a->q_head, elt) && runs_ok(a->q_out, a->q_out_row, a->q_out_head, elt);
  if (a->k) runs = runs && runs_ok(a->k, a->k_row, a->k_head, elt);
  if (a->k && !kv) runs = runs && runs_ok(a->k_out, a->k_out_row, a->k_out_head, elt);
  if (a->v) runs = runs && runs_ok(a->v, a->v_row, a->v_head, elt);
  memcpy(d.turn, plan->turn, sizeof(d.turn));
  d.mscale = plan->mscale; d.sign = a->inverse ? -1.f : 1.f;
  d.rot_dim = plan->rot_dim; d.interleaved = plan->interleaved; d.head_dim = plan->head_dim;
  d.n_rows = a->n_rows; d.H = a->q ? a->n_heads : 0; d.KVH = a->k ? a->n_kv_heads : 0;
  const long long heads = (long long)d.H + d.KVH + (a->v ? d.KVH : 0);
  if (heads > 65535) return fail(EAGLE_EINVAL, "rope: too many heads");
  {
    const Heads q{a->q, a->n_rows, a->q_row, a->n_heads, a->q_head, plan->head_dim, elt}, k{a->k, a->n_rows, a->k_row, a->n_kv_heads, a->k_head, plan->head_dim, elt};
    const Heads v{a->v, a->n_rows, a->v_row, a->n_kv_heads, a->v_head, plan->head_dim, elt}, q_out{a->q ? a->q_out : nullptr, a->n_rows, a->q_out_row, a->n_heads, a->q_out_head, plan->head_dim, elt};
    const Heads k_out{a->k && !kv ? a->k_out : nullptr, a->n_rows, a->k_out_row, a->n_kv_heads, a->k_out_head, plan->head_dim, elt};
    if (torn(q_out, q) || torn(k_out, k)) return fail(EAGLE_EINVAL, "rope: an output lies on part of its input: it must be the input or apart from it");
    if (share_elements(q_out, k) || share_elements(q_out, v) || share_elements(k_out, q) || share_elements(q_out, k_out)) return fail(EAGLE_EINVAL, "rope: an output lies on another tensor of the call");
  }
  d.n_heads_all = (int)heads;
  d.q = a->q; d.k = a->k; d.v = a->v; d.q_out = a->q_out; d.k_out = a->k_out;
  d.q_row = a->q_row; d.q_head = a->q_head; d.k_row = a->k_row; d.k_head = a->k_head; d.v_row = a->v_row; d.v_head = a->v_head;
  d.q_out_row = a->q_out_row; d.q_out_head = a->q_out_head; d.k_out_row = a->k_out_row; d.k_out_head = a->k_out_head;
  d.positions = a->positions; d.has_chunk = chunk != nullptr; d.has_kv = kv != nullptr;
  const int VE = runs ? 16 / elt : 1;
  const int units = (plan->head_dim + 2 * VE - 1) / (2 * VE), least = std::max(1, 256 / units);
  const int parts = std::max(1, std::min(1024 / a->n_rows, (d.n_heads_all + least - 1) / least));   // (few rows: their heads in parts, of at least a unit a thread)
  d.heads_per_wg = (d.n_heads_all + parts - 1) / parts;
  const dim3 grid(a->n_rows, (d.n_heads_all + d.heads_per_wg - 1) / d.heads_per_wg);
  const hipStream_t stream = (hipStream_t)hip_stream;
  const bool cf = kv && kv->dtype == EAGLE_F32;
  if (a->dtype == EAGLE_F32) { if (cf) launch_rope<float, float>(d, runs, grid, stream); else launch_rope<float, bf16_t>(d, runs, grid, stream); }
  else { if (cf) launch_rope<bf16_t, float>(d, runs, grid, stream); else launch_rope<bf16_t, bf16_t>(d, runs, grid, stream); }
  LAUNCH_CHECK();
  return EAGLE_OK;
}

// ---------------------------------------------------------------------------- attention over a paged cache
static int check_attention(const eagle_attention_args* a, const eagle_chunk* chunk, const eagle_paged_kv* kv, ChunkAttnDev* d) {
  if (!a) return fail(EAGLE_EINVAL, "null argument");
  int rc;
  memset(d, 0, sizeof(*d));
  if ((rc = check_chunk(chunk, &d->chunk)) || (rc = check_kv(kv, &d->kv))) return rc;
  if (!is_type(a->dtype)) return fail(EAGLE_EINVAL, "attention: dtype must be EAGLE_F32 or EAGLE_BF16");
  if (a->dtype == EAGLE_BF16 && kv->dtype != EAGLE_BF16) return fail(EAGLE_EINVAL, "attention: bf16 queries need a bf16 cache");
  if (a->n_heads < 1 || a->n_heads > 65535 || a->n_heads % kv->n_kv_heads) return fail(EAGLE_EINVAL, "attention: n_heads must be a multiple of the cache's heads");
  if (kv->head_dim % 8 || kv->head_dim > 128) return fail(EAGLE_EINVAL, "attention: head_dim must be a multiple of 8, at most 128");
  if (!std::isfinite(a->scale) || !(a->softcap >= 0.f) || !std::isfinite(a->softcap)) return fail(EAGLE_EINVAL, "attention: scale must be finite, softcap >= 0 and finite");
  if (!std::isfinite(a->scale * 2.885390f) || (a->softcap > 0.f && (a->softcap < FLT_MIN || !std::isfinite(a->scale * 2.885390f / a->softcap))))
    return fail(EAGLE_EINVAL, "attention: scale, or scale / softcap, is too large");
  if (a->window < 0) return fail(EAGLE_EINVAL, "attention: window must be >= 0");
  if (chunk->n_rows > 0 && (!a->q || !a->out)) return fail(EAGLE_EINVAL, "attention: q or out is null");
  if ((chunk->n_rows > 1 && a->out_row == 0) || (a->n_heads > 1 && a->out_head == 0)) return fail(EAGLE_EINVAL, "attention: rows or heads of out lie on each other");
  // (bounds that a caller leaves wide are drawn in, so that they cost no work-groups and no number overflows)
  d->chunk.max_rows = std::min(chunk->max_rows, std::max(1, chunk->n_rows));
  d->chunk.max_keys = (int)std::min((long long)chunk->max_keys, (long long)kv->pages_per_seq * kv->page_tokens);
  if ((long long)d->chunk.max_rows * (a->n_heads / kv->n_kv_heads) > 1 << 30) return fail(EAGLE_EINVAL, "attention: too many rows a kv head");
  const int elt = elt_of(a->dtype), kelt = elt_of(kv->dtype);
  if (chunk->n_rows > 0 && torn(Heads{a->out, chunk->n_rows, a->out_row, a->n_heads, a->out_head, kv->head_dim, elt}, Heads{a->q, chunk->n_rows, a->q_row, a->n_heads, a->q_head, kv->head_dim, elt}))
    return fail(EAGLE_EINVAL, "attention: out lies on part of q: it must be q or apart from it");
  if (!runs_ok(a->q, a->q_row, a->q_head, elt)) return fail(EAGLE_EINVAL, "attention: q's rows and heads must start on multiples of 16 bytes");
  if (!aligned(a->out, 16) || a->out_row % 8 || a->out_head % 8) return fail(EAGLE_EINVAL, "attention: out's rows and heads must start on multiples of 16 bytes and 8 elements");
  if (kv->token_stride > 1 << 24) return fail(EAGLE_EINVAL, "attention: the cache's token_stride must be at most 2^24");
  if (!aligned(kv->k, 16) || !aligned(kv->v, 16) || kv->page_stride * kelt % 16 || kv->head_stride * kelt % 16 || kv->token_stride * kelt % 16)
    return fail(EAGLE_EINVAL, "attention: the cache's tokens must start on multiples of 16 bytes");
  d->q = a->q; d->out = a->out; d->q_row = a->q_row; d->q_head = a->q_head; d->out_row = a->out_row; d->out_head = a->out_head;
  d->H = a->n_heads; d->window = std::min(a->window, 1 << 30); d->slopes = a->slopes; d->prefix = a->prefix; d->softcap = a->softcap;
  d->scale = std::fabs(a->scale);
  d->q_flip = std::signbit(a->scale) ? 0x80008000u : 0u;
  d->lane_pages = kv->page_tokens < 8;
  return EAGLE_OK;
}

// WIDE beyond 32 columns, where a narrow block would read the cache a second time (64 sequences of 1k to 16k tokens, 8 heads a kv head, with joining, narrow / wide.  bf16: 32 columns 451 / 464,
// 40 486 / 485, 48 496 / 487, 64 511 / 489.  fp32 queries would stay narrow a little longer where there are as many sequences: 32 columns 533 / 624 over bf16, 1035 / 2109 over fp32; 64 columns
// 705 / 805, 1679 / 2196.)
// Where sequences, kv heads and column blocks make fewer work-groups than these, the tokens are split; a part has a few tiles at least (the narrow shape: whole rounds of its four waves),
// and there are at most as many parts as k_chunk_attn_join has lanes.
// Narrow, 64 sequences of 1k to 16k tokens, 64 / 8 heads, us with 1 to 8 parts at most.  bf16: 434, 417, 414, 439, 407, 407, 408, 414; fp32 over bf16 with 1, 2, 4, 6, 8: 531, 578, 613, 489, 537; over
// fp32 993, 1173, 1309, 986, 1124.  (Not in order: the sequences' own numbers of parts, hence the rounds of work-groups, change with the bound; six is the least of all three.)  Sixteen of those
// sequences, bf16, with 1, 2, 4, 6, 8, 12, 16, 25: 215, 173, 172, 180, 171, 179, 177, 181; this bound makes it 25.  One token over 701 keys, 32 heads, fp32, 22 tiles: parts of 4 tiles 17.6, of 5 23.0, of 3 29.4.  Wide: one a CU (four trees of 26 nodes on 8 kv heads, fp32 queries, 37 tiles: 8 parts 27, 10 parts 32 to 38; 2011 fp32 rows on 32 heads, 512 work-groups: whole
// 327, in two 339 and 26 more for joining).
constexpr int ATTN_WIDE_WGS = 256, ATTN_NARROW_WGS = 3200, ATTN_MIN_TILES = 4, ATTN_MAX_PARTS = 64;

// Columns and parts of a call; returns the bytes of workspace, at most `limit` of them if that is possible.
static size_t plan_attention(ChunkAttnDev* d, int kv_dtype, size_t limit, bool* wide) {
  const int g = d->H / d->kv.n_kv_heads;
  const long long cols = (long long)d->chunk.max_rows * g;
  *wide = cols > 32;
  const int KT = *wide && kv_dtype == EAGLE_BF16 ? 64 : 32, round = *wide ? 1 : 4;
  d->col_blocks = (int)((cols + (*wide ? 127 : 31)) / (*wide ? 128 : 32));
  const long long units = (long long)d->col_blocks * d->kv.n_kv_heads * d->chunk.n_seqs, tiles = ((long long)d->chunk.max_keys + KT - 1) / KT;
  long long parts = std::min((*wide ? ATTN_WIDE_WGS : ATTN_NARROW_WGS) / units, (tiles + ATTN_MIN_TILES - 1) / ATTN_MIN_TILES);
  parts = std::max(1ll, std::min(parts, (long long)ATTN_MAX_PARTS));
  const size_t pairs = (size_t)d->chunk.n_rows * d->H, PART = d->kv.head_dim <= 64 ? 64 : 128;
  for (;; --parts) {
    d->split_tiles = (int)((tiles + parts * round - 1) / (parts * round) * round);
    d->splits = (int)((tiles + d->split_tiles - 1) / d->split_tiles);
    if (d->splits == 1) return 256;
    const size_t bytes = (pairs * d->splits * 8 + 255) / 256 * 256 + pairs * d->splits * PART * 4;
    if (bytes <= limit) return bytes;
  }
}

extern "C" size_t eagle_chunk_attention_workspace(const eagle_attention_args* a, const eagle_chunk* chunk, const eagle_paged_kv* kv) {
  ChunkAttnDev d;
  bool wide;
  if (check_attention(a, chunk, kv, &d)) return 0;
  return plan_attention(&d, kv->dtype, SIZE_MAX, &wide);
}

template <typename T, typename CT, int DH, bool WIDE, bool MODS>
static int launch_attention(ChunkAttnDev d, hipStream_t stream) {
  typedef ChunkAttn<T, CT, DH, WIDE, MODS> P;
  auto kernel = k_chunk_attn<P, T, CT>;
  const int blocks = d.kv.n_kv_heads * d.col_blocks;
  d.turn = P::WAVES == 2 && d.chunk.n_seqs == 1 && d.splits == 1 && blocks <= 512 ? std::max(1, 256 / d.kv.n_kv_heads) : d.col_blocks;
  kernel<<<dim3(d.kv.n_kv_heads * d.col_blocks * d.splits, d.chunk.n_seqs), 256, 0, stream>>>(d);
  LAUNCH_CHECK();
  if (d.splits > 1) {
    k_chunk_attn_join<P, T><<<dim3(d.chunk.n_rows, (d.H + 3) / 4), 256, 0, stream>>>(d);
    LAUNCH_CHECK();
  }
  return EAGLE_OK;
}
template <typename T, typename CT>
static int launch_attention(const ChunkAttnDev& d, bool wide, bool mods, hipStream_t stream) {
#define ATTEND(DH, WIDE) return mods ? launch_attention<T, CT, DH, WIDE, true>(d, stream) : launch_attention<T, CT, DH, WIDE, false>(d, stream)
  if (d.kv.head_dim > 96) { if (wide) ATTEND(128, true); else ATTEND(128, false); }
  if (d.kv.head_dim > 64) { if (wide) ATTEND(96, true); else ATTEND(96, false); }
  if (wide) ATTEND(64, true); else ATTEND(64, false);
#undef ATTEND
}

int chunk_attention(const eagle_attention_args* a, const eagle_chunk* chunk, const eagle_paged_kv* kv, void* workspace, size_t workspace_bytes, bool fit, hipStream_t stream) {
  ChunkAttnDev d;
  int rc = check_attention(a, chunk, kv, &d);
  if (rc) return rc;
  bool wide;
  const size_t need = plan_attention(&d, kv->dtype, fit ? workspace_bytes : SIZE_MAX, &wide);
  if (!workspace || !aligned(workspace, 256)) return fail(EAGLE_EINVAL, "attention: workspace must be a 256-byte aligned device pointer");
  if (workspace_bytes < need) return fail(EAGLE_ENOMEM, "attention: workspace of %zu bytes is smaller than the %zu needed", workspace_bytes, need);
  if (chunk->n_rows == 0) return EAGLE_OK;
  if (d.chunk.n_seqs > 65535 || (long long)d.kv.n_kv_heads * d.col_blocks * d.splits > 0x7FFFFFFF) return fail(EAGLE_EINVAL, "attention: more than 65535 sequences, or too many rows");
  const size_t pairs = (size_t)d.chunk.n_rows * d.H * d.splits;
  d.part_ml = (float*)workspace;
  d.part_o = (float*)((char*)workspace + (pairs * 8 + 255) / 256 * 256);
  const bool mods = d.softcap > 0.f || d.slopes || d.scale == 0.f;   // (a scale of 0 times a masked score)
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
