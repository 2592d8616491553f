// Attention over a paged cache on the host: checks, split, launches, for every type of cache.
#pragma once
#include "checks.h"
#include "chunk_attn.h"

#include <cfloat>
#include <cstring>

// What is common to every type of cache (d->kv says where it lies), of elements of kelt bytes.
static int check_attention(const eagle_attention_args* a, const eagle_chunk* chunk, int kelt, ChunkAttnDev* d) {
  const PagedDev* kv = &d->kv;
  int rc;
  if ((rc = check_chunk(chunk, &d->chunk))) return rc;
  if (!is_type(a->dtype)) return fail(EAGLE_EINVAL, "attention: dtype must be EAGLE_F32 or EAGLE_BF16");
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
  d->chunk.max_keys = (int)std::min((long long)chunk->max_keys, (long long)kv->pages_per_seq << kv->page_shift);
  if ((long long)d->chunk.max_rows * (a->n_heads / kv->n_kv_heads) > 1 << 30) return fail(EAGLE_EINVAL, "attention: too many rows a kv head");
  const int elt = elt_of(a->dtype);
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
  d->lane_pages = kv->page_shift < 3;
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
// Codes: the narrow shape up to 8192 columns, since a wave's tiles are then its own, without barriers, and what it reads beyond once comes from the L2 (D 128, a causal prompt on 8 kv heads, wide / narrow:
// 1024 columns 15.8 / 10.0, 4096 40.5 / 31.4, 8192 77 / 77, 16384 209 / 222; with a cap 17.8 / 10.0, 47 / 32, 91 / 82, 252 / 249; fp32 queries 25 / 22, 67 / 47, 137 / 128, 392 / 427; int8 and bf16 16 / 10,
// 41 / 32, 80 / 83, 208 / 251).  Two work-groups a CU where there are not as many units anyway (four trees of 26 nodes, fp32: 512 work-groups 33, 1024 38, 3200 59; 16 of them 103, 122, 130), else as above
// (64 sequences of 1k to 16k tokens: 242, 242, 220).
constexpr int ATTN_CODED_COLS = 8192, ATTN_CODED_WGS = 512;
constexpr int ATTN_WIDE_WGS = 256, ATTN_NARROW_WGS = 3200, ATTN_MIN_TILES = 4, ATTN_MAX_PARTS = 64;

// Columns and parts of a call; returns the bytes of workspace, at most `limit` of them if that is possible.
static size_t plan_attention(ChunkAttnDev* d, int dtype, int kelt, size_t limit, bool* wide) {
  const int g = d->H / d->kv.n_kv_heads;
  const long long cols = (long long)d->chunk.max_rows * g;
  *wide = cols > (kelt == 1 ? ATTN_CODED_COLS : 32);
  const int KT = tile_tokens(*wide, dtype == EAGLE_F32, kelt), round = *wide ? 1 : 4;
  d->col_blocks = (int)((cols + (*wide ? 127 : 31)) / (*wide ? 128 : 32));
  const long long units = (long long)d->col_blocks * d->kv.n_kv_heads * d->chunk.n_seqs, tiles = ((long long)d->chunk.max_keys + KT - 1) / KT;
  const int wgs = *wide ? ATTN_WIDE_WGS : kelt == 1 && units < ATTN_CODED_WGS ? ATTN_CODED_WGS : ATTN_NARROW_WGS;
  long long parts = std::min(wgs / units, (tiles + ATTN_MIN_TILES - 1) / ATTN_MIN_TILES);
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

// Splits the tokens, and checks and divides the workspace; `fit`: over fewer work-groups rather than refuse a small one.
static int place_attention(ChunkAttnDev* d, const eagle_attention_args* a, int kelt, void* workspace, size_t workspace_bytes, bool fit, bool* wide, bool* mods) {
  const size_t need = plan_attention(d, a->dtype, kelt, fit ? workspace_bytes : SIZE_MAX, wide);
  if (!workspace || !aligned(workspace, 256)) return fail(EAGLE_EINVAL, "attention: workspace must be a 256-byte aligned device pointer");
  if (workspace_bytes < need) return fail(EAGLE_ENOMEM, "attention: workspace of %zu bytes is smaller than the %zu needed", workspace_bytes, need);
  if (d->chunk.n_rows == 0) return EAGLE_OK;
  if (d->chunk.n_seqs > 65535 || (long long)d->kv.n_kv_heads * d->col_blocks * d->splits > 0x7FFFFFFF) return fail(EAGLE_EINVAL, "attention: more than 65535 sequences, or too many rows");
  const size_t pairs = (size_t)d->chunk.n_rows * d->H * d->splits;
  d->part_ml = (float*)workspace;
  d->part_o = (float*)((char*)workspace + (pairs * 8 + 255) / 256 * 256);
  *mods = d->softcap > 0.f || d->slopes || d->scale == 0.f;   // (a scale of 0 times a masked score)
  return EAGLE_OK;
}
