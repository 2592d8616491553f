// What the entry points of the operators check, and what they share on the host.
#pragma once
#include "operators.h"
#include "rows.h"
#include "codes.h"

#include <cmath>
#include <algorithm>

static inline bool is_type(int t) { return t == EAGLE_F32 || t == EAGLE_BF16; }
static inline int elt_of(int t) { return t == EAGLE_F32 ? 4 : 2; }
static inline bool aligned(const void* p, size_t n) { return (uintptr_t)p % n == 0; }

static inline int check_chunk(const eagle_chunk* c, ChunkDev* d) {
  if (!c) return fail(EAGLE_EINVAL, "chunk is null");
  if (c->n_seqs < 1 || c->n_rows < 0 || c->max_rows < 1 || c->max_keys < 1) return fail(EAGLE_EINVAL, "chunk: n_seqs, max_rows and max_keys must be >= 1, n_rows >= 0");
  if (c->n_rows > 1 << 30 || c->max_rows > 1 << 30 || c->max_keys > 1 << 30) return fail(EAGLE_EINVAL, "chunk: n_rows, max_rows and max_keys must be at most 2^30");
  if (!c->row_start || !c->key_len) return fail(EAGLE_EINVAL, "chunk: row_start or key_len is null");
  if (c->n_rows > 0 && !c->tree_base != !c->tree_mask) return fail(EAGLE_EINVAL, "chunk: tree_base and tree_mask belong together");
  *d = ChunkDev{c->n_seqs, c->n_rows, c->max_rows, c->max_keys, c->row_start, c->key_len, c->tree_base, (const unsigned long long*)c->tree_mask};
  return EAGLE_OK;
}
static inline int check_kv(const eagle_paged_kv* k, PagedDev* d) {
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
static inline int check_coded(const eagle_coded_kv* k, CodedDev* d) {
  if (!k) return fail(EAGLE_EINVAL, "kv is null");
  if (!k->k || !k->v || !k->k_scale || !k->v_scale || !k->page_table) return fail(EAGLE_EINVAL, "kv: k, v, k_scale, v_scale or page_table is null");
  if (k->dtype != EAGLE_E4M3 && k->dtype != EAGLE_INT8) return fail(EAGLE_EINVAL, "kv: dtype must be EAGLE_E4M3 or EAGLE_INT8");
  if (k->n_kv_heads < 1 || k->head_dim < 1 || k->n_pages < 1 || k->pages_per_seq < 1) return fail(EAGLE_EINVAL, "kv: n_kv_heads, head_dim, n_pages and pages_per_seq must be >= 1");
  if (k->block_tokens < 16 || k->block_tokens > 128 || (k->block_tokens & (k->block_tokens - 1))) return fail(EAGLE_EINVAL, "kv: block_tokens must be 16, 32, 64 or 128");
  if (k->page_tokens < k->block_tokens || (k->page_tokens & (k->page_tokens - 1))) return fail(EAGLE_EINVAL, "kv: page_tokens must be a power of two, at least block_tokens");
  if (k->page_stride < 1 || k->head_stride < 1 || k->token_stride < 1 || k->scale_page < 1 || k->scale_head < 1) return fail(EAGLE_EINVAL, "kv: strides must be positive");
  if (k->table_stride < k->pages_per_seq) return fail(EAGLE_EINVAL, "kv: table_stride %lld is smaller than pages_per_seq %d", (long long)k->table_stride, k->pages_per_seq);
  if (!aligned(k->k_scale, 4) || !aligned(k->v_scale, 4)) return fail(EAGLE_EINVAL, "kv: scales must start on multiples of 4 bytes");
  int page = 0, block = 0;
  while ((1 << page) < k->page_tokens) ++page;
  while ((1 << block) < k->block_tokens) ++block;
  *d = CodedDev{(uint8_t*)k->k, (uint8_t*)k->v, k->k_scale, k->v_scale, k->n_kv_heads, k->head_dim, page, block, k->n_pages, k->pages_per_seq, k->page_stride, k->head_stride, k->token_stride,
                k->table_stride, k->scale_page, k->scale_head, k->page_table};
  return EAGLE_OK;
}
// Whether runs of 16 bytes (of an element of `elt` bytes) may be moved at every (row, head).
static inline bool runs_ok(const void* p, int64_t row, int64_t head, int elt) { return aligned(p, 16) && row * elt % 16 == 0 && head * elt % 16 == 0; }

// Rows of heads of consecutive elements: (row, head) begins at p + (row * row_stride + head * head_stride) * elt.
struct Heads { const void* p; int64_t rows, row, heads, head; int dim, elt; };
static inline bool same_place(const Heads& a, const Heads& b) { return a.p == b.p && (a.rows == 1 || a.row == b.row) && (a.heads == 1 || a.head == b.head); }
// Whether a and b share an element, as far as that is easily seen: strides that differ say nothing (callers keep such tensors apart).  At most two divisions a head, where the ranges overlap.
static inline bool share_elements(Heads a, Heads b) {
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
static inline bool torn(const Heads& out, const Heads& in) { return !same_place(out, in) && share_elements(out, in); }
