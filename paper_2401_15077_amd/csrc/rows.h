// New tokens of a batch over a paged cache, as the operators on the caller's tensors see them: which sequence a row belongs to, where its
// token lies, what it sees.
#pragma once
#include "common.h"

struct ChunkDev {
  int n_seqs, n_rows, max_rows, max_keys;
  const int *row_start, *key_len, *tree_base;
  const unsigned long long* tree_mask;
};
struct PagedDev {
  void *k, *v;
  int n_kv_heads, head_dim, page_shift, n_pages, pages_per_seq;
  long long page_stride, head_stride, token_stride, table_stride;
  const int* page_table;
};

// The sequence that owns row r (-1: none), for a whole wave: 64 boundaries are compared at a time, so up to 64 sequences cost one load.
__device__ inline int wave_row_seq(const int* __restrict__ row_start, int n_seqs, int r) {
  const int lane = threadIdx.x & 63;
  int s = 0;
  for (int i = 0; i < n_seqs; i += 64) {
    const bool behind = i + lane < n_seqs && row_start[i + lane + 1] <= r;
    s += __popcll(__ballot(behind));
  }
  return s < n_seqs && row_start[0] <= r ? s : -1;
}

// Tokens of sequence s that may be read: its length within what the host said and the page table has.
__device__ inline int chunk_keys(const ChunkDev& c, const PagedDev& kv, int s) {
  const long long room = (long long)kv.pages_per_seq << kv.page_shift;
  return (int)max(0ll, min((long long)min(c.key_len[s], c.max_keys), room));
}

// Page of token t (0 <= t < chunk_keys) of sequence s, -1 where it is not there.
__device__ inline int token_page(const PagedDev& kv, int s, int t) {
  const int p = kv.page_table[(size_t)s * kv.table_stride + (t >> kv.page_shift)];
  return (unsigned)p < (unsigned)kv.n_pages ? p : -1;
}
