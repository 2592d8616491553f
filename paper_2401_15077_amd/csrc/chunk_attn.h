// Attention of a chunk of new tokens over a paged cache.
#pragma once
#include "rows.h"
#include "rope.h"

struct ChunkAttnDev {
  const void* q; void* out;
  long long q_row, q_head, out_row, out_head;
  int H, window;
  float scale, softcap;
  const float* slopes; const int* prefix;
  ChunkDev chunk; PagedDev kv;
};

// A work-group a row and head; a thread a token for the scores, a thread an element for the sums.
template <typename T, typename CT>
__global__ __launch_bounds__(256) void k_chunk_attn(const ChunkAttnDev A) {
  __shared__ float qs[128], ps[256], sh[16];
  __shared__ long long cell_s[256];
  const int r = blockIdx.x, h = blockIdx.y, tid = threadIdx.x, dh = A.kv.head_dim;
  const int s = wave_row_seq(A.chunk.row_start, A.chunk.n_seqs, r);
  if (s < 0 || r - A.chunk.row_start[s] >= A.chunk.max_rows) return;
  const int keys = chunk_keys(A.chunk, A.kv, s), kvh = h / (A.H / A.kv.n_kv_heads);
  const bool tree = A.chunk.tree_mask;
  const unsigned long long m = tree ? A.chunk.tree_mask[r] : 0;
  const int base = tree ? A.chunk.tree_base[s] : 0;
  const int own = tree ? base + __popcll(m) - 1 : A.chunk.key_len[s] - A.chunk.row_start[s + 1] + r;
  const int prefix = A.prefix ? (tree ? min(A.prefix[s], base) : A.prefix[s]) : 0;
  if (tid < dh) load_run<1>((const T*)A.q + r * A.q_row + h * A.q_head + tid, qs + tid);
  __syncthreads();
  float m_run = -INFINITY, l = 0.f, o = 0.f;
  for (int j0 = 0; j0 < keys; j0 += 256) {
    const int j = j0 + tid;
    float x = -INFINITY;
    long long cell = -1;
    if (j < keys) {
      const int page = token_page(A.kv, s, j);
      bool seen;
      int pos = j;
      if (tree) {
        const int u = j - base;
        seen = u < 0 || (u < 64 && (m >> u & 1));
        if (u >= 0) pos = base + __popcll(m & ((u < 64 ? 1ull << u : 0ull) - 1));
      } else seen = j <= own;
      const int dist = own - pos;
      seen = (seen && (A.window <= 0 || dist < A.window)) || j < prefix;
      if (seen && page >= 0) {
        cell = page * A.kv.page_stride + kvh * A.kv.head_stride + (j & ((1 << A.kv.page_shift) - 1)) * A.kv.token_stride;
        float acc = 0.f;
        for (int d = 0; d < dh; ++d) { float kx; load_run<1>((const CT*)A.kv.k + cell + d, &kx); acc = fmaf(qs[d], kx, acc); }
        x = acc * A.scale;
        if (A.softcap > 0.f) x = A.softcap * tanhf(x / A.softcap);
        if (A.slopes) x -= A.slopes[h] * (float)abs(dist);
      }
    }
    float mx = x;
    for (int i = 32; i; i >>= 1) mx = fmaxf(mx, __shfl_xor(mx, i, 64));
    __syncthreads();
    if ((tid & 63) == 0) sh[tid >> 6] = mx;
    __syncthreads();
    const float m_new = fmaxf(m_run, fmaxf(fmaxf(sh[0], sh[1]), fmaxf(sh[2], sh[3])));
    const float p = cell >= 0 ? expf(x - (m_new > -INFINITY ? m_new : 0.f)) : 0.f;
    const float f = m_run > -INFINITY ? expf(m_run - m_new) : 0.f;
    ps[tid] = p; cell_s[tid] = cell;
    __syncthreads();
    m_run = m_new;
    l *= f; o *= f;
    for (int i = 0; i < 256; ++i)
      if (cell_s[i] >= 0) {
        l += ps[i];
        if (tid < dh) { float v; load_run<1>((const CT*)A.kv.v + cell_s[i] + tid, &v); o = fmaf(ps[i], v, o); }
      }
  }
  if (tid < dh) { o = l == 0.f ? 0.f : o / l; store_run<1>((T*)A.out + r * A.out_row + h * A.out_head + tid, &o); }
}
