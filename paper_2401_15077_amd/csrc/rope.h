// Rotary positions of queries and keys, and the append of keys and values to a paged cache.
#pragma once
#include "rows.h"

struct RopeDev {
  unsigned long long turn[128];            // pair p: fraction of a turn a position, times 2^64
  float mscale, sign;                      // sign -1: the transposed map
  int rot_dim, interleaved, head_dim;
  int n_rows, H, KVH, heads_per_wg, n_heads_all;   // n_heads_all: H query heads, KVH key heads, and KVH value heads if v is given
  const void *q, *k, *v;
  void *q_out, *k_out;
  long long q_row, q_head, k_row, k_head, v_row, v_head, q_out_row, q_out_head, k_out_row, k_out_head;
  const int* positions;
  int has_chunk, has_kv;
  ChunkDev chunk; PagedDev kv;
};

// Cosine and sine of position * turn.  The product wraps at whole turns by itself (mod 2^64) and is exact, so a position of 10^9 costs no accuracy: what is
// left is the 2^-65 turn that `turn` was rounded by, times the position.  The nearest quarter turn is taken off in integers, the rest (at most an eighth,
// |x| <= pi / 4) is exact in 32 bits but for one rounding, and the Taylor polynomials up to x^11 / x^10 leave out less than 10^-9.
__device__ inline float2 cos_sin_turn(unsigned long long turn, int position) {
  const unsigned long long t = turn * (unsigned long long)(long long)position + (1ull << 31);
  const int x32 = (int)(uint32_t)(t >> 32);                       // signed fraction of a turn, 2^-32 each
  const uint32_t quarter = ((uint32_t)x32 + (1u << 29)) >> 30;
  const int rest = (int)((uint32_t)x32 - (quarter << 30));
  const float x = (float)rest * 1.46291807926715968e-9f;          // 2 pi / 2^32
  const float z = x * x;
  float s = -2.50521083854417188e-8f, c = -2.75573192239858907e-7f;
  s = fmaf(s, z, 2.75573192239858907e-6f); c = fmaf(c, z, 2.48015873015873016e-5f);
  s = fmaf(s, z, -1.98412698412698413e-4f); c = fmaf(c, z, -1.38888888888888889e-3f);
  s = fmaf(s, z, 8.33333333333333333e-3f); c = fmaf(c, z, 4.16666666666666667e-2f);
  s = fmaf(s, z, -1.66666666666666667e-1f); c = fmaf(c, z, -0.5f);
  s = fmaf(s * z, x, x); c = fmaf(c, z, 1.0f);
  const float a = quarter & 1 ? s : c, b = quarter & 1 ? c : s;   // quarters turn (c, s) into (c, s), (-s, c), (-c, -s), (s, -c)
  return make_float2((quarter + 1) & 2 ? -a : a, quarter & 2 ? -b : b);
}

template <int VE> __device__ inline void load_run(const float* p, float* x) {
  if constexpr (VE == 4) { const f32x4 v = *(const f32x4*)p; x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w; }
  else x[0] = *p;
}
template <int VE> __device__ inline void load_run(const bf16_t* p, float* x) {
  if constexpr (VE == 8) {
    const u32x4 v = *(const u32x4*)p;
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = __builtin_bit_cast(float, v[i] << 16); x[2 * i + 1] = __builtin_bit_cast(float, v[i] & 0xFFFF0000u); }
  } else x[0] = bf16_to_f32(*p);
}
__device__ inline uint32_t bf16_pair(float a, float b) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 h = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, h);
}
template <int VE> __device__ inline void store_run(float* p, const float* x) {
  if constexpr (VE == 1) *p = x[0];
  else
#pragma unroll
    for (int i = 0; i < VE; i += 4) *(f32x4*)(p + i) = f32x4{x[i], x[i + 1], x[i + 2], x[i + 3]};
}
template <int VE> __device__ inline void store_run(bf16_t* p, const float* x) {
  if constexpr (VE == 1) *p = f32_to_bf16(x[0]);
  else if constexpr (VE == 4) *(u32x2*)p = u32x2{bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3])};
  else *(u32x4*)p = u32x4{bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3]), bf16_pair(x[4], x[5]), bf16_pair(x[6], x[7])};
}

// A work-group takes a row and heads_per_wg of its heads.  First a wave finds out about the row, then the threads work out the cosines and
// sines of the row's pairs, once for all heads (in LDS), then every thread moves runs of VE elements, two at a time: the two members of VE pairs (half
// layout), or VE pairs side by side (interleaved), or what is not rotated.  VE = 16 bytes' worth where strides and sizes allow, else 1.
// Bound by HBM, and by latency for a few rows: 8191 rows of 64 + 8 + 8 heads of 128 in bf16 take 63 us, 5.3 TB/s read and written (four rows a work-group 78: fewer, longer chains of loads;
// elements instead of runs 190); 2011 fp32 rows of 64 + 8 heads in a loop over the same tensors 25; 104 rows of 32 + 8 + 8 heads 5.6 (four a work-group 8.1).
template <typename T, typename CT, int VE>
__global__ __launch_bounds__(256) void k_rope(const RopeDev A) {
  __shared__ float2 cs[128];
  __shared__ int s_pos;
  __shared__ long long s_cell;                                    // the row's place in the cache: element offset of kv head 0, -1 none, -2: not a row of any sequence
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int r = blockIdx.x;
  if (wave == 0) {
    int pos = A.positions ? A.positions[r] : 0;
    long long cell = -1;
    if (A.has_chunk) {
      const int s = wave_row_seq(A.chunk.row_start, A.chunk.n_seqs, r);
      if (s < 0 || r - max(0, A.chunk.row_start[s]) >= A.chunk.max_rows) cell = -2;
      else {
        int token, p;
        if (A.chunk.tree_mask) {
          const unsigned long long m = A.chunk.tree_mask[r];
          const int base = A.chunk.tree_base[s];
          token = m ? base + 63 - __builtin_clzll(m) : -1; p = base + __popcll(m) - 1;
        } else token = p = A.chunk.key_len[s] - A.chunk.row_start[s + 1] + r;
        if (!A.positions) pos = p;
        if (A.has_kv && token >= 0 && token < min((long long)A.chunk.max_keys, (long long)A.kv.pages_per_seq << A.kv.page_shift)) {
          const int page = token_page(A.kv, s, token);
          if (page >= 0) cell = page * A.kv.page_stride + (token & ((1 << A.kv.page_shift) - 1)) * A.kv.token_stride;
        }
      }
    }
    if (lane == 0) { s_pos = pos; s_cell = cell; }
  }
  __syncthreads();
  const int half = A.rot_dim >> 1;
  const long long cell = s_cell;
  if (cell == -2) return;
  for (int p = tid; p < half; p += 256) {
    float2 c = cos_sin_turn(A.turn[p], s_pos);
    c.x *= A.mscale; c.y *= A.mscale * A.sign;
    cs[p] = c;
  }
  __syncthreads();
  const int rot_units = half / VE, units = rot_units + (A.head_dim - A.rot_dim + 2 * VE - 1) / (2 * VE);   // (VE > 1: half is a multiple of VE)
  const int h0 = blockIdx.y * A.heads_per_wg, nh = min(A.heads_per_wg, A.n_heads_all - h0);
  for (int i = tid; i < nh * units; i += 256) {
    const int h = h0 + i / units, u = i % units;
    const bool is_q = h < A.H, is_k = !is_q && h < A.H + A.KVH;
    const int kh = is_q ? h : h - A.H - (is_k ? 0 : A.KVH);       // head within q, k or v
    if (!is_q && A.has_kv && cell < 0) continue;
    const T* src = is_q ? (const T*)A.q + r * A.q_row + kh * A.q_head : is_k ? (const T*)A.k + r * A.k_row + kh * A.k_head : (const T*)A.v + r * A.v_row + kh * A.v_head;
    const bool rotated = u < rot_units && (is_q || is_k);
    // the two runs of the unit
    int e0, e1;
    if (u >= rot_units) { e0 = A.rot_dim + (u - rot_units) * 2 * VE; e1 = e0 + VE; }
    else if (A.interleaved) { e0 = u * 2 * VE; e1 = e0 + VE; }
    else { e0 = u * VE; e1 = half + e0; }
    const bool two = e1 < A.head_dim;
    float a[VE], b[VE];
    load_run<VE>(src + e0, a);
    if (two) load_run<VE>(src + e1, b);
    if (rotated) {
      const float2* c = cs + u * VE;
      if (A.interleaved && VE > 1) {
#pragma unroll
        for (int j = 0; j < VE; j += 2) {
          const float2 c0 = c[j / 2], c1 = c[VE / 2 + j / 2];
          const float x0 = a[j], y0 = a[(j + 1) % VE], x1 = b[j], y1 = b[(j + 1) % VE];
          a[j] = x0 * c0.x - y0 * c0.y; a[(j + 1) % VE] = y0 * c0.x + x0 * c0.y;
          b[j] = x1 * c1.x - y1 * c1.y; b[(j + 1) % VE] = y1 * c1.x + x1 * c1.y;
        }
      } else {
#pragma unroll
        for (int j = 0; j < VE; ++j) {
          const float x = a[j], y = b[j];
          a[j] = x * c[j].x - y * c[j].y; b[j] = y * c[j].x + x * c[j].y;
        }
      }
    }
    if (is_q || !A.has_kv) {
      T* dst = is_q ? (T*)A.q_out + r * A.q_out_row + kh * A.q_out_head : (T*)A.k_out + r * A.k_out_row + kh * A.k_out_head;
      store_run<VE>(dst + e0, a);
      if (two) store_run<VE>(dst + e1, b);
    } else {
      CT* dst = (CT*)(is_k ? A.kv.k : A.kv.v) + cell + kh * A.kv.head_stride;
      store_run<VE>(dst + e0, a);
      if (two) store_run<VE>(dst + e1, b);
    }
  }
}
