// Rotary positions of queries and keys, and the append of keys and values to a paged cache of 8-bit codes.
#pragma once
#include "rope.h"
#include "codes.h"

struct AppendDev {
  RopeDev rope;                            // of the queries (KVH 0), and what says how the keys turn
  CodedDev kv;
  const void *k, *v;
  long long k_row, k_head, v_row, v_head;
  int KVH, seq_blocks;                     // trees: blocks of a sequence at most
  int kv_groups;                           // work-groups that append (each a block, kv head, keys or values): below i there are i * kv_share / 2^32 of them, until there are all
  unsigned long long kv_share;
};

// Cosine and sine of position * turn in 64 bits: as cos_sin_turn takes whole and quarter turns off, with the series' terms up to x^17 and x^16, which leave out less than 2^-63 of a sine and 2^-58 of a
// cosine (|x| <= pi / 4; a term more would be lost in the sum's own roundings of 2^-53).  The turn is rounded to a multiple of 2^-64: the angle is off by less than 2^-62 a position.
__device__ inline double2 cos_sin_turn64(unsigned long long turn, int position) {
  const unsigned long long t = turn * (unsigned long long)(long long)position;
  const unsigned long long quarter = (t + (1ull << 61)) >> 62;
  const double x = (double)(long long)(t - (quarter << 62)) * 3.4061215800865545e-19;   // 2 pi / 2^64
  const double z = x * x;
  double s = 2.8114572543455206e-15, c = 4.7794773323873853e-14;                        // 1 / 17!, 1 / 16!
  s = fma(s, z, -7.6471637318198165e-13); c = fma(c, z, -1.1470745597729725e-11);
  s = fma(s, z, 1.6059043836821613e-10); c = fma(c, z, 2.0876756987868099e-9);
  s = fma(s, z, -2.505210838544172e-8); c = fma(c, z, -2.755731922398589e-7);
  s = fma(s, z, 2.7557319223985893e-6); c = fma(c, z, 2.4801587301587302e-5);
  s = fma(s, z, -1.9841269841269841e-4); c = fma(c, z, -1.3888888888888889e-3);
  s = fma(s, z, 8.3333333333333333e-3); c = fma(c, z, 4.1666666666666667e-2);
  s = fma(s, z, -1.6666666666666667e-1); c = fma(c, z, -0.5);
  s = fma(s * z, x, x); c = fma(c, z, 1.0);
  const double a = quarter & 1 ? s : c, b = quarter & 1 ? c : s;
  return make_double2((quarter + 1) & 2 ? -a : a, quarter & 2 ? -b : b);
}

// a <= largest * 2^e: the least e (a > 0, finite).  largest = m 2^x with 0.5 <= m < 1.
template <bool E4M3> __device__ inline int least_exponent(double a) {
  int e;
  const double f = frexp(a, &e);
  return E4M3 ? e - 9 + (f > 0.875) : e - 7 + (f > 0.9921875);
}

// Some work-groups append: one takes the new tokens of one block of a kv head, keys or values (it has to know the largest of them before it can write one).  The others rotate the queries, as
// rope_row says.
// Everything from the angle to the code is worked out in 64 bits and rounded to odd once for the conversion.  So a code is what the definition says, but where the exact number lies as near to the border
// between two codes as the angle's error and a few roundings of 2^-53 move it: there it may be the neighbour.
//
// What bounds it: 8191 rows, 64 / 8 heads of 128, bf16, take 84 us for 318 MB, where a copy of as much takes 66.  Keys and values keep the vector unit busy (64-bit operations issue as 32-bit ones do
// here; in 32 bits with a 64-bit way out for what falls near a border they took 13 more), queries the memory, so the two kinds are spread among each other, and five waves a SIMD hide what either
// waits for: with four (all of a run's angles at once) 92, with six (by spilling) 89 to 121.  Queries in a launch of their own, or heads in a loop of a work-group that keeps angles: 121 to 129, then.
// One row 8.5, 104 rows 10: the chain from lengths to page, tokens, largest, scale and code.
template <typename T, bool E4M3, int VE>
__global__ __launch_bounds__(256) void k_rope_coded(const AppendDev A) {
  const RopeDev& P = A.rope;
  const int nth = min((int)(blockIdx.x * A.kv_share >> 32), A.kv_groups);
  if (min((int)((blockIdx.x + 1) * A.kv_share >> 32), A.kv_groups) == nth) {
    const int i = blockIdx.x - nth;
    rope_row<T, T, VE>(P, i % P.n_rows, i / P.n_rows);
    return;
  }
  constexpr double M = LARGEST_CODE<E4M3>;
  __shared__ int s_row[128], s_slot[128], s_pos[128], s_n, s_rows;
  __shared__ int s_held[128];                                     // tree: the slot is written
  __shared__ double s_max[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const bool values = A.v && (nth & 1);
  int id = A.v ? nth >> 1 : nth;
  const int kvh = id % A.KVH;
  id /= A.KVH;
  // the block: sequence and number
  const ChunkDev& C = P.chunk;
  const int shift = A.kv.block_shift, B = 1 << shift;
  const long long room = (long long)A.kv.pages_per_seq << A.kv.page_shift;
  auto rows_of = [&](int s, int* r0, int* n_all) {
    *r0 = min(max(0, C.row_start[s]), C.n_rows);
    *n_all = max(0, min(C.row_start[s + 1], C.n_rows) - *r0);
  };
  int s = -1, block = 0;
  if (C.tree_mask) {
    s = id / A.seq_blocks;
    const int base = C.tree_base[s];
    if (base < 0 || base > 1 << 30) return;
    block = (base >> shift) + id % A.seq_blocks;
  } else {
    int before = 0;
    for (int i = 0; i < C.n_seqs && s < 0; i += 64) {
      int count = 0, first = 0;
      if (i + lane < C.n_seqs) {
        int r0, n_all;
        rows_of(i + lane, &r0, &n_all);
        const int keys = min(max(0, C.key_len[i + lane]), 1 << 30);
        const long long lo = max(0, keys - n_all), hi = min(min((long long)keys - n_all + min(n_all, C.max_rows), room), (long long)C.max_keys);
        first = (int)(lo >> shift);
        if (lo < hi) count = (int)((hi - 1) >> shift) - first + 1;
      }
      int sum = count;
      for (int o = 1; o < 64; o <<= 1) { const int x = __shfl_up(sum, o, 64); if (lane >= o) sum += x; }
      const uint64_t behind = __ballot(i + lane < C.n_seqs && before + sum > id);
      if (behind) {
        const int l = __builtin_ctzll(behind);
        s = i + l;
        block = __shfl(first, l, 64) + id - before - (__shfl(sum, l, 64) - __shfl(count, l, 64));
      }
      before += __shfl(sum, 63, 64);
    }
    if (s < 0) return;
  }
  const long long t0 = (long long)block << shift;                 // its first token
  if (t0 < 0 || t0 >= room) return;
  const int page = token_page(A.kv, s, (int)t0);
  if (page < 0) return;
  uint8_t* codes = (values ? A.kv.v : A.kv.k) + page * A.kv.page_stride + kvh * A.kv.head_stride + (t0 & ((1ll << A.kv.page_shift) - 1)) * A.kv.token_stride;
  float* scale_at = (values ? A.kv.v_scale : A.kv.k_scale) + page * A.kv.scale_page + kvh * A.kv.scale_head + ((t0 & ((1ll << A.kv.page_shift) - 1)) >> shift);
  const float old_scale = *scale_at;
  // the rows that go there
  int r0, n_all;
  rows_of(s, &r0, &n_all);
  const int keys = min(max(0, C.key_len[s]), 1 << 30), n_rows = min(n_all, C.max_rows);
  const long long end = min((long long)min(C.max_keys, keys), room);   // tokens from here on are not stored (a tree's nodes may lie behind the sequence's last token)
  const int held = (int)max(0ll, min((long long)B, min((long long)keys, room) - t0));   // slots of tokens of the sequence
  if (tid < 128) s_held[tid] = 0;
  if (tid == 0) s_n = 0;
  __syncthreads();
  if (C.tree_mask) {
    const int base = C.tree_base[s];
    for (int i = tid; i < n_rows; i += 256) {
      const unsigned long long m = C.tree_mask[r0 + i];
      const long long t = m ? (long long)base + 63 - __builtin_clzll(m) : -1;
      if (t >= t0 && t < t0 + B && t < end && !atomicExch(&s_held[t - t0], 1)) {
        const int j = atomicAdd(&s_n, 1);
        s_row[j] = r0 + i; s_slot[j] = (int)(t - t0);
        s_pos[j] = P.positions ? P.positions[r0 + i] : base + __popcll(m) - 1;
      }
    }
  } else {
    const long long lo = max(t0, (long long)keys - n_all), hi = min(min(t0 + B, (long long)keys - n_all + n_rows), end);
    if (tid < B && t0 + tid >= lo && t0 + tid < hi) {
      const int j = tid - (int)(lo - t0), r = r0 + (int)(t0 + tid - (keys - n_all));
      s_held[tid] = 1;
      s_row[j] = r; s_slot[j] = tid;
      s_pos[j] = P.positions ? P.positions[r] : (int)(t0 + tid);
    }
    if (tid == 0) s_n = (int)max(0ll, hi - lo);
  }
  __syncthreads();
  const int n = s_n;
  if (n == 0) return;
  const bool others = __syncthreads_or(tid < held && !s_held[tid]);

  const int half = P.rot_dim >> 1, rot_units = half / VE, units = rot_units + (P.head_dim - P.rot_dim + 2 * VE - 1) / (2 * VE), all = n * units;
  const T* src = values ? (const T*)A.v + kvh * A.v_head : (const T*)A.k + kvh * A.k_head;
  const long long src_row = values ? A.v_row : A.k_row;
  // Unit i: two runs of VE elements of a token.
  struct Place { int e0, e1; bool two; };
  auto place = [&](int u) -> Place {
    Place p;
    if (u >= rot_units) { p.e0 = P.rot_dim + (u - rot_units) * 2 * VE; p.e1 = p.e0 + VE; }
    else if (P.interleaved) { p.e0 = u * 2 * VE; p.e1 = p.e0 + VE; }
    else { p.e0 = u * VE; p.e1 = half + p.e0; }
    p.two = p.e1 < P.head_dim;
    return p;
  };
  auto unit = [&](int i, double* a, double* b) {
    const int t = i / units, u = i % units;
    const Place p = place(u);
    const T* x = src + s_row[t] * src_row;
    float fa[VE], fb[VE];
    load_run<VE>(x + p.e0, fa);
#pragma unroll
    for (int j = 0; j < VE; ++j) fb[j] = 0.f;
    if (p.two) load_run<VE>(x + p.e1, fb);
#pragma unroll
    for (int j = 0; j < VE; ++j) { a[j] = fa[j]; b[j] = fb[j]; }
    if (values || u >= rot_units) return;
    const int pos = s_pos[t];
    auto turned = [](double& x, double& y, double2 c) { const double x0 = x; x = x0 * c.x - y * c.y; y = y * c.x + x0 * c.y; };
#pragma unroll
    for (int j = 0; j < VE; ++j) {
      double2 c = cos_sin_turn64(P.turn[u * VE + j], pos);
      c.x *= P.mscale; c.y *= P.mscale;
      if (P.interleaved && VE > 1) {
        double* x = 2 * j < VE ? a + 2 * j : b + 2 * j - VE;
        turned(x[0], x[1], c);
      } else turned(a[j], b[j], c);
      __builtin_amdgcn_sched_barrier(0);                          // (an angle at a time: all of them at once take the registers of a further wave of five)
    }
  };
  double a[VE], b[VE], top = 0.0;
  auto largest = [&](const double* x) {
#pragma unroll
    for (int j = 0; j < VE; ++j) { const double m = fabs(x[j]); top = ((m > top) & (m < INFINITY)) ? m : top; }
  };
#pragma unroll 1
  for (int i = tid; i < all; i += 256) {
    unit(i, a, b);
    largest(a); largest(b);
  }
  for (int o = 32; o; o >>= 1) { const double x = __shfl_xor(top, o, 64); top = x > top ? x : top; }
  if (lane == 0) s_max[wave] = top;
  __syncthreads();
  top = s_max[0];
  for (int i = 1; i < 4; ++i) top = s_max[i] > top ? s_max[i] : top;
  // the scale
  const bool kept = others && old_scale > 0.f && old_scale < INFINITY;
  int e = -100, grown = 0;
  double scale;
  if (!kept) {
    if (top > 0.0) e = min(max(least_exponent<E4M3>(top), -100), 100);
    scale = ldexp(1.0, e);
  } else {
    int ea, es, el;
    const double fs = frexp((double)old_scale, &es), fl = frexp(M * (double)old_scale, &el);
    if (top > 0.0) { const double fa = frexp(top, &ea); grown = max(0, ea - el + (fa > fl)); }
    grown = min(grown, max(0, 100 - (es - (fs == 0.5))));         // (the scale stays within 2^100)
    scale = ldexp((double)old_scale, grown);
  }
  if (tid == 0 && (!kept || grown > 0)) *scale_at = (float)scale;
  const double inv = 1.0 / scale, bound = 2.0 * M * scale;
  auto code = [&](double x) -> float {
    x = x > bound ? bound : x;
    x = x < -bound ? -bound : x;
    double y = x * inv;
    y = fma(fma(-y, scale, x), inv, y);                           // (put right by what the quotient leaves, so that a tie is a tie)
    return odd_f32(y);
  };
  auto put = [&](uint8_t* p, const float* y) {
    if constexpr (VE == 1) {
      const float z[4] = {y[0], 0.f, 0.f, 0.f};
      *p = (uint8_t)encode4<E4M3>(z);
    } else if constexpr (VE == 4) *(uint32_t*)p = encode4<E4M3>(y);
    else *(u32x2*)p = u32x2{encode4<E4M3>(y), encode4<E4M3>(y + 4)};
  };
#pragma unroll 1
  for (int i = tid; i < all; i += 256) {
    if (all > 256) unit(i, a, b);
    const Place p = place(i % units);
    uint8_t* to = codes + s_slot[i / units] * A.kv.token_stride;
    float y[VE];
#pragma unroll
    for (int j = 0; j < VE; ++j) y[j] = code(a[j]);
    put(to + p.e0, y);
    if (!p.two) continue;
#pragma unroll
    for (int j = 0; j < VE; ++j) y[j] = code(b[j]);
    put(to + p.e1, y);
  }
  if (!others || (kept && grown == 0)) return;
  // the block's other tokens: their codes in the new scale, or 0 where the old one stood for nothing
  const double shrink = kept ? ldexp(1.0, -grown) : 0.0;
  const int runs = P.head_dim / VE;
#pragma unroll 1
  for (int i = tid; i < held * runs; i += 256) {
    const int slot = i / runs;
    if (s_held[slot]) continue;
    uint8_t* p = codes + slot * A.kv.token_stride + (i % runs) * VE;
    uint32_t u[2] = {0, 0};
    if constexpr (VE == 1) u[0] = *p;
    else if constexpr (VE == 4) u[0] = *(const uint32_t*)p;
    else { const u32x2 w = *(const u32x2*)p; u[0] = w.x; u[1] = w.y; }
    float x[8];
    decode4<E4M3>(u[0], x);
    decode4<E4M3>(u[1], x + 4);
    float y[VE];
#pragma unroll
    for (int j = 0; j < VE; ++j) y[j] = kept ? odd_f32(x[j] * shrink) : 0.f;
    put(p, y);
  }
}
