// Penalties for repeated tokens, biases and masks on rows of logits.
#pragma once
#include "rows.h"
#include "rope.h"

struct RulesDev {
  int n_rows, vocab, n_masks, n_seqs, n_bias, max_tokens;
  const void* in; void* out;
  long long in_stride, out_stride, mask_stride, token_stride;
  const int *row_start, *path_token, *allowed_row, *tokens, *n_tokens, *n_prompt, *bias_start, *bias_token;
  const unsigned long long* path_mask;
  const uint32_t* allowed;
  const float *repetition, *presence, *frequency, *bias_value;
};

// A work-group takes one row and one slice of the vocabulary, PIECES runs of VE logits a thread.  It asks for the logits first; while they are on their way it counts the row's text in LDS,
// one word a token of the slice: SEEN = stands in the prompt, BIASED = has an entry, below them how often it stands behind the prompt.  That is one walk over the token list, with no hash
// table or sorting, and integer additions in any order give one result.  Then the logits pass through: the words of a run are one or two reads of LDS, and most are 0.  A logit with a
// bias leaves its penalised value in its word instead, in fp32, and is finished from there by the thread that holds the entry.
// Of several entries for a token the last counts.  That a token has several shows when BIASED is set twice; only then the list is taken from its end, one entry a thread at a time, and of those
// at hand the largest index wins.
// Bound by HBM and, where texts are long, by the vector unit: 160 rows of 100003 bf16 logits with texts of 4500 tokens, masks and 150 entries 25.5 us, of which logits and masks alone take 15 to
// 16, the text's walk and the penalties of whole runs 8, entries 2; 104 rows of 32000 fp32 logits along trees 9.9 (kernel; without runs 40 and 13.4).
// VE elements at a time where a row of `in` and of `out` start at the same place of a 16-byte piece; the first and last pieces may be partly outside the row.
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(4)));
constexpr uint32_t RULES_SEEN = 0x80000000u, RULES_BIASED = 0x40000000u, RULES_TAKEN = 0xFFFFFFFFu;
template <typename T, int VE, int PIECES>
__global__ __launch_bounds__(512) void k_logit_rules(const RulesDev A) {
  extern __shared__ __attribute__((aligned(16))) uint32_t count[];   // [slice], then one word: a token has several entries
  const int tid = threadIdx.x, nt = blockDim.x, r = blockIdx.y, V = A.vocab, slice = nt * VE * PIECES;
  int seq = r;
  if (A.row_start) {
    seq = wave_row_seq(A.row_start, A.n_seqs, r);
    if (seq < 0) return;
  }
  const T* in = (const T*)A.in + r * A.in_stride;
  T* out = (T*)A.out + r * A.out_stride;
  const int shift = VE > 1 ? (int)((uintptr_t)in / sizeof(T) % VE) : 0;   // elements of the first piece in front of the row
  const int t0 = (int)blockIdx.x * slice - shift, t1 = min(t0 + slice, V);   // the slice: tokens t0 .. t1 - 1, those that exist
  if (t0 >= V) return;
  uint4 raw[PIECES];
#pragma unroll
  for (int p = 0; p < PIECES; ++p) {
    const int t = t0 + (p * nt + tid) * VE;
    if (VE > 1 && t >= 0 && t + VE <= t1) raw[p] = *(const uint4*)(in + t);
  }
  const int first = A.row_start ? A.row_start[seq] : seq, last = A.row_start ? A.row_start[seq + 1] : seq + 1;
  const int n = A.tokens ? max(0, min(A.n_tokens[seq], A.max_tokens)) : 0, prompt = A.n_prompt ? A.n_prompt[seq] : 0;
  float rep = A.repetition ? A.repetition[seq] : 1.f;
  rep = rep > 0.f ? fmaxf(rep, 1.17549435e-38f) : 1.f;             // (a subnormal one's reciprocal may be infinite)
  const float pres = A.presence ? A.presence[seq] : 0.f, freq = A.frequency ? A.frequency[seq] : 0.f;
  const uint32_t* mask = nullptr;
  if (A.allowed) {
    const int m = A.allowed_row ? A.allowed_row[r] : r;
    if ((unsigned)m < (unsigned)A.n_masks) mask = A.allowed + m * A.mask_stride;
  }
  const int b0 = A.bias_token ? max(0, A.bias_start[seq]) : 0, b1 = A.bias_token ? min(A.n_bias, A.bias_start[seq + 1]) : 0;
  const int* text = A.tokens + seq * A.token_stride;
  u32x4_any t[4];                                                  // 16 tokens of the text: four fours, the first at i0 + 4 tid
  auto ask = [&](int i0) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int i = i0 + (u * nt + tid) * 4;
      t[u] = u32x4_any{~0u, ~0u, ~0u, ~0u};
      if (i + 4 <= n) t[u] = *(const u32x4_any*)(text + i);
    }
  };
  ask(0);
  int rest = -1;                                                   // and the up to three behind the last four, a thread each
  if (tid < (n & 3)) rest = text[(n & ~3) + tid];
  int entry_token = -1;
  float entry_value = 0.f;
  if (b0 + tid < b1) { entry_token = A.bias_token[b0 + tid]; entry_value = A.bias_value[b0 + tid]; }
  uint32_t* several = count + slice;
  for (int i = tid * 4; i < slice; i += nt * 4) *(u32x4*)(count + i) = u32x4{0, 0, 0, 0};
  if (tid == 0) *several = 0;
  __syncthreads();
  const int low = max(t0, 0);
  auto here = [&](int t) { return (unsigned)t - (unsigned)low < (unsigned)(t1 - low); };
  auto tally = [&](int i, int k) {
    if (!here(k)) return;
    if (i < prompt) atomicOr(count + (k - t0), RULES_SEEN);
    else atomicAdd(count + (k - t0), 1u);
  };
  for (int i0 = 0; i0 + 4 <= n; i0 += 16 * nt) {
    if (i0) ask(i0);
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int j = 0; j < 4; ++j) tally(i0 + (u * nt + tid) * 4 + j, (int)t[u][j]);
  }
  tally((n & ~3) + tid, rest);
  if (A.path_mask && tid < 64) {
    const long long node = (long long)first + tid;
    if (A.path_mask[r] >> tid & 1 && node < last && node < A.n_rows && node >= 0) {
      const int t = A.path_token[node];
      if (here(t)) atomicAdd(count + (t - t0), 1u);
    }
  }
  for (int i = b0 + tid; i < b1; i += nt) {
    const int t = i < b0 + nt ? entry_token : A.bias_token[i];
    if (here(t) && atomicOr(count + (t - t0), RULES_BIASED) & RULES_BIASED) *several = 1;
  }
  __syncthreads();
  const float inv = 1.f / rep;
  auto penalised = [&](uint32_t c, float x) -> float {             // without branches: x / rep by its reciprocal, put right by what the quotient leaves
    const float f = (float)(c & ~(RULES_SEEN | RULES_BIASED)), q = x * inv, e = fmaf(-q, rep, x), div = fabsf(e) < INFINITY ? fmaf(e, inv, q) : q;
    const float y = x > 0.f ? div : x * rep;
    x = c & ~RULES_BIASED ? y : x;
    return f > 0.f ? x - (pres + freq * f) : x;
  };
  auto allows = [&](int t) { return !mask || mask[t >> 5] >> (t & 31) & 1u; };
  auto leave = [&](int t, float x) { count[t - t0] = x == x ? __builtin_bit_cast(uint32_t, x) : 0x7FC00000u; };   // (no value is RULES_TAKEN)
  auto one = [&](int t) {
    const uint32_t c = count[t - t0];
    float x;
    load_run<1>(in + t, &x);
    if (c) x = penalised(c, x);
    if (c & RULES_BIASED) { leave(t, x); return; }
    if (!allows(t)) x = -INFINITY;
    store_run<1>(out + t, &x);
  };
  if constexpr (VE == 1) {
#pragma unroll
    for (int p = 0; p < PIECES; ++p)
      if (t0 + p * nt + tid < t1) one(t0 + p * nt + tid);
  } else {
    const int words = (V + 31) >> 5;
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      const int t = t0 + (p * nt + tid) * VE;
      if (t < 0 || t + VE > t1) {
        for (int j = max(t, 0); j < min(t + VE, t1); ++j) one(j);
        continue;
      }
      uint32_t c[VE], any = 0, ok = (1u << VE) - 1u;
#pragma unroll
      for (int j = 0; j < VE; j += 4) {
        const u32x4 w = *(const u32x4*)(count + (t - t0) + j);
        c[j] = w.x; c[j + 1] = w.y; c[j + 2] = w.z; c[j + 3] = w.w;
        any |= w.x | w.y | w.z | w.w;
      }
      if (mask) {
        const uint64_t w = (uint64_t)mask[min((t >> 5) + 1, words - 1)] << 32 | mask[t >> 5];
        ok &= (uint32_t)(w >> (t & 31));
      }
      float x[VE];
      load_run<VE>((const T*)(raw + p), x);
      if (any) {
#pragma unroll
        for (int j = 0; j < VE; ++j) x[j] = penalised(c[j], x[j]);
        if (any & RULES_BIASED) {
#pragma unroll
          for (int j = 0; j < VE; ++j)
            if (c[j] & RULES_BIASED) leave(t + j, x[j]);
        }
      }
#pragma unroll
      for (int j = 0; j < VE; ++j) x[j] = ok >> j & 1u ? x[j] : -INFINITY;
      store_run<VE>(out + t, x);
    }
  }
  if (b0 >= b1) return;
  __syncthreads();
  auto finish = [&](int t, uint32_t word, float value) {
    float x = __builtin_bit_cast(float, word) + value;
    if (!allows(t)) x = -INFINITY;
    store_run<1>(out + t, &x);
  };
  if (!*several) {
    for (int i = b0 + tid; i < b1; i += nt) {
      const int t = i < b0 + nt ? entry_token : A.bias_token[i];
      if (here(t)) finish(t, count[t - t0], i < b0 + nt ? entry_value : A.bias_value[i]);
    }
    return;
  }
  for (int c0 = b1 - nt; c0 > b0 - nt; c0 -= nt) {                 // entries c0 .. c0 + nt - 1, from the end
    const int i = c0 + tid, t = i >= b0 ? A.bias_token[i] : -1;
    const bool mine = here(t) && count[t - t0] != RULES_TAKEN;
    uint32_t* c = count + (mine ? t - t0 : 0);
    const uint32_t word = *c;
    if (!__syncthreads_or(mine)) continue;
    if (mine) *c = 0;
    __syncthreads();
    if (mine) atomicMax(c, (uint32_t)i + 1u);
    __syncthreads();
    const bool wins = mine && *c == (uint32_t)i + 1u;
    __syncthreads();
    if (wins) { finish(t, word, A.bias_value[i]); *c = RULES_TAKEN; }
    __syncthreads();
  }
}
