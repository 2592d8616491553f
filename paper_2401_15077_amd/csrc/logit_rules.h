// Penalties for repeated tokens, biases and masks on rows of logits.
#pragma once
#include "rows.h"
#include "rope.h"

struct RulesDev {
  int n_rows, vocab, n_masks, n_seqs, n_bias, slice;
  const void* in; void* out;
  long long in_stride, out_stride, mask_stride, token_stride;
  const int *row_start, *path_token, *allowed_row, *tokens, *n_tokens, *n_prompt, *bias_start, *bias_token;
  const unsigned long long* path_mask;
  const uint32_t* allowed;
  const float *repetition, *presence, *frequency, *bias_value;
};

// A work-group takes one row and one slice of the vocabulary.  It counts the row's text in LDS -- one word a token of the slice: bit 31 = stands in the text,
// below it how often behind the prompt -- by walking the token list once, and then streams its logits through.  Counting needs no hash table or sorting, and integer
// additions in any order give one result.  Of several bias entries for a token the last counts: the largest index wins, whatever the order.
// VE elements at a time where a row of `in` and of `out` start at the same place of a 16-byte piece; the first and last pieces may be partly outside the row.
template <typename T, int VE>
__global__ __launch_bounds__(512) void k_logit_rules(const RulesDev A) {
  extern __shared__ __attribute__((aligned(16))) uint32_t count[];   // [slice], then with biases [slice]: index of the entry + 1
  const int tid = threadIdx.x, nt = blockDim.x, r = blockIdx.y, V = A.vocab;
  int seq = r;
  if (A.row_start) {
    seq = wave_row_seq(A.row_start, A.n_seqs, r);
    if (seq < 0) return;
  }
  const T* in = (const T*)A.in + r * A.in_stride;
  T* out = (T*)A.out + r * A.out_stride;
  const int shift = VE > 1 ? (int)((uintptr_t)in / sizeof(T) % VE) : 0;   // elements of the first piece in front of the row
  const int t0 = (int)blockIdx.x * A.slice - shift;                // the slice: tokens t0 .. t0 + slice - 1, those that exist
  if (t0 >= V) return;
  uint32_t* bias_at = count + A.slice;
  for (int i = tid; i < A.slice * (A.bias_token ? 2 : 1); i += nt) count[i] = 0;
  __syncthreads();
  if (A.tokens) {
    const int n = (int)min((long long)A.n_tokens[seq], A.token_stride), prompt = A.n_prompt ? A.n_prompt[seq] : 0;
    const int* text = A.tokens + seq * A.token_stride;
    for (int i0 = 0; i0 < n; i0 += 8 * nt) {
      int t[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) t[u] = i0 + u * nt + tid < n ? text[i0 + u * nt + tid] : -1;
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if ((unsigned)t[u] < (unsigned)V && (unsigned)(t[u] - t0) < (unsigned)A.slice) {
          uint32_t* c = count + (t[u] - t0);
          if (i0 + u * nt + tid < prompt) atomicOr(c, 0x80000000u);
          else { atomicAdd(c, 1u); atomicOr(c, 0x80000000u); }
        }
    }
  }
  if (A.path_mask && tid < 64) {
    const unsigned long long m = A.path_mask[r];
    const int node = (A.row_start ? A.row_start[seq] : seq) + tid;
    if (m >> tid & 1 && node < (A.row_start ? A.row_start[seq + 1] : seq + 1) && node < A.n_rows) {
      const int t = A.path_token[node];
      if ((unsigned)t < (unsigned)V && (unsigned)(t - t0) < (unsigned)A.slice) { atomicAdd(count + (t - t0), 1u); atomicOr(count + (t - t0), 0x80000000u); }
    }
  }
  if (A.bias_token) {
    const int b0 = max(0, A.bias_start[seq]), b1 = min(A.n_bias, A.bias_start[seq + 1]);
    for (int i = b0 + tid; i < b1; i += nt) {
      const int t = A.bias_token[i];
      if ((unsigned)t < (unsigned)V && (unsigned)(t - t0) < (unsigned)A.slice) atomicMax(bias_at + (t - t0), (uint32_t)i + 1u);
    }
  }
  __syncthreads();
  float rep = A.repetition ? A.repetition[seq] : 1.f;
  if (!(rep > 0.f)) rep = 1.f;
  const float pres = A.presence ? A.presence[seq] : 0.f, freq = A.frequency ? A.frequency[seq] : 0.f;
  const uint32_t* mask = nullptr;
  if (A.allowed) {
    const int m = A.allowed_row ? A.allowed_row[r] : r;
    if ((unsigned)m < (unsigned)A.n_masks) mask = A.allowed + m * A.mask_stride;
  }
  auto one = [&](int t, float x) -> float {
    const uint32_t c = count[t - t0];
    if (c) {
      const uint32_t n = c & 0x7FFFFFFFu;
      x = x > 0.f ? x / rep : x * rep;
      if (n) x -= pres + freq * (float)n;
    }
    if (A.bias_token) {
      const uint32_t b = bias_at[t - t0];
      if (b) x += A.bias_value[b - 1];
    }
    if (mask && !(mask[t >> 5] >> (t & 31) & 1u)) x = -INFINITY;
    return x;
  };
  const int t1 = min(t0 + A.slice, V);
  for (int t = t0 + tid * VE; t < t1; t += nt * VE) {
    float x[VE];
    if (VE == 1 || (t >= 0 && t + VE <= t1)) {
      load_run<VE>(in + t, x);
#pragma unroll
      for (int j = 0; j < VE; ++j) x[j] = one(t + j, x[j]);
      store_run<VE>(out + t, x);
    } else {
      for (int j = 0; j < VE; ++j)
        if (t + j >= 0 && t + j < t1) {
          load_run<1>(in + t + j, x);
          x[0] = one(t + j, x[0]);
          store_run<1>(out + t + j, x);
        }
    }
  }
}
