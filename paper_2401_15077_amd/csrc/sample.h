// The choice of a token from a row of logits: temperature, top-k, top-p, min-p, from a given random number.
#pragma once
#include "rows.h"
#include "rope.h"

typedef unsigned long long u64;

struct SampleDev {
  int n_rows, vocab, bits;                 // weights are multiples of 2^-bits of the largest one
  const void* logits;
  long long stride;
  const float *uniform, *temperature, *top_p, *min_p;
  const int* top_k;
  int* token; float* logprob;
};

// The order of the tokens, by value, descending, equal ones by index, as the order of 64-bit numbers.
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t b = x == 0.f ? 0u : __builtin_bit_cast(uint32_t, x);     // (-0 is 0)
  return ~(b ^ ((uint32_t)((int)b >> 31) | 0x80000000u));
}
__device__ __forceinline__ float value_of(uint32_t order) {
  const uint32_t a = ~order;
  return __builtin_bit_cast(float, a & 0x80000000u ? a ^ 0x80000000u : ~a);
}
__device__ __forceinline__ u64 place_of(float x, int i) { return (u64)order_of(x) << 32 | (uint32_t)i; }

// A work-group takes a row.  Nothing is sorted: what is looked for is the token in whose share of the running mass (or count) a given number falls.  A histogram of the masses over buckets of
// equal width in log(weight), which keep the order, says the bucket; its tokens are listed, by histograms over ever smaller ranges of (value, index) until few are left, and those are ranked
// pair by pair.  Masses are whole numbers (of 2^-bits of the largest weight) in 64 bits, so sums come out the same in any order.
constexpr int SAMPLE_BUCKETS = 4096, SAMPLE_LIST = 1024, SAMPLE_PAIRS = 128, SAMPLE_TOP = 256;
template <typename T>
__global__ __launch_bounds__(1024) void k_sample(const SampleDev A) {
  __shared__ u64 hist[SAMPLE_BUCKETS], sub[SAMPLE_BUCKETS], list[2][SAMPLE_LIST], mass[SAMPLE_TOP], s_wave[16], s_low, s_high, s_found[3];
  __shared__ int s_n, s_bucket;
  constexpr int VE = 16 / sizeof(T);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, V = A.vocab, r = blockIdx.x;
  const T* row = (const T*)A.logits + r * A.stride;
  auto each = [&](auto f) {                                       // f(logit, token) of the row, NaN as -inf
    auto clean = [](float x) { return x == x ? x : -INFINITY; };
    const int head = min(V, (int)((16 - (uintptr_t)row % 16) % 16 / sizeof(T))), body = (V - head) / VE;
    float x[VE];
    if (tid < head) { load_run<1>(row + tid, x); f(clean(x[0]), tid); }
    for (int i = tid; i < body; i += 1024) {
      load_run<VE>(row + head + i * VE, x);
#pragma unroll
      for (int j = 0; j < VE; ++j) f(clean(x[j]), head + i * VE + j);
    }
    const int t = head + body * VE + tid;
    if (t < V) { load_run<1>(row + t, x); f(clean(x[0]), t); }
  };
  auto sum_all = [&](u64 x) -> u64 {                              // of the work-group
    for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o, 64);
    __syncthreads();
    if (lane == 0) s_wave[wave] = x;
    __syncthreads();
    x = 0;
    for (int i = 0; i < 16; ++i) x += s_wave[i];
    return x;
  };
  float top = -INFINITY;
  each([&](float x, int) { top = fmaxf(top, x); });
  for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
  float* s_top = (float*)s_wave;
  if (lane == 0) s_top[wave] = top;
  __syncthreads();
  for (int i = 0; i < 16; ++i) top = fmaxf(top, s_top[i]);
  const float temperature = A.temperature ? A.temperature[r] : 1.f;
  auto answer = [&](int token, float logprob) {
    if (tid > 0) return;
    A.token[r] = token;
    if (A.logprob) A.logprob[r] = logprob;
  };
  if (top == -INFINITY) { answer(-1, -INFINITY); return; }
  if (!(temperature > 0.f)) {                                     // the first of the largest
    u64 best = ~0ull;
    each([&](float x, int t) { if (x == top) best = min(best, (u64)t); });
    if (tid == 0) s_low = ~0ull;
    __syncthreads();
    atomicMin(&s_low, best);
    __syncthreads();
    answer((int)s_low, 0.f);
    return;
  }
  const double rate = 1.0 / (double)temperature, one = ldexp(1.0, A.bits);
  auto weight = [&](float x) -> u64 {
    if (x == -INFINITY) return 0;
    if (top == INFINITY) return x == top ? 1ull << A.bits : 0ull;
    return (u64)(exp(((double)x - (double)top) * rate) * one + 0.5);
  };
  const float slope = fminf((float)(rate * (1.4426950408889634 * SAMPLE_BUCKETS / 32)), 3.4e38f);   // the last bucket begins 2^-32 below the largest weight
  auto bucket = [&](float x) -> int { return x == -INFINITY ? SAMPLE_BUCKETS - 1 : x == top ? 0 : (int)fminf((top - x) * slope, SAMPLE_BUCKETS - 1.f); };
  auto clear = [&](u64* h) {
    for (int i = tid; i < SAMPLE_BUCKETS; i += 1024) h[i] = 0;
    __syncthreads();
  };
  // The bucket that the number falls into and what is in front of it.
  auto find = [&](const u64* h, u64 target, u64* before) -> int {
    constexpr int EACH = SAMPLE_BUCKETS / 1024;
    u64 x[EACH], sum = 0;
    __syncthreads();
    for (int i = 0; i < EACH; ++i) { x[i] = h[tid * EACH + i]; sum += x[i]; }
    u64 upto = sum;
    for (int o = 1; o < 64; o <<= 1) { const u64 y = __shfl_up(upto, o, 64); if (lane >= o) upto += y; }
    if (lane == 63) s_wave[wave] = upto;
    __syncthreads();
    for (int i = 0; i < wave; ++i) upto += s_wave[i];
    u64 at = upto - sum;
    if (at <= target && target < upto) {
      int i = 0;
      while (target >= at + x[i]) at += x[i++];
      s_bucket = tid * EACH + i;
      s_found[0] = at;
    }
    __syncthreads();
    *before = s_found[0];
    return s_bucket;
  };
  struct Found { u64 place, before, share; };
  // The token in whose share (its weight, or 1) of the tokens up to `limit` the number falls; h: histogram of those shares.
  auto select = [&](const u64* h, u64 target, bool by_mass, u64 limit) -> Found {
    auto share = [&](float x) -> u64 { return by_mass ? weight(x) : 1ull; };
    u64 before;
    const int b = find(h, target, &before);
    u64 in_front = before, low = 0, high = 0;
    bool ranged = false;
    int n;
    for (;;) {                                                    // list the bucket's tokens, or those of the range
      if (tid == 0) { s_n = 0; s_low = ~0ull; s_high = 0; }
      __syncthreads();
      u64 lo = ~0ull, hi = 0;
      each([&](float x, int t) {
        const u64 p = place_of(x, t);
        if (p > limit || (ranged ? p < low || p > high : bucket(x) != b)) return;
        const int i = atomicAdd(&s_n, 1);
        if (i < SAMPLE_LIST) list[0][i] = p;
        lo = min(lo, p); hi = max(hi, p);
      });
      if (hi) { atomicMin(&s_low, lo); atomicMax(&s_high, hi); }
      __syncthreads();
      n = s_n; low = s_low; high = s_high;
      if (n <= SAMPLE_LIST) break;
      int shift = 0;
      while ((high - low) >> shift >= SAMPLE_BUCKETS) ++shift;
      clear(sub);
      each([&](float x, int t) {
        const u64 p = place_of(x, t);
        if (p >= low && p <= high && p <= limit) atomicAdd(&sub[(p - low) >> shift], share(x));
      });
      const int c = find(sub, target - in_front, &before);
      in_front += before;
      low += (u64)c << shift;
      high = min(high, low + ((1ull << shift) - 1));
      ranged = true;
    }
    int from = 0;
    while (n > SAMPLE_PAIRS) {                                    // the same on the list
      int shift = 0;
      while ((high - low) >> shift >= SAMPLE_BUCKETS) ++shift;
      clear(sub);
      const u64 p = tid < n ? list[from][tid] : 0;
      if (tid < n) atomicAdd(&sub[(p - low) >> shift], share(value_of((uint32_t)(p >> 32))));
      const int c = find(sub, target - in_front, &before);
      in_front += before;
      if (tid == 0) s_n = 0;
      __syncthreads();
      low += (u64)c << shift;
      high = min(high, low + ((1ull << shift) - 1));
      if (tid < n && p >= low && p <= high) list[from ^ 1][atomicAdd(&s_n, 1)] = p;
      __syncthreads();
      n = s_n;
      from ^= 1;
      __syncthreads();
    }
    // what lies in front of each of the few, eight threads each
    if (tid < n) mass[tid] = share(value_of((uint32_t)(list[from][tid] >> 32)));
    __syncthreads();
    const int mine = tid >> 3;
    const u64 p = mine < n ? list[from][mine] : 0;
    u64 at = 0;
    for (int j = tid & 7; j < n; j += 8) at += list[from][j] < p ? mass[j] : 0;
    for (int o = 4; o; o >>= 1) at += __shfl_xor(at, o, 64);
    at += in_front;
    if (mine < n && (tid & 7) == 0 && at <= target && target < at + mass[mine]) { s_found[0] = p; s_found[1] = at; s_found[2] = mass[mine]; }
    __syncthreads();
    const Found f{s_found[0], s_found[1], s_found[2]};
    __syncthreads();
    return f;
  };
  auto histogram = [&](bool by_mass, u64 limit) {
    clear(hist);
    each([&](float x, int t) {
      if (limit != ~0ull && place_of(x, t) > limit) return;
      const u64 w = by_mass ? weight(x) : 1ull;
      if (w) atomicAdd(&hist[bucket(x)], w);
    });
    __syncthreads();
  };
  const int k = A.top_k ? A.top_k[r] : 0;
  const float p = A.top_p ? A.top_p[r] : 1.f, least = A.min_p ? A.min_p[r] : 0.f, uniform = A.uniform[r];
  const double u = uniform > 0.f ? fmin((double)uniform, 1.0) : 0.0;
  const double log_least = least > 0.f ? log((double)least) : 0.0;
  auto heavy = [&](float x) { return x == top || (top != INFINITY && ((double)x - (double)top) * rate >= log_least); };   // min-p keeps it
  u64 limit = ~0ull;
  if (k > 0 && k < V) {
    histogram(false, ~0ull);
    limit = select(hist, (u64)k - 1, false, ~0ull).place;
  }
  histogram(true, limit);
  u64 total = 0;
  for (int i = tid; i < SAMPLE_BUCKETS; i += 1024) total += hist[i];
  total = sum_all(total);
  u64 kept = total;
  if (p < 1.f) {
    const u64 need = (u64)ceil(fmax((double)p, 0.0) * (double)total);
    const Found f = select(hist, need > 0 ? need - 1 : 0, true, limit);
    kept = f.before + f.share;
  }
  if (least > 0.f) {
    u64 m = 0;
    each([&](float x, int t) { if (heavy(x) && (limit == ~0ull || place_of(x, t) <= limit)) m += weight(x); });
    m = sum_all(m);
    kept = min(kept, max(m, 1ull << A.bits));
  }
  const u64 target = min((u64)(u * (double)kept), kept - 1);
  const Found f = select(hist, target, true, limit);
  const float x = value_of((uint32_t)(f.place >> 32));
  const double t = top == INFINITY ? 0.0 : ((double)x - (double)top) * rate;
  answer((int)(uint32_t)f.place, (float)(t - log((double)kept / one)));
}
