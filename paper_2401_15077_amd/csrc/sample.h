// The choice of a token from a row of logits: temperature, top-k, top-p, min-p, from a given random number.
#pragma once
#include "rows.h"
#include "rope.h"
#include "wave.h"
#include <type_traits>

struct SampleDev {
  int vocab, bits, unit;                   // masses are multiples of 2^-bits of the largest weight, parts of 2^-unit
  const void* logits;
  long long stride;
  const float *uniform, *temperature, *top_p, *min_p;
  const int* top_k;
  int* token; float* logprob;
  double part[4];                          // 2^-x/64 in units: the terms of its series, the first one with 2^52
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

// Nothing is sorted: what is looked for is the token in whose share of the running mass (or count) a given number falls.  A histogram over buckets of equal width in log(weight), which keep the
// order, says the bucket; its tokens are listed, through histograms over ever smaller ranges of (value, index) where they are many, and the last few are ranked pair by pair.  Where top-k or
// min-p leaves few tokens, these are listed and ranked at once.
//
// A weight is 2^(-y / 64), y = (largest - logit) * 64 log2(e) / temperature, bucket b the nearest whole number to y, and what is added up is 2^((b - y) / 64) in whole multiples of 2^-unit, so
// that no order of additions changes a sum: eight operations in 64 bits a logit, since y has to be known to far more than 24, and an atomic addition in LDS.  The 1 and three terms of the exponential
// series leave out 4 * 10^-11 of a weight.  A bucket's sum times 2^(-b / 64) is its mass, in multiples of 2^-bits of the largest weight.  The last bucket holds what lies 2^-64 below, which is as
// good as nothing.
//
// A row is one work-group of 16 waves, which holds the CU's LDS and registers, in one launch.  What bounds it: the work-group's chain of passes and barriers, not memory (160 rows of 100003, bf16,
// are 32 MB and take 47 us; of one row's time 4 are the largest, 17 the histogram, 2.5 finding buckets and their edges, 9 the pass that lists, 8 the two rankings).  With all filters 104 rows of
// 32000 in fp32 take 25, one row of 32000 13, three rows of 128256 35.  Rows divided over several work-groups need a launch for every pass: three rows of 128256 32, but one of 16384 26 in place of
// 16 and one of 32000 with top-p 41 in place of 27.  What is the same for a row (parameters, the edges of buckets) is worked out by one wave: sixteen that do so at once take each other's time
// (1.1 us an edge).
constexpr int SAMPLE_BUCKETS = 4096, SAMPLE_LIST = 1024, SAMPLE_PAIRS = 128, SAMPLE_FEW = 256;

// What a row asks for; step: buckets a unit of logits, farthest: what the last bucket lies below the largest, reach: what the least weight does.
struct SampleRow {
  int greedy, top_k, top_p, min_p, k;
  double rate, p, log_least, u, step, farthest, reach;
};
// The same in every lane: kept in scalar registers.
__device__ __forceinline__ double uniform(double x) {
  const u64 b = __builtin_bit_cast(u64, x);
  return __builtin_bit_cast(double, (u64)(uint32_t)__builtin_amdgcn_readfirstlane((int)(b >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)b));
}
__device__ __forceinline__ u64 uniform(u64 x) { return __builtin_bit_cast(u64, uniform(__builtin_bit_cast(double, x))); }
__device__ __forceinline__ float uniform(float x) { return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, x))); }
__device__ inline SampleRow sample_row(int vocab, float temperature, int k, float p, float least, float u) {
  SampleRow q;
  q.k = k;
  q.greedy = !(temperature > 0.f);
  q.top_k = k > 0 && k < vocab; q.top_p = p < 1.f; q.min_p = least > 0.f;
  q.rate = 1.0 / (double)temperature;
  q.p = fmax((double)p, 0.0);
  q.log_least = q.min_p ? log((double)least) : 0.0;
  q.u = u > 0.f ? fmin((double)u, 1.0) : 0.0;
  q.step = fmax(q.rate * (64 * 1.4426950408889634), 1e-290);
  q.farthest = (SAMPLE_BUCKETS - 1) / q.step;
  q.reach = q.log_least / q.rate;
  return q;
}

// f(logits, first token, how many) of tokens first .. last - 1 of a row for the work-group's threads, a run at a time, in no order.  A run past the end is NaN.
template <typename T, int NT, typename F>
__device__ __forceinline__ void each_run(const T* row, int first, int last, F f) {
  constexpr int VE = 16 / sizeof(T), GROUP = 16 / VE;
  const int tid = threadIdx.x, n = last - first, head = min(n, (int)((16 - (uintptr_t)(row + first) % 16) % 16 / sizeof(T))), body = (n - head) / VE;
  const uint4* p = (const uint4*)(row + first + head);
  if (body > 0) {
    uint4 raw[GROUP];
    auto ask = [&](int i0) {
#pragma unroll
      for (int u = 0; u < GROUP; ++u) raw[u] = p[min(i0 + u * NT, body - 1)];
    };
    ask(tid);
#pragma unroll 1
    for (int i0 = tid; i0 - tid < body; i0 += NT * GROUP) {
      uint4 now[GROUP];
#pragma unroll
      for (int u = 0; u < GROUP; ++u) now[u] = raw[u];
      if (i0 - tid + NT * GROUP > body) {
#pragma unroll
        for (int u = 0; u < GROUP; ++u)
          if (i0 + u * NT >= body) now[u] = uint4{~0u, ~0u, ~0u, ~0u};
      }
      ask(i0 + NT * GROUP);
#pragma unroll
      for (int u = 0; u < GROUP; ++u) {
        float x[VE];
        load_run<VE>((const T*)(now + u), x);
        f(x, first + head + (i0 + u * NT) * VE, std::integral_constant<int, VE>());
        __builtin_amdgcn_sched_barrier(0);                        // (a run after the other: all at once would take more registers than there are)
      }
    }
  }
  // what is in front of the first run and behind the last: a token each for some threads
  const int t = tid < head ? first + tid : first + head + body * VE + (tid - 32);
  if (tid < head || (tid >= 32 && t < last)) {
    float x[1];
    load_run<1>(row + t, x);
    f(x, t, std::integral_constant<int, 1>());
  }
}

template <typename T>
__global__ __launch_bounds__(1024) void k_sample(const SampleDev A) {
  __shared__ u64 hist[SAMPLE_BUCKETS + 64], sub[SAMPLE_BUCKETS], list[2][SAMPLE_LIST], mass[SAMPLE_FEW], s_wave[16], s_low, s_high, s_found[3];
  __shared__ double root[64];                                     // powers of 2^(-1 / 64)
  __shared__ int noted[SAMPLE_LIST], s_n, s_bucket;
  __shared__ uint32_t s_edge[4];
  __shared__ SampleRow s_row;
  int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), V = A.vocab, r = blockIdx.x;
  const T* row = (const T*)A.logits + r * A.stride;
  const float temperature = A.temperature ? A.temperature[r] : 1.f, p_of_row = A.top_p ? A.top_p[r] : 1.f, min_of_row = A.min_p ? A.min_p[r] : 0.f, u_of_row = A.uniform[r];
  const int k_of_row = A.top_k ? A.top_k[r] : 0;
  auto runs = [&](auto f) { each_run<T, 1024>(row, 0, V, f); };
  // f(first token, bits of those from `least` to `most`, least <= most) of the runs that have such; few are expected.
  auto between = [&](float least, float most, auto f) {
    runs([&](const float* x, int t, auto n) {
      uint32_t hits = 0;
#pragma unroll
      for (int j = 0; j < decltype(n)::value; ++j) hits |= __builtin_amdgcn_fmed3f(x[j], least, most) == x[j] ? 1u << j : 0u;
      if (hits) f(t, hits);
    });
  };
  auto logit = [&](int t) { float x; load_run<1>(row + t, &x); return x; };
  auto each_bit = [&](int t, uint32_t hits, auto f) {             // f(logit, token)
    for (; hits; hits &= hits - 1) f(logit(t + __builtin_ctz(hits)), t + __builtin_ctz(hits));
  };
  auto answer = [&](int token, float logprob) {
    A.token[r] = token;
    if (A.logprob) A.logprob[r] = logprob;
  };
  for (int i = 2 * tid; i < SAMPLE_BUCKETS; i += 2048) *(ulonglong2*)(hist + i) = ulonglong2{0, 0};
  float top = -INFINITY;
  runs([&](const float* x, int, auto n) {
#pragma unroll
    for (int j = 0; j < decltype(n)::value; ++j) top = fmaxf(top, x[j]);
  });
  const float best_here = top;                                    // of this thread's tokens
  {
    const u64 first = wave_min(order_of(top));
    // (what is the same for all is worked out by a wave or two: sixteen would take each other's time)
    if (wave == 1) root[lane] = exp2(lane * (-1.0 / 64.0));
    if (wave == 2) { const SampleRow q = sample_row(V, temperature, k_of_row, p_of_row, min_of_row, u_of_row); if (lane == 0) s_row = q; }
    if (lane == 0) s_wave[wave] = first;
    if (tid == 0) { s_low = ~0ull; s_n = 0; }
    __syncthreads();
    u64 least = ~0ull;
    for (int i = 0; i < 16; ++i) least = min(least, s_wave[i]);
    top = uniform(value_of((uint32_t)least));
  }
  SampleRow Q = s_row;
  Q.greedy = __builtin_amdgcn_readfirstlane(Q.greedy); Q.top_k = __builtin_amdgcn_readfirstlane(Q.top_k); Q.top_p = __builtin_amdgcn_readfirstlane(Q.top_p);
  Q.min_p = __builtin_amdgcn_readfirstlane(Q.min_p); Q.k = __builtin_amdgcn_readfirstlane(Q.k);
  Q.rate = uniform(Q.rate); Q.p = uniform(Q.p); Q.log_least = uniform(Q.log_least); Q.u = uniform(Q.u);
  if (top == -INFINITY) {
    if (tid == 0) answer(-1, -INFINITY);
    return;
  }
  if (Q.greedy) {                                                 // the first of the largest
    u64 best = ~0ull;
    between(top, top, [&](int t, uint32_t hits) { best = min(best, (u64)(t + __builtin_ctz(hits))); });
    if (best != ~0ull) atomicMin(&s_low, best);
    __syncthreads();
    if (tid == 0) answer((int)s_low, 0.f);
    return;
  }
  if (top == INFINITY) {                                          // those alone, all alike: the n-th of them
    u64 n = 0;
    between(top, top, [&](int, uint32_t hits) { n += __popc(hits); });
    n = wave_sum(n);
    __syncthreads();
    if (lane == 0) s_wave[wave] = n;
    __syncthreads();
    n = 0;
    for (int i = 0; i < 16; ++i) n += s_wave[i];
    if (Q.top_k) n = min(n, (u64)Q.k);
    if (Q.top_p) n = min(n, max(1ull, (u64)ceil(Q.p * (double)n)));
    if (Q.min_p && Q.log_least > 0.0) n = 1;
    u64 left = min((u64)(Q.u * (double)n), n - 1);
    for (int t0 = 0; t0 < V; t0 += 1024) {
      float x = 0.f;
      if (t0 + tid < V) load_run<1>(row + t0 + tid, &x);
      const uint64_t those = __ballot(x == top);
      __syncthreads();
      if (lane == 0) s_wave[wave] = __popcll(those);
      __syncthreads();
      u64 before = 0, all = 0;
      for (int i = 0; i < 16; ++i) { if (i < wave) before += s_wave[i]; all += s_wave[i]; }
      if (x == top && before + __popcll(those & ((1ull << lane) - 1)) == left) answer(t0 + tid, (float)-log((double)n));
      if (left < all) return;
      left -= all;
    }
    return;
  }

  const double step = uniform(Q.step), farthest = uniform(Q.farthest), magic = 6755399441055744.0;   // 1.5 * 2^52: what is added to it is rounded to a whole number
  const double top64 = uniform((double)top);
  struct Bucket { int b; double rest; };
  auto bucket_of = [&](double d) -> Bucket {                      // b and y - b
    const double k = fma(d, step, magic);
    return Bucket{(int)(uint32_t)__builtin_bit_cast(u64, k), fma(d, step, magic - k)};
  };
  auto bucket = [&](float x) { return bucket_of(fmin(top64 - (double)x, farthest)); };
  // 2^(-rest / 64): three terms behind the 1 leave out 4 * 10^-11.  The last sum is one with 2^52, so it ends on a whole number, in the lower 52 bits; what is above them is left to whoever adds up.
  const double first = A.part[0], c1 = A.part[1], c2 = A.part[2], c3 = A.part[3];
  auto part_above = [&](double rest) -> u64 { return __builtin_bit_cast(u64, fma(fma(fma(rest, c3, c2), rest, c1), rest, first)); };
  constexpr u64 LOWER = 0xFFFFFFFFFFFFFull;
  auto part = [&](double rest) -> u64 { return part_above(rest) & LOWER; };
  // Adds the parts of a run's tokens (or 1 each) to their buckets; what is far below, and NaN, goes to a place of the lane's behind them.
  const float low = uniform((float)(top64 - farthest) - (fabsf(top) + (float)fmin(farthest, 1e30)) * 1e-6f);   // (a little below what is far below)
  auto add_run = [&](const float* x, auto n, bool by_mass) {
    constexpr int N = decltype(n)::value;
    float most = x[0];
#pragma unroll
    for (int j = 1; j < N; ++j) most = fmaxf(most, x[j]);
    if (!(most >= low)) return;
    if (by_mass) {
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const double d = top64 - (double)x[j];
        const Bucket b = bucket_of(d);
        atomicAdd(&hist[d < farthest ? b.b : SAMPLE_BUCKETS + lane], part_above(b.rest));
      }
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const double d = top64 - (double)x[j];
        atomicAdd(&hist[d < farthest ? bucket_of(d).b : SAMPLE_BUCKETS + lane], 1ull);
      }
    }
  };
  auto exponent = [&](float x) -> double { return ((double)x - top64) * Q.rate; };   // ln(weight)
  auto heavy = [&](float x) { return exponent(x) >= Q.log_least; };                  // min-p keeps it
  // a little below the least that min-p keeps (at a temperature that is infinite, no bound)
  const float scaled = (float)(top64 + uniform(Q.reach)), cut = uniform(Q.rate > 0.0 ? fminf(top, scaled - fabsf(scaled) * 1e-6f - 1e-30f) : -INFINITY);

  auto scale_of = [&](int b) { return ldexp(root[b & 63], A.bits - A.unit - (b >> 6)); };   // a part of bucket b as a mass
  auto clear = [&](u64* h) {
    for (int i = 2 * tid; i < SAMPLE_BUCKETS; i += 2048) *(ulonglong2*)(h + i) = ulonglong2{0, 0};
    __syncthreads();
  };
  // The running sums of a histogram, four buckets a thread.
  constexpr int EACH = SAMPLE_BUCKETS / 1024;
  struct Sums { u64 at, x[EACH], total; };
  auto scan = [&](const u64* h, bool masses) -> Sums {
    Sums s;
    u64 sum = 0, any = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      s.x[i] = h[tid * EACH + i] & LOWER;
      any |= s.x[i];
    }
    if (any) {                                                    // (most of the buckets are empty)
#pragma unroll
      for (int i = 0; i < EACH; ++i) {
        if (masses) s.x[i] = (u64)((double)s.x[i] * scale_of(tid * EACH + i));
        sum += s.x[i];
      }
    }
    u64 upto = wave_scan(sum, 0, Add());
    if (lane == 63) s_wave[wave] = upto;
    __syncthreads();
    u64 total = 0;
    for (int i = 0; i < 16; ++i) { const u64 y = s_wave[i]; if (i < wave) upto += y; total += y; }
    s.at = upto - sum; s.total = uniform(total);
    return s;
  };
  // The bucket that the number falls into -> s_bucket, what is in front of it -> s_found[0], what it holds -> s_found[1].
  auto find = [&](const Sums& s, u64 target) {
    u64 at = s.at;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      if (at <= target && target < at + s.x[i]) { s_bucket = tid * EACH + i; s_found[0] = at; s_found[1] = s.x[i]; }
      at += s.x[i];
    }
    __syncthreads();
  };
  // The first place in the order whose bucket is at least b, for a whole wave.
  auto edge = [&](int b) -> uint32_t {
    uint32_t lo = order_of(top), hi = order_of(-INFINITY) + 1;
    if (b <= 0) return lo;
    while (hi - lo > 1) {
      const uint32_t by = (hi - lo + 63) / 64, at = lo + by * (lane + 1);
      const uint64_t yes = __ballot(at >= hi || bucket(value_of(at)).b >= b);
      const int f = __builtin_ctzll(yes | 1ull << 63);
      const uint32_t next = lo + by * (f + 1);
      lo += by * f;
      hi = min(hi, next);
    }
    return (uint32_t)__builtin_amdgcn_readfirstlane((int)hi);
  };
  // Those of two or four buckets, a wave each (all sixteen looking for the same would take each other's time: 1.1 us an edge).
  struct Edges { uint32_t at[4]; };
  auto edges = [&](int b0, int b1, int b2, int b3) -> Edges {
    const int b = wave == 0 ? b0 : wave == 1 ? b1 : wave == 2 ? b2 : b3;
    if (wave < 4 && b >= 0) { const uint32_t e = edge(b); if (lane == 0) s_edge[wave] = e; }
    __syncthreads();
    Edges e;
    for (int i = 0; i < 4; ++i) e.at[i] = (uint32_t)__builtin_amdgcn_readfirstlane((int)s_edge[i]);
    __syncthreads();
    return e;
  };
  auto mass_of = [&](float x) -> u64 {
    const Bucket b = bucket(x);
    return b.b < SAMPLE_BUCKETS - 1 ? (u64)((double)part(b.rest) * scale_of(b.b)) : 0ull;
  };
  struct Found { u64 place, before, share; };
  // Of the tokens up to `limit` from place `begin` up to `end` (a bucket's), the one in whose share (its part, or 1) the number falls.
  // given >= 0: these are among the `given` tokens in `noted`.
  auto select = [&](uint32_t begin, uint32_t end, u64 target, bool by_mass, u64 limit, int given) -> Found {
    auto share = [&](u64 place) -> u64 { return by_mass ? part(bucket(value_of((uint32_t)(place >> 32))).rest) : 1ull; };
    u64 low = (u64)begin << 32, high = min(limit, ((u64)end << 32) - 1), in_front = 0;
    auto narrow = [&](int shift) {                                // to the bucket of `sub` that the number falls into
      const Sums s = scan(sub, false);
      find(s, target - in_front);
      in_front += uniform(s_found[0]);
      low += (u64)__builtin_amdgcn_readfirstlane(s_bucket) << shift;
      high = min(high, low + ((1ull << shift) - 1));
    };
    auto width = [&]() -> int {
      const u64 range = high - low;
      return max(0, 64 - __builtin_clzll(range | 1) - 12);        // (range >> width < 4096)
    };
    // f(logits, first token, bits of those in the range) of every run: where a value's tokens lie on both sides of an end
    auto in_range = [&](auto f) {
      runs([&](const float* x, int t, auto n) {
        uint32_t hits = 0;
#pragma unroll
        for (int j = 0; j < decltype(n)::value; ++j) {
          const u64 p = place_of(x[j], t + j);
          hits |= x[j] == x[j] && p >= low && p <= high ? 1u << j : 0u;
        }
        if (hits) f(t, hits);
      });
    };
    auto note = [&](int t, uint32_t hits) {
      int i = atomicAdd(&s_n, __popc(hits));
      for (; hits && i < SAMPLE_LIST; hits &= hits - 1) noted[i++] = t + __builtin_ctz(hits);
    };
    int n = given;
    if (given >= 0) {
      if (tid == 0) { s_low = ~0ull; s_high = 0; }
    } else for (bool ranged = false;; ranged = true) {                   // (every turn leaves a 2048th of the range at most, so that one of SAMPLE_LIST tokens is reached)
      if (tid == 0) { s_n = 0; s_low = ~0ull; s_high = 0; }
      __syncthreads();
      if (!ranged) between(value_of((uint32_t)(high >> 32)), value_of((uint32_t)(low >> 32)), note);
      else in_range(note);
      __syncthreads();
      n = __builtin_amdgcn_readfirstlane(s_n);
      if (n <= SAMPLE_LIST) break;
      const int shift = width();
      clear(sub);
      in_range([&](int t, uint32_t hits) {
        for (; hits; hits &= hits - 1) {
          const u64 p = place_of(logit(t + __builtin_ctz(hits)), t + __builtin_ctz(hits));
          atomicAdd(&sub[(p - low) >> shift], share(p));
        }
      });
      narrow(shift);
    }
    {
      const int t = tid < n ? noted[tid] : 0;
      const u64 p = place_of(logit(t), t);
      const bool mine = tid < n && p >= low && p <= high;         // (of the last value some may lie behind the limit, and what is given may be of other buckets)
      u64 lo = mine ? p : ~0ull, hi = mine ? p : 0;
      lo = wave_min(lo);
      hi = wave_max(hi);
      __syncthreads();
      if (tid == 0) s_n = 0;
      if (lane == 0 && hi) { atomicMin(&s_low, lo); atomicMax(&s_high, hi); }
      __syncthreads();
      if (mine) list[0][atomicAdd(&s_n, 1)] = p;
      __syncthreads();
      n = __builtin_amdgcn_readfirstlane(s_n);
      if (n > 0) { low = uniform(s_low); high = uniform(s_high); }
    }
    int from = 0;
    while (n > SAMPLE_PAIRS) {                                    // the same on the list
      const int shift = width();
      clear(sub);
      const u64 p = tid < n ? list[from][tid] : 0;
      if (tid < n) atomicAdd(&sub[(p - low) >> shift], share(p));
      narrow(shift);
      if (tid == 0) s_n = 0;
      __syncthreads();
      if (tid < n && p >= low && p <= high) list[from ^ 1][atomicAdd(&s_n, 1)] = p;
      __syncthreads();
      n = __builtin_amdgcn_readfirstlane(s_n);
      from ^= 1;
      __syncthreads();
    }
    // what lies in front of each of the few, eight threads each
    if (tid < n) mass[tid] = share(list[from][tid]);
    __syncthreads();
    const int mine = tid >> 3;
    const u64 p = mine < n ? list[from][mine] : 0;
    u64 at = 0;
    for (int j = tid & 7; j < n; j += 8) at += list[from][j] < p ? mass[j] : 0;
    at += moved<0xB1>(at, 0);                                     // lanes two by two, four by four, and eight by eight
    at += moved<0x4E>(at, 0);
    at += moved<0x141>(at, 0);
    at += in_front;
    if (mine < n && (tid & 7) == 0 && at <= target && target < at + mass[mine]) { s_found[0] = p; s_found[1] = at; s_found[2] = mass[mine]; }
    __syncthreads();
    const Found f{uniform(s_found[0]), uniform(s_found[1]), uniform(s_found[2])};
    __syncthreads();
    return f;
  };
  u64 chosen = ~0ull, kept = 0;                                   // the thread that has it: the token's place, and the mass of all that are kept
  // All of at most SAMPLE_FEW tokens in list[0], or the first `most` of them in order, are what top-p, min-p and the number choose from.
  auto few = [&](int n, int most) {
    const int mine = tid >> 2;
    const u64 p = mine < n ? list[0][mine] : 0;
    int rank = 0;
    for (int j = tid & 3; j < n; j += 4) rank += list[0][j] < p;
    rank += (int)moved<0xB1>(rank, 0);
    rank += (int)moved<0x4E>(rank, 0);
    const float x = value_of((uint32_t)(p >> 32));
    if (mine < n && (tid & 3) == 0) {
      list[1][rank] = p;
      mass[rank] = rank < most ? mass_of(x) : 0ull;
    }
    __syncthreads();
    if (wave > 0) return;
    u64 m[4], sum = 0, strong = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int j = 4 * lane + i;
      m[i] = j < n ? mass[j] : 0;
      sum += m[i];
      if (Q.min_p && m[i] && heavy(value_of((uint32_t)(list[1][j] >> 32)))) strong += m[i];
    }
    const u64 upto = wave_scan(sum, 0, Add());
    kept = last_lane(upto);
    if (Q.top_p) {
      const u64 need = max(1ull, (u64)ceil(Q.p * (double)kept));
      u64 at = upto - sum, least = ~0ull;
#pragma unroll
      for (int i = 3; i >= 0; --i) {                              // (from the end: the least running sum that reaches it)
        u64 run = at;
#pragma unroll
        for (int j = 0; j <= i; ++j) run += m[j];
        if (run >= need) least = run;
      }
      kept = min(kept, wave_min(least));
    }
    if (Q.min_p) {
      kept = min(kept, max(wave_sum(strong), 1ull << A.bits));
    }
    const u64 target = min((u64)(Q.u * (double)kept), kept - 1);
    u64 at = upto - sum;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (at <= target && target < at + m[i]) chosen = list[1][4 * lane + i];
      at += m[i];
    }
  };
  auto gather = [&](float least) -> int {                         // tokens of at least this value: into list[0], if they are few enough
    if (tid == 0) s_n = 0;
    __syncthreads();
    between(least, top, [&](int t, uint32_t hits) {
      int i = atomicAdd(&s_n, __popc(hits));
      for (; hits && i < SAMPLE_FEW; hits &= hits - 1) noted[i++] = t + __builtin_ctz(hits);
    });
    __syncthreads();
    const int n = __builtin_amdgcn_readfirstlane(s_n);
    if (tid < min(n, SAMPLE_FEW)) list[0][tid] = place_of(logit(noted[tid]), noted[tid]);
    __syncthreads();
    return n;
  };

  // Three boundaries, one after the other: the last token of top-k, the last of top-p, the token itself.
  enum { LAST_K, LAST_P, TOKEN };
  u64 limit = ~0ull, heavy_mass = ~0ull;
  int given = -1, given_from = 0, given_to = -1;                  // tokens in `noted`: those of buckets given_from to given_to among them
  Sums s;
  bool cleared = true;                                            // (hist is, from the start)
  bool by_threads = Q.top_k && Q.k <= SAMPLE_FEW, tried = false;
  float least = !Q.top_k && Q.min_p && !Q.top_p ? cut : NAN;      // tokens from here on may be few (NaN: not known)
#pragma unroll 1
  for (int stage = Q.top_k ? LAST_K : LAST_P;; ++stage) {
    asm volatile("" : "+v"(tid));                                  // (what can be had from the thread's number in an instruction or two is not kept: it would be spilled)
    lane = tid & 63;
    u64 target = (u64)Q.k - 1;
    if (stage != TOKEN) {
      if (least == least) {
        const int n = gather(least);
        if (n <= SAMPLE_FEW) { few(n, Q.top_k ? Q.k : V); break; }
        __syncthreads();
        least = NAN;
      }
      if (!cleared) clear(hist);
      cleared = false;
      if (by_threads) {
        if (top64 - (double)best_here < farthest) atomicAdd(&hist[bucket(best_here).b], 1ull);
      } else if (limit == ~0ull) runs([&](const float* x, int, auto n) { add_run(x, n, stage == LAST_P); });
      else runs([&](const float* x, int t, auto n) {
        float y[decltype(n)::value];
#pragma unroll
        for (int j = 0; j < decltype(n)::value; ++j) y[j] = place_of(x[j], t + j) <= limit ? x[j] : NAN;
        add_run(y, n, true);
      });
      s = scan(hist, stage == LAST_P);
    }
    if (by_threads) {
      // The k-th largest of the threads' own largest tokens is no larger than the k-th of all, and hardly smaller: what is not below its bucket is listed.
      by_threads = false;
      if (target < s.total) {
        find(s, target);
        least = value_of(edges(__builtin_amdgcn_readfirstlane(s_bucket) + 1, -1, -1, -1).at[0] - 1);
      }
      __syncthreads();
      stage = LAST_K - 1;
      continue;
    }
    if (stage == LAST_K) {
      if (target >= s.total) continue;                            // (the last of them weighs nothing: no bound)
    } else if (stage == LAST_P) {
      kept = s.total;
      if (Q.min_p) {
        // The buckets in front of the one that the least weight falls into are kept, and of this one and its neighbours what is heavy enough.
        const int at = (int)fmax(0.0, fmin(-Q.log_least * (64 * 1.4426950408889634) + 0.5, SAMPLE_BUCKETS - 1.0)), from = max(0, at - 1);
        if (tid == 0) s_found[2] = 0;
        __syncthreads();
        if (tid == from / EACH) {
          u64 m = s.at;
#pragma unroll
          for (int i = 0; i < EACH; ++i) m += i < from % EACH ? s.x[i] : 0;
          atomicAdd(&s_found[2], m);
        }
        u64 m = 0;
        const Edges e = edges(from, min(at + 2, SAMPLE_BUCKETS), -1, -1);
        if (e.at[0] < e.at[1]) between(value_of(e.at[1] - 1), value_of(e.at[0]), [&](int t, uint32_t hits) {   // (numbers may lie further apart than these buckets: then none falls into them)
          each_bit(t, hits, [&](float x, int i) { if (heavy(x) && place_of(x, i) <= limit) m += mass_of(x); });
        });
        m = wave_sum(m);
        if (lane == 0) atomicAdd(&s_found[2], m);
        __syncthreads();
        heavy_mass = uniform(max(s_found[2], 1ull << A.bits));
        __syncthreads();
      }
      if (!Q.top_p) stage = TOKEN;
      else target = uniform(min(max(1ull, (u64)ceil(Q.p * (double)kept)), kept) - 1);
    }
    if (stage == TOKEN) {
      kept = min(kept, heavy_mass);
      target = uniform(min((u64)(Q.u * (double)kept), kept - 1));
    }
    find(s, target);
    const int b = __builtin_amdgcn_readfirstlane(s_bucket);
    const u64 before = uniform(s_found[0]), inside = uniform(hist[b] & LOWER);
    if (stage == LAST_K && before + inside <= SAMPLE_FEW && !tried) {
      tried = true;
      least = value_of(edges(b + 1, -1, -1, -1).at[0] - 1);
      stage = LAST_K - 1;
      continue;
    }
    // inside the bucket the number counts in the bucket's own units
    const double scale = stage == LAST_K ? 1.0 : scale_of(b);
    Edges e;
    if (stage == LAST_P) {
      // What is kept is known but for this bucket's mass, so the token's bucket is known too, or two or three that it may be: their tokens are noted on the way.
      const u64 least_kept = min(before + 1, heavy_mass), most_kept = min(before + uniform(s_found[1]), heavy_mass);
      __syncthreads();
      find(s, min((u64)(Q.u * (double)least_kept), least_kept - 1));
      given_from = __builtin_amdgcn_readfirstlane(s_bucket);
      __syncthreads();
      find(s, min((u64)(Q.u * (double)most_kept), most_kept - 1));
      given_to = __builtin_amdgcn_readfirstlane(s_bucket);
      if (tid == 0) s_n = 0;
      e = edges(b, b + 1, given_from, given_to + 1);
      const float most = value_of(e.at[0]), least = value_of(e.at[1] - 1), most_u = value_of(e.at[2]), least_u = value_of(e.at[3] - 1);
      runs([&](const float* x, int t, auto n) {
        uint32_t hits = 0;
#pragma unroll
        for (int j = 0; j < decltype(n)::value; ++j)
          hits |= __builtin_amdgcn_fmed3f(x[j], least, most) == x[j] || __builtin_amdgcn_fmed3f(x[j], least_u, most_u) == x[j] ? 1u << j : 0u;
        if (!hits) return;
        int i = atomicAdd(&s_n, __popc(hits));
        for (; hits && i < SAMPLE_LIST; hits &= hits - 1) noted[i++] = t + __builtin_ctz(hits);
      });
      __syncthreads();
      given = __builtin_amdgcn_readfirstlane(s_n);
      if (given > SAMPLE_LIST) given = -1;
    } else e = edges(b, b + 1, -1, -1);
    const bool noted_here = given >= 0 && (stage == LAST_P || (stage == TOKEN && b >= given_from && b <= given_to));
    const Found f = select(e.at[0], e.at[1], min((u64)((double)(target - before) / scale), inside - 1), stage != LAST_K, limit, noted_here ? given : -1);
    if (stage == LAST_K) limit = f.place;
    else if (stage == LAST_P) kept = uniform(min(kept, before + (u64)((double)(f.before + f.share) * scale)));
    else {
      if (tid == 0) chosen = f.place;
      break;
    }
  }
  if (chosen != ~0ull) answer((int)(uint32_t)chosen, (float)(exponent(value_of((uint32_t)(chosen >> 32))) - log(ldexp((double)kept, -A.bits))));
}
