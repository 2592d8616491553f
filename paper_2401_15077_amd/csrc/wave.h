// Scans and reductions over a wave of 64.
#pragma once
#include "common.h"

typedef unsigned long long u64;

// Sums and the like over a wave, by moves between neighbouring lanes (a step of a shuffle through LDS takes ten times as long).  What comes from outside the row of 16 is `none`.
template <int MOVE, int ROWS = 0xF> __device__ __forceinline__ u64 moved(u64 x, u64 none) {
  const uint32_t lo = __builtin_amdgcn_update_dpp((int)none, (int)x, MOVE, ROWS, 0xF, false), hi = __builtin_amdgcn_update_dpp((int)(none >> 32), (int)(x >> 32), MOVE, ROWS, 0xF, false);
  return (u64)hi << 32 | lo;
}
// Lane l: f over lanes 0 .. l.  (Lanes 1, 2, 4, 8 back; the last lane of a row into the next; of the lower half into the upper.)
template <typename F> __device__ __forceinline__ u64 wave_scan(u64 x, u64 none, F f) {
  x = f(x, moved<0x111>(x, none));
  x = f(x, moved<0x112>(x, none));
  x = f(x, moved<0x114>(x, none));
  x = f(x, moved<0x118>(x, none));
  x = f(x, moved<0x142, 0xA>(x, none));
  return f(x, moved<0x143, 0xC>(x, none));
}
__device__ __forceinline__ u64 last_lane(u64 x) {
  return (u64)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), 63) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}
struct Add { __device__ u64 operator()(u64 a, u64 b) const { return a + b; } };
struct Least { __device__ u64 operator()(u64 a, u64 b) const { return min(a, b); } };
struct Most { __device__ u64 operator()(u64 a, u64 b) const { return max(a, b); } };
__device__ __forceinline__ u64 wave_sum(u64 x) { return last_lane(wave_scan(x, 0, Add())); }
__device__ __forceinline__ u64 wave_min(u64 x) { return last_lane(wave_scan(x, ~0ull, Least())); }
__device__ __forceinline__ u64 wave_max(u64 x) { return last_lane(wave_scan(x, 0, Most())); }
