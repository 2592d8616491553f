// A paged cache of 8-bit codes: e4m3 (a sign, four bits of exponent, three of mantissa, no infinity) or int8, with an fp32 scale for each block of tokens of a kv head.
#pragma once
#include "rows.h"

struct CodedDev {
  uint8_t *k, *v;
  float *k_scale, *v_scale;
  int n_kv_heads, head_dim, page_shift, block_shift, n_pages, pages_per_seq;
  long long page_stride, head_stride, token_stride, table_stride, scale_page, scale_head;
  const int* page_table;
};

template <bool E4M3> constexpr float LARGEST_CODE = E4M3 ? 448.f : 127.f;

// A number for which every rounding to at most 24 bits gives what the 64-bit number gives: what does not fit is remembered in the last bit (rounding to odd).
__device__ __forceinline__ float odd_f32(double x) {
  unsigned long long u = __builtin_bit_cast(unsigned long long, x);
  u = (u & ~0x1FFFFFFFull) | ((u & 0x1FFFFFFFull) ? 0x20000000ull : 0ull);
  return (float)__builtin_bit_cast(double, u);
}
// Codes of four numbers: to nearest, ties to even, within the largest code; NaN is NaN in e4m3 and 0 in int8.
template <bool E4M3> __device__ __forceinline__ uint32_t encode4(const float* x) {
  constexpr float M = LARGEST_CODE<E4M3>;
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {                                   // (one choice after the other: nested they become branches)
    y[i] = x[i] > M ? M : x[i];
    y[i] = y[i] < -M ? -M : y[i];
  }
  if constexpr (E4M3) {
    int u = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], u, true);
  } else {
    uint32_t u = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) u |= ((uint32_t)(int)rintf(y[i] == y[i] ? y[i] : 0.f) & 0xFFu) << (8 * i);
    return u;
  }
}
// The numbers that four codes stand for (without their scale).
template <bool E4M3> __device__ __forceinline__ void decode4(uint32_t u, float* x) {
  if constexpr (E4M3) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)u, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)u, true);
    x[0] = lo.x; x[1] = lo.y; x[2] = hi.x; x[3] = hi.y;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (float)(int)(int8_t)(u >> (8 * i));
  }
}
