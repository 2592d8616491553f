// libeagle: the choice of a token (host side): argument checks, launches.
#include "checks.h"
#include "sample.h"

#include <cstring>

static bool meet(const void* a, size_t n, const void* b, size_t m) { return a && b && (uintptr_t)a < (uintptr_t)b + m && (uintptr_t)b < (uintptr_t)a + n; }

static int check_sample(const eagle_sample_args* a) {
  if (!a) return fail(EAGLE_EINVAL, "null argument");
  if (!is_type(a->dtype)) return fail(EAGLE_EINVAL, "sample: dtype must be EAGLE_F32 or EAGLE_BF16");
  if (a->n_rows < 0 || a->n_rows > 1 << 24 || a->vocab < 1 || a->vocab > 1 << 30) return fail(EAGLE_EINVAL, "sample: n_rows must be 0..2^24, vocab 1..2^30");
  if (a->n_rows == 0) return EAGLE_OK;
  if (!a->logits || !a->uniform || !a->token) return fail(EAGLE_EINVAL, "sample: logits, uniform or token is null");
  if (a->n_rows > 1 && a->stride < a->vocab) return fail(EAGLE_EINVAL, "sample: rows of %d entries need a stride of at least that", a->vocab);
  const int elt = elt_of(a->dtype);
  for (const void* p : {(const void*)a->uniform, (const void*)a->temperature, (const void*)a->top_k, (const void*)a->top_p, (const void*)a->min_p, (const void*)a->token, (const void*)a->logprob})
    if (!aligned(p, 4)) return fail(EAGLE_EINVAL, "sample: arrays must start on multiples of 4 bytes");
  if (!aligned(a->logits, elt)) return fail(EAGLE_EINVAL, "sample: logits must start on a multiple of an element");
  const size_t R = a->n_rows, all = (((size_t)R - 1) * (R > 1 ? a->stride : 0) + a->vocab) * elt;
  const void* out[2] = {a->token, a->logprob};
  const void* in[5] = {a->uniform, a->temperature, a->top_k, a->top_p, a->min_p};
  for (const void* o : out) {
    if (meet(o, 4 * R, a->logits, all)) return fail(EAGLE_EINVAL, "sample: an output lies on the logits");
    for (const void* i : in)
      if (meet(o, 4 * R, i, 4 * R)) return fail(EAGLE_EINVAL, "sample: an output lies on an input");
  }
  if (meet(a->token, 4 * R, a->logprob, 4 * R)) return fail(EAGLE_EINVAL, "sample: token and logprob lie on each other");
  return EAGLE_OK;
}

extern "C" size_t eagle_sample_workspace(const eagle_sample_args* a) {
  if (check_sample(a)) return 0;
  return 256;                                                     // (reserved: a row is one work-group, which has all it needs in LDS)
}

extern "C" int eagle_sample(const eagle_sample_args* a, void* workspace, size_t workspace_bytes, void* hip_stream) {
  int rc = check_sample(a);
  if (rc || a->n_rows == 0) return rc;
  const size_t need = eagle_sample_workspace(a);
  if (!workspace || !aligned(workspace, 256)) return fail(EAGLE_EINVAL, "sample: workspace must be a 256-byte aligned device pointer");
  if (workspace_bytes < need) return fail(EAGLE_ENOMEM, "sample: workspace of %zu bytes is smaller than the %zu needed", workspace_bytes, need);
  int bits = 62;                                                  // (as many weights of at most 2^bits add up to at most 2^62, and parts to less than 2^52)
  while ((long long)a->vocab > 1ll << (62 - bits)) --bits;
  const double one = std::ldexp(1.0, bits - 11), L = 0.010830424696249145;   // ln 2 / 64
  const SampleDev d{a->vocab, bits, bits - 11, a->logits, a->stride, a->uniform, a->temperature, a->top_p, a->min_p, a->top_k, a->token, a->logprob,
                    {one + 4503599627370496.0, -L * one, L * L / 2 * one, -L * L * L / 6 * one}};
  const hipStream_t stream = (hipStream_t)hip_stream;
  if (a->dtype == EAGLE_F32) k_sample<float><<<a->n_rows, 1024, 0, stream>>>(d);
  else k_sample<bf16_t><<<a->n_rows, 1024, 0, stream>>>(d);
  LAUNCH_CHECK();
  return EAGLE_OK;
}
