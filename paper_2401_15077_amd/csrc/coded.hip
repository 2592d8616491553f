// libeagle: attention over a paged cache of 8-bit codes (host side).
#include "attention.h"

static int check_coded_attention(const eagle_attention_args* a, const eagle_chunk* chunk, const eagle_coded_kv* kv, ChunkAttnDev* d) {
  if (!a) return fail(EAGLE_EINVAL, "null argument");
  int rc;
  CodedDev c;
  memset(d, 0, sizeof(*d));
  if ((rc = check_coded(kv, &c))) return rc;
  if (kv->head_dim % 16) return fail(EAGLE_EINVAL, "attention: over codes head_dim must be a multiple of 16");
  d->kv = PagedDev{c.k, c.v, c.n_kv_heads, c.head_dim, c.page_shift, c.n_pages, c.pages_per_seq, c.page_stride, c.head_stride, c.token_stride, c.table_stride, c.page_table};
  d->k_scale = c.k_scale; d->v_scale = c.v_scale; d->scale_page = c.scale_page; d->scale_head = c.scale_head; d->block_shift = c.block_shift;
  return check_attention(a, chunk, 1, d);
}

extern "C" size_t eagle_chunk_attention_coded_workspace(const eagle_attention_args* a, const eagle_chunk* chunk, const eagle_coded_kv* kv) {
  ChunkAttnDev d;
  bool wide;
  if (check_coded_attention(a, chunk, kv, &d)) return 0;
  return plan_attention(&d, a->dtype, 1, SIZE_MAX, &wide);
}

extern "C" int eagle_chunk_attention_coded(const eagle_attention_args* a, const eagle_chunk* chunk, const eagle_coded_kv* kv, void* workspace, size_t workspace_bytes, void* hip_stream) {
  ChunkAttnDev d;
  int rc = check_coded_attention(a, chunk, kv, &d);
  if (rc) return rc;
  bool wide, mods;
  if ((rc = place_attention(&d, a, 1, workspace, workspace_bytes, false, &wide, &mods)) || chunk->n_rows == 0) return rc;
  const hipStream_t stream = (hipStream_t)hip_stream;
  if (kv->dtype == EAGLE_E4M3) return a->dtype == EAGLE_F32 ? launch_attention<float, e4m3_t>(d, wide, mods, stream) : launch_attention<bf16_t, e4m3_t>(d, wide, mods, stream);
  return a->dtype == EAGLE_F32 ? launch_attention<float, int8_code_t>(d, wide, mods, stream) : launch_attention<bf16_t, int8_code_t>(d, wide, mods, stream);
}
