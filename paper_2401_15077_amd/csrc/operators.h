// What the context's passes share with the operators on the caller's own tensors.
#pragma once
#include "host.h"

// eagle_chunk_attention; `fit`: split the tokens over fewer work-groups rather than refuse a small workspace.
__attribute__((visibility("hidden"))) int chunk_attention(const eagle_attention_args* args, const eagle_chunk* chunk, const eagle_paged_kv* kv, void* workspace, size_t bytes, bool fit,
                                                          hipStream_t stream);
