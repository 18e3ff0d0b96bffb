// operators.h -- launchers of the operators that answer with a tuned decoder (internal, not ABI).  They take
// the ABI's argument blocks, checked by operators.cu.
#pragma once

#include "../../include/ringada.h"
#include "kernels.h"

namespace ra {

// the slots that a sequence of the cache can have
inline int64_t cache_capacity(const ra_kv_cache& c) { return (int64_t)c.max_pages * c.page_size; }
// the longest sequence of a call: max_len, at most the table's capacity
inline int call_max_len(const ra_kv_cache& c, int max_len) {
  const int64_t cap = cache_capacity(c);
  return (int)(max_len > 0 && max_len < cap ? max_len : cap);
}

cudaError_t kv_append(const ra_kv_append_args& a, cudaStream_t st);
cudaError_t kv_evict(const ra_kv_evict_args& a, cudaStream_t st);
size_t attention_decode_workspace(const ra_attention_decode_args& a);
cudaError_t attention_decode(const ra_attention_decode_args& a, cudaStream_t st);
size_t attention_window_workspace(const ra_attention_window_args& a);
cudaError_t attention_window_fwd_simt(const ra_attention_window_args& a, cudaStream_t st);
cudaError_t attention_window_fwd_tc(const ra_attention_window_args& a, cudaStream_t st);
size_t attention_window_workspace_tc(const ra_attention_window_args& a);
cudaError_t attention_window_bwd_tc(const ra_attention_window_args& a, cudaStream_t st);
cudaError_t attention_window_bwd_simt(const ra_attention_window_args& a, cudaStream_t st);
size_t verify_draft_workspace(const ra_verify_draft_args& a);
cudaError_t verify_draft(const ra_verify_draft_args& a, cudaStream_t st);

}  // namespace ra
