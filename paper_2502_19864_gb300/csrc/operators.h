// operators.h -- launchers of the operators that answer with a tuned decoder and train its weights (internal, not ABI).  They take
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

// What calls need to find zero in a workspace, and leave zero, lies at its start, at a place and of a size that no shape and
// no operator moves: the decode's join counters, one a CTA, then the verification's slots, one for each sequence that
// is cut over several CTAs.  Everything else comes behind, and may hold anything.
constexpr int WS_COUNTERS = 1024, WS_SLOTS = 768;
constexpr size_t WS_SLOTS_AT = WS_COUNTERS * 4, WS_ZERO = WS_SLOTS_AT + WS_SLOTS * 16;  // 16 KB

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

size_t norm_workspace(const ra_norm_args& a);
cudaError_t norm_fwd(const ra_norm_args& a, cudaStream_t st);
cudaError_t norm_bwd(const ra_norm_args& a, cudaStream_t st);
size_t vocab_loss_workspace(const ra_vocab_loss_args& a);
cudaError_t vocab_loss_fwd(const ra_vocab_loss_args& a, cudaStream_t st);
cudaError_t vocab_loss_bwd(const ra_vocab_loss_args& a, cudaStream_t st);
size_t orthogonalize_workspace(const ra_orthogonalize_args& a);
cudaError_t orthogonalize(const ra_orthogonalize_args& a, cudaStream_t st);

// What the launchers choose for a block's sizes, for tests that ask which form a size runs:
//   loss: few fp32 tokens; planes; pieces of the vocabulary, words of one; CTAs and columns of a tile of the forward's logits, the
//   backward's, the gradients; ranges of K of dx and of dW
//   orthogonalisation: smaller side up to 64; CTAs, columns, halves and ranges of S in the first step and in the others, and of Q; CTAs
//   and columns of X in the first step and in the others
void vocab_loss_plan(const ra_vocab_loss_args& a, int32_t (&out)[12]);
void orthogonalize_plan(const ra_orthogonalize_args& a, int32_t (&out)[17]);

}  // namespace ra
