// operators.cu -- C ABI of the operators that answer with a tuned decoder and that train all of its weights: argument
// checks, then the launch.
#include <algorithm>
#include <cmath>

#include "operators.h"

using namespace ra;

namespace {

// what a launcher returns: cudaErrorNotSupported for a size that its kernels do not take
ra_status launched(cudaError_t e) {
  return e == cudaSuccess ? RA_OK : e == cudaErrorNotSupported ? RA_ERR_SHAPE : RA_ERR_CUDA;
}
bool aligned(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
int vec(int dtype) { return dtype == RA_BF16 ? 8 : 4; }  // values of 16 bytes
// (the largest score is the largest product, scaled)
bool good_scale(float s) { return s > 0.f && std::isfinite(s); }
// rows of head_dim values, `heads` to a token, at a 16-byte aligned base
ra_status check_rows(const void* p, int64_t stride, int heads, int head_dim, int dtype) {
  if (!p || !aligned(p, 16)) return RA_ERR_ARG;
  if (stride < (int64_t)heads * head_dim || stride % vec(dtype)) return RA_ERR_SHAPE;
  if ((int64_t)heads * head_dim > INT32_MAX) return RA_ERR_SHAPE;  // (a head's place in its token is counted in 32 bits)
  return RA_OK;
}
ra_status check_cache(const ra_kv_cache& c) {
  if (!c.k_dev || !c.v_dev || !c.block_table_dev || !aligned(c.k_dev, 16) || !aligned(c.v_dev, 16)) return RA_ERR_ARG;
  if (c.dtype != RA_F32 && c.dtype != RA_BF16) return RA_ERR_ARG;
  if (c.n_pages < 1 || c.max_pages < 1 || c.page_size < 1 || c.n_kv_heads < 1) return RA_ERR_ARG;
  if (c.head_dim < 1 || c.head_dim > 256 || c.head_dim % vec(c.dtype)) return RA_ERR_SHAPE;
  // slots are counted in 32 bits, and shares of them run past a sequence's end (in the selection by up to 2016)
  if (cache_capacity(c) > INT32_MAX - 4096) return RA_ERR_SHAPE;
  return RA_OK;
}
ra_status check_workspace(const void* p, size_t bytes, size_t need) {
  if (need == 0) return RA_OK;
  if (!p || !aligned(p, 256)) return RA_ERR_ARG;
  return bytes < need ? RA_ERR_NOMEM : RA_OK;
}
#define TRY(x)                    \
  do {                            \
    ra_status _r = (x);           \
    if (_r != RA_OK) return _r;   \
  } while (0)

ra_status check_append(const ra_kv_append_args& a) {
  TRY(check_cache(a.cache));
  const ra_kv_cache& c = a.cache;
  if (!a.lens_dev || a.batch < 0 || a.n_new < 1) return RA_ERR_ARG;
  TRY(check_rows(a.k_dev, a.k_stride, c.n_kv_heads, c.head_dim, c.dtype));
  TRY(check_rows(a.v_dev, a.v_stride, c.n_kv_heads, c.head_dim, c.dtype));
  if (a.q_dev || a.q_out_dev) {
    if (a.n_heads < 1 || a.n_heads % c.n_kv_heads) return RA_ERR_ARG;
    TRY(check_rows(a.q_dev, a.q_stride, a.n_heads, c.head_dim, c.dtype));
    TRY(check_rows(a.q_out_dev, a.q_out_stride, a.n_heads, c.head_dim, c.dtype));
  }
  if (a.rope_dev && (a.rope_len < 1 || !aligned(a.rope_dev, 16))) return RA_ERR_ARG;
  if ((int64_t)a.batch * a.n_new > INT32_MAX) return RA_ERR_SHAPE;  // (tokens are counted in 32 bits)
  return RA_OK;
}
ra_status check_decode(const ra_attention_decode_args& a) {
  TRY(check_cache(a.cache));
  const ra_kv_cache& c = a.cache;
  if (!a.lens_dev || a.batch < 0 || a.n_new < 1 || a.n_heads < 1 || a.n_heads % c.n_kv_heads || a.window < 0 ||
      a.sinks < 0 || a.max_len < 0 || !good_scale(a.scale))
    return RA_ERR_ARG;
  TRY(check_rows(a.q_dev, a.q_stride, a.n_heads, c.head_dim, c.dtype));
  TRY(check_rows(a.out_dev, a.out_stride, a.n_heads, c.head_dim, c.dtype));
  if (a.weights_in_dev && !a.weights_out_dev) return RA_ERR_ARG;
  if (a.weights_out_dev && a.weights_stride < call_max_len(c, a.max_len)) return RA_ERR_SHAPE;
  // rows of queries, and the tiles that they are cut into, are counted in 32 bits
  if ((int64_t)a.batch * a.n_new * a.n_heads > (1 << 28)) return RA_ERR_SHAPE;
  if ((int64_t)a.n_new * a.n_heads * (c.head_dim / 4) > INT32_MAX - 1024) return RA_ERR_SHAPE;  // ... and a sequence's outputs, in fours
  return RA_OK;
}
ra_status check_evict(const ra_kv_evict_args& a) {
  TRY(check_cache(a.src));
  TRY(check_cache(a.dst));
  if (!a.lens_dev || !a.weights_dev || !a.lens_out_dev || !a.kept_dev || a.batch < 0 || a.max_len < 0 || a.budget < 1 ||
      a.first < 0 || a.recent < 0 || (int64_t)a.first + a.recent > a.budget)
    return RA_ERR_ARG;
  if (a.src.n_kv_heads != a.dst.n_kv_heads || a.src.head_dim != a.dst.head_dim || a.src.dtype != a.dst.dtype ||
      cache_capacity(a.dst) < a.budget || a.weights_stride < call_max_len(a.src, a.max_len) ||
      (a.weights_out_dev && a.weights_out_stride < a.budget))
    return RA_ERR_SHAPE;
  if ((int64_t)a.batch * a.src.n_kv_heads > INT32_MAX) return RA_ERR_SHAPE;
  return RA_OK;
}
ra_status check_window(const ra_attention_window_args& a, bool backward) {
  if (a.dtype != RA_F32 && a.dtype != RA_BF16) return RA_ERR_ARG;
  if (a.batch < 0 || a.seq < 0 || a.n_heads < 1 || a.n_kv_heads < 1 || a.n_heads % a.n_kv_heads || a.window < 0 ||
      a.sinks < 0 || !good_scale(a.scale))
    return RA_ERR_ARG;
  const bool dims = a.dtype == RA_BF16 ? a.head_dim == 64 || a.head_dim == 128
                                       : a.head_dim >= 4 && a.head_dim <= 128 && a.head_dim % 4 == 0;
  if (!dims) return RA_ERR_SHAPE;
  // tokens, and (sequence, head) pairs, are counted in 32 bits
  if ((int64_t)a.batch * a.seq > INT32_MAX - 256 || (int64_t)a.batch * a.n_heads > INT32_MAX) return RA_ERR_SHAPE;
  TRY(check_rows(a.q_dev, a.q_stride, a.n_heads, a.head_dim, a.dtype));
  TRY(check_rows(a.k_dev, a.k_stride, a.n_kv_heads, a.head_dim, a.dtype));
  TRY(check_rows(a.v_dev, a.v_stride, a.n_kv_heads, a.head_dim, a.dtype));
  TRY(check_rows(a.out_dev, a.out_stride, a.n_heads, a.head_dim, a.dtype));
  if (backward) {
    if (!a.lse_dev) return RA_ERR_ARG;
    TRY(check_rows(a.dout_dev, a.dout_stride, a.n_heads, a.head_dim, a.dtype));
    TRY(check_rows(a.dq_dev, a.dq_stride, a.n_heads, a.head_dim, a.dtype));
    TRY(check_rows(a.dk_dev, a.dk_stride, a.n_kv_heads, a.head_dim, a.dtype));
    TRY(check_rows(a.dv_dev, a.dv_stride, a.n_kv_heads, a.head_dim, a.dtype));
    TRY(check_workspace(a.workspace_dev, a.workspace_bytes, attention_window_workspace(a)));
  }
  return RA_OK;
}
// (of a negative size the check says what is wrong)
bool no_tokens(const ra_attention_window_args& a) { return a.batch >= 0 && a.seq >= 0 && (a.batch == 0 || a.seq == 0); }
ra_status check_verify(const ra_verify_draft_args& a) {
  if (a.dtype != RA_F32 && a.dtype != RA_BF16) return RA_ERR_ARG;
  if (a.batch < 0 || a.n_draft < 0 || a.vocab < 1 || !a.target_dev || !a.noise_dev || !a.accepted_dev ||
      !a.out_tokens_dev)
    return RA_ERR_ARG;
  if (a.n_draft > 0 && (!a.draft_dev || !a.tokens_dev || !a.uniform_dev)) return RA_ERR_ARG;
  if (a.n_draft > (1 << 28) || a.vocab > (1 << 30)) return RA_ERR_SHAPE;  // (both are walked in strides, in 32 bits)
  const size_t es = a.dtype == RA_BF16 ? 2 : 4;
  if (!aligned(a.target_dev, es) || !aligned(a.draft_dev, es)) return RA_ERR_ARG;
  if (a.target_stride < a.vocab || (a.n_draft > 0 && a.draft_stride < a.vocab)) return RA_ERR_SHAPE;
  return RA_OK;
}

// rows of `cols` values at any boundary that their type allows
ra_status check_loose(const void* p, int64_t stride, int64_t cols, int dtype) {
  if (!p || !aligned(p, dtype == RA_BF16 ? 2 : 4)) return RA_ERR_ARG;
  return stride < cols ? RA_ERR_SHAPE : RA_OK;
}
bool no_less_than_zero(float v) { return v >= 0.f && std::isfinite(v); }
ra_status check_norm(const ra_norm_args& a, bool backward) {
  if (a.dtype != RA_F32 && a.dtype != RA_BF16) return RA_ERR_ARG;
  if (a.w_dtype != a.dtype && a.w_dtype != RA_F32) return RA_ERR_ARG;
  if (a.kind != RA_NORM_LAYER && a.kind != RA_NORM_RMS) return RA_ERR_ARG;
  if (a.rows < 0 || a.hidden < 1 || !no_less_than_zero(a.eps)) return RA_ERR_ARG;
  if (a.hidden > 32768) return RA_ERR_SHAPE;
  const size_t wes = a.w_dtype == RA_BF16 ? 2 : 4;
  if (!aligned(a.gamma_dev, wes) || !aligned(a.beta_dev, wes) || !aligned(a.mean_dev, 4) || !aligned(a.rstd_dev, 4))
    return RA_ERR_ARG;
  if (a.rows == 0) return RA_OK;
  if (!backward || !a.residual_dev) TRY(check_loose(a.x_dev, a.x_stride, a.hidden, a.dtype));
  if (a.sum_dev) TRY(check_loose(a.sum_dev, a.sum_stride, a.hidden, a.dtype));
  if (!backward) {
    if (a.residual_dev) TRY(check_loose(a.residual_dev, a.residual_stride, a.hidden, a.dtype));
    return check_loose(a.y_dev, a.y_stride, a.hidden, a.dtype);
  }
  if (a.residual_dev && !a.sum_dev) return RA_ERR_ARG;  // (what was normalised was not kept)
  if (!a.rstd_dev || (a.kind == RA_NORM_LAYER && !a.mean_dev)) return RA_ERR_ARG;
  TRY(check_loose(a.dy_dev, a.dy_stride, a.hidden, a.dtype));
  if (a.dsum_dev) TRY(check_loose(a.dsum_dev, a.dsum_stride, a.hidden, a.dtype));
  if (a.dx_dev) TRY(check_loose(a.dx_dev, a.dx_stride, a.hidden, a.dtype));
  return aligned(a.dgamma_dev, wes) && aligned(a.dbeta_dev, wes) ? RA_OK : RA_ERR_ARG;
}
ra_status check_vocab(const ra_vocab_loss_args& a, bool backward) {
  if (a.dtype != RA_F32 && a.dtype != RA_BF16) return RA_ERR_ARG;
  if (a.tokens < 0 || a.vocab < 1 || a.hidden < 1) return RA_ERR_ARG;
  // tokens, words and values are counted in 32 bits, with room for whole tiles
  if (a.hidden % vec(a.dtype) || a.hidden > (1 << 20) || a.tokens > (1 << 24) || a.vocab > (1 << 24)) return RA_ERR_SHAPE;
  // ... and so are the tiles of the products
  if ((int64_t)a.tokens * a.vocab > (1ll << 40) || (int64_t)std::max(a.tokens, a.vocab) * a.hidden > (1ll << 37)) return RA_ERR_SHAPE;
  if (backward && a.dw_dev) TRY(check_rows(a.dw_dev, a.dw_stride, 1, a.hidden, a.dtype));
  if (a.tokens == 0) return RA_OK;
  TRY(check_rows(a.x_dev, a.x_stride, 1, a.hidden, a.dtype));
  TRY(check_rows(a.w_dev, a.w_stride, 1, a.hidden, a.dtype));
  if (!a.labels_dev || !aligned(a.labels_dev, 4) || !aligned(a.lse_dev, 4)) return RA_ERR_ARG;
  if (!backward && (!a.loss_dev || !aligned(a.loss_dev, 4))) return RA_ERR_ARG;
  if (backward) {
    if (!a.lse_dev || !a.dloss_dev || !aligned(a.dloss_dev, 4)) return RA_ERR_ARG;
    if (a.dx_dev) TRY(check_rows(a.dx_dev, a.dx_stride, 1, a.hidden, a.dtype));
  }
  return RA_OK;
}
ra_status check_orthogonalize(const ra_orthogonalize_args& a) {
  if (a.dtype != RA_F32 && a.dtype != RA_BF16) return RA_ERR_ARG;
  if (a.n_matrices < 0 || a.rows < 1 || a.cols < 1 || a.steps < 0 || !no_less_than_zero(a.eps) || !std::isfinite(a.a) ||
      !std::isfinite(a.b) || !std::isfinite(a.c))
    return RA_ERR_ARG;
  if (a.rows > 32768 || a.cols > 32768 || a.steps > 64 || a.n_matrices > 65535) return RA_ERR_SHAPE;
  TRY(check_loose(a.x_dev, a.x_stride, a.cols, a.dtype));
  TRY(check_loose(a.out_dev, a.out_stride, a.cols, a.dtype));
  // matrices of their own: one behind the other, or side by side
  auto apart = [&](int64_t stride, int64_t matrix) {
    return matrix >= (a.rows - 1) * stride + a.cols || (matrix >= a.cols && stride >= (a.n_matrices - 1) * matrix + a.cols);
  };
  if (a.n_matrices > 1 && (!apart(a.x_stride, a.x_matrix_stride) || !apart(a.out_stride, a.out_matrix_stride))) return RA_ERR_SHAPE;
  return RA_OK;
}

}  // namespace

extern "C" {

ra_status ra_kv_append(const ra_kv_append_args* args, ra_stream_t stream) {
  if (!args) return RA_ERR_ARG;
  if (args->batch == 0) return RA_OK;
  TRY(check_append(*args));
  if (!tc_available()) return RA_ERR_UNSUPPORTED;
  return launched(kv_append(*args, (cudaStream_t)stream));
}

size_t ra_attention_decode_workspace_bytes(const ra_attention_decode_args* args) {
  if (args && args->batch == 0) return WS_ZERO;
  return args && check_decode(*args) == RA_OK ? attention_decode_workspace(*args) : 0;
}
ra_status ra_attention_decode(const ra_attention_decode_args* args, ra_stream_t stream) {
  if (!args) return RA_ERR_ARG;
  if (args->batch == 0) return RA_OK;
  TRY(check_decode(*args));
  TRY(check_workspace(args->workspace_dev, args->workspace_bytes, attention_decode_workspace(*args)));
  if (!tc_available()) return RA_ERR_UNSUPPORTED;
  return launched(attention_decode(*args, (cudaStream_t)stream));
}

ra_status ra_kv_evict(const ra_kv_evict_args* args, ra_stream_t stream) {
  if (!args) return RA_ERR_ARG;
  if (args->batch == 0) return RA_OK;
  TRY(check_evict(*args));
  if (!tc_available()) return RA_ERR_UNSUPPORTED;
  return launched(kv_evict(*args, (cudaStream_t)stream));
}

size_t ra_attention_window_workspace_bytes(const ra_attention_window_args* args) {
  if (args && no_tokens(*args)) return WS_ZERO;
  return args && check_window(*args, false) == RA_OK ? attention_window_workspace(*args) : 0;
}
ra_status ra_attention_window_forward(const ra_attention_window_args* args, ra_stream_t stream) {
  if (!args) return RA_ERR_ARG;
  if (no_tokens(*args)) return RA_OK;
  TRY(check_window(*args, false));
  if (!tc_available()) return RA_ERR_UNSUPPORTED;
  return launched(args->dtype == RA_BF16 ? attention_window_fwd_tc(*args, (cudaStream_t)stream)
                                         : attention_window_fwd_simt(*args, (cudaStream_t)stream));
}
ra_status ra_attention_window_backward(const ra_attention_window_args* args, ra_stream_t stream) {
  if (!args) return RA_ERR_ARG;
  if (no_tokens(*args)) return RA_OK;
  TRY(check_window(*args, true));
  if (!tc_available()) return RA_ERR_UNSUPPORTED;
  return launched(args->dtype == RA_BF16 ? attention_window_bwd_tc(*args, (cudaStream_t)stream)
                                         : attention_window_bwd_simt(*args, (cudaStream_t)stream));
}

size_t ra_verify_draft_workspace_bytes(const ra_verify_draft_args* args) {
  if (args && args->batch == 0) return WS_ZERO;
  return args && check_verify(*args) == RA_OK ? verify_draft_workspace(*args) : 0;
}
ra_status ra_verify_draft(const ra_verify_draft_args* args, ra_stream_t stream) {
  if (!args) return RA_ERR_ARG;
  if (args->batch == 0) return RA_OK;
  TRY(check_verify(*args));
  TRY(check_workspace(args->workspace_dev, args->workspace_bytes, verify_draft_workspace(*args)));
  if (!tc_available()) return RA_ERR_UNSUPPORTED;
  return launched(verify_draft(*args, (cudaStream_t)stream));
}

size_t ra_norm_workspace_bytes(const ra_norm_args* args) {
  return args && (check_norm(*args, false) == RA_OK || check_norm(*args, true) == RA_OK) ? norm_workspace(*args) : 0;
}
ra_status ra_norm_forward(const ra_norm_args* args, ra_stream_t stream) {
  if (!args) return RA_ERR_ARG;
  if (args->rows == 0) return RA_OK;
  TRY(check_norm(*args, false));
  if (!tc_available()) return RA_ERR_UNSUPPORTED;
  return launched(norm_fwd(*args, (cudaStream_t)stream));
}
ra_status ra_norm_backward(const ra_norm_args* args, ra_stream_t stream) {
  if (!args) return RA_ERR_ARG;
  TRY(check_norm(*args, true));
  if (args->rows > 0) TRY(check_workspace(args->workspace_dev, args->workspace_bytes, norm_workspace(*args)));
  if (!args->dx_dev && !args->dgamma_dev && !args->dbeta_dev) return RA_OK;
  if (!tc_available()) return RA_ERR_UNSUPPORTED;
  return launched(norm_bwd(*args, (cudaStream_t)stream));
}

size_t ra_vocab_loss_workspace_bytes(const ra_vocab_loss_args* args) {
  return args && (check_vocab(*args, false) == RA_OK || check_vocab(*args, true) == RA_OK) ? vocab_loss_workspace(*args) : 0;
}
ra_status ra_vocab_loss_forward(const ra_vocab_loss_args* args, ra_stream_t stream) {
  if (!args) return RA_ERR_ARG;
  if (args->tokens == 0) return RA_OK;
  TRY(check_vocab(*args, false));
  TRY(check_workspace(args->workspace_dev, args->workspace_bytes, vocab_loss_workspace(*args)));
  if (!tc_available()) return RA_ERR_UNSUPPORTED;
  return launched(vocab_loss_fwd(*args, (cudaStream_t)stream));
}
ra_status ra_vocab_loss_backward(const ra_vocab_loss_args* args, ra_stream_t stream) {
  if (!args) return RA_ERR_ARG;
  TRY(check_vocab(*args, true));
  if (args->tokens > 0) TRY(check_workspace(args->workspace_dev, args->workspace_bytes, vocab_loss_workspace(*args)));
  if (!args->dx_dev && !args->dw_dev) return RA_OK;
  if (args->tokens == 0 && !args->dw_dev) return RA_OK;
  if (!tc_available()) return RA_ERR_UNSUPPORTED;
  return launched(vocab_loss_bwd(*args, (cudaStream_t)stream));
}

size_t ra_orthogonalize_workspace_bytes(const ra_orthogonalize_args* args) {
  if (args && args->n_matrices == 0) return WS_ZERO;
  return args && check_orthogonalize(*args) == RA_OK ? orthogonalize_workspace(*args) : 0;
}
ra_status ra_orthogonalize(const ra_orthogonalize_args* args, ra_stream_t stream) {
  if (!args) return RA_ERR_ARG;
  if (args->n_matrices == 0) return RA_OK;
  TRY(check_orthogonalize(*args));
  TRY(check_workspace(args->workspace_dev, args->workspace_bytes, orthogonalize_workspace(*args)));
  if (!tc_available()) return RA_ERR_UNSUPPORTED;
  return launched(orthogonalize(*args, (cudaStream_t)stream));
}

// (not in the header: what the launchers choose, for tests)
ra_status ra_internal_vocab_loss_plan(const ra_vocab_loss_args* args, int32_t (&out)[12]) {
  if (!args || args->tokens == 0) return RA_ERR_ARG;
  TRY(check_vocab(*args, false));
  vocab_loss_plan(*args, out);
  return RA_OK;
}
ra_status ra_internal_orthogonalize_plan(const ra_orthogonalize_args* args, int32_t (&out)[17]) {
  if (!args || args->n_matrices == 0) return RA_ERR_ARG;
  TRY(check_orthogonalize(*args));
  orthogonalize_plan(*args, out);
  return RA_OK;
}

}  // extern "C"
