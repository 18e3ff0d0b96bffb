// k_vocab_loss.cu -- cross-entropy over a vocabulary from hidden states, without keeping logits.
//
// Forward: tiles of logits z = x W^T; of each tile's rows the maximum and the sum of exp(z - maximum) go to the
// workspace, with the label's logit, and a second kernel joins them: lse = m + log(sum), loss = lse - z[label].
// Backward, piece by piece of the vocabulary: the piece's logits again, dz = dloss (exp(z - lse) - onehot) into the
// workspace, then dw of the piece = dz^T x and dx += dz W.
#include "common.cuh"
#include "operators.h"
#include "simt_tile.cuh"

namespace ra {
namespace {

constexpr int TILE = 64;

struct Plan {
  int tiles;         // of the vocabulary
  int piece;         // words of a piece
  size_t stats, label, dz, dx, bytes;
};
Plan plan(const ra_vocab_loss_args& a) {
  Plan p;
  p.tiles = (a.vocab + TILE - 1) / TILE;
  int64_t piece = (64ll << 20) / 4 / (a.tokens > 0 ? a.tokens : 1) / TILE * TILE;
  if (piece < TILE) piece = TILE;
  if (piece > (int64_t)p.tiles * TILE) piece = (int64_t)p.tiles * TILE;
  p.piece = (int)piece;
  size_t at = WS_ZERO;
  auto take = [&](size_t n) {
    const size_t r = at;
    at += (n + 255) / 256 * 256;
    return r;
  };
  p.stats = take((size_t)p.tiles * a.tokens * sizeof(float2));
  p.label = take((size_t)a.tokens * sizeof(float));
  p.dz = take((size_t)a.tokens * p.piece * sizeof(float));
  p.dx = take((size_t)a.tokens * a.hidden * sizeof(float));
  p.bytes = at;
  return p;
}

// the label of a token that is counted, else -1
__device__ __forceinline__ int label_of(const ra_vocab_loss_args& a, int t) {
  const int l = a.labels_dev[t];
  if (l >= a.vocab) set_dev_error(a.err_dev, RA_DEVERR_BOUNDS);
  return l < 0 || l >= a.vocab ? -1 : l;
}

template <typename T>
__device__ __forceinline__ void logits(const ra_vocab_loss_args& a, SimtTile& sh, float (&acc)[4][4], int m0, int n0) {
  const T* x = static_cast<const T*>(a.x_dev);
  const T* w = static_cast<const T*>(a.w_dev);
  simt_tile<true, true>(
      sh, acc, m0, n0, 0, a.hidden,
      [&](int m, int k) { return m < a.tokens && (uint32_t)a.labels_dev[m] < (uint32_t)a.vocab ? to_f(x[m * a.x_stride + k]) : 0.f; },
      [&](int n, int k) { return n < a.vocab ? to_f(w[n * a.w_stride + k]) : 0.f; });
}

template <typename T>
__global__ void __launch_bounds__(ST_THREADS) vocab_stats_kernel(const ra_vocab_loss_args a, float2* stats, float* label) {
  __shared__ SimtTile sh;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4, m0 = blockIdx.y * TILE, n0 = blockIdx.x * TILE;
  float acc[4][4] = {};
  logits<T>(a, sh, acc, m0, n0);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int t = m0 + 4 * ty + i;
    float m = -INFINITY;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (n0 + 4 * tx + j < a.vocab) m = fmaxf(m, acc[i][j]);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    float l = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (n0 + 4 * tx + j < a.vocab) l += expf(acc[i][j] - m);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
    if (t >= a.tokens) continue;
    if (tx == 0) stats[(int64_t)blockIdx.x * a.tokens + t] = make_float2(m, l);
    const int c = label_of(a, t) - n0 - 4 * tx;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (c == j) label[t] = acc[i][j];
  }
}

__global__ void __launch_bounds__(128) vocab_join_kernel(const ra_vocab_loss_args a, const float2* stats, const float* label, int tiles) {
  const int t = blockIdx.x * 128 + threadIdx.x;
  if (t >= a.tokens) return;
  float lse = 0.f, loss = 0.f;
  if (label_of(a, t) >= 0) {
    float m = -INFINITY, l = 0.f;
    for (int i = 0; i < tiles; ++i) m = fmaxf(m, stats[(int64_t)i * a.tokens + t].x);
    for (int i = 0; i < tiles; ++i) {
      const float2 s = stats[(int64_t)i * a.tokens + t];
      l += s.y * expf(s.x - m);
    }
    lse = m + logf(l);
    loss = lse - label[t];
  }
  a.loss_dev[t] = loss;
  if (a.lse_dev) a.lse_dev[t] = lse;
}

template <typename T>
__global__ void __launch_bounds__(ST_THREADS) vocab_dz_kernel(const ra_vocab_loss_args a, float* dz, int v0, int width, int pitch) {
  __shared__ SimtTile sh;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4, m0 = blockIdx.y * TILE, n0 = blockIdx.x * TILE;
  float acc[4][4] = {};
  logits<T>(a, sh, acc, m0, v0 + n0);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int t = m0 + 4 * ty + i;
    if (t >= a.tokens) continue;
    const int label = label_of(a, t);
    const float lse = a.lse_dev[t], scale = a.dloss_dev[t];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int c = n0 + 4 * tx + j;
      if (c < width)
        dz[(int64_t)t * pitch + c] = label < 0 ? 0.f : scale * (expf(acc[i][j] - lse) - (v0 + c == label ? 1.f : 0.f));
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(ST_THREADS) vocab_dw_kernel(const ra_vocab_loss_args a, const float* dz, int v0, int width, int pitch) {
  __shared__ SimtTile sh;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4, m0 = blockIdx.y * TILE, n0 = blockIdx.x * TILE;
  const T* x = static_cast<const T*>(a.x_dev);
  float acc[4][4] = {};
  simt_tile<false, false>(
      sh, acc, m0, n0, 0, a.tokens, [&](int m, int k) { return m < width ? dz[(int64_t)k * pitch + m] : 0.f; },
      [&](int n, int k) { return n < a.hidden && (uint32_t)a.labels_dev[k] < (uint32_t)a.vocab ? to_f(x[k * a.x_stride + n]) : 0.f; });
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int v = m0 + 4 * ty + i, c = n0 + 4 * tx + j;
      if (v < width && c < a.hidden) static_cast<T*>(a.dw_dev)[(v0 + v) * a.dw_stride + c] = from_f<T>(acc[i][j]);
    }
}

template <typename T>
__global__ void __launch_bounds__(ST_THREADS) vocab_dx_kernel(const ra_vocab_loss_args a, const float* dz, float* sum, int v0, int width, int pitch) {
  __shared__ SimtTile sh;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4, m0 = blockIdx.y * TILE, n0 = blockIdx.x * TILE;
  const T* w = static_cast<const T*>(a.w_dev);
  float acc[4][4] = {};
  simt_tile<true, false>(
      sh, acc, m0, n0, 0, width, [&](int m, int k) { return m < a.tokens ? dz[(int64_t)m * pitch + k] : 0.f; },
      [&](int n, int k) { return n < a.hidden ? to_f(w[(v0 + k) * a.w_stride + n]) : 0.f; });
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int t = m0 + 4 * ty + i, c = n0 + 4 * tx + j;
      if (t >= a.tokens || c >= a.hidden) continue;
      float s = acc[i][j];
      if (v0 > 0) s += sum[(int64_t)t * a.hidden + c];
      if (v0 + width < a.vocab) sum[(int64_t)t * a.hidden + c] = s;
      else static_cast<T*>(a.dx_dev)[t * a.dx_stride + c] = label_of(a, t) < 0 ? from_f<T>(0.f) : from_f<T>(s);
    }
}

int tiles_of(int n) { return (n + TILE - 1) / TILE; }

template <typename T>
cudaError_t forward(const ra_vocab_loss_args& a, cudaStream_t st) {
  const Plan p = plan(a);
  char* ws = static_cast<char*>(a.workspace_dev);
  float2* stats = reinterpret_cast<float2*>(ws + p.stats);
  float* label = reinterpret_cast<float*>(ws + p.label);
  vocab_stats_kernel<T><<<dim3(p.tiles, tiles_of(a.tokens)), ST_THREADS, 0, st>>>(a, stats, label);
  vocab_join_kernel<<<(a.tokens + 127) / 128, 128, 0, st>>>(a, stats, label, p.tiles);
  note_launch(2);
  return cudaGetLastError();
}
template <typename T>
cudaError_t backward(const ra_vocab_loss_args& a, cudaStream_t st) {
  const Plan p = plan(a);
  char* ws = static_cast<char*>(a.workspace_dev);
  float* dz = reinterpret_cast<float*>(ws + p.dz);
  for (int v0 = 0; v0 < a.vocab; v0 += p.piece) {
    const int width = a.vocab - v0 < p.piece ? a.vocab - v0 : p.piece;
    vocab_dz_kernel<T><<<dim3(tiles_of(width), tiles_of(a.tokens)), ST_THREADS, 0, st>>>(a, dz, v0, width, p.piece);
    if (a.dw_dev) vocab_dw_kernel<T><<<dim3(tiles_of(a.hidden), tiles_of(width)), ST_THREADS, 0, st>>>(a, dz, v0, width, p.piece);
    if (a.dx_dev)
      vocab_dx_kernel<T><<<dim3(tiles_of(a.hidden), tiles_of(a.tokens)), ST_THREADS, 0, st>>>(
          a, dz, reinterpret_cast<float*>(ws + p.dx), v0, width, p.piece);
    note_launch(3);
  }
  return cudaGetLastError();
}

}  // namespace

size_t vocab_loss_workspace(const ra_vocab_loss_args& a) { return plan(a).bytes; }
cudaError_t vocab_loss_fwd(const ra_vocab_loss_args& a, cudaStream_t st) {
  return a.dtype == RA_BF16 ? forward<bf16>(a, st) : forward<float>(a, st);
}
cudaError_t vocab_loss_bwd(const ra_vocab_loss_args& a, cudaStream_t st) {
  if (a.tokens == 0) {
    const size_t es = a.dtype == RA_BF16 ? 2 : 4;
    return cudaMemset2DAsync(a.dw_dev, a.dw_stride * es, 0, a.hidden * es, a.vocab, st);
  }
  return a.dtype == RA_BF16 ? backward<bf16>(a, st) : backward<float>(a, st);
}

}  // namespace ra
