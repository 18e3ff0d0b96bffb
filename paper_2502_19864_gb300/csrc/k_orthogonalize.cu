// k_orthogonalize.cu -- orthogonalisation of updates by Newton-Schulz products.
//
// X = x / (|x| + eps); then `steps` times X <- a X + (b S + c S^2) X with S = X X^T (rows <= cols), or, which is the same
// polynomial of X, X <- a X + X (b S + c S^2) with S = X^T X: S has the smaller of the two sides.
#include "common.cuh"
#include "operators.h"
#include "simt_tile.cuh"

namespace ra {
namespace {

constexpr int TILE = 64;
constexpr int NORM_CTAS = 64;  // parts of a matrix's sum of squares

struct Plan {
  int low;
  size_t norms, x, y, s, b, bytes;
};
Plan plan(const ra_orthogonalize_args& a) {
  Plan p;
  p.low = a.rows < a.cols ? a.rows : a.cols;
  size_t at = WS_ZERO;
  auto take = [&](size_t n) {
    const size_t r = at;
    at += (n + 255) / 256 * 256;
    return r;
  };
  const size_t n = (size_t)a.n_matrices * a.rows * a.cols * 4, s = (size_t)a.n_matrices * p.low * p.low * 4;
  p.norms = take((size_t)a.n_matrices * NORM_CTAS * 3 * 4);
  p.x = take(n);
  p.y = take(n);
  p.s = take(s);
  p.b = take(s);
  p.bytes = at;
  return p;
}

// Sums of squares of the elements by their size, scaled so that none overflows or vanishes: those above 2^50 by 2^-140, those
// below 2^-50 by 2^140, and the others.
__global__ void __launch_bounds__(256) orth_norm_kernel(const ra_orthogonalize_args a, float* norms) {
  const int m = blockIdx.y;
  const int64_t base = m * a.x_matrix_stride, n = (int64_t)a.rows * a.cols;
  float s[3] = {0.f, 0.f, 0.f};
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t at = base + i / a.cols * a.x_stride + i % a.cols;
    const float v = a.dtype == RA_BF16 ? to_f(static_cast<const bf16*>(a.x_dev)[at]) : static_cast<const float*>(a.x_dev)[at];
    const float av = fabsf(v);
    const int k = av > 0x1p50f ? 0 : av < 0x1p-50f ? 2 : 1;
    const float w = v * (k == 0 ? 0x1p-70f : k == 2 ? 0x1p70f : 1.f);
    if (k == 0) s[0] = fmaf(w, w, s[0]);
    else if (k == 2) s[2] = fmaf(w, w, s[2]);
    else s[1] = fmaf(w, w, s[1]);
  }
  __shared__ float sh[8][3];
#pragma unroll
  for (int k = 0; k < 3; ++k) s[k] = warp_sum(s[k]);
  if ((threadIdx.x & 31) == 0)
    for (int k = 0; k < 3; ++k) sh[threadIdx.x >> 5][k] = s[k];
  __syncthreads();
  if (threadIdx.x < 3) {
    float t = 0.f;
    for (int w = 0; w < 8; ++w) t += sh[w][threadIdx.x];
    norms[((int64_t)m * gridDim.x + blockIdx.x) * 3 + threadIdx.x] = t;
  }
}

__global__ void __launch_bounds__(256) orth_start_kernel(const ra_orthogonalize_args a, const float* norms, float* x) {
  const int m = blockIdx.y;
  __shared__ double scale;
  if (threadIdx.x == 0) {
    double t = 0.;
    for (int i = 0; i < NORM_CTAS; ++i) {
      const float* s = norms + ((int64_t)m * NORM_CTAS + i) * 3;
      t += (double)s[0] * 0x1p140 + (double)s[1] + (double)s[2] * 0x1p-140;
    }
    scale = isfinite(t) ? 1. / (sqrt(t) + (double)a.eps) : (double)NAN;  // (a value that is not finite takes the whole matrix)
  }
  __syncthreads();
  const double sc = scale;
  const int64_t base = m * a.x_matrix_stride, n = (int64_t)a.rows * a.cols;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t at = base + i / a.cols * a.x_stride + i % a.cols;
    const float v = a.dtype == RA_BF16 ? to_f(static_cast<const bf16*>(a.x_dev)[at]) : static_cast<const float*>(a.x_dev)[at];
    x[m * n + i] = v == 0.f && !isnan(sc) ? 0.f : (float)((double)v * sc);
  }
}

// S = X X^T, or X^T X
template <bool WIDE>
__global__ void __launch_bounds__(ST_THREADS) orth_gram_kernel(const ra_orthogonalize_args a, const float* x, float* s, int low, int high) {
  __shared__ SimtTile sh;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4, m0 = blockIdx.y * TILE, n0 = blockIdx.x * TILE;
  x += (int64_t)blockIdx.z * a.rows * a.cols;
  s += (int64_t)blockIdx.z * low * low;
  float acc[4][4] = {};
  auto at = [&](int m, int k) { return m < low ? x[WIDE ? (int64_t)m * a.cols + k : (int64_t)k * a.cols + m] : 0.f; };
  simt_tile<WIDE, WIDE>(sh, acc, m0, n0, 0, high, at, at);
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j)
      if (m0 + 4 * ty + i < low && n0 + 4 * tx + j < low) s[(int64_t)(m0 + 4 * ty + i) * low + n0 + 4 * tx + j] = acc[i][j];
}
// B = b S + c S S (S is symmetric)
__global__ void __launch_bounds__(ST_THREADS) orth_square_kernel(const ra_orthogonalize_args a, const float* s, float* b, int low) {
  __shared__ SimtTile sh;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4, m0 = blockIdx.y * TILE, n0 = blockIdx.x * TILE;
  s += (int64_t)blockIdx.z * low * low;
  b += (int64_t)blockIdx.z * low * low;
  float acc[4][4] = {};
  auto at = [&](int m, int k) { return m < low ? s[(int64_t)m * low + k] : 0.f; };
  simt_tile<true, true>(sh, acc, m0, n0, 0, low, at, at);
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const int64_t e = (int64_t)(m0 + 4 * ty + i) * low + n0 + 4 * tx + j;
      if (m0 + 4 * ty + i < low && n0 + 4 * tx + j < low) b[e] = a.b * s[e] + a.c * acc[i][j];
    }
}
// Y = a X + B X, or a X + X B
template <bool WIDE>
__global__ void __launch_bounds__(ST_THREADS) orth_apply_kernel(const ra_orthogonalize_args a, const float* x, const float* b, float* y, int low) {
  __shared__ SimtTile sh;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4, m0 = blockIdx.y * TILE, n0 = blockIdx.x * TILE;
  x += (int64_t)blockIdx.z * a.rows * a.cols;
  y += (int64_t)blockIdx.z * a.rows * a.cols;
  b += (int64_t)blockIdx.z * low * low;
  float acc[4][4] = {};
  auto rows = [&](int m, int k) { return m < a.rows ? (WIDE ? b[(int64_t)m * low + k] : x[(int64_t)m * a.cols + k]) : 0.f; };
  auto cols = [&](int n, int k) { return n < a.cols ? (WIDE ? x[(int64_t)k * a.cols + n] : b[(int64_t)k * low + n]) : 0.f; };
  simt_tile<true, false>(sh, acc, m0, n0, 0, low, rows, cols);
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const int64_t e = (int64_t)(m0 + 4 * ty + i) * a.cols + n0 + 4 * tx + j;
      if (m0 + 4 * ty + i < a.rows && n0 + 4 * tx + j < a.cols) y[e] = a.a * x[e] + acc[i][j];
    }
}
__global__ void __launch_bounds__(256) orth_end_kernel(const ra_orthogonalize_args a, const float* x) {
  const int m = blockIdx.y;
  const int64_t base = m * a.out_matrix_stride, n = (int64_t)a.rows * a.cols;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t at = base + i / a.cols * a.out_stride + i % a.cols;
    const float v = x[m * n + i];
    if (a.dtype == RA_BF16) static_cast<bf16*>(a.out_dev)[at] = from_f<bf16>(v);
    else static_cast<float*>(a.out_dev)[at] = v;
  }
}

int tiles_of(int n) { return (n + TILE - 1) / TILE; }

template <bool WIDE>
cudaError_t run(const ra_orthogonalize_args& a, cudaStream_t st) {
  const Plan p = plan(a);
  char* ws = static_cast<char*>(a.workspace_dev);
  auto f = [&](size_t at) { return reinterpret_cast<float*>(ws + at); };
  const int high = a.rows < a.cols ? a.cols : a.rows, n = a.n_matrices;
  float *x = f(p.x), *y = f(p.y);
  orth_norm_kernel<<<dim3(NORM_CTAS, n), 256, 0, st>>>(a, f(p.norms));
  orth_start_kernel<<<dim3(NORM_CTAS, n), 256, 0, st>>>(a, f(p.norms), x);
  const dim3 sq(tiles_of(p.low), tiles_of(p.low), n);
  for (int i = 0; i < a.steps; ++i) {
    orth_gram_kernel<WIDE><<<sq, ST_THREADS, 0, st>>>(a, x, f(p.s), p.low, high);
    orth_square_kernel<<<sq, ST_THREADS, 0, st>>>(a, f(p.s), f(p.b), p.low);
    orth_apply_kernel<WIDE><<<dim3(tiles_of(a.cols), tiles_of(a.rows), n), ST_THREADS, 0, st>>>(a, x, f(p.b), y, p.low);
    float* t = x;
    x = y;
    y = t;
  }
  orth_end_kernel<<<dim3(NORM_CTAS, n), 256, 0, st>>>(a, x);
  note_launch(3 + 3 * a.steps);
  return cudaGetLastError();
}

}  // namespace

size_t orthogonalize_workspace(const ra_orthogonalize_args& a) { return plan(a).bytes; }
cudaError_t orthogonalize(const ra_orthogonalize_args& a, cudaStream_t st) {
  return a.rows <= a.cols ? run<true>(a, st) : run<false>(a, st);
}

}  // namespace ra
