// k_orthogonalize.cu -- orthogonalisation of updates by Newton-Schulz products.
//
// X = x / (|x| + eps); then `steps` times X <- (a I + S (b I + c S)) X with S = X X^T (rows <= cols), or, which is the same
// polynomial of X, X <- X (a I + S (b I + c S)) with S = X^T X: S has the smaller of the two sides.  A step is three
// products on the tensor cores: S, of which S and T = b I + c S are kept; Q = a I + S T; and X.
//
// Operands are planes of bf16 (products.cuh).  For fp32 three, the significand whole.  For bf16 matrices two, 17 bits: a
// step raises what lies along small singular values by up to 3.4445 while the large ones stay, so that an error of the first
// steps grows with them, about 140-fold by the last; 2^-17 is then a quarter of the output's own rounding at
// worst, where one plane's 2^-9 would be as large as what is computed.
//
// Bound: the products, 2 low^2 high + low^3 multiply-adds a step, three (six) times over for the planes.
#include <algorithm>

#include "common.cuh"
#include "operators.h"
#include "products.cuh"

namespace ra {
namespace {

using prod::parts_of;
using prod::Pick;
using prod::Store;
using prod::Tile;
using prod::Unit;
using prod::up;

constexpr int NORM_CTAS = 64;  // parts of a matrix's sum of squares, at most

template <typename T> __device__ __forceinline__ float value(const void* p, int64_t at) { return to_f(static_cast<const T*>(p)[at]); }

// Sums of squares of the elements by their size, scaled so that none overflows or vanishes: those above 2^50 by 2^-140, those
// below 2^-50 by 2^140, and the others.
template <typename T>
__global__ void __launch_bounds__(256) orth_norm_kernel(const ra_orthogonalize_args a, float* norms) {
  pdl_wait();
  pdl_trigger();
  const int m = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  float s[3] = {0.f, 0.f, 0.f};
  for (int r = blockIdx.x * 8 + warp; r < a.rows; r += gridDim.x * 8) {
    const int64_t base = m * a.x_matrix_stride + r * a.x_stride;
#pragma unroll 8
    for (int c = lane; c < a.cols; c += 32) {
      const float v = value<T>(a.x_dev, base + c), av = fabsf(v);
      const bool big = av > 0x1p50f, small = av < 0x1p-50f;
      const float w = v * (big ? 0x1p-70f : small ? 0x1p70f : 1.f), q = w * w;
      s[0] += big ? q : 0.f;
      s[1] += big || small ? 0.f : q;
      s[2] += small ? q : 0.f;
    }
  }
  __shared__ float sh[8][3];
#pragma unroll
  for (int k = 0; k < 3; ++k) s[k] = warp_sum(s[k]);
  if (lane == 0)
    for (int k = 0; k < 3; ++k) sh[warp][k] = s[k];
  __syncthreads();
  if (threadIdx.x < 3) {
    float t = 0.f;
    for (int w = 0; w < 8; ++w) t += sh[w][threadIdx.x];
    norms[((int64_t)m * gridDim.x + blockIdx.x) * 3 + threadIdx.x] = t;
  }
}

// 1 / (|x| + eps) as two powers of two and a factor in [1, 2); NaN where |x| is not finite, so that a value that is not finite
// takes its whole matrix
struct Scale {
  float p, q, f;
  __device__ __forceinline__ float operator()(float v) const { return v == 0.f && f == f ? 0.f : v * p * f * q; }
};
// (by a warp)
__device__ __forceinline__ Scale scale_of(const float* norms, int parts, float eps) {
  double t = 0.;
  for (int i = threadIdx.x & 31; i < parts; i += 32) t += (double)norms[3 * i] * 0x1p140 + (double)norms[3 * i + 1] + (double)norms[3 * i + 2] * 0x1p-140;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
  if (!isfinite(t)) return {1.f, 1.f, NAN};
  const double s = 1. / (sqrt(t) + (double)eps);
  if (!isfinite(s)) return {1.f, 1.f, 1.f};  // (all zeros, and eps too)
  int e;
  const double f = 2. * frexp(s, &e);
  --e;
  return {ldexpf(1.f, e / 2), ldexpf(1.f, e - e / 2), (float)f};
}

// The scaled matrices in planes [n][planes][rows][pitch]; or (planes 0) into out
template <typename T>
__global__ void __launch_bounds__(256) orth_start_kernel(const ra_orthogonalize_args a, const float* norms, int parts, bf16* x, int planes, int pitch) {
  __shared__ Scale sh;
  pdl_wait();
  pdl_trigger();
  const int m = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (warp == 0) {
    const Scale mine = scale_of(norms + (int64_t)m * parts * 3, parts, a.eps);
    if (lane == 0) sh = mine;
  }
  __syncthreads();
  const Scale s = sh;
  const int64_t plane = (int64_t)a.rows * pitch;
  for (int r = blockIdx.x * 8 + warp; r < a.rows; r += gridDim.x * 8) {
    const int64_t base = m * a.x_matrix_stride + r * a.x_stride;
    if (planes == 0) {
      for (int c = lane; c < a.cols; c += 32)
        static_cast<T*>(a.out_dev)[m * a.out_matrix_stride + r * a.out_stride + c] = from_f<T>(s(value<T>(a.x_dev, base + c)));
      continue;
    }
    bf16* d = x + ((int64_t)m * planes * a.rows + r) * pitch;
#pragma unroll 4
    for (int c = lane; c < pitch; c += 32) {
      float v = c < a.cols ? s(value<T>(a.x_dev, base + c)) : 0.f;
      if (planes == 2) {
        d[c] = __float2bfloat16_rn(prod::plane_round(v));
        d[plane + c] = __float2bfloat16_rn(v);
      } else {
#pragma unroll
        for (int k = 0; k < 3; ++k) d[k * plane + c] = __float2bfloat16_rn(prod::plane_trunc(v));
      }
    }
  }
}

struct OrthArgs {
  CUtensorMap a, b;        // the product's operands
  CUtensorMap o, o2, out;  // where it goes: planes, T's planes, the result
  prod::Shape shape;
  unsigned* err;
  void* dst;
  int64_t dst_stride, dst_matrix_stride;
  int rows, cols;          // of the product
  int k, n, planes, cg, dtype;
  bool a_mn, b_mn, last, map_out;
  float add, add2, mul2;   // o = P + add I and, if wanted, o2 = mul2 P + add2 I
  bool second;
};
#define MAP(m, ...)                                                    \
  do {                                                                 \
    if (!tma_map_3d(&(m), __VA_ARGS__)) return cudaErrorInvalidValue;  \
  } while (0)
#define DO(x)                                \
  do {                                       \
    const cudaError_t _e = (x);              \
    if (_e != cudaSuccess) return _e;        \
  } while (0)

struct Step {
  using Args = OrthArgs;
  static __host__ __device__ __forceinline__ int tiles(const Args& p, int& mt, int& nt) {
    mt = (p.rows + prod::BM * p.cg - 1) / (prod::BM * p.cg);
    nt = (p.cols + p.shape.bn - 1) / p.shape.bn;
    return mt * nt;
  }
  static __device__ __forceinline__ int count(const Args& p) {
    int mt, nt;
    return p.n * tiles(p, mt, nt);
  }
  static __device__ __forceinline__ void unit(const Args& p, int u, Unit& w) {
    int m_n, n_n, mt, nt;
    const int each = tiles(p, m_n, n_n);
    w.z = u / each;
    prod::tile_of(u % each, m_n, n_n, mt, nt);
    w.a = &p.a;
    w.b = &p.b;
    w.m0 = w.ar = mt * prod::BM * p.cg;
    w.n0 = w.br = nt * p.shape.bn;
    w.ak = w.bk = w.kb0 = w.job = 0;
    w.az = w.bz = w.z * p.planes;
    w.kb1 = (p.k + prod::BK - 1) / prod::BK;
    w.a_mn = p.a_mn;
    w.b_mn = p.b_mn;
  }
  static __device__ __forceinline__ void finish(const Args& p, const Unit& w, const Tile& t, Store& st, float (&v)[4][32]) {
    const int row0 = w.m0 + t.rank * prod::BM + t.quad * 32, row = row0 + t.lane;
    if (row0 >= p.rows) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int col = w.n0 + 32 * (t.half + 2 * i);
      if (i >= t.chunks || col >= p.cols) break;
      if (p.last) {
        if (p.map_out) {
          if (p.dtype == RA_BF16) st.bf16_row(&p.out, [&](int j) { return v[i][j]; }, col, row0, w.z);
          else st.f32_row(&p.out, v[i], col, row0, w.z, false, p.cols);
        } else if (row < p.rows) {
          const int64_t at = w.z * p.dst_matrix_stride + row * p.dst_stride + col;
#pragma unroll
          for (int j = 0; j < 32; ++j)
            if (col + j < p.cols) {
              if (p.dtype == RA_BF16) static_cast<bf16*>(p.dst)[at + j] = __float2bfloat16_rn(v[i][j]);
              else static_cast<float*>(p.dst)[at + j] = v[i][j];
            }
        }
        continue;
      }
      // (the identity's part: nothing behind the last row)
      const int diag = row < p.rows ? row - col : -1;
      st.planes_row(&p.o, [&](int j) { return v[i][j] + (j == diag ? p.add : 0.f); }, col, row0, w.z * p.planes, p.planes);
      if (p.second)
        st.planes_row(&p.o2, [&](int j) { return p.mul2 * v[i][j] + (j == diag ? p.add2 : 0.f); }, col, row0, w.z * p.planes, p.planes);
    }
  }
};

struct Plan {
  int planes, low, high, pitch, low_pitch, parts;
  size_t norms, x[2], s, t, q, bytes;
};
Plan plan(const ra_orthogonalize_args& a) {
  Plan p = {};
  p.planes = a.dtype == RA_F32 ? 3 : 2;
  p.low = std::min(a.rows, a.cols);
  p.high = std::max(a.rows, a.cols);
  p.pitch = up(a.cols, 8);
  p.low_pitch = up(p.low, 8);
  p.parts = std::min(NORM_CTAS, parts_of(a.rows, 8));
  size_t at = WS_ZERO;
  auto take = [&](size_t n) {
    const size_t r = at;
    at += (n + 255) / 256 * 256;
    return r;
  };
  const size_t n = (size_t)a.n_matrices * p.planes * 2;
  p.norms = take((size_t)a.n_matrices * p.parts * 3 * 4);
  for (size_t& x : p.x) x = take(n * a.rows * p.pitch);
  p.s = take(n * p.low * p.low_pitch);
  p.t = take(n * p.low * p.low_pitch);
  p.q = take(n * p.low * p.low_pitch);
  p.bytes = at;
  return p;
}

template <typename T>
cudaError_t run(const ra_orthogonalize_args& a, cudaStream_t st) {
  const Plan p = plan(a);
  char* ws = static_cast<char*>(a.workspace_dev);
  const int n = a.n_matrices, nz = n * p.planes;
  const bool wide = a.rows <= a.cols;
  float* norms = reinterpret_cast<float*>(ws + p.norms);
  note_launch(2);
  DO(launch_pdl(orth_norm_kernel<T>, dim3(p.parts, n), dim3(256), 0, st, a, norms));
  DO(launch_pdl(orth_start_kernel<T>, dim3(std::min(parts_of(a.rows, 8), std::max(64, 1216 / n)), n), dim3(256), 0, st, a, (const float*)norms, p.parts,
                reinterpret_cast<bf16*>(ws + p.x[0]), a.steps ? p.planes : 0, p.pitch));
  if (a.steps == 0) return cudaSuccess;

  const int terms = prod::terms_of(p.planes).n, chunk = p.planes == 3 ? 4 : 32;
  OrthArgs g = {};
  g.err = a.err_dev;
  g.n = n;
  g.planes = p.planes;
  g.dtype = a.dtype;
  auto shape = [&](OrthArgs& s, int rows, int cols, int k) {
    const Pick c = prod::pick(rows, cols, n, parts_of(k, prod::BK) * terms);
    s.rows = rows;
    s.cols = cols;
    s.k = k;
    s.cg = c.cg;
    s.shape = prod::shape_of(c.bn, c.cg, p.planes, chunk);
  };
  auto go = [&](const OrthArgs& s) {
    int mt, nt;
    const int64_t units = (int64_t)n * Step::tiles(s, mt, nt);
    const int u = (int)std::min<int64_t>(units, 1 << 20);
    return s.cg == 2 ? prod::launch<Step, 2>(s, u, st) : prod::launch<Step, 1>(s, u, st);
  };
  const int es = a.dtype == RA_BF16 ? 2 : 4;
  OrthArgs gram = g, square = g, apply = g;
  shape(gram, p.low, p.low, p.high);
  gram.a_mn = gram.b_mn = !wide;
  gram.second = true;
  gram.add2 = a.b;
  gram.mul2 = a.c;
  MAP(gram.o, ws + p.s, DT_BF16, nz, p.low, p.low_pitch, p.low_pitch, 32, 32);
  MAP(gram.o2, ws + p.t, DT_BF16, nz, p.low, p.low_pitch, p.low_pitch, 32, 32);
  shape(square, p.low, p.low, p.low);
  square.add = a.a;
  MAP(square.a, ws + p.s, DT_BF16, nz, p.low, p.low_pitch, p.low_pitch, 64, prod::BM);
  MAP(square.b, ws + p.t, DT_BF16, nz, p.low, p.low_pitch, p.low_pitch, 64, square.shape.bn / square.cg);
  MAP(square.o, ws + p.q, DT_BF16, nz, p.low, p.low_pitch, p.low_pitch, 32, 32);
  shape(apply, a.rows, a.cols, p.low);
  apply.b_mn = wide;
  if (wide) MAP(apply.a, ws + p.q, DT_BF16, nz, p.low, p.low_pitch, p.low_pitch, 64, prod::BM);
  else MAP(apply.b, ws + p.q, DT_BF16, nz, p.low, p.low_pitch, p.low_pitch, 64, apply.shape.bn / apply.cg);
  apply.dst = a.out_dev;
  apply.dst_stride = a.out_stride;
  apply.dst_matrix_stride = a.out_matrix_stride;
  // the result by TMA where its rows are at 16-byte boundaries and its matrices one after the other
  apply.map_out = ((uintptr_t)a.out_dev & 15) == 0 && a.out_stride * es % 16 == 0 && (int64_t)a.cols * es % 16 == 0 &&
                  (n == 1 || a.out_matrix_stride == a.rows * a.out_stride);
  if (apply.map_out) MAP(apply.out, a.out_dev, a.dtype, n, a.rows, a.cols, a.out_stride, a.dtype == RA_BF16 ? 32 : 16, 32);
  for (int i = 0; i < a.steps; ++i) {
    const char* x = ws + p.x[i & 1];
    if (wide) {
      MAP(gram.a, x, DT_BF16, nz, a.rows, p.pitch, p.pitch, 64, prod::BM);
      MAP(gram.b, x, DT_BF16, nz, a.rows, p.pitch, p.pitch, 64, gram.shape.bn / gram.cg);
      MAP(apply.b, x, DT_BF16, nz, a.rows, p.pitch, p.pitch, 64, 64);
    } else {
      MAP(gram.a, x, DT_BF16, nz, a.rows, p.pitch, p.pitch, 64, 64);
      gram.b = gram.a;
      MAP(apply.a, x, DT_BF16, nz, a.rows, p.pitch, p.pitch, 64, prod::BM);
    }
    MAP(apply.o, ws + p.x[(i + 1) & 1], DT_BF16, nz, a.rows, p.pitch, p.pitch, 32, 32);
    apply.last = i + 1 == a.steps;
    DO(go(gram));
    DO(go(square));
    DO(go(apply));
  }
  return cudaSuccess;
}

}  // namespace

size_t orthogonalize_workspace(const ra_orthogonalize_args& a) { return plan(a).bytes; }
cudaError_t orthogonalize(const ra_orthogonalize_args& a, cudaStream_t st) {
  return a.dtype == RA_BF16 ? run<bf16>(a, st) : run<float>(a, st);
}

}  // namespace ra
