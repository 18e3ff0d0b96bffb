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

constexpr int NORM_CTAS = 512;  // parts of a matrix's sum of squares, at most

// VEC elements at c, c + 1, .. of a row (VEC 1: at any place)
template <typename T, int VEC>
__device__ __forceinline__ void elements(const T* p, float* v) {
  if constexpr (VEC == 1) {
    v[0] = to_f(*p);
  } else {
    const uint4 x = *reinterpret_cast<const uint4*>(p);
    const T* h = reinterpret_cast<const T*>(&x);
#pragma unroll
    for (int i = 0; i < VEC; ++i) v[i] = to_f(h[i]);
  }
}

// Sums of squares of the elements by their size, scaled so that none overflows or vanishes: those above 2^50 by 2^-140, those
// below 2^-50 by 2^140, and the others.  A warp a row.
template <typename T, int VEC>
__global__ void __launch_bounds__(256) orth_norm_kernel(const ra_orthogonalize_args a, float* norms) {
  pdl_wait();
  pdl_trigger();
  const int m = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  float s[3] = {0.f, 0.f, 0.f};
  for (int r = blockIdx.x * 8 + warp; r < a.rows; r += gridDim.x * 8) {
    const T* row = static_cast<const T*>(a.x_dev) + m * a.x_matrix_stride + r * a.x_stride;
#pragma unroll 4
    for (int c = lane * VEC; c < a.cols; c += 32 * VEC) {
      float v[VEC];
      elements<T, VEC>(row + c, v);
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const float av = fabsf(v[i]);
        const bool big = av > 0x1p50f, small = av < 0x1p-50f;
        const float w = v[i] * (big ? 0x1p-70f : small ? 0x1p70f : 1.f), q = w * w;
        s[0] += big ? q : 0.f;
        s[1] += big || small ? 0.f : q;
        s[2] += small ? q : 0.f;
      }
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
  __device__ __forceinline__ float power(float v) const { return v * p * q; }
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

// The scaled matrices in planes [n][planes][rows][pitch].  One plane (bf16): scaled by the power of two alone, exactly; the
// factor, which goes to factors[m], is left to the first step's products.  No plane: into out.
template <typename T, int VEC>
__global__ void __launch_bounds__(256) orth_start_kernel(const ra_orthogonalize_args a, const float* norms, int parts, float* factors, bf16* x, int planes, int pitch) {
  __shared__ Scale sh;
  pdl_wait();
  pdl_trigger();
  const int m = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (warp == 0) {
    const Scale mine = scale_of(norms + (int64_t)m * parts * 3, parts, a.eps);
    if (lane == 0) {
      sh = mine;
      if (blockIdx.x == 0) factors[m] = mine.f;
    }
  }
  __syncthreads();
  const Scale s = sh;
  const int64_t plane = (int64_t)a.rows * pitch;
  for (int r = blockIdx.x * 8 + warp; r < a.rows; r += gridDim.x * 8) {
    const T* row = static_cast<const T*>(a.x_dev) + m * a.x_matrix_stride + r * a.x_stride;
    if (planes == 0) {
      for (int c = lane; c < a.cols; c += 32)
        static_cast<T*>(a.out_dev)[m * a.out_matrix_stride + r * a.out_stride + c] = from_f<T>(s(to_f(row[c])));
      continue;
    }
    bf16* d = x + ((int64_t)m * planes * a.rows + r) * pitch;
#pragma unroll 4
    for (int c = lane * VEC; c < pitch; c += 32 * VEC) {  // (cols is a multiple of VEC)
      float v[VEC];
#pragma unroll
      for (int i = 0; i < VEC; ++i) v[i] = 0.f;
      if (c < a.cols) elements<T, VEC>(row + c, v);
      auto store = [&](int k, const bf16* h) {
        if constexpr (VEC == 1) d[k * plane + c] = h[0];
        else if constexpr (VEC == 4) *reinterpret_cast<uint2*>(d + k * plane + c) = *reinterpret_cast<const uint2*>(h);
        else *reinterpret_cast<uint4*>(d + k * plane + c) = *reinterpret_cast<const uint4*>(h);
      };
      __align__(16) bf16 h[VEC];
      if (planes == 1) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) h[i] = __float2bfloat16_rn(s.power(v[i]));
        store(0, h);
      } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = s(v[i]);
#pragma unroll
        for (int k = 0; k < 3; ++k) {
#pragma unroll
          for (int i = 0; i < VEC; ++i) {
            h[i] = __float2bfloat16_rz(v[i]);
            prod::plane_trunc(v[i]);
          }
          store(k, h);
        }
      }
    }
  }
}

struct OrthArgs {
  CUtensorMap a, b, out;   // the product's operands; the result
  prod::Shape shape;
  unsigned* err;
  const float* factors;    // of the first step's matrices: P is scaled by the power'th power of its factor
  bf16 *o, *o2;            // P + add I and, if wanted, mul2 P + add2 I in planes [n][planes][rows][pitch]
  int pitch, power;
  void* dst;
  int64_t dst_stride, dst_matrix_stride;
  int rows, cols;          // of the product
  int k, n, pa, pb, cg, dtype;
  bool a_mn, b_mn, sym, last, map_out;
  float add, add2, mul2;
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

template <int PLANES>
struct Step {
  using Args = OrthArgs;
  // of a symmetric product (square tiles) those on and above the diagonal, column by column of tiles
  static __host__ __device__ __forceinline__ int tiles(const Args& p, int& mt, int& nt) {
    mt = (p.rows + prod::BM * p.cg - 1) / (prod::BM * p.cg);
    nt = (p.cols + p.shape.bn - 1) / p.shape.bn;
    return p.sym ? nt * (nt + 1) / 2 : mt * nt;
  }
  static __device__ __forceinline__ int count(const Args& p) {
    int mt, nt;
    return p.n * tiles(p, mt, nt);
  }
  static __device__ __forceinline__ void unit(const Args& p, int u, Unit& w) {
    int m_n, n_n, mt, nt;
    const int each = tiles(p, m_n, n_n);
    w.z = u / each;
    u %= each;
    if (p.sym) {
      nt = (int)((sqrtf(8.f * u + 1.f) - 1.f) * 0.5f);
      while (nt * (nt + 1) / 2 > u) --nt;
      while ((nt + 1) * (nt + 2) / 2 <= u) ++nt;
      mt = u - nt * (nt + 1) / 2;
    } else {
      prod::tile_of(u, m_n, n_n, mt, nt);
    }
    w.a = &p.a;
    w.b = &p.b;
    w.m0 = w.ar = mt * prod::BM * p.cg;
    w.n0 = w.br = nt * p.shape.bn;
    w.ak = w.bk = w.kb0 = 0;
    w.job = p.sym && mt != nt;  // its mirror image too
    w.az = w.z * p.pa;
    w.bz = w.z * p.pb;
    w.kb1 = (p.k + prod::BK - 1) / prod::BK;
    w.a_mn = p.a_mn;
    w.b_mn = p.b_mn;
  }
  template <typename F>
  static __device__ __forceinline__ void put(const Args& p, const Unit& w, bf16* to, F f, int row, int col, int lane) {
    const int64_t plane = (int64_t)p.rows * p.pitch;
    bf16* base = to + (int64_t)w.z * PLANES * plane;
    prod::planes_out<PLANES>(base + (int64_t)row * p.pitch + col, plane, f, row < p.rows, p.pitch - col);
    if (w.job) prod::planes_mirrored<PLANES>(base + (int64_t)col * p.pitch + (row & ~1), plane, f, p.pitch, p.rows - col, row < p.pitch, lane);
  }
  static __device__ __forceinline__ void finish(const Args& p, const Unit& w, const Tile& t, Store& st, float (&v)[4][32]) {
    const int row0 = w.m0 + t.rank * prod::BM + t.quad * 32, row = row0 + t.lane;
    if (row0 >= p.rows) return;
    float f = 1.f;
    if (p.power) {
      f = p.factors[w.z];
      if (p.power == 2) f *= f;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int col = w.n0 + 32 * (t.half + 2 * i);
      if (i >= t.chunks || col >= p.cols) break;
      if (p.power)
#pragma unroll
        for (int j = 0; j < 32; ++j) v[i][j] *= f;
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
      put(p, w, p.o, [&](int j) { return v[i][j] + (j == diag ? p.add : 0.f); }, row, col, t.lane);
      if (p.o2) put(p, w, p.o2, [&](int j) { return p.mul2 * v[i][j] + (j == diag ? p.add2 : 0.f); }, row, col, t.lane);
    }
  }
};

struct Plan {
  int planes, low, high, pitch, low_pitch, parts;
  size_t norms, factors, x[2], s, t, q, bytes;
};
Plan plan(const ra_orthogonalize_args& a) {
  Plan p = {};
  p.planes = a.dtype == RA_F32 ? 3 : 2;
  p.low = std::min(a.rows, a.cols);
  p.high = std::max(a.rows, a.cols);
  p.pitch = up(a.cols, 8);
  p.low_pitch = up(p.low, 8);
  p.parts = std::min(std::max(1, NORM_CTAS / a.n_matrices), parts_of(a.rows, 8));
  size_t at = WS_ZERO;
  auto take = [&](size_t n) {
    const size_t r = at;
    at += (n + 255) / 256 * 256;
    return r;
  };
  const size_t n = (size_t)a.n_matrices * p.planes * 2;
  p.norms = take((size_t)a.n_matrices * p.parts * 3 * 4);
  p.factors = take((size_t)a.n_matrices * 4);
  for (size_t& x : p.x) x = take(n * a.rows * p.pitch);
  p.s = take(n * p.low * p.low_pitch);
  p.t = take(n * p.low * p.low_pitch);
  p.q = take(n * p.low * p.low_pitch);
  p.bytes = at;
  return p;
}

// ... of a symmetric product: square tiles, about half of them
Pick pick_sym(int rows, int n, int blocks) {
  auto time = [&](Pick k) {
    const int64_t t = parts_of(rows, k.bn);
    return (double)parts_of(n * t * (t + 1) / 2, prod::SMS / k.cg) * (blocks * prod::block_time(k) + 1.5) + (k.cg == 2 ? 1. : 0.);
  };
  const Pick one = {1, 128}, two = {2, 256};
  return rows > 128 && time(two) < time(one) ? two : one;
}

template <typename T>
cudaError_t run(const ra_orthogonalize_args& a, cudaStream_t st) {
  const Plan p = plan(a);
  char* ws = static_cast<char*>(a.workspace_dev);
  const int n = a.n_matrices, nz = n * p.planes;
  const bool wide = a.rows <= a.cols;
  float *norms = reinterpret_cast<float*>(ws + p.norms), *factors = reinterpret_cast<float*>(ws + p.factors);
  bf16* x[2] = {reinterpret_cast<bf16*>(ws + p.x[0]), reinterpret_cast<bf16*>(ws + p.x[1])};
  bf16 *s = reinterpret_cast<bf16*>(ws + p.s), *t = reinterpret_cast<bf16*>(ws + p.t), *q = reinterpret_cast<bf16*>(ws + p.q);
  constexpr int es = sizeof(T), V = 16 / es;
  // bf16 matrices are one plane as they come
  const int first = a.steps == 0 ? 0 : es == 2 ? 1 : 3;
  {
    const bool vec = ((uintptr_t)a.x_dev & 15) == 0 && a.cols % V == 0 && a.x_stride % V == 0 && (n == 1 || a.x_matrix_stride % V == 0);
    const dim3 ng(p.parts, n), sg(std::min(parts_of(a.rows, 8), std::max(16, 2432 / n)), n);
    note_launch(2);
    DO(launch_pdl(vec ? orth_norm_kernel<T, V> : orth_norm_kernel<T, 1>, ng, dim3(256), 0, st, a, norms));
    DO(launch_pdl(vec ? orth_start_kernel<T, V> : orth_start_kernel<T, 1>, sg, dim3(256), 0, st, a, (const float*)norms, p.parts, factors, x[0], first,
                  p.pitch));
  }
  if (a.steps == 0) return cudaSuccess;

  const int chunk = p.planes == 3 ? 4 : 32;
  OrthArgs g = {};
  g.err = a.err_dev;
  g.factors = factors;
  g.n = n;
  g.dtype = a.dtype;
  auto shape = [&](OrthArgs& s, int rows, int cols, int k, int pa, int pb, bool sym) {
    const prod::Terms terms = prod::terms_of(pa, pb);
    const int blocks = parts_of(k, prod::BK) * terms.n;
    const Pick c = sym ? pick_sym(rows, n, blocks) : prod::pick(rows, cols, n, blocks);
    s.rows = rows;
    s.cols = cols;
    s.k = k;
    s.pa = pa;
    s.pb = pb;
    s.sym = sym;
    s.cg = c.cg;
    s.shape = prod::shape_of(c.bn, c.cg, terms, chunk);
  };
  auto go = [&](const OrthArgs& s) {
    int mt, nt;
    using S = Step<es == 2 ? 2 : 3>;
    const int u = (int)std::min<int64_t>((int64_t)n * S::tiles(s, mt, nt), 1 << 20);
    return s.cg == 2 ? prod::launch<S, 2>(s, u, st) : prod::launch<S, 1>(s, u, st);
  };
  OrthArgs square = g;
  shape(square, p.low, p.low, p.low, p.planes, p.planes, true);
  square.add = a.a;
  square.o = q;
  square.pitch = p.low_pitch;
  MAP(square.a, s, DT_BF16, nz, p.low, p.low_pitch, p.low_pitch, 64, prod::BM);
  MAP(square.b, t, DT_BF16, nz, p.low, p.low_pitch, p.low_pitch, 64, square.shape.bn / square.cg);
  for (int i = 0; i < a.steps; ++i) {
    const int px = i == 0 ? first : p.planes;
    const bf16* from = x[i & 1];
    OrthArgs gram = g, apply = g;
    shape(gram, p.low, p.low, p.high, px, px, true);
    gram.a_mn = gram.b_mn = !wide;
    gram.power = px == 1 ? 2 : 0;
    gram.o = s;
    gram.o2 = t;
    gram.add2 = a.b;
    gram.mul2 = a.c;
    gram.pitch = p.low_pitch;
    shape(apply, a.rows, a.cols, p.low, wide ? p.planes : px, wide ? px : p.planes, false);
    apply.b_mn = wide;
    apply.power = px == 1 ? 1 : 0;
    apply.o = x[(i + 1) & 1];
    apply.pitch = p.pitch;
    if (wide) {
      MAP(gram.a, from, DT_BF16, n * px, a.rows, p.pitch, p.pitch, 64, prod::BM);
      MAP(gram.b, from, DT_BF16, n * px, a.rows, p.pitch, p.pitch, 64, gram.shape.bn / gram.cg);
      MAP(apply.a, q, DT_BF16, nz, p.low, p.low_pitch, p.low_pitch, 64, prod::BM);
      MAP(apply.b, from, DT_BF16, n * px, a.rows, p.pitch, p.pitch, 64, 64);
    } else {
      MAP(gram.a, from, DT_BF16, n * px, a.rows, p.pitch, p.pitch, 64, 64);
      gram.b = gram.a;
      MAP(apply.a, from, DT_BF16, n * px, a.rows, p.pitch, p.pitch, 64, prod::BM);
      MAP(apply.b, q, DT_BF16, nz, p.low, p.low_pitch, p.low_pitch, 64, apply.shape.bn / apply.cg);
    }
    if ((apply.last = i + 1 == a.steps)) {
      apply.dst = a.out_dev;
      apply.dst_stride = a.out_stride;
      apply.dst_matrix_stride = a.out_matrix_stride;
      // by TMA where rows are at 16-byte boundaries and matrices one after the other
      apply.map_out = ((uintptr_t)a.out_dev & 15) == 0 && a.out_stride * es % 16 == 0 && (int64_t)a.cols * es % 16 == 0 &&
                      (n == 1 || a.out_matrix_stride == a.rows * a.out_stride);
      if (apply.map_out) MAP(apply.out, a.out_dev, a.dtype, n, a.rows, a.cols, a.out_stride, es == 2 ? 32 : 16, 32);
    }
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
