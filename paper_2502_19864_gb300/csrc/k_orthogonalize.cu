// k_orthogonalize.cu -- orthogonalisation of updates by Newton-Schulz products.
//
// X = x / (|x| + eps); then `steps` times X <- (a I + S (b I + c S)) X with S = X X^T (rows <= cols), or, which is the same
// polynomial of X, X <- X (a I + S (b I + c S)) with S = X^T X: S has the smaller of the two sides.  A step is three
// products on the tensor cores: S; Q = a I + b S + c S S; and X.
//
// Operands are planes of bf16 (products.cuh).  For fp32 three, the significand whole.  For bf16 matrices two, 17 bits: a
// step raises what lies along small singular values by up to 3.4445 while the large ones stay, so that an error of the first
// steps grows with them, about 140-fold by the last; 2^-17 is then a quarter of the output's own rounding at
// worst, where one plane's 2^-9 would be as large as what is computed.
//
// Bound: the products, 1.5 low^2 high + low^3 / 2 multiply-adds a step with the symmetric ones' halves, three (six) times over for
// the planes; of small matrices the launches.  2048 x 5632 in bf16 0.80 ms for five steps, 2 x 777 x 1000 in fp32 0.31 ms.
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

// Sums of squares by the elements' size, scaled so that none overflows or vanishes: those above 2^50 by 2^-140, those below 2^-50
// by 2^140 (s[2]), and the others (s[1])
__device__ __forceinline__ void add_square(float v, float (&s)[3]) {
  const float av = fabsf(v);
  const bool big = av > 0x1p50f, small = av < 0x1p-50f;
  const float w = v * (big ? 0x1p-70f : small ? 0x1p70f : 1.f), q = w * w;
  s[0] += big ? q : 0.f;
  s[1] += big || small ? 0.f : q;
  s[2] += small ? q : 0.f;
}
// N elements' squares, as they are where their sum has room on both sides
template <int N>
__device__ __forceinline__ void add_squares(const float* v, float (&s)[3]) {
  float q = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) q = fmaf(v[i], v[i], q);
  if (q > 0x1p-60f && q < 0x1p100f) {
    s[1] += q;
  } else {
#pragma unroll 1
    for (int i = 0; i < N; ++i) add_square(v[i], s);
  }
}
// ... of a matrix's parts.  A warp a row.
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
      add_squares<VEC>(v, s);
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
  float p, q, f, fq;  // (the powers, the factor, and the factor times the second power)
  __device__ __forceinline__ float power(float v) const { return v * p * q; }
  __device__ __forceinline__ float operator()(float v) const { return v * p * fq; }
};
// (by a warp)
__device__ __forceinline__ Scale scale_of(const float* norms, int parts, float eps) {
  double t = 0.;
  for (int i = threadIdx.x & 31; i < parts; i += 32) t += (double)norms[3 * i] * 0x1p140 + (double)norms[3 * i + 1] + (double)norms[3 * i + 2] * 0x1p-140;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
  if (!isfinite(t)) return {1.f, 1.f, NAN, NAN};
  const double s = 1. / (sqrt(t) + (double)eps);
  if (!isfinite(s)) return {1.f, 1.f, 1.f, 1.f};  // (all zeros, and eps too)
  int e;
  const double f = 2. * frexp(s, &e);
  --e;
  const float q = ldexpf(1.f, e - e / 2);
  return {ldexpf(1.f, e / 2), q, (float)f, (float)f * q};
}

// The scaled matrices in planes [n][planes][rows][pitch], zeros behind cols up to width.  One plane (bf16): scaled by the power of two alone, exactly; the
// factor, which goes to factors[m], is left to the first step's products.  No plane: into out.
template <typename T, int VEC>
__global__ void __launch_bounds__(256) orth_start_kernel(const ra_orthogonalize_args a, const float* norms, int parts, float* factors, bf16* x, int planes, int width, int pitch) {
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
    for (int c = lane * VEC; c < width; c += 32 * VEC) {  // (cols is a multiple of VEC)
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
  CUtensorMap a, b, out;   // the product's operands; the result, or its planes [n][planes][rows][pitch]
  prod::Shape shape;
  unsigned* err;
  const float* factors;    // of the first step's matrices: P is scaled by the power'th power of its factor
  const bf16* with;        // not NULL: the result is mul P + mul_with W + add I, W in planes like its own; else P
  bf16* o;                 // (the ranges' sums': its planes)
  int width, pitch, power;  // (width: the columns that are written, to a multiple of 8)
  void* dst;
  int64_t dst_stride, dst_matrix_stride;
  int rows, cols;          // of the product
  int k, n, cg, dtype;
  bool a_mn, b_mn, sym, last, map_out;
  float add, mul, mul_with;
  // a symmetric product of few tiles: K in `splits` ranges of `blocks` k-blocks, whose sums go to sums [splits][n][rows][sums_pitch]
  int splits, blocks, sums_pitch;
  const float* sums;
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

// PLANES: of what is kept; A_PLANES, B_PLANES: of the operands
template <int PLANES, int A_PLANES, int B_PLANES>
struct Step {
  static constexpr int PA = A_PLANES, PB = B_PLANES;
  // (bf16: what an accumulator of 32768 products loses, 3.5e-5 of them, is of the size of what two planes leave out)
  static constexpr bool PARTS = true, ONE = PLANES == 2;
  using Args = OrthArgs;
  // of a symmetric product (square tiles) those on and above the diagonal, column by column of tiles
  static __host__ __device__ __forceinline__ int tiles(const Args& p, int& mt, int& nt) {
    mt = (p.rows + prod::BM * p.cg - 1) / (prod::BM * p.cg);
    nt = (p.cols + p.shape.bn - 1) / p.shape.bn;
    return p.sym ? nt * (nt + 1) / 2 : mt * nt;
  }
  static __device__ __forceinline__ void prefetch(const Args& p) {
    prod::prefetch_map(&p.a);
    prod::prefetch_map(&p.b);
  }
  static __device__ __forceinline__ int count(const Args& p) {
    int mt, nt;
    return p.n * tiles(p, mt, nt) * p.splits;
  }
  static __device__ __forceinline__ void unit(const Args& p, int u, Unit& w) {
    int m_n, n_n, mt, nt;
    const int each = tiles(p, m_n, n_n), range = u % p.splits;
    u /= p.splits;
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
    w.kb0 = range * p.blocks;
    w.ak = w.bk = 0;
    w.job = p.splits > 1 ? range : p.sym && mt != nt;  // the range; or: its mirror image too
    w.az = w.z * PA;
    w.bz = w.z * PB;
    w.kb1 = min(w.kb0 + p.blocks, (p.k + prod::BK - 1) / prod::BK);
    w.a_mn = p.a_mn;
    w.b_mn = p.b_mn;
  }
  static __device__ __forceinline__ void part(const Args& p, const Unit& w, const Tile& t, Store& st, int i, float (&v)[32]) {
    const int row0 = w.m0 + t.rank * prod::BM + t.quad * 32, row = row0 + t.lane, col = w.n0 + 32 * (t.half + 2 * i);
    if (row0 >= p.rows || col >= p.cols) return;
    if (p.power) {
      float f = p.factors[w.z];
      if (p.power == 2) f *= f;
#pragma unroll
      for (int j = 0; j < 32; ++j) v[j] *= f;
    }
    if (p.splits > 1) {
      st.f32_row(&p.out, v, col, row0, w.job * p.n + w.z, false, p.sums_pitch);
      return;
    }
    if (p.last) {
      if (p.map_out) {
        if (p.dtype == RA_BF16) st.bf16_row(&p.out, [&](int j) { return v[j]; }, col, row0, w.z);
        else st.f32_row(&p.out, v, col, row0, w.z, false, p.cols);
      } else {
        const int64_t at = w.z * p.dst_matrix_stride + row0 * p.dst_stride + col + t.lane;
        st.by_columns(v, [&](int r, float x) {
          if (row0 + r >= p.rows || col + t.lane >= p.cols) return;
          if (p.dtype == RA_BF16) static_cast<bf16*>(p.dst)[at + r * p.dst_stride] = __float2bfloat16_rn(x);
          else static_cast<float*>(p.dst)[at + r * p.dst_stride] = x;
        });
      }
      return;
    }
    if (p.with) {
      const bf16* from = p.with + (int64_t)w.z * PLANES * p.rows * p.pitch + (int64_t)row0 * p.pitch + col;
      uint32_t h[PLANES][16];
#pragma unroll
      for (int k = 0; k < PLANES; ++k)  // (a warp's load: 64 bytes of eight rows)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int r = (t.lane & ~3) + q, c = 8 * (t.lane & 3);
          uint4 u = make_uint4(0, 0, 0, 0);
          if (row0 + r < p.rows && col + c < p.width) u = *reinterpret_cast<const uint4*>(from + ((int64_t)k * p.rows + r) * p.pitch + c);
          h[k][4 * q] = u.x, h[k][4 * q + 1] = u.y, h[k][4 * q + 2] = u.z, h[k][4 * q + 3] = u.w;
        }
      float x[32];
#pragma unroll
      for (int k = PLANES - 1; k >= 0; --k) {
        tc::transpose4(h[k], t.lane);
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const float lo = __uint_as_float(h[k][j] << 16), hi = __uint_as_float(h[k][j] & 0xffff0000u);
          x[2 * j] = k + 1 < PLANES ? x[2 * j] + lo : lo;
          x[2 * j + 1] = k + 1 < PLANES ? x[2 * j + 1] + hi : hi;
        }
      }
      const int diag = row < p.rows ? row - col : -1;  // (nothing behind the last row)
#pragma unroll
      for (int j = 0; j < 32; ++j) v[j] = fmaf(p.mul, v[j], fmaf(p.mul_with, x[j], j == diag ? p.add : 0.f));
    }
    auto at = [&](int j) { return v[j]; };
    st.planes<PLANES, false>(&p.out, at, col, row0, w.z * PLANES);
    if (w.job) st.planes<PLANES, true>(&p.out, at, row0, col, w.z * PLANES);
  }
};

// The symmetric product from the ranges' sums, in order: a CTA a 32 x 32 block on or above the diagonal, and its mirror image
template <int PLANES>
__global__ void __launch_bounds__(256) orth_join_kernel(const OrthArgs p) {
  __shared__ float tile[32][33];
  pdl_wait();
  pdl_trigger();
  int bj = (int)((sqrtf(8.f * blockIdx.x + 1.f) - 1.f) * 0.5f);
  while (bj * (bj + 1) / 2 > (int)blockIdx.x) --bj;
  while ((bj + 1) * (bj + 2) / 2 <= (int)blockIdx.x) ++bj;
  const int bi = (int)blockIdx.x - bj * (bj + 1) / 2, z = blockIdx.y, r = threadIdx.x >> 3, c = 4 * (threadIdx.x & 7);
  const int64_t plane = (int64_t)p.rows * p.pitch, range = (int64_t)p.n * p.rows * p.sums_pitch;
  auto put = [&](const float* v, int row, int col) {
    if (row >= p.rows || col >= p.width) return;
    const int64_t at = (int64_t)z * PLANES * plane + (int64_t)row * p.pitch + col;
    float x[4] = {v[0], v[1], v[2], v[3]};
    if (p.with) {
      float w[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = PLANES - 1; k >= 0; --k) {
        const uint2 h = *reinterpret_cast<const uint2*>(p.with + at + k * plane);
        w[0] += __uint_as_float(h.x << 16), w[1] += __uint_as_float(h.x & 0xffff0000u);
        w[2] += __uint_as_float(h.y << 16), w[3] += __uint_as_float(h.y & 0xffff0000u);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = fmaf(p.mul, x[j], fmaf(p.mul_with, w[j], row == col + j ? p.add : 0.f));
    }
    uint32_t lo[PLANES], hi[PLANES];
    prod::planes_of<PLANES>(x[0], x[1], lo);
    prod::planes_of<PLANES>(x[2], x[3], hi);
    bf16* to = p.o + at;
#pragma unroll
    for (int k = 0; k < PLANES; ++k) *reinterpret_cast<uint2*>(to + k * plane) = make_uint2(lo[k], hi[k]);
  };
  float v[4] = {0.f, 0.f, 0.f, 0.f};
  if (32 * bi + r < p.rows) {
    const float* from = p.sums + ((int64_t)z * p.rows + 32 * bi + r) * p.sums_pitch + 32 * bj + c;
#pragma unroll 4
    for (int s = 0; s < p.splits; ++s) {
      const float4 x = *reinterpret_cast<const float4*>(from + s * range);
      v[0] += x.x, v[1] += x.y, v[2] += x.z, v[3] += x.w;
    }
  }
  put(v, 32 * bi + r, 32 * bj + c);
  if (bi == bj) return;
#pragma unroll
  for (int j = 0; j < 4; ++j) tile[r][c + j] = v[j];
  __syncthreads();
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = tile[c + j][r];
  put(v, 32 * bj + r, 32 * bi + c);
}

// ---- matrices whose smaller side is at most 64 --------------------------------------------------
// An adapter's matrix stays on chip through all steps: a cluster of up to eight CTAs has one matrix, each CTA `blocks` blocks
// of 64 of the longer side's indexes (rows, say; a wide matrix comes transposed), in planes in shared memory,
// [block][64 rows][64 of the shorter side], 128-byte swizzled.  S is the sum of the CTAs' products X^T X, which they leave
// for one another in shared memory and each adds up, in the same order; S T and X Q each CTA does by itself.  The same storage is an
// MN-major operand of X^T X and a K-major one of X Q.
// Bound: latency.  A step is three products' issue and read-out and one meeting of the cluster: 48 of 1024 x 64 in bf16 take 6.6 us a
// step and 46 us in all (three launches of the products above a step: 200 us in all), 8 of 128 x 16 in fp32 29 us (91 us).
constexpr int SMALL = 64, SMALL_THREADS = 512, SMALL_BLOCK = SMALL * 128;  // bytes of a block's plane
constexpr int PART_PITCH = SMALL + 4;                                      // of S in fp32: rows four banks apart
constexpr int PART_BYTES = SMALL * PART_PITCH * 4;
template <int PL>
constexpr int small_blocks() { return PL == 2 ? 9 : 5; }  // that shared memory holds
template <int PL>
constexpr int small_smem() { return PL * (small_blocks<PL>() + 2) * SMALL_BLOCK + 2 * PART_BYTES + 1024; }

struct SmallArgs {
  ra_orthogonalize_args a;
  int blocks, ctas;  // of a CTA; of a cluster
  bool tall, vec_in, vec_out;
  prod::Terms terms;
};

template <typename T, int PL>
__global__ void __launch_bounds__(SMALL_THREADS, 1) orth_small_kernel(const __grid_constant__ SmallArgs p) {
  using namespace tc;
  extern __shared__ uint8_t raw[];
  __shared__ __align__(8) uint64_t bar;
  __shared__ uint32_t tmem_sh;
  __shared__ volatile int abort_sh;
  __shared__ float norm_sh[3], norms_sh[8 * 3], warp_sh[16][3];
  __shared__ Scale scale_sh;
  constexpr int V = 16 / (int)sizeof(T);
  const ra_orthogonalize_args& a = p.a;
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~static_cast<uintptr_t>(1023));
  const int tid = threadIdx.x, warp = warp_index(), lane = tid & 31, quad = warp & 3, grp = warp >> 2;  // (16 of 64 columns)
  const int HB = p.blocks, CS = p.ctas, rank = (int)blockIdx.x % CS, m = (int)blockIdx.x / CS;
  const int low = p.tall ? a.cols : a.rows, high = p.tall ? a.rows : a.cols, rows = HB * SMALL, first = rank * rows;
  uint8_t *xs = smem, *ss = xs + PL * HB * SMALL_BLOCK, *ts = ss + PL * SMALL_BLOCK;
  float* part = reinterpret_cast<float*>(ts + PL * SMALL_BLOCK);
  const uint32_t xa = smem_u32(xs), sa = smem_u32(ss), ta = smem_u32(ts);

  if (tid == 0) {
    mbar_init(&bar, 1);
    abort_sh = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_sh)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_sh;
  pdl_wait();
  pdl_trigger();

  // ---- the matrix, in units of eight of a row's elements; where they are 32 bytes or less at a 16-byte boundary, a thread's all
  // at once on their way, and held until the norm is there; else four at a time, twice
  const T* x = static_cast<const T*>(a.x_dev) + m * a.x_matrix_stride;
  const int units = rows * 8;
  const bool hold = p.tall && p.vec_in;
  constexpr int HELD = small_blocks<PL>() * 512 / SMALL_THREADS, PIECES = 8 / V;
  uint4 held[HELD][PIECES];
  auto place = [&](int u, int& r, int& j) {
    r = p.tall ? u >> 3 : u % rows;  // (neighbours in memory to neighbouring threads)
    j = p.tall ? u & 7 : u / rows;
  };
  auto scattered = [&](int u, float (&v)[8]) {
    int r, j;
    place(u, r, j);
    const int hi = first + r, lo = 8 * j;
#pragma unroll
    for (int c = 0; c < 8; ++c)
      v[c] = u < units && hi < high && lo + c < low ? to_f(x[p.tall ? hi * a.x_stride + lo + c : (lo + c) * a.x_stride + hi]) : 0.f;
  };
  float s3[3] = {0.f, 0.f, 0.f};
  if (hold) {
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
      const int u = tid + i * SMALL_THREADS, hi = first + (u >> 3), lo = 8 * (u & 7);
#pragma unroll
      for (int q = 0; q < PIECES; ++q) {
        held[i][q] = make_uint4(0, 0, 0, 0);
        if (u < units && hi < high && lo + V * q < low) held[i][q] = *reinterpret_cast<const uint4*>(x + hi * a.x_stride + lo + V * q);
      }
    }
#pragma unroll
    for (int i = 0; i < HELD; ++i)
#pragma unroll
      for (int q = 0; q < PIECES; ++q) {
        const T* h = reinterpret_cast<const T*>(&held[i][q]);
        float v[V];
#pragma unroll
        for (int c = 0; c < V; ++c) v[c] = to_f(h[c]);
        if (tid + i * SMALL_THREADS < units) add_squares<V>(v, s3);
      }
  } else {
    for (int u0 = tid; u0 < units; u0 += 4 * SMALL_THREADS) {
      float v[4][8];
#pragma unroll
      for (int i = 0; i < 4; ++i) scattered(u0 + i * SMALL_THREADS, v[i]);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (u0 + i * SMALL_THREADS < units) add_squares<8>(v[i], s3);
    }
  }
#pragma unroll
  for (int k = 0; k < 3; ++k) s3[k] = warp_sum(s3[k]);
  if (lane == 0)
    for (int k = 0; k < 3; ++k) warp_sh[warp][k] = s3[k];
  __syncthreads();
  if (tid < 3) {
    float t = 0.f;
    for (int w = 0; w < SMALL_THREADS / 32; ++w) t += warp_sh[w][tid];
    norm_sh[tid] = t;
  }
  auto meet = [&]() {  // the cluster's writes to shared memory are seen by all of it
    if (CS > 1) {
      cluster_arrive();
      cluster_wait();
    } else {
      __syncthreads();
    }
  };
  auto far = [&](const float* q, int of) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(peer_addr(smem_u32(q), of)) : "memory");
    return v;
  };
  meet();
  if (tid < 3 * CS) norms_sh[tid] = CS > 1 ? far(norm_sh + tid % 3, tid / 3) : norm_sh[tid];
  __syncthreads();
  if (warp == 0) {
    const Scale mine = scale_of(norms_sh, CS, a.eps);
    if (lane == 0) scale_sh = mine;
  }
  __syncthreads();
  const Scale scale = scale_sh;
  // eight values' planes to chunk j of row r of a 64-row block
  auto planes8 = [&](uint8_t* to, int step, int r, int j, const float* v) {
    uint32_t w[4][PL];
#pragma unroll
    for (int i = 0; i < 4; ++i) prod::planes_of<PL>(v[2 * i], v[2 * i + 1], w[i]);
#pragma unroll
    for (int k = 0; k < PL; ++k) *reinterpret_cast<uint4*>(to + k * step + swz(r, j)) = make_uint4(w[0][k], w[1][k], w[2][k], w[3][k]);
  };
  auto keep = [&](int u, float (&v)[8]) {
    int r, j;
    place(u, r, j);
    if (u >= units) return;
#pragma unroll
    for (int c = 0; c < 8; ++c) v[c] = scale(v[c]);
    planes8(xs + (r >> 6) * SMALL_BLOCK, HB * SMALL_BLOCK, r & 63, j, v);
  };
  if (hold) {
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
      float v[8];
#pragma unroll
      for (int q = 0; q < PIECES; ++q) {
        const T* h = reinterpret_cast<const T*>(&held[i][q]);
#pragma unroll
        for (int c = 0; c < V; ++c) v[V * q + c] = to_f(h[c]);
      }
      keep(tid + i * SMALL_THREADS, v);
    }
  } else {
    for (int u0 = tid; u0 < units; u0 += 4 * SMALL_THREADS) {
      float v[4][8];
#pragma unroll
      for (int i = 0; i < 4; ++i) scattered(u0 + i * SMALL_THREADS, v[i]);
#pragma unroll
      for (int i = 0; i < 4; ++i) keep(u0 + i * SMALL_THREADS, v[i]);
    }
  }

  uint32_t phase = 0;
  // what the threads wrote is an operand now; one thread issues f's products, all wait for them
  auto terms = [&](auto f) {
    for (int t = 0; t < p.terms.n; ++t) f(t, (int)(p.terms.a >> (2 * t) & 3u), (int)(p.terms.b >> (2 * t) & 3u));
  };
  auto products = [&](auto f) {
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    tc_fence_before();
    __syncthreads();
    if (warp == 0 && elect_one()) {
      tc_fence_after();
      f();
      umma_commit(&bar);
    }
    __syncwarp();
    mbar_wait(&bar, phase, &abort_sh, a.err_dev);
    phase ^= 1u;
    tc_fence_after();
  };
  constexpr uint32_t MN = idesc_bf16_abmn(128, SMALL), KK = idesc_bf16(128, SMALL);
  constexpr uint32_t C_S = 0, C_Q = PL == 2 ? 128 : 256, C_X = C_Q + 64;  // (C_X + 64 pairs <= 512)
  const int r = quad * 32 + lane;  // S and Q are with quads 0 and 1
  const uint32_t at = tmem + ((uint32_t)(quad * 32) << 16) + (uint32_t)(16 * grp);
  float* const parts[2] = {part, part + SMALL * PART_PITCH};
  const int pairs = (HB + 1) / 2;
  for (int step = 0; step < a.steps; ++step) {
    // planes 0 and 1 (64 rows of the product each) by all planes (64 columns each) at once, and plane 2 by plane 0
    products([&]() {
      const uint32_t plane = HB * SMALL_BLOCK;
      for (int b = 0; b < HB; ++b)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t at = xa + b * SMALL_BLOCK + k * 2048;
          umma_bf16(tmem + C_S, sdesc_mn_sw128_lbo(at, plane), sdesc_mn_sw128_lbo(at, plane), idesc_bf16_abmn(128, 64 * PL), (uint32_t)(b | k));
          if (PL == 3)
            umma_bf16(tmem + C_S + 64 * PL, sdesc_mn_sw128_lbo(at + 2 * plane, SMALL_BLOCK), sdesc_mn_sw128(at), MN, (uint32_t)(b | k));
        }
    });
    float v[16];
    float *mine = parts[step & 1], *low_rows = reinterpret_cast<float*>(ss);  // (Q is done with)
    {
      float y[16];
      tmem_ld16(at + C_S + 64, v);
      if (PL == 3 && quad < 2) {
        tmem_ld16(at + C_S + 64 * (PL - 1), y);
#pragma unroll
        for (int j = 0; j < 16; ++j) v[j] += y[j];
        tmem_ld16(at + C_S + 64 * PL, y);
#pragma unroll
        for (int j = 0; j < 16; ++j) v[j] += y[j];
      }
      tmem_ld16(at + C_S, y);
#pragma unroll
      for (int j = 0; j < 16; ++j) v[j] += y[j];
    }
    if (quad >= 2)
#pragma unroll
      for (int j = 0; j < 16; j += 4)
        *reinterpret_cast<float4*>(low_rows + (r - SMALL) * PART_PITCH + 16 * grp + j) = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
    __syncthreads();
    if (quad < 2)
#pragma unroll
      for (int j = 0; j < 16; j += 4) {
        const float4 y = *reinterpret_cast<const float4*>(low_rows + r * PART_PITCH + 16 * grp + j);
        v[j] += y.x;
        v[j + 1] += y.y;
        v[j + 2] += y.z;
        v[j + 3] += y.w;
        if (CS > 1) *reinterpret_cast<float4*>(mine + r * PART_PITCH + 16 * grp + j) = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
      }
    meet();
    if (CS > 1) {
      // the CTAs' sums, neighbouring threads on neighbouring pieces (a row a thread takes 32 lines of another SM's memory an
      // instruction: 2.5 us a CTA of the cluster), and back through this CTA's memory to the rows' threads
      constexpr int PIECES4 = SMALL * PART_PITCH / 4, EACH = (PIECES4 + SMALL_THREADS - 1) / SMALL_THREADS;
      float4 sum[EACH] = {};
#pragma unroll 2
      for (int c = 0; c < CS; ++c) {
        const uint32_t from = peer_addr(smem_u32(mine), c);
        float4 y[EACH];
#pragma unroll
        for (int i = 0; i < EACH; ++i)
          if (tid + i * SMALL_THREADS < PIECES4)
            asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(y[i].x), "=f"(y[i].y), "=f"(y[i].z), "=f"(y[i].w) : "r"(from + 16 * (tid + i * SMALL_THREADS)));
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
          sum[i].x += y[i].x;
          sum[i].y += y[i].y;
          sum[i].z += y[i].z;
          sum[i].w += y[i].w;
        }
      }
#pragma unroll
      for (int i = 0; i < EACH; ++i)
        if (tid + i * SMALL_THREADS < PIECES4) *reinterpret_cast<float4*>(low_rows + 4 * (tid + i * SMALL_THREADS)) = sum[i];
      __syncthreads();
      if (quad < 2)
#pragma unroll
        for (int j = 0; j < 16; j += 4) {
          const float4 y = *reinterpret_cast<const float4*>(low_rows + r * PART_PITCH + 16 * grp + j);
          v[j] = y.x;
          v[j + 1] = y.y;
          v[j + 2] = y.z;
          v[j + 3] = y.w;
        }
      __syncthreads();
    }
    const int diag = r < low ? r - 16 * grp : -1;
    if (quad < 2) {
#pragma unroll
      for (int q = 0; q < 2; ++q) planes8(ss, SMALL_BLOCK, r, 2 * grp + q, v + 8 * q);
#pragma unroll
      for (int j = 0; j < 16; ++j) v[j] = a.c * v[j] + (j == diag ? a.b : 0.f);
#pragma unroll
      for (int q = 0; q < 2; ++q) planes8(ts, SMALL_BLOCK, r, 2 * grp + q, v + 8 * q);
    }
    products([&]() {  // (S and T are symmetric; rows 64.. of the product are of what lies behind S's plane)
      terms([&](int t, int pa, int pb) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          umma_bf16(tmem + C_Q, sdesc_mn_sw128_lbo(sa + pa * SMALL_BLOCK + k * 2048, SMALL_BLOCK), sdesc_mn_sw128(ta + pb * SMALL_BLOCK + k * 2048), MN,
                    (uint32_t)(t | k));
      });
    });
    if (quad < 2) {
      tmem_ld16(at + C_Q, v);
#pragma unroll
      for (int j = 0; j < 16; ++j) v[j] += j == diag ? a.a : 0.f;
#pragma unroll
      for (int q = 0; q < 2; ++q) planes8(ss, SMALL_BLOCK, r, 2 * grp + q, v + 8 * q);  // Q, where S was
    }
    products([&]() {
      terms([&](int t, int pa, int pb) {
        for (int b = 0; b < pairs; ++b)
#pragma unroll
          for (int k = 0; k < 4; ++k)
            umma_bf16(tmem + C_X + 64 * b, sdesc_sw128(xa + (pa * HB + 2 * b) * SMALL_BLOCK + k * 32), sdesc_sw128(sa + pb * SMALL_BLOCK + k * 32), KK,
                      (uint32_t)(t | k));
      });
    });
    const bool last = step + 1 == a.steps;
    T* out = static_cast<T*>(a.out_dev) + m * a.out_matrix_stride;
    for (int b = 0; b < pairs; ++b) {
      __syncwarp();
      tmem_ld16(at + C_X + 64 * b, v);
      const int row = b * 128 + r;
      if (row >= rows) continue;
      if (!last) {
#pragma unroll
        for (int q = 0; q < 2; ++q) planes8(xs + (row >> 6) * SMALL_BLOCK, HB * SMALL_BLOCK, row & 63, 2 * grp + q, v + 8 * q);
        continue;
      }
      const int hi = first + row;
      if (hi >= high) continue;
      if (p.tall && p.vec_out) {
        T* o = out + hi * a.out_stride + 16 * grp;
#pragma unroll
        for (int j = 0; j < 16; j += V)
          if (16 * grp + j < low) {
            __align__(16) T h[V];
#pragma unroll
            for (int i = 0; i < V; ++i) h[i] = from_f<T>(v[j + i]);
            *reinterpret_cast<uint4*>(o + j) = *reinterpret_cast<const uint4*>(h);
          }
      } else {
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const int lo = 16 * grp + j;
          if (lo < low) out[p.tall ? hi * a.out_stride + lo : lo * a.out_stride + hi] = from_f<T>(v[j]);
        }
      }
    }
  }
  tc_fence_before();
  meet();  // (no CTA leaves while another reads its sums)
  if (warp == 0) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
  }
}

bool small_fits(const ra_orthogonalize_args& a) {
  const int most = a.dtype == RA_BF16 ? small_blocks<2>() : small_blocks<3>();
  return std::min(a.rows, a.cols) <= SMALL && parts_of(std::max(a.rows, a.cols), SMALL) <= 8 * most && a.steps > 0;
}

template <typename T, int PL>
cudaError_t run_small(const ra_orthogonalize_args& a, cudaStream_t st) {
  auto k = orth_small_kernel<T, PL>;
  // (all of shared memory, whatever the plan: one CTA an SM, whose TMEM no other waits for)
  constexpr int smem = small_smem<PL>();
  auto config = [&](cudaLaunchConfig_t& cfg, cudaLaunchAttribute* at, int ctas) {
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = ctas;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.gridDim = dim3((unsigned)a.n_matrices * ctas);
    cfg.blockDim = dim3(SMALL_THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = at;
    cfg.numAttrs = 1;
  };
  struct Fit {
    cudaError_t error;
    int clusters[9];  // of each size, that run at the same time
  };
  static const Fit fit = [&] {
    Fit f = {allow_smem(k, smem), {}};
    for (int c = 1; c <= 8 && f.error == cudaSuccess; ++c) {
      cudaLaunchConfig_t cfg = {};
      cudaLaunchAttribute at[1];
      config(cfg, at, c);
      cfg.gridDim = dim3((unsigned)c);
      f.error = cudaOccupancyMaxActiveClusters(&f.clusters[c], k, &cfg);
    }
    return f;
  }();
  if (fit.error != cudaSuccess) return fit.error;
  // CTAs of a cluster and blocks of a CTA by the measured time: rounds of clusters, each of about 5 us and 1 a block to begin with, and
  // 3 us, 0.35 a block and 0.5 a CTA a step (1024 x 64 in bf16: two CTAs 7.2 us a step, four 6.2, eight 7.6)
  int ctas = 0, blocks = 0;
  double best = 1e30;
  const int all = parts_of(std::max(a.rows, a.cols), SMALL);
  for (int c = 1; c <= 8; ++c) {
    const int b = parts_of(all, c);
    if (b > small_blocks<PL>() || parts_of(all, b) != c || fit.clusters[c] < 1) continue;
    const double t = (double)parts_of(a.n_matrices, fit.clusters[c]) * (5. + b + a.steps * (3. + 0.35 * b + 0.5 * c + (c > 1 ? 1. : 0.)));
    if (t < best) {
      best = t;
      ctas = c;
      blocks = b;
    }
  }
  if (ctas == 0) return cudaErrorNotSupported;
  constexpr int V = 16 / (int)sizeof(T);
  auto aligned = [&](const void* p, int64_t stride, int64_t matrix) {
    return ((uintptr_t)p & 15) == 0 && stride % V == 0 && (a.n_matrices == 1 || matrix % V == 0) && a.cols % V == 0;
  };
  SmallArgs p = {a, blocks, ctas, a.rows > a.cols, aligned(a.x_dev, a.x_stride, a.x_matrix_stride), aligned(a.out_dev, a.out_stride, a.out_matrix_stride),
                 prod::terms_of(PL, PL)};
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute at[2];
  config(cfg, at, ctas);
  at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.numAttrs = 2;
  note_launch(1);
  return cudaLaunchKernelEx(&cfg, k, p);
}

// What an epilogue takes for 128 x 128, in microseconds a plane of it, of two or three: stored (with its mirror image twice that), read as much (of the part of a tile that is there)
constexpr double plane_time(int kept) { return kept == 2 ? 0.8 : 1.5; }
// A symmetric product: all tiles, or (sym) square ones on and above the diagonal, which takes rounds off and costs the
// mirrored stores: 2048 x 2048 of K = 5632 in two planes 98 -> 73 us, two of 777 x 777 in three planes 49 -> 60.  `reads`: planes are read too
double time_sym(Pick k, int rows, int n, int blocks, double out) {
  const int64_t t = parts_of(rows, k.bn);
  return prod::time_of_tiles(k, n * t * (t + 1) / 2, blocks, t > 1 ? 2. * out : out);
}
struct Square {
  Pick pick;
  bool sym;
  double time;
};
Square pick_sym(int rows, int n, int blocks, int planes, int kept, bool reads) {
  const double part = (double)rows / up(rows, prod::BM), write = kept * plane_time(kept) * part * part, read = reads ? write : 0.;
  auto time = [&](Pick k) { return time_sym(k, rows, n, blocks, write) + read * k.bn / 128.; };
  const Pick one = {1, 128}, two = {2, 256}, best = rows > 128 && prod::takes(two, planes, planes) && time(two) < time(one) ? two : one;
  const Pick all = prod::pick(rows, rows, n, blocks, planes, planes, write + read);
  const double half = time(best), whole = prod::time_of(all, rows, rows, n, blocks, write + read);
  return half < whole ? Square{best, true, half} : Square{all, false, whole};
}

struct Plan {
  int planes, low, high, parts;
  // columns to a multiple of 8, what TMA reads of a row; rows at 128 bytes, the boxes' rows (at 16, each would touch two lines)
  int width, pitch, low_width, low_pitch;
  size_t norms, factors, x[2], s, q, sums, bytes;
};
// The tiles of a symmetric product and the k-blocks of a range, of operands in `planes`, kept in `kept`.  K in ranges where its tiles
// leave SMs idle (S of 3892 x 390 in fp32: 81 us a step in one range, 20 in ten and their join)
struct Ranges {
  Square how;
  int range, splits;
};
Ranges ranges_of(int rows, int k, int n, int planes, int kept, bool reads) {
  const int kbs = parts_of(k, prod::BK), terms = prod::terms_of(planes, planes).n;
  const int64_t side = parts_of(rows, prod::BM), tiles = n * side * (side + 1) / 2;
  Ranges g = {pick_sym(rows, n, kbs * terms, planes, kept, reads), kbs, 1};
  for (int splits = 2; splits <= 16 && splits <= kbs; ++splits) {
    const int each = parts_of(kbs, splits), ranges = parts_of(kbs, each);
    const Pick tile = {1, prod::BM};
    const double t = prod::time_of_tiles(tile, tiles * ranges, each * terms, 1.5) + (reads ? 8. : 6.);  // (stored as they are; the join)
    if (t < g.how.time) g = {{tile, true, t}, each, ranges};
  }
  return g;
}
// The planes of the matrices in a step, as they come (bf16 ones are one plane) or as they are kept
int planes_in(const Plan& p, bool first) { return first && p.planes == 2 ? 1 : p.planes; }
Ranges gram_of(const ra_orthogonalize_args& a, const Plan& p, bool first) { return ranges_of(p.low, p.high, a.n_matrices, planes_in(p, first), p.planes, false); }
Ranges square_of(const ra_orthogonalize_args& a, const Plan& p) { return ranges_of(p.low, p.low, a.n_matrices, p.planes, p.planes, true); }
Plan plan(const ra_orthogonalize_args& a) {
  Plan p = {};
  p.planes = a.dtype == RA_F32 ? 3 : 2;
  p.low = std::min(a.rows, a.cols);
  p.high = std::max(a.rows, a.cols);
  p.width = up(a.cols, 8);
  p.pitch = up(a.cols, 64);
  p.low_width = up(p.low, 8);
  p.low_pitch = up(p.low, 64);
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
  p.q = take(n * p.low * p.low_pitch);
  int splits = square_of(a, p).splits;
  for (bool first : {true, false}) splits = std::max(splits, gram_of(a, p, first).splits);
  p.sums = take(splits > 1 ? (size_t)splits * a.n_matrices * p.low * up(p.low, 32) * 4 : 0);
  p.bytes = at;
  return p;
}

Pick apply_of(const ra_orthogonalize_args& a, const Plan& p, bool first) {
  const int px = planes_in(p, first), pa = a.rows <= a.cols ? p.planes : px, pb = a.rows <= a.cols ? px : p.planes;
  return prod::pick(a.rows, a.cols, a.n_matrices, parts_of(p.low, prod::BK) * prod::terms_of(pa, pb).n, pa, pb, p.planes * plane_time(p.planes));
}

template <typename T>
cudaError_t run(const ra_orthogonalize_args& a, cudaStream_t st) {
  const Plan p = plan(a);
  char* ws = static_cast<char*>(a.workspace_dev);
  const int n = a.n_matrices, nz = n * p.planes;
  const bool wide = a.rows <= a.cols;
  float *norms = reinterpret_cast<float*>(ws + p.norms), *factors = reinterpret_cast<float*>(ws + p.factors);
  bf16* x[2] = {reinterpret_cast<bf16*>(ws + p.x[0]), reinterpret_cast<bf16*>(ws + p.x[1])};
  bf16 *s = reinterpret_cast<bf16*>(ws + p.s), *q = reinterpret_cast<bf16*>(ws + p.q);
  constexpr int es = sizeof(T), V = 16 / es;
  // bf16 matrices are one plane as they come
  const int first = a.steps == 0 ? 0 : es == 2 ? 1 : 3;
  {
    const bool vec = ((uintptr_t)a.x_dev & 15) == 0 && a.cols % V == 0 && a.x_stride % V == 0 && (n == 1 || a.x_matrix_stride % V == 0);
    const dim3 ng(p.parts, n), sg(std::min(parts_of(a.rows, 8), std::max(16, 2432 / n)), n);
    note_launch(2);
    DO(launch_pdl(vec ? orth_norm_kernel<T, V> : orth_norm_kernel<T, 1>, ng, dim3(256), 0, st, a, norms));
    DO(launch_pdl(vec ? orth_start_kernel<T, V> : orth_start_kernel<T, 1>, sg, dim3(256), 0, st, a, (const float*)norms, p.parts, factors, x[0], first,
                  p.width, p.pitch));
  }
  if (a.steps == 0) return cudaSuccess;

  const int chunk = p.planes == 3 ? 4 : 512;
  OrthArgs g = {};
  g.err = a.err_dev;
  g.factors = factors;
  g.n = n;
  g.dtype = a.dtype;
  g.splits = 1;
  auto shape = [&](OrthArgs& s, int rows, int cols, int k, int pa, int pb, Pick c, bool sym) {
    s.rows = rows;
    s.cols = cols;
    s.k = k;
    s.sym = sym;
    s.blocks = parts_of(k, prod::BK);
    s.cg = c.cg;
    s.shape = prod::shape_of(c.bn, c.cg, pa, pb, chunk);
  };
  constexpr int PL = es == 2 ? 2 : 3, ONE = es == 2 ? 1 : 3;  // planes of what is kept, and of the matrices as they come
  auto go = [&](const OrthArgs& s, auto step) {
    using S = decltype(step);
    int mt, nt;
    const int u = (int)std::min<int64_t>((int64_t)n * S::tiles(s, mt, nt) * s.splits, 1 << 20);
    return prod::launch<S>(s, s.cg, u, st);
  };
  OrthArgs square = g;
  // a symmetric product into `to`
  auto symmetric = [&](OrthArgs& s, int k, int planes, bf16* to, const Ranges& r) {
    shape(s, p.low, p.low, k, planes, planes, r.how.pick, r.how.sym);
    s.splits = r.splits;
    s.blocks = r.range;
    s.sums = reinterpret_cast<const float*>(ws + p.sums);
    s.sums_pitch = up(p.low, 32);
    s.o = to;
    s.width = p.low_width;
    s.pitch = p.low_pitch;
    if (s.splits > 1) MAP(s.out, s.sums, RA_F32, n * s.splits, p.low, s.sums_pitch, s.sums_pitch, 16, 32);
    else MAP(s.out, to, DT_BF16, nz, p.low, p.low_width, p.low_pitch, 32, 32);
    return cudaSuccess;
  };
  auto join = [&](const OrthArgs& s) {
    if (s.splits == 1) return cudaSuccess;
    const int side = parts_of(p.low, 32);
    note_launch(1);
    return launch_pdl(orth_join_kernel<PL>, dim3(side * (side + 1) / 2, n), dim3(256), 0, st, s);
  };
  DO(symmetric(square, p.low, p.planes, q, square_of(a, p)));
  square.add = a.a;
  square.mul = a.c;
  square.mul_with = a.b;
  square.with = s;
  MAP(square.a, s, DT_BF16, nz, p.low, p.low_width, p.low_pitch, 64, prod::BM);
  MAP(square.b, s, DT_BF16, nz, p.low, p.low_width, p.low_pitch, 64, square.shape.bn / square.cg);
  for (int i = 0; i < a.steps; ++i) {
    const int px = i == 0 ? first : p.planes;
    const bf16* from = x[i & 1];
    OrthArgs gram = g, apply = g;
    DO(symmetric(gram, p.high, px, s, gram_of(a, p, i == 0)));
    gram.a_mn = gram.b_mn = !wide;
    gram.power = px == 1 ? 2 : 0;
    const int pa = wide ? p.planes : px, pb = wide ? px : p.planes;
    shape(apply, a.rows, a.cols, p.low, pa, pb, apply_of(a, p, i == 0), false);
    MAP(apply.out, x[(i + 1) & 1], DT_BF16, nz, a.rows, p.width, p.pitch, 32, 32);
    apply.b_mn = wide;
    apply.power = px == 1 ? 1 : 0;
    apply.width = p.width;
    apply.pitch = p.pitch;
    if (wide) {
      MAP(gram.a, from, DT_BF16, n * px, a.rows, p.width, p.pitch, 64, prod::BM);
      MAP(gram.b, from, DT_BF16, n * px, a.rows, p.width, p.pitch, 64, gram.shape.bn / gram.cg);
      MAP(apply.a, q, DT_BF16, nz, p.low, p.low_width, p.low_pitch, 64, prod::BM);
      MAP(apply.b, from, DT_BF16, n * px, a.rows, p.width, p.pitch, 64, 64);
    } else {
      MAP(gram.a, from, DT_BF16, n * px, a.rows, p.width, p.pitch, 64, 64);
      gram.b = gram.a;
      MAP(apply.a, from, DT_BF16, n * px, a.rows, p.width, p.pitch, 64, prod::BM);
      MAP(apply.b, q, DT_BF16, nz, p.low, p.low_width, p.low_pitch, 64, apply.shape.bn / apply.cg);
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
    using Full = Step<PL, PL, PL>;
    DO(px == PL ? go(gram, Full()) : go(gram, Step<PL, ONE, ONE>()));
    DO(join(gram));
    DO(go(square, Full()));
    DO(join(square));
    DO(px == PL ? go(apply, Full()) : wide ? go(apply, Step<PL, PL, ONE>()) : go(apply, Step<PL, ONE, PL>()));
  }
  return cudaSuccess;
}

}  // namespace

void orthogonalize_plan(const ra_orthogonalize_args& a, int32_t (&out)[17]) {
  const Plan p = plan(a);
  const Ranges s0 = gram_of(a, p, true), s = gram_of(a, p, false), q = square_of(a, p);
  const Pick x0 = apply_of(a, p, true), x = apply_of(a, p, false);
  int32_t* at = out;
  *at++ = small_fits(a);
  for (const Ranges* r : {&s0, &s, &q})
    for (int v : {r->how.pick.cg, r->how.pick.bn, (int)r->how.sym, r->splits}) *at++ = v;
  for (const Pick* k : {&x0, &x})
    for (int v : {k->cg, k->bn}) *at++ = v;
}
size_t orthogonalize_workspace(const ra_orthogonalize_args& a) { return small_fits(a) ? WS_ZERO : plan(a).bytes; }
cudaError_t orthogonalize(const ra_orthogonalize_args& a, cudaStream_t st) {
  if (small_fits(a)) return a.dtype == RA_BF16 ? run_small<bf16, 2>(a, st) : run_small<float, 3>(a, st);
  return a.dtype == RA_BF16 ? run<bf16>(a, st) : run<float>(a, st);
}

}  // namespace ra
