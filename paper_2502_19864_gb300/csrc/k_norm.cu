// k_norm.cu -- LayerNorm and RMSNorm with a residual's sum, and their backward with the weights' gradients.
//
// Forward, for each row z = x + residual of n values: mean m, then the deviations d = z - m; the rounding of m is
// taken out again by the deviations' own mean, so that rows far from zero keep their digits:
//   rstd = 1 / sqrt(mean(d^2) - mean(d)^2 + eps), y = (d - mean(d)) rstd gamma + beta.
// Backward, with u = (z - m) rstd and g = dy gamma: dx = rstd (g - mean(g) - u mean(g u)) + dsum, and the sums over rows
// dgamma = sum dy u, dbeta = sum dy, which each CTA keeps in registers over its rows; the CTAs' partial sums are added in
// a second kernel, in a fixed order.
//
// Bound: bytes.  A row is read once, held in registers (or, on its way through a ring, in shared memory) through the reductions
// and written once.  A CTA's threads share a row (one of up to 256 values: a warp's, eight warps a CTA), eight (16, 32) values each, and
// take ROWS rows at a time, so that enough loads are on their way and a barrier serves them all; two values an instruction, as the
// instructions' issue is the next bound (28 a value without: 165 us, with 137).
// Forward and backward of 65536 x 1024 in bf16 take 137 us (4.9 TB/s), of 8192 x 2048 with its residual 52 us (5.2 TB/s), of
// 16271 x 1334, in pieces of 4 bytes, 135 us (2.5 TB/s).
// Rows over 8192 values have 32 a thread and the 64 registers of 1024 threads.  The forward has room: 4096 x 8200 in bf16 with its
// residual 64 us (4.2 TB/s), 2048 x 32768 117 us (4.6).  The backward, which holds the weights, their sums and three inputs, spills 1.0 to
// 1.9 KB a thread: 200 us (1.3 TB/s, where 4096 x 8192 takes 52) and 449; in fp32 440 and 790.
#include <algorithm>

#include "common.cuh"
#include "operators.h"

namespace ra {
namespace {

constexpr int NORM_MAX_CTAS = 608;  // four an SM of 152: the backward's partial sums

// VEC values at a place that is a multiple of their bytes, as they come from memory.  keep(): what was computed of them before is
// computed again after, and not held in registers of its own in between
template <typename T, int VEC> struct Raw;
template <> struct Raw<float, 4> {
  float4 v;
  __device__ __forceinline__ void load(const float* p) { v = *reinterpret_cast<const float4*>(p); }
  __device__ __forceinline__ void get(float* f) const { f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w; }
  __device__ __forceinline__ void keep() { asm volatile("" : "+f"(v.x), "+f"(v.y), "+f"(v.z), "+f"(v.w)); }
};
template <> struct Raw<bf16, 8> {
  uint4 v;
  __device__ __forceinline__ void load(const bf16* p) { v = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void get(float* f) const {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  __device__ __forceinline__ void keep() { asm volatile("" : "+r"(v.x), "+r"(v.y), "+r"(v.z), "+r"(v.w)); }
};
template <> struct Raw<float, 2> {
  float2 v;
  __device__ __forceinline__ void load(const float* p) { v = *reinterpret_cast<const float2*>(p); }
  __device__ __forceinline__ void get(float* f) const { f[0] = v.x; f[1] = v.y; }
  __device__ __forceinline__ void keep() { asm volatile("" : "+f"(v.x), "+f"(v.y)); }
};
template <> struct Raw<bf16, 4> {
  uint2 v;
  __device__ __forceinline__ void load(const bf16* p) { v = *reinterpret_cast<const uint2*>(p); }
  __device__ __forceinline__ void get(float* f) const {
    f[0] = __uint_as_float(v.x << 16); f[1] = __uint_as_float(v.x & 0xffff0000u);
    f[2] = __uint_as_float(v.y << 16); f[3] = __uint_as_float(v.y & 0xffff0000u);
  }
  __device__ __forceinline__ void keep() { asm volatile("" : "+r"(v.x), "+r"(v.y)); }
};
template <> struct Raw<bf16, 2> {
  uint32_t v;
  __device__ __forceinline__ void load(const bf16* p) { v = *reinterpret_cast<const uint32_t*>(p); }
  __device__ __forceinline__ void get(float* f) const { f[0] = __uint_as_float(v << 16); f[1] = __uint_as_float(v & 0xffff0000u); }
  __device__ __forceinline__ void keep() { asm volatile("" : "+r"(v)); }
};
template <> struct Raw<float, 8> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = reinterpret_cast<const float4*>(p)[0];
    b = reinterpret_cast<const float4*>(p)[1];
  }
  __device__ __forceinline__ void get(float* f) const {
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
    f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  }
};
template <typename T> struct Raw<T, 1> {
  T v;
  __device__ __forceinline__ void load(const T* p) { v = *p; }
  __device__ __forceinline__ void get(float* f) const { f[0] = to_f(v); }
  __device__ __forceinline__ void keep() {}
};
template <int VEC> __device__ __forceinline__ void put(float* p, const float* v) {
  if constexpr (VEC == 1) *p = v[0];
  else if constexpr (VEC == 2) *reinterpret_cast<float2*>(p) = make_float2(v[0], v[1]);
  else *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
}
template <int VEC> __device__ __forceinline__ void put(bf16* p, const float* v) {
  if constexpr (VEC == 1) {
    *p = __float2bfloat16_rn(v[0]);
  } else {
    uint32_t w[VEC / 2];
#pragma unroll
    for (int i = 0; i < VEC / 2; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    if constexpr (VEC == 2) *reinterpret_cast<uint32_t*>(p) = w[0];
    else if constexpr (VEC == 4) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    else *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// d = a b + c, d = a + b, d = a b of VEC values, two to an instruction; operands that are one value for all as such
template <int VEC> __device__ __forceinline__ void vfma(float* d, const float* a, const float* b, const float* c) {
  if constexpr (VEC == 1) d[0] = fmaf(a[0], b[0], c[0]);
  else
#pragma unroll
    for (int j = 0; j < VEC; j += 2) {
      const float2 r = __ffma2_rn(make_float2(a[j], a[j + 1]), make_float2(b[j], b[j + 1]), make_float2(c[j], c[j + 1]));
      d[j] = r.x;
      d[j + 1] = r.y;
    }
}
template <int VEC> __device__ __forceinline__ void vfma1(float* d, const float* a, float b, float c) {
  if constexpr (VEC == 1) d[0] = fmaf(a[0], b, c);
  else
#pragma unroll
    for (int j = 0; j < VEC; j += 2) {
      const float2 r = __ffma2_rn(make_float2(a[j], a[j + 1]), make_float2(b, b), make_float2(c, c));
      d[j] = r.x;
      d[j + 1] = r.y;
    }
}
template <int VEC> __device__ __forceinline__ void vfmas(float* d, const float* a, float b, const float* c) {
  if constexpr (VEC == 1) d[0] = fmaf(a[0], b, c[0]);
  else
#pragma unroll
    for (int j = 0; j < VEC; j += 2) {
      const float2 r = __ffma2_rn(make_float2(a[j], a[j + 1]), make_float2(b, b), make_float2(c[j], c[j + 1]));
      d[j] = r.x;
      d[j + 1] = r.y;
    }
}
template <int VEC> __device__ __forceinline__ void vadd(float* d, const float* a, const float* b) {
  if constexpr (VEC == 1) d[0] = a[0] + b[0];
  else
#pragma unroll
    for (int j = 0; j < VEC; j += 2) {
      const float2 r = __fadd2_rn(make_float2(a[j], a[j + 1]), make_float2(b[j], b[j + 1]));
      d[j] = r.x;
      d[j + 1] = r.y;
    }
}
template <int VEC> __device__ __forceinline__ void vmul(float* d, const float* a, const float* b) {
  if constexpr (VEC == 1) d[0] = a[0] * b[0];
  else
#pragma unroll
    for (int j = 0; j < VEC; j += 2) {
      const float2 r = __fmul2_rn(make_float2(a[j], a[j + 1]), make_float2(b[j], b[j + 1]));
      d[j] = r.x;
      d[j + 1] = r.y;
    }
}
// 1 / sqrt(v): the special function unit's (2 ulp) and a step of Newton's method
__device__ __forceinline__ float inv_sqrt(float v) {
  const float y = rsqrtf(v);
  const float r = y * fmaf(-0.5f * v * y, y, 1.5f);
  return y > 0.f && y < INFINITY ? r : y;  // (of 0, infinity and NaN the unit's answer)
}

// DEPTH groups of ROWS rows in shared memory on their way from the inputs, BYTES (VEC values) a thread at a place of its own, so
// that no thread waits for another's copies
template <int BYTES>
__device__ __forceinline__ void copy(void* smem, const void* p) {
  if constexpr (BYTES == 16)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(smem)), "l"(p) : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"((uint32_t)__cvta_generic_to_shared(smem)), "l"(p), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Sums of K (a power of two) values over the CTA, for every thread, in a fixed order.  A warp halves the values it carries
// with the lanes that share them, so that K values cost K + 4 - log2(K) exchanges.  sh holds two parts of 32 K floats,
// used in turn by successive calls (`turn`), so that one barrier a call is enough.
template <int K>
__device__ __forceinline__ void block_sum(float (&v)[K], float* sh, int turn) {
  const int lane = threadIdx.x & 31, warps = (int)blockDim.x >> 5;
  int o = 16, idx = 0;
#pragma unroll
  for (int k = K / 2; k >= 1; k >>= 1, o >>= 1) {
    const bool high = lane & o;
#pragma unroll
    for (int i = 0; i < k; ++i) {
      const float give = high ? v[i] : v[i + k], keep = high ? v[i + k] : v[i];
      v[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
    }
    idx += high ? k : 0;
  }
#pragma unroll
  for (int p = 16 / K; p >= 1; p >>= 1) v[0] += __shfl_xor_sync(0xffffffffu, v[0], p);
  if (warps == 1) {
    const float mine = v[0];
    // value i is with the lanes whose high bits are i
#pragma unroll
    for (int i = 0; i < K; ++i) v[i] = __shfl_sync(0xffffffffu, mine, i * (32 / K));
    return;
  }
  float* at = sh + (turn & 1) * 32 * K;
  if ((lane & (32 / K - 1)) == 0) at[(threadIdx.x >> 5) * K + idx] = v[0];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < K; ++i) v[i] = at[i];
  for (int w = 1; w < warps; ++w)
#pragma unroll
    for (int i = 0; i < K; ++i) v[i] += at[w * K + i];
}

// the most threads of a CTA by its values a thread: 8 take rows up to 8192 values one by one, up to 2048 four at a time;
// 16 rows up to 8192; 32 the longest
constexpr int max_threads(int n, int rows) { return n == 8 && rows == 1 ? 1024 : n == 8 ? 256 : n == 16 ? 512 : 1024; }
constexpr int min_ctas(int n, int rows, bool backward) { return n == 8 && rows > 1 ? (backward ? 2 : 3) : 1; }

template <typename T, typename W, int VEC, int NV, int ROWS, int DEPTH>
__global__ void __launch_bounds__(max_threads(VEC * NV, ROWS), min_ctas(VEC * NV, ROWS, false)) norm_fwd_kernel(const __grid_constant__ ra_norm_args a) {
  __shared__ __align__(16) float sh1[2 * 32 * ROWS], sh2[2 * 32 * 2 * ROWS];
  constexpr int N = VEC * NV, PIECE = VEC * (int)sizeof(T);
  const int t = threadIdx.x, G = blockDim.x, H = a.hidden;
  const bool layer = a.kind == RA_NORM_LAYER;
  const float inv = 1.f / (float)H;
  const W* gamma = static_cast<const W*>(a.gamma_dev);
  const W* beta = static_cast<const W*>(a.beta_dev);
  pdl_wait();
  pdl_trigger();
  extern __shared__ __align__(16) uint8_t ring[];  // [blockDim.y][DEPTH][inputs][ROWS][NV][G] pieces
  const int inputs = a.residual_dev ? 2 : 1;
  const int64_t first = ((int64_t)blockIdx.x * blockDim.y + threadIdx.y) * ROWS, step = (int64_t)gridDim.x * blockDim.y * ROWS;
  uint8_t* own = ring + threadIdx.y * (DEPTH * inputs * ROWS * NV * G * PIECE);
  auto place = [&](int slot, int in, int r, int i) { return own + ((((slot * inputs + in) * ROWS + r) * NV + i) * G + t) * PIECE; };
  auto fetch = [&](int64_t row0, int slot) {
    if constexpr (DEPTH > 0) {
#pragma unroll
      for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          const int c = (i * G + t) * VEC;
          if (c < H && row0 + r < a.rows) {
            copy<PIECE>(place(slot, 0, r, i), static_cast<const T*>(a.x_dev) + (row0 + r) * a.x_stride + c);
            if (inputs > 1) copy<PIECE>(place(slot, 1, r, i), static_cast<const T*>(a.residual_dev) + (row0 + r) * a.residual_stride + c);
          }
        }
      copies_end();
    }
  };
  auto from = [&](const T* p, int slot, int in, int r, int i) {
    Raw<T, VEC> v;
    if constexpr (DEPTH > 0) v.load(reinterpret_cast<const T*>(place(slot, in, r, i)));
    else v.load(p);
    return v;
  };
  int turn = 0, slot = 0;
  if constexpr (DEPTH > 0)
    for (int d = 0; d + 1 < DEPTH; ++d) fetch(first + d * step, d);
  for (int64_t row0 = first; row0 < a.rows; row0 += step, ++turn) {
    if constexpr (DEPTH > 0) {
      fetch(row0 + (DEPTH - 1) * step, slot == 0 ? DEPTH - 1 : slot - 1);
      copies_wait<DEPTH - 1>();
    }
    float z[ROWS][N];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const T* x = static_cast<const T*>(a.x_dev) + (row0 + r) * a.x_stride;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = (i * G + t) * VEC;
#pragma unroll
        for (int j = 0; j < VEC; ++j) z[r][i * VEC + j] = 0.f;
        if (c < H && row0 + r < a.rows) from(x + c, slot, 0, r, i).get(z[r] + i * VEC);
      }
    }
    if (a.residual_dev) {
#pragma unroll
      for (int r = 0; r < ROWS; ++r) {
        const T* p = static_cast<const T*>(a.residual_dev) + (row0 + r) * a.residual_stride;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          const int c = (i * G + t) * VEC;
          if (c < H && row0 + r < a.rows) {
            float f[VEC];
            from(p + c, slot, 1, r, i).get(f);
            vadd<VEC>(z[r] + i * VEC, z[r] + i * VEC, f);
          }
        }
      }
      if (a.sum_dev)
#pragma unroll
        for (int r = 0; r < ROWS; ++r)
#pragma unroll
          for (int i = 0; i < NV; ++i) {
            const int c = (i * G + t) * VEC;
            if (c < H && row0 + r < a.rows) put<VEC>(static_cast<T*>(a.sum_dev) + (row0 + r) * a.sum_stride + c, z[r] + i * VEC);
          }
    }
    constexpr int P = N > 1 ? 2 : 1;  // sums in pairs
    float mean[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) mean[r] = 0.f;
    if (layer) {
#pragma unroll
      for (int r = 0; r < ROWS; ++r) {
        float m[P] = {};
#pragma unroll
        for (int i = 0; i < N; i += P) vadd<P>(m, m, z[r] + i);
        mean[r] = m[0] + (P > 1 ? m[P - 1] : 0.f);
      }
      block_sum(mean, sh1, turn);
#pragma unroll
      for (int r = 0; r < ROWS; ++r) {
        mean[r] *= inv;
#pragma unroll
        for (int i = 0; i < NV; ++i)
          if ((i * G + t) * VEC < H) vfma1<VEC>(z[r] + i * VEC, z[r] + i * VEC, 1.f, -mean[r]);
      }
    }
    float s[2 * ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      float q[P] = {}, m[P] = {};
#pragma unroll
      for (int i = 0; i < N; i += P) {
        vfma<P>(q, z[r] + i, z[r] + i, q);
        if (layer) vadd<P>(m, m, z[r] + i);
      }
      s[2 * r] = q[0] + (P > 1 ? q[P - 1] : 0.f);
      s[2 * r + 1] = m[0] + (P > 1 ? m[P - 1] : 0.f);
    }
    block_sum(s, sh2, turn);
    float off[ROWS], rstd[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      off[r] = layer ? s[2 * r + 1] * inv : 0.f;
      mean[r] += off[r];
      const float var = fmaf(-off[r], off[r], s[2 * r] * inv);
      rstd[r] = inv_sqrt((var < 0.f ? 0.f : var) + a.eps);  // (a NaN stays)
      if (t == 0 && row0 + r < a.rows) {
        if (a.mean_dev && layer) a.mean_dev[row0 + r] = mean[r];
        if (a.rstd_dev) a.rstd_dev[row0 + r] = rstd[r];
      }
      off[r] *= -rstd[r];
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * G + t) * VEC;
      if (c >= H) continue;
      float w[VEC], b[VEC];
#pragma unroll
      for (int j = 0; j < VEC; ++j) w[j] = 1.f, b[j] = 0.f;
      Raw<W, VEC> v;
      if (gamma) {
        v.load(gamma + c);
        v.get(w);
      }
      if (beta) {
        v.load(beta + c);
        v.get(b);
      }
#pragma unroll
      for (int r = 0; r < ROWS; ++r) {
        float f[VEC];
        vfma1<VEC>(f, z[r] + i * VEC, rstd[r], off[r]);
        vfma<VEC>(f, f, w, b);
        if (row0 + r < a.rows) put<VEC>(static_cast<T*>(a.y_dev) + (row0 + r) * a.y_stride + c, f);
      }
    }
    if (DEPTH > 0) slot = slot + 1 == DEPTH ? 0 : slot + 1;
  }
}

// sums [2][ctas][hidden]: each CTA's part of dgamma, then of dbeta
template <typename T, typename W, int VEC, int NV, int ROWS, int DEPTH>
__global__ void __launch_bounds__(max_threads(VEC * NV, ROWS), min_ctas(VEC * NV, ROWS, true)) norm_bwd_kernel(const __grid_constant__ ra_norm_args a, float* sums) {
  __shared__ __align__(16) float sh[2 * 32 * 2 * ROWS];
  constexpr int N = VEC * NV, PIECE = VEC * (int)sizeof(T);
  const int t = threadIdx.x, G = blockDim.x, H = a.hidden;
  const bool layer = a.kind == RA_NORM_LAYER;
  const float inv = 1.f / (float)H;
  const W* gamma = static_cast<const W*>(a.gamma_dev);
  const T* zsrc = static_cast<const T*>(a.residual_dev ? a.sum_dev : a.x_dev);
  const int64_t zstride = a.residual_dev ? a.sum_stride : a.x_stride;
  pdl_wait();
  pdl_trigger();
  float dg[N], db[N], w[N];
#pragma unroll
  for (int i = 0; i < N; ++i) dg[i] = db[i] = 0.f, w[i] = 1.f;
  if (gamma)
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * G + t) * VEC;
      Raw<W, VEC> v;
      if (c < H) {
        v.load(gamma + c);
        v.get(w + i * VEC);
      }
    }
  extern __shared__ __align__(16) uint8_t ring[];  // [blockDim.y][DEPTH][inputs][ROWS][NV][G] pieces
  const bool more = a.dsum_dev && a.dx_dev;
  const int inputs = more ? 3 : 2;
  const int64_t first = ((int64_t)blockIdx.x * blockDim.y + threadIdx.y) * ROWS, step = (int64_t)gridDim.x * blockDim.y * ROWS;
  uint8_t* own = ring + threadIdx.y * (DEPTH * inputs * ROWS * NV * G * PIECE);
  auto source = [&](int in, int64_t row, int c) {
    return in == 0 ? zsrc + row * zstride + c
                   : in == 1 ? static_cast<const T*>(a.dy_dev) + row * a.dy_stride + c : static_cast<const T*>(a.dsum_dev) + row * a.dsum_stride + c;
  };
  auto place = [&](int slot, int in, int r, int i) { return own + ((((slot * inputs + in) * ROWS + r) * NV + i) * G + t) * PIECE; };
  auto fetch = [&](int64_t row0, int slot) {
    if constexpr (DEPTH > 0) {
#pragma unroll
      for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          const int c = (i * G + t) * VEC;
          if (c < H && row0 + r < a.rows) {
            copy<PIECE>(place(slot, 0, r, i), source(0, row0 + r, c));
            copy<PIECE>(place(slot, 1, r, i), source(1, row0 + r, c));
            if (more) copy<PIECE>(place(slot, 2, r, i), source(2, row0 + r, c));
          }
        }
      copies_end();
    }
  };
  int turn = 0, slot = 0;
  if constexpr (DEPTH > 0)
    for (int d = 0; d + 1 < DEPTH; ++d) fetch(first + d * step, d);
  for (int64_t row0 = first; row0 < a.rows; row0 += step, ++turn) {
    // (without a ring the rows are held as they came)
    Raw<T, VEC> held[DEPTH > 0 ? 1 : 3][DEPTH > 0 ? 1 : ROWS][DEPTH > 0 ? 1 : NV];
    float mean[ROWS], rstd[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      mean[r] = layer && row0 + r < a.rows ? a.mean_dev[row0 + r] : 0.f;
      rstd[r] = row0 + r < a.rows ? a.rstd_dev[row0 + r] : 0.f;
    }
    if constexpr (DEPTH > 0) {
      fetch(row0 + (DEPTH - 1) * step, slot == 0 ? DEPTH - 1 : slot - 1);
      copies_wait<DEPTH - 1>();
    } else {
#pragma unroll
      for (int in = 0; in < 3; ++in)
        if (in < inputs)
#pragma unroll
          for (int r = 0; r < ROWS; ++r)
#pragma unroll
            for (int i = 0; i < NV; ++i) {
              const int c = (i * G + t) * VEC;
              if (c < H && row0 + r < a.rows) held[in][r][i].load(source(in, row0 + r, c));
            }
    }
    auto get = [&](int slot, int in, int r, int i, float* f) {
      if constexpr (DEPTH > 0) {
        Raw<T, VEC> v;
        v.load(reinterpret_cast<const T*>(place(slot, in, r, i)));
        v.get(f);
      } else {
        held[in][r][i].keep();
        held[in][r][i].get(f);
      }
    };
    float s[2 * ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      mean[r] *= -rstd[r];  // (u = z rstd - mean rstd)
      constexpr int P = VEC > 1 ? 2 : 1;
      float s0[P] = {}, s1[P] = {};
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if ((i * G + t) * VEC < H && row0 + r < a.rows) {
          float u[VEC], g[VEC];
          get(slot, 0, r, i, u);
          get(slot, 1, r, i, g);
          vfma1<VEC>(u, u, rstd[r], mean[r]);
          vfma<VEC>(dg + i * VEC, g, u, dg + i * VEC);
          vadd<VEC>(db + i * VEC, g, db + i * VEC);
          vmul<VEC>(g, g, w + i * VEC);
#pragma unroll
          for (int j = 0; j < VEC; j += P) {
            vadd<P>(s0, s0, g + j);
            vfma<P>(s1, g + j, u + j, s1);
          }
        }
      s[2 * r] = s0[0] + (P > 1 ? s0[P - 1] : 0.f);
      s[2 * r + 1] = s1[0] + (P > 1 ? s1[P - 1] : 0.f);
    }
    const int here = slot;
    if (DEPTH > 0) slot = slot + 1 == DEPTH ? 0 : slot + 1;
    if (!a.dx_dev) continue;
    block_sum(s, sh, turn);
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const float mg = layer ? s[2 * r] * inv * -rstd[r] : 0.f, mgu = s[2 * r + 1] * inv * -rstd[r];
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = (i * G + t) * VEC;
        if (c < H && row0 + r < a.rows) {
          float u[VEC], g[VEC], e[VEC];
          get(here, 0, r, i, u);
          get(here, 1, r, i, g);
          vfma1<VEC>(u, u, rstd[r], mean[r]);
          vmul<VEC>(g, g, w + i * VEC);
          vfma1<VEC>(u, u, mgu, mg);
          vfmas<VEC>(g, g, rstd[r], u);
          if (more) {
            get(here, 2, r, i, e);
            vadd<VEC>(g, g, e);
          }
          put<VEC>(static_cast<T*>(a.dx_dev) + (row0 + r) * a.dx_stride + c, g);
        }
      }
    }
  }
  if (blockDim.y > 1) {  // the warps' sums in turn
    float* part = reinterpret_cast<float*>(ring);
    const int all = N * G;
    copies_wait<0>();
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const int c = (i * G + t) * VEC + j;
        part[2 * threadIdx.y * all + c] = dg[i * VEC + j];
        part[(2 * threadIdx.y + 1) * all + c] = db[i * VEC + j];
      }
    __syncthreads();
    for (int k = threadIdx.y * G + t; k < 2 * H; k += blockDim.y * G) {
      const int c = k < H ? k : k - H + all;
      float v = 0.f;
      for (int y = 0; y < (int)blockDim.y; ++y) v += part[2 * y * all + c];
      if (k < H ? a.dgamma_dev != nullptr : a.dbeta_dev != nullptr)
        sums[k < H ? (int64_t)blockIdx.x * H + k : (int64_t)(gridDim.x + blockIdx.x) * H + (k - H)] = v;
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      const int c = (i * G + t) * VEC + j;
      if (c < H) {
        if (a.dgamma_dev) sums[(int64_t)blockIdx.x * H + c] = dg[i * VEC + j];
        if (a.dbeta_dev) sums[(int64_t)(gridDim.x + blockIdx.x) * H + c] = db[i * VEC + j];
      }
    }
}

// dgamma and dbeta of 32 columns from `ctas` partial sums: 32 warps take every 32nd, eight at once on their way, then the
// warps' sums in turn
template <typename W>
__global__ void __launch_bounds__(1024) norm_weights_kernel(const float* sums, W* dgamma, W* dbeta, int ctas, int H) {
  __shared__ float sh[32][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  W* out = blockIdx.y ? dbeta : dgamma;
  pdl_wait();
  pdl_trigger();
  if (!out) return;
  const float* at = sums + (int64_t)blockIdx.y * ctas * H;
  float s = 0.f;
  if (c < H)
    for (int i0 = warp; i0 < ctas; i0 += 256) {
      float v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = i0 + 32 * k < ctas ? at[(int64_t)(i0 + 32 * k) * H + c] : 0.f;
#pragma unroll
      for (int k = 0; k < 8; ++k) s += v[k];
    }
  sh[warp][lane] = s;
  __syncthreads();
  s = warp_sum(sh[lane][warp]);  // column `warp`
  if (lane == 0 && blockIdx.x * 32 + warp < H) out[blockIdx.x * 32 + warp] = from_f<W>(s);
}

int bwd_ctas(const ra_norm_args& a) { return std::min(a.rows, NORM_MAX_CTAS); }

// CTAs of `threads` with `smem` bytes each that an SM holds, as far as those decide
int ctas_an_sm(int threads, int smem) { return std::max(1, std::min(2048 / threads, smem ? 227 * 1024 / (smem + 4096) : 32)); }

template <bool BACK, typename T, typename W, int VEC, int NV, int ROWS, int DEPTH = 0>
cudaError_t launch(const ra_norm_args& a, cudaStream_t st) {
  const int vecs = (a.hidden + VEC - 1) / VEC;
  const int threads = ((vecs + NV - 1) / NV + 31) / 32 * 32;
  const int groups = (int)(((int64_t)a.rows + ROWS - 1) / ROWS), sms = device_sm_count();
  // Rows of one warp: up to eight warps a CTA with rows of their own, as far as two CTAs an SM have as many (24071 x 40 in fp32
  // backward 19 us, with a warp a CTA 33)
  const int ys = threads == 32 && ROWS > 1 ? std::max(1, std::min(8, groups / (2 * sms))) : 1;
  const int wide = (groups + ys - 1) / ys;
  constexpr int each = DEPTH * ROWS * NV * VEC * (int)sizeof(T);  // bytes of the ring a thread and input
  constexpr int most = std::min((BACK ? 3 : 2) * each * max_threads(VEC * NV, ROWS), MAX_DYNAMIC_SMEM - 4096);
  auto k = [] {
    if constexpr (BACK) return norm_bwd_kernel<T, W, VEC, NV, ROWS, DEPTH>;
    else return norm_fwd_kernel<T, W, VEC, NV, ROWS, DEPTH>;
  }();
  if (DEPTH > 0) {
    static const cudaError_t attr = allow_smem(k, most);
    if (attr != cudaSuccess) return attr;
  }
  note_launch(1);
  if constexpr (!BACK) {
    const int smem = ys * threads * each * (a.residual_dev ? 2 : 1);
    return launch_pdl(k, dim3(std::min(wide, sms * ctas_an_sm(threads * ys, smem))), dim3(threads, ys), smem, st, a);
  } else {
    const int ring = ys * threads * each * (a.dsum_dev && a.dx_dev ? 3 : 2);
    const int smem = std::max(ring, ys > 1 ? ys * threads * 2 * VEC * NV * (int)sizeof(float) : 0);  // (the warps' sums after it)
    const int ctas = std::min(std::min(wide, NORM_MAX_CTAS), sms * (DEPTH > 0 ? ctas_an_sm(threads * ys, smem) : 4));
    float* sums = reinterpret_cast<float*>(static_cast<char*>(a.workspace_dev) + WS_ZERO);
    const cudaError_t e = launch_pdl(k, dim3(ctas), dim3(threads, ys), smem, st, a, sums);
    if (e != cudaSuccess || (!a.dgamma_dev && !a.dbeta_dev)) return e;
    note_launch(1);
    return launch_pdl(norm_weights_kernel<W>, dim3((a.hidden + 31) / 32, a.dbeta_dev ? 2 : 1), dim3(1024), 0, st,
                      (const float*)sums, (W*)a.dgamma_dev, (W*)a.dbeta_dev, ctas, (int)a.hidden);
  }
}

// rows of the ring by their values' size, and its groups (65536 x 1024 and 8192 x 2048 trained: 140 and 54 us when these were measured, 137
// and 52 now; two rows and three groups 154 and 62, three groups 145 and 60; without a ring 173 and 82)
constexpr int RING_ROWS = 8, RING_DEPTH = 2;

// The widest accesses that all rows and weights allow, up to 16 bytes
template <typename T>
int widest(const ra_norm_args& a, bool backward) {
  constexpr int es = sizeof(T);
  const int wes = a.w_dtype == RA_BF16 ? 2 : 4;
  int v = 16 / es;
  auto rows = [&](const void* p, int64_t stride) {
    while (p && v > 1 && (((uintptr_t)p & (v * es - 1)) || stride % v)) v /= 2;
  };
  auto weights = [&](const void* p) {
    while (p && v > 1 && ((uintptr_t)p & (std::min(16, v * wes) - 1))) v /= 2;
  };
  while (a.hidden % v) v /= 2;
  weights(a.gamma_dev);
  weights(a.beta_dev);
  if (!backward || !a.residual_dev) rows(a.x_dev, a.x_stride);
  rows(a.sum_dev, a.sum_stride);
  if (backward) {
    rows(a.dy_dev, a.dy_stride);
    rows(a.dsum_dev, a.dsum_stride);
    rows(a.dx_dev, a.dx_stride);
  } else {
    rows(a.residual_dev, a.residual_stride);
    rows(a.y_dev, a.y_stride);
  }
  return v;
}

// VEC values an access; several rows at a time where there are enough of them for every SM, backward through a ring where they are
// in pieces of 4 bytes at least, forward where they are in 16 (8192 x 8192 with its residual 91 us, without 142; in pieces of 4
// 11793 x 2302 takes 70 us with it and 54 without).  Backward by single 2-byte values, rows longer than 2048 go one by one, as two
// have no room in the registers (11793 x 2299: 139 us, 300 so)
template <bool BACK, typename T, typename W, int VEC>
cudaError_t by_size(const ra_norm_args& a, cudaStream_t st) {
  constexpr int piece = VEC * (int)sizeof(T), NV = 8 / VEC, DEPTH = piece >= (BACK ? 4 : 16) ? RING_DEPTH : 0;
  const bool many = a.rows >= 4 * 608;
  if (a.hidden <= 2048 && many) return launch<BACK, T, W, VEC, NV, RING_ROWS / (int)sizeof(T), DEPTH>(a, st);
  if constexpr (!BACK || DEPTH > 0)
    if (a.hidden <= 8192 && many) return launch<BACK, T, W, VEC, 2 * NV, RING_ROWS / 2 / (int)sizeof(T), DEPTH>(a, st);
  if (a.hidden <= 8192) return launch<BACK, T, W, VEC, NV, 1>(a, st);
  return launch<BACK, T, W, VEC, 4 * NV, 1>(a, st);
}
template <bool BACK, typename T, typename W>
cudaError_t dispatch(const ra_norm_args& a, cudaStream_t st) {
  const int vec = widest<T>(a, BACK);
  if constexpr (sizeof(T) == 2)
    if (vec == 8) return by_size<BACK, T, W, 8>(a, st);
  return vec == 4 ? by_size<BACK, T, W, 4>(a, st) : vec == 2 ? by_size<BACK, T, W, 2>(a, st) : by_size<BACK, T, W, 1>(a, st);
}
template <bool BACK>
cudaError_t any(const ra_norm_args& a, cudaStream_t st) {
  if (a.dtype == RA_F32) return dispatch<BACK, float, float>(a, st);
  return a.w_dtype == RA_F32 ? dispatch<BACK, bf16, float>(a, st) : dispatch<BACK, bf16, bf16>(a, st);
}

}  // namespace

size_t norm_workspace(const ra_norm_args& a) { return WS_ZERO + (size_t)bwd_ctas(a) * 2 * a.hidden * sizeof(float); }
cudaError_t norm_fwd(const ra_norm_args& a, cudaStream_t st) { return any<false>(a, st); }
cudaError_t norm_bwd(const ra_norm_args& a, cudaStream_t st) {
  if (a.rows == 0) {
    const size_t n = (size_t)a.hidden * (a.w_dtype == RA_BF16 ? 2 : 4);
    cudaError_t e = a.dgamma_dev ? cudaMemsetAsync(a.dgamma_dev, 0, n, st) : cudaSuccess;
    if (e == cudaSuccess && a.dbeta_dev) e = cudaMemsetAsync(a.dbeta_dev, 0, n, st);
    return e;
  }
  return any<true>(a, st);
}

}  // namespace ra
