// k_norm.cu -- LayerNorm and RMSNorm with a residual's sum, and their backward with the weights' gradients.
//
// Forward, for each row z = x + residual of n values: mean m, then the deviations d = z - m; the rounding of m is
// taken out again by the deviations' own mean, so that rows far from zero keep their digits:
//   rstd = 1 / sqrt(mean(d^2) - mean(d)^2 + eps), y = (d - mean(d)) rstd gamma + beta.
// Backward, with u = (z - m) rstd and g = dy gamma: dx = rstd (g - mean(g) - u mean(g u)) + dsum, and the sums over rows
// dgamma = sum dy u, dbeta = sum dy, which each CTA keeps in registers over its rows; the CTAs' partial sums are added in
// a second kernel, in a fixed order.
//
// Bound: bytes.  A row is read once, held in registers through both reductions and written once.
#include "common.cuh"
#include "operators.h"

namespace ra {
namespace {

constexpr int NORM_MAX_CTAS = 608;  // four an SM of 152: the backward's partial sums

// VEC values at a VEC-aligned place (VEC 1: anywhere)
template <typename T, int VEC> struct Pack;
template <> struct Pack<float, 4> {
  static __device__ __forceinline__ void load(const float* p, float* v) {
    const float4 x = *reinterpret_cast<const float4*>(p);
    v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
  }
  static __device__ __forceinline__ void store(float* p, const float* v) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  }
};
template <> struct Pack<float, 8> {
  static __device__ __forceinline__ void load(const float* p, float* v) {
    Pack<float, 4>::load(p, v);
    Pack<float, 4>::load(p + 4, v + 4);
  }
  static __device__ __forceinline__ void store(float* p, const float* v) {
    Pack<float, 4>::store(p, v);
    Pack<float, 4>::store(p + 4, v + 4);
  }
};
template <> struct Pack<bf16, 8> {
  static __device__ __forceinline__ void load(const bf16* p, float* v) {
    const uint4 x = *reinterpret_cast<const uint4*>(p);
    const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&x);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = __bfloat1622float2(h[i]);
      v[2 * i] = f.x;
      v[2 * i + 1] = f.y;
    }
  }
  static __device__ __forceinline__ void store(bf16* p, const float* v) {
    uint4 x;
    __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&x);
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
    *reinterpret_cast<uint4*>(p) = x;
  }
};
template <typename T> struct Pack<T, 1> {
  static __device__ __forceinline__ void load(const T* p, float* v) { v[0] = to_f(p[0]); }
  static __device__ __forceinline__ void store(T* p, const float* v) { p[0] = from_f<T>(v[0]); }
};

// Sums of K values over the CTA, for every thread, in a fixed order.  `sh` holds 2 x 32 x K floats, used in turn by
// successive calls (`turn`), so that one barrier a call is enough.
template <int K>
__device__ __forceinline__ void block_sum(float (&v)[K], float* sh, int turn) {
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = warp_sum(v[k]);
  const int warps = (int)blockDim.x >> 5;
  if (warps == 1) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  float* at = sh + (turn & 1) * 32 * K;
  if (lane == 0)
#pragma unroll
    for (int k = 0; k < K; ++k) at[warp * K + k] = v[k];
  __syncthreads();
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = warp_sum(lane < warps ? at[lane * K + k] : 0.f);
}

// the most threads of a CTA: those of 8 and 32 values a thread take the longest rows of their kind
constexpr int max_threads(int n) { return n == 16 ? 512 : 1024; }

template <typename T, typename W, int VEC, int NV>
__global__ void __launch_bounds__(max_threads(VEC * NV)) norm_fwd_kernel(const ra_norm_args a) {
  __shared__ float sh[64];
  constexpr int N = VEC * NV;
  const int t = threadIdx.x, G = blockDim.x, H = a.hidden;
  const bool layer = a.kind == RA_NORM_LAYER;
  const float inv = 1.f / (float)H;
  const W* gamma = static_cast<const W*>(a.gamma_dev);
  const W* beta = static_cast<const W*>(a.beta_dev);
  pdl_wait();
  pdl_trigger();
  int turn = 0;
  for (int row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T* x = static_cast<const T*>(a.x_dev) + row * a.x_stride;
    float z[N];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * G + t) * VEC;
#pragma unroll
      for (int j = 0; j < VEC; ++j) z[i * VEC + j] = 0.f;
      if (c < H) Pack<T, VEC>::load(x + c, z + i * VEC);
    }
    if (a.residual_dev) {
      const T* r = static_cast<const T*>(a.residual_dev) + row * a.residual_stride;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = (i * G + t) * VEC;
        if (c < H) {
          float v[VEC];
          Pack<T, VEC>::load(r + c, v);
#pragma unroll
          for (int j = 0; j < VEC; ++j) z[i * VEC + j] += v[j];
        }
      }
      if (a.sum_dev) {
        T* s = static_cast<T*>(a.sum_dev) + row * a.sum_stride;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          const int c = (i * G + t) * VEC;
          if (c < H) Pack<T, VEC>::store(s + c, z + i * VEC);
        }
      }
    }
    float mean = 0.f;
    if (layer) {
      float s[1] = {0.f};
#pragma unroll
      for (int i = 0; i < N; ++i) s[0] += z[i];
      block_sum(s, sh, turn++);
      mean = s[0] * inv;
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if ((i * G + t) * VEC < H)
#pragma unroll
          for (int j = 0; j < VEC; ++j) z[i * VEC + j] -= mean;
    }
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < N; ++i) {
      s[0] = fmaf(z[i], z[i], s[0]);
      s[1] += z[i];
    }
    __shared__ float sh2[128];
    block_sum(s, sh2, turn);
    float off = 0.f;
    if (layer) {
      off = s[1] * inv;
      mean += off;
    }
    const float rstd = 1.f / sqrtf(fmaxf(s[0] * inv - off * off, 0.f) + a.eps);
    if (t == 0) {
      if (a.mean_dev && layer) a.mean_dev[row] = mean;
      if (a.rstd_dev) a.rstd_dev[row] = rstd;
    }
    T* y = static_cast<T*>(a.y_dev) + row * a.y_stride;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * G + t) * VEC;
      if (c < H) {
        float v[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) v[j] = (z[i * VEC + j] - off) * rstd;
        if (gamma) {
          float w[VEC];
          Pack<W, VEC>::load(gamma + c, w);
#pragma unroll
          for (int j = 0; j < VEC; ++j) v[j] *= w[j];
        }
        if (beta) {
          float w[VEC];
          Pack<W, VEC>::load(beta + c, w);
#pragma unroll
          for (int j = 0; j < VEC; ++j) v[j] += w[j];
        }
        Pack<T, VEC>::store(y + c, v);
      }
    }
    if (!layer) ++turn;
  }
}

// sums [2][ctas][hidden]: each CTA's part of dgamma, then of dbeta
template <typename T, typename W, int VEC, int NV>
__global__ void __launch_bounds__(max_threads(VEC * NV)) norm_bwd_kernel(const ra_norm_args a, float* sums) {
  __shared__ float sh[128];
  constexpr int N = VEC * NV;
  const int t = threadIdx.x, G = blockDim.x, H = a.hidden;
  const bool layer = a.kind == RA_NORM_LAYER;
  const float inv = 1.f / (float)H;
  const W* gamma = static_cast<const W*>(a.gamma_dev);
  const char* zsrc = static_cast<const char*>(a.residual_dev ? a.sum_dev : a.x_dev);
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
      if (c < H) Pack<W, VEC>::load(gamma + c, w + i * VEC);
    }
  int turn = 0;
  for (int row = blockIdx.x; row < a.rows; row += gridDim.x, ++turn) {
    const T* x = reinterpret_cast<const T*>(zsrc) + row * zstride;
    const T* dy = static_cast<const T*>(a.dy_dev) + row * a.dy_stride;
    const float mean = layer ? a.mean_dev[row] : 0.f, rstd = a.rstd_dev[row];
    float u[N], g[N];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * G + t) * VEC;
#pragma unroll
      for (int j = 0; j < VEC; ++j) u[i * VEC + j] = mean, g[i * VEC + j] = 0.f;
      if (c < H) {
        Pack<T, VEC>::load(x + c, u + i * VEC);
        Pack<T, VEC>::load(dy + c, g + i * VEC);
      }
    }
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < N; ++i) {
      u[i] = (u[i] - mean) * rstd;
      dg[i] = fmaf(g[i], u[i], dg[i]);
      db[i] += g[i];
      g[i] *= w[i];
      s[0] += g[i];
      s[1] = fmaf(g[i], u[i], s[1]);
    }
    if (!a.dx_dev) continue;
    block_sum(s, sh, turn);
    const float mg = layer ? s[0] * inv : 0.f, mgu = s[1] * inv;
    const T* ds = a.dsum_dev ? static_cast<const T*>(a.dsum_dev) + row * a.dsum_stride : nullptr;
    T* dx = static_cast<T*>(a.dx_dev) + row * a.dx_stride;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * G + t) * VEC;
      if (c < H) {
        float v[VEC], d[VEC];
        if (ds) Pack<T, VEC>::load(ds + c, d);
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          v[j] = (g[i * VEC + j] - mg - u[i * VEC + j] * mgu) * rstd;
          if (ds) v[j] += d[j];
        }
        Pack<T, VEC>::store(dx + c, v);
      }
    }
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

// dgamma and dbeta of 32 columns from `ctas` partial sums: 16 warps take every 16th, then the warps' sums in turn
template <typename W>
__global__ void __launch_bounds__(512) norm_weights_kernel(const float* sums, W* dgamma, W* dbeta, int ctas, int H) {
  __shared__ float sh[16][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  W* out = blockIdx.y ? dbeta : dgamma;
  pdl_wait();
  pdl_trigger();
  if (!out) return;
  const float* at = sums + (int64_t)blockIdx.y * ctas * H;
  float s = 0.f;
  if (c < H)
#pragma unroll 8
    for (int i = warp; i < ctas; i += 16) s += at[(int64_t)i * H + c];
  sh[warp][lane] = s;
  __syncthreads();
  if (warp == 0 && c < H) {
    s = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) s += sh[i][lane];
    out[c] = from_f<W>(s);
  }
}

int bwd_ctas(const ra_norm_args& a) { return a.rows < NORM_MAX_CTAS ? a.rows : NORM_MAX_CTAS; }

template <typename T, typename W, int VEC, int NV>
cudaError_t launch(const ra_norm_args& a, bool backward, cudaStream_t st) {
  const int vecs = (a.hidden + VEC - 1) / VEC;
  const int threads = ((vecs + NV - 1) / NV + 31) / 32 * 32;
  note_launch(1);
  if (!backward) {
    const int most = 8 * device_sm_count();
    return launch_pdl(norm_fwd_kernel<T, W, VEC, NV>, dim3(a.rows < most ? a.rows : most), dim3(threads), 0, st, a);
  }
  const int ctas = bwd_ctas(a);
  float* sums = reinterpret_cast<float*>(static_cast<char*>(a.workspace_dev) + WS_ZERO);
  cudaError_t e = launch_pdl(norm_bwd_kernel<T, W, VEC, NV>, dim3(ctas), dim3(threads), 0, st, a, sums);
  if (e != cudaSuccess || (!a.dgamma_dev && !a.dbeta_dev)) return e;
  note_launch(1);
  return launch_pdl(norm_weights_kernel<W>, dim3((a.hidden + 31) / 32, a.dbeta_dev ? 2 : 1), dim3(512), 0, st,
                    (const float*)sums, (W*)a.dgamma_dev, (W*)a.dbeta_dev, ctas, (int)a.hidden);
}

bool at16(const void* p, int64_t stride, int es) { return !p || (((uintptr_t)p & 15) == 0 && stride * es % 16 == 0); }

template <typename T, typename W>
cudaError_t dispatch(const ra_norm_args& a, bool backward, cudaStream_t st) {
  constexpr int es = sizeof(T), V = 16 / es;
  bool wide = a.hidden % V == 0 && at16(a.gamma_dev, 0, es) && at16(a.beta_dev, 0, es);
  if (!backward || !a.residual_dev) wide = wide && at16(a.x_dev, a.x_stride, es);
  wide = wide && at16(a.sum_dev, a.sum_stride, es);
  if (backward)
    wide = wide && at16(a.dy_dev, a.dy_stride, es) && at16(a.dsum_dev, a.dsum_stride, es) && at16(a.dx_dev, a.dx_stride, es);
  else
    wide = wide && at16(a.residual_dev, a.residual_stride, es) && at16(a.y_dev, a.y_stride, es);
  if (wide) {
    const int vecs = a.hidden / V;
    if (vecs <= 64) return launch<T, W, V, 1>(a, backward, st);
    if (a.hidden <= 8192) return launch<T, W, V, 16 / V>(a, backward, st);
    return launch<T, W, V, 32 / V>(a, backward, st);
  }
  if (a.hidden <= 8192) return launch<T, W, 1, 8>(a, backward, st);
  return launch<T, W, 1, 32>(a, backward, st);
}

cudaError_t any(const ra_norm_args& a, bool backward, cudaStream_t st) {
  if (a.dtype == RA_F32) return dispatch<float, float>(a, backward, st);
  return a.w_dtype == RA_F32 ? dispatch<bf16, float>(a, backward, st) : dispatch<bf16, bf16>(a, backward, st);
}

}  // namespace

size_t norm_workspace(const ra_norm_args& a) { return WS_ZERO + (size_t)bwd_ctas(a) * 2 * a.hidden * sizeof(float); }
cudaError_t norm_fwd(const ra_norm_args& a, cudaStream_t st) { return any(a, false, st); }
cudaError_t norm_bwd(const ra_norm_args& a, cudaStream_t st) {
  if (a.rows == 0) {
    const size_t n = (size_t)a.hidden * (a.w_dtype == RA_BF16 ? 2 : 4);
    cudaError_t e = a.dgamma_dev ? cudaMemsetAsync(a.dgamma_dev, 0, n, st) : cudaSuccess;
    if (e == cudaSuccess && a.dbeta_dev) e = cudaMemsetAsync(a.dbeta_dev, 0, n, st);
    return e;
  }
  return any(a, true, st);
}

}  // namespace ra
