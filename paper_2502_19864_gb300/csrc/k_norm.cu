// k_norm.cu -- LayerNorm and RMSNorm with a residual's sum, and their backward with the weights' gradients.
//
// Forward, for each row z = x + residual of n values: mean m, then the deviations d = z - m; the rounding of m is
// taken out again by the deviations' own mean, so that rows far from zero keep their digits:
//   rstd = 1 / sqrt(mean(d^2) - mean(d)^2 + eps), y = (d - mean(d)) rstd gamma + beta.
// Backward, with u = (z - m) rstd and g = dy gamma: dx = rstd (g - mean(g) - u mean(g u)) + dsum, and the sums over rows
// dgamma = sum dy u, dbeta = sum dy, which each CTA keeps in registers over its rows; the CTAs' partial sums are added in
// a second kernel, in a fixed order.
//
// Bound: bytes.  A row is read once, held in registers through the reductions and written once.  A CTA's threads share a
// row, eight (16, 32) values each, and take ROWS rows at a time, so that enough loads are on their way and a barrier
// serves them all.
#include <algorithm>

#include "common.cuh"
#include "operators.h"

namespace ra {
namespace {

constexpr int NORM_MAX_CTAS = 608;  // four an SM of 152: the backward's partial sums

// VEC values at a 16-byte aligned place (VEC 1: anywhere), as they come from memory.  keep(): what was computed of them before is
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
  if (VEC == 1) *p = v[0];
  else *reinterpret_cast<float4*>(p) = make_float4(v[0], v[VEC > 1 ? 1 : 0], v[VEC > 1 ? 2 : 0], v[VEC > 1 ? 3 : 0]);
}
template <int VEC> __device__ __forceinline__ void put(bf16* p, const float* v) {
  if (VEC == 1) {
    *p = __float2bfloat16_rn(v[0]);
  } else {
    uint4 x;
    __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&x);
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = __floats2bfloat162_rn(v[VEC > 1 ? 2 * i : 0], v[VEC > 1 ? 2 * i + 1 : 0]);
    *reinterpret_cast<uint4*>(p) = x;
  }
}

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
constexpr int min_ctas(int n, int rows) { return n == 8 && rows > 1 ? 2 : 1; }

template <typename T, typename W, int VEC, int NV, int ROWS>
__global__ void __launch_bounds__(max_threads(VEC * NV, ROWS), min_ctas(VEC * NV, ROWS)) norm_fwd_kernel(const __grid_constant__ ra_norm_args a) {
  __shared__ __align__(16) float sh1[2 * 32 * ROWS], sh2[2 * 32 * 2 * ROWS];
  constexpr int N = VEC * NV;
  const int t = threadIdx.x, G = blockDim.x, H = a.hidden;
  const bool layer = a.kind == RA_NORM_LAYER;
  const float inv = 1.f / (float)H;
  const W* gamma = static_cast<const W*>(a.gamma_dev);
  const W* beta = static_cast<const W*>(a.beta_dev);
  pdl_wait();
  pdl_trigger();
  int turn = 0;
  for (int64_t row0 = (int64_t)blockIdx.x * ROWS; row0 < a.rows; row0 += (int64_t)gridDim.x * ROWS, ++turn) {
    float z[ROWS][N];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const T* x = static_cast<const T*>(a.x_dev) + (row0 + r) * a.x_stride;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = (i * G + t) * VEC;
#pragma unroll
        for (int j = 0; j < VEC; ++j) z[r][i * VEC + j] = 0.f;
        if (c < H && row0 + r < a.rows) {
          Raw<T, VEC> v;
          v.load(x + c);
          v.get(z[r] + i * VEC);
        }
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
            Raw<T, VEC> v;
            v.load(p + c);
            v.get(f);
#pragma unroll
            for (int j = 0; j < VEC; ++j) z[r][i * VEC + j] += f[j];
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
    float mean[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) mean[r] = 0.f;
    if (layer) {
#pragma unroll
      for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int i = 0; i < N; ++i) mean[r] += z[r][i];
      block_sum(mean, sh1, turn);
#pragma unroll
      for (int r = 0; r < ROWS; ++r) {
        mean[r] *= inv;
#pragma unroll
        for (int i = 0; i < NV; ++i)
          if ((i * G + t) * VEC < H)
#pragma unroll
            for (int j = 0; j < VEC; ++j) z[r][i * VEC + j] -= mean[r];
      }
    }
    float s[2 * ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      s[2 * r] = s[2 * r + 1] = 0.f;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        s[2 * r] = fmaf(z[r][i], z[r][i], s[2 * r]);
        s[2 * r + 1] += z[r][i];
      }
    }
    block_sum(s, sh2, turn);
    float off[ROWS], rstd[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      off[r] = layer ? s[2 * r + 1] * inv : 0.f;
      mean[r] += off[r];
      rstd[r] = 1.f / sqrtf(fmaxf(s[2 * r] * inv - off[r] * off[r], 0.f) + a.eps);
      if (s[2 * r] != s[2 * r]) rstd[r] = s[2 * r];  // (fmaxf would lose a NaN)
      if (t == 0 && row0 + r < a.rows) {
        if (a.mean_dev && layer) a.mean_dev[row0 + r] = mean[r];
        if (a.rstd_dev) a.rstd_dev[row0 + r] = rstd[r];
      }
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
#pragma unroll
        for (int j = 0; j < VEC; ++j) f[j] = fmaf((z[r][i * VEC + j] - off[r]) * rstd[r], w[j], b[j]);
        if (row0 + r < a.rows) put<VEC>(static_cast<T*>(a.y_dev) + (row0 + r) * a.y_stride + c, f);
      }
    }
  }
}

// sums [2][ctas][hidden]: each CTA's part of dgamma, then of dbeta
template <typename T, typename W, int VEC, int NV, int ROWS>
__global__ void __launch_bounds__(max_threads(VEC * NV, ROWS), min_ctas(VEC * NV, ROWS)) norm_bwd_kernel(const __grid_constant__ ra_norm_args a, float* sums) {
  __shared__ __align__(16) float sh[2 * 32 * 2 * ROWS];
  constexpr int N = VEC * NV;
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
  int turn = 0;
  for (int64_t row0 = (int64_t)blockIdx.x * ROWS; row0 < a.rows; row0 += (int64_t)gridDim.x * ROWS, ++turn) {
    Raw<T, VEC> x[ROWS][NV], y[ROWS][NV], d[ROWS][NV];
    float mean[ROWS], rstd[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const int64_t row = row0 + r;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = (i * G + t) * VEC;
        if (c < H && row < a.rows) {
          x[r][i].load(zsrc + row * zstride + c);
          y[r][i].load(static_cast<const T*>(a.dy_dev) + row * a.dy_stride + c);
        }
      }
      mean[r] = layer && row < a.rows ? a.mean_dev[row] : 0.f;
      rstd[r] = row < a.rows ? a.rstd_dev[row] : 0.f;
    }
    if (a.dsum_dev && a.dx_dev)  // (on their way through the reductions)
#pragma unroll
      for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          const int c = (i * G + t) * VEC;
          if (c < H && row0 + r < a.rows) d[r][i].load(static_cast<const T*>(a.dsum_dev) + (row0 + r) * a.dsum_stride + c);
        }
    float s[2 * ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      s[2 * r] = s[2 * r + 1] = 0.f;
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if ((i * G + t) * VEC < H && row0 + r < a.rows) {
          float u[VEC], g[VEC];
          x[r][i].get(u);
          y[r][i].get(g);
#pragma unroll
          for (int j = 0; j < VEC; ++j) {
            const int k = i * VEC + j;
            u[j] = (u[j] - mean[r]) * rstd[r];
            dg[k] = fmaf(g[j], u[j], dg[k]);
            db[k] += g[j];
            g[j] *= w[k];
            s[2 * r] += g[j];
            s[2 * r + 1] = fmaf(g[j], u[j], s[2 * r + 1]);
          }
        }
    }
    if (!a.dx_dev) continue;
    block_sum(s, sh, turn);
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const float mg = layer ? s[2 * r] * inv : 0.f, mgu = s[2 * r + 1] * inv;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = (i * G + t) * VEC;
        if (c < H && row0 + r < a.rows) {
          float u[VEC], g[VEC], e[VEC];
          x[r][i].keep();
          y[r][i].keep();
          x[r][i].get(u);
          y[r][i].get(g);
          if (a.dsum_dev) d[r][i].get(e);
#pragma unroll
          for (int j = 0; j < VEC; ++j) {
            u[j] = (u[j] - mean[r]) * rstd[r];
            g[j] = (g[j] * w[i * VEC + j] - mg - u[j] * mgu) * rstd[r];
            if (a.dsum_dev) g[j] += e[j];
          }
          put<VEC>(static_cast<T*>(a.dx_dev) + (row0 + r) * a.dx_stride + c, g);
        }
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

int bwd_ctas(const ra_norm_args& a) { return std::min(a.rows, NORM_MAX_CTAS); }

template <typename T, typename W, int VEC, int NV, int ROWS>
cudaError_t launch(const ra_norm_args& a, bool backward, cudaStream_t st) {
  const int vecs = (a.hidden + VEC - 1) / VEC;
  const int threads = ((vecs + NV - 1) / NV + 31) / 32 * 32;
  const int groups = (a.rows + ROWS - 1) / ROWS;
  note_launch(1);
  if (!backward) {
    const int most = device_sm_count() * std::max(1, std::min(32, 2048 / threads));
    return launch_pdl(norm_fwd_kernel<T, W, VEC, NV, ROWS>, dim3(std::min(groups, most)), dim3(threads), 0, st, a);
  }
  const int ctas = std::min(groups, NORM_MAX_CTAS);
  float* sums = reinterpret_cast<float*>(static_cast<char*>(a.workspace_dev) + WS_ZERO);
  cudaError_t e = launch_pdl(norm_bwd_kernel<T, W, VEC, NV, ROWS>, dim3(ctas), dim3(threads), 0, st, a, sums);
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
  // several rows at a time where there are enough of them for every SM
  const bool many = a.rows >= 4 * 608;
  if (wide) {
    if (a.hidden <= 2048) return many ? launch<T, W, V, 8 / V, 16 / es / 2>(a, backward, st) : launch<T, W, V, 8 / V, 1>(a, backward, st);
    if (a.hidden <= 8192) return many ? launch<T, W, V, 16 / V, 4 / es>(a, backward, st) : launch<T, W, V, 8 / V, 1>(a, backward, st);
    return launch<T, W, V, 32 / V, 1>(a, backward, st);
  }
  if (a.hidden <= 8192) return a.hidden <= 2048 && many ? launch<T, W, 1, 8, 16 / es / 2>(a, backward, st) : launch<T, W, 1, 8, 1>(a, backward, st);
  return launch<T, W, 1, 32, 1>(a, backward, st);
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
