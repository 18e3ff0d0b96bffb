// k_attention_window.cu -- causal attention with a sliding window and first tokens that stay visible, over whole
// sequences, in fp32 arithmetic: the forward and the backward of fp32 inputs (products of operands rounded to tf32 would be 1e-3 off).
//
// Query i sees key j when j <= i and (i - j < W or j < sinks), both below the sequence's length:
//   forward   o_i = sum_j p_ij v_j, p_ij = exp(scale q_i k_j - lse_i), by blocks of 64 keys with a running maximum
//             and sum;
//   backward  dV_j = sum_i p_ij dO_i;  dS_ij = p_ij (dO_i v_j - D_i), D_i = dO_i o_i;  dQ_i = scale sum_j dS_ij k_j;
//             dK_j = scale sum_i dS_ij q_i, the sums over i over all query heads that share the key.
// A query CTA holds 32 queries and walks the blocks of 64 keys that any of them sees: those of the window and those that
// hold sinks.  A key CTA holds 32 keys and walks, head by head of its group, the blocks of 64 queries that see any of them:
// dK and dV are sums in a fixed order.  Keys that are sinks are seen by every later query; where that makes their blocks
// much longer than a window, several CTAs share a block's queries and a last kernel adds their parts in order.  A kernel
// before them computes D, so that both passes of the backward run in one launch.  Rows past the sequence's end are loaded as
// zeros, whatever memory holds there.
// A warp has four held rows: a thread keeps their scores with 2 of the 64 streamed rows and their outputs in DH / 32
// columns.  What bounds it is the latency of a step at the sizes that fp32 models have, not a pipe: 32 held rows and eight
// warps (64 rows and as many warps: 228 us for 3 sequences of 333 tokens, 4 heads of 64 on 2, window 100, forward and
// backward; four warps of 4 x 4 scores a thread: 102 us; this, the passes one after the other: 77 us), the next step's rows on
// their way, and both passes at once: 55 us.
#include "common.cuh"
#include "operators.h"
#include "paged.cuh"

namespace ra {
namespace {

constexpr int BH = 32, BT = 64, NT = 256, PP = BT + 4;  // rows held and streamed, threads, floats of a row of X
constexpr float kLog2e = 1.4426950408889634f;

template <int DH>
struct Plan {
  static constexpr int DP = DH + 4;  // padded rows: eight lanes' 16 bytes of eight rows fall in distinct banks
  static constexpr int HELD = BH * DP, TILE = BT * DP;
  static constexpr int FWD_BYTES = (HELD + 4 * TILE + BH * PP) * 4, BWD_BYTES = (2 * HELD + 4 * TILE + BH * PP + 4 * BT) * 4;
};

// ROWS rows from r0 on of one head, zeros from row `len` on and past head_dim, on their way (cp.async)
template <int DH, int ROWS>
__device__ __forceinline__ void load_rows(float* dst, const float* src, int64_t stride, int r0, int len, int head_dim) {
  const uint32_t to = (uint32_t)__cvta_generic_to_shared(dst);
  for (int i = threadIdx.x; i < ROWS * DH / 4; i += NT) {
    const int r = i / (DH / 4), c = (i - r * (DH / 4)) * 4;
    const bool live = r0 + r < len && c < head_dim;
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to + (r * Plan<DH>::DP + c) * 4),
                 "l"(live ? src + (int64_t)(r0 + r) * stride + c : src), "r"(live ? 16 : 0) : "memory");
  }
}
// 64 floats from r0 on, zeros from `len` on
__device__ __forceinline__ void load_stats(float* dst, const float* src, int r0, int len) {
  const int i = threadIdx.x;
  if (i < BT) {
    const bool live = r0 + i < len;
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst + i)),
                 "l"(live ? src + r0 + i : src), "r"(live ? 4 : 0) : "memory");
  }
}
__device__ __forceinline__ void loads_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void loads_done() { asm volatile("cp.async.wait_all;" ::: "memory"); }
// all but the newest group of this thread's loads have landed
__device__ __forceinline__ void loads_before_newest() { asm volatile("cp.async.wait_group 1;" ::: "memory"); }

// acc[i][j] = A[4 ty + i] . B[tx + 32 j]
template <int DH>
__device__ __forceinline__ void dot_rows(float (&acc)[4][2], const float* A, const float* B, int ty, int tx) {
  float2 s[4][2];  // even and odd dims
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) s[i][j] = f2(0.f);
#pragma unroll 8
  for (int d = 0; d < DH; d += 4) {
    float4 a[4], b[2];
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = *reinterpret_cast<const float4*>(A + (4 * ty + i) * Plan<DH>::DP + d);
#pragma unroll
    for (int j = 0; j < 2; ++j) b[j] = *reinterpret_cast<const float4*>(B + (tx + 32 * j) * Plan<DH>::DP + d);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        s[i][j] = __ffma2_rn(make_float2(a[i].x, a[i].y), make_float2(b[j].x, b[j].y), s[i][j]);
        s[i][j] = __ffma2_rn(make_float2(a[i].z, a[i].w), make_float2(b[j].z, b[j].w), s[i][j]);
      }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) acc[i][j] = s[i][j].x + s[i][j].y;
}
// out[i][c] += sum_k X[4 ty + i][k] B[k][tx + 32 c]
template <int DH>
__device__ __forceinline__ void times_rows(float (&out)[4][DH / 32], const float* X, const float* B, int ty, int tx) {
#pragma unroll 4
  for (int k = 0; k < BT; k += 4) {
    float x[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) *reinterpret_cast<float4*>(x[i]) = *reinterpret_cast<const float4*>(X + (4 * ty + i) * PP + k);
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int c = 0; c < DH / 32; ++c) {
        const float b = B[(k + u) * Plan<DH>::DP + tx + 32 * c];
#pragma unroll
        for (int i = 0; i < 4; ++i) out[i][c] = fmaf(x[i][u], b, out[i][c]);
      }
  }
}
template <int DH>
__device__ __forceinline__ void store_rows(float* dst, int64_t stride, const float (&o)[4][DH / 32], const float (&f)[4],
                                           int r0, int rows, int head_dim, int ty, int tx) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = r0 + 4 * ty + i;
    if (r >= rows) continue;
#pragma unroll
    for (int c = 0; c < DH / 32; ++c)
      if (tx + 32 * c < head_dim) dst[(int64_t)r * stride + tx + 32 * c] = o[i][c] * f[i];
  }
}

struct Geometry {  // of a CTA's (block, sequence, head)
  int blk, b, head, len;
};
__device__ __forceinline__ Geometry geometry(const ra_attention_window_args& a, int heads, int n_blk, int64_t id) {
  Geometry g;
  g.blk = n_blk - 1 - (int)(id % n_blk);
  const int bh = (int)(id / n_blk);
  g.b = bh / heads;
  g.head = bh - g.b * heads;
  int len = a.lens_dev ? a.lens_dev[g.b] : a.seq;
  if (len < 0 || len > a.seq) {
    set_dev_error(a.err_dev, RA_DEVERR_BOUNDS);
    len = len < 0 ? 0 : a.seq;
  }
  g.len = len;
  return g;
}
// whether query i sees key j (W: at least 1; both within the sequence)
__device__ __forceinline__ bool sees(int i, int j, int W, int sinks, int len) {
  return j <= i && (i - j < W || j < sinks) && i < len;
}

// The key blocks that the queries r0 .. last see: those with sinks, [0, ns), then [lo, hi]
struct KeyBlocks {
  int ns, lo, n;
  __device__ __forceinline__ int at(int i) const { return i < ns ? i : i - ns + lo; }
};
__device__ __forceinline__ KeyBlocks key_blocks(int r0, int last, int W, int sinks) {
  KeyBlocks k;
  const int hi = last / BT, first = r0 - W + 1, sink_blocks = sinks / BT + (sinks % BT != 0);
  k.lo = first > 0 ? first / BT : 0;
  k.ns = sink_blocks < hi + 1 ? sink_blocks : hi + 1;
  if (k.lo < k.ns) k.lo = k.ns;
  k.n = k.ns + (hi >= k.lo ? hi - k.lo + 1 : 0);
  return k;
}

template <int DH>
__global__ void __launch_bounds__(NT) window_fwd_simt_kernel(const __grid_constant__ ra_attention_window_args a, int W, int n_blk) {
  extern __shared__ __align__(16) float sm[];
  using P = Plan<DH>;
  float *Q = sm, *KV = Q + P::HELD, *X = KV + 4 * P::TILE;  // (two buffers of K and V)
  pdl_wait();
  pdl_trigger();
  const Geometry g = geometry(a, a.n_heads, n_blk, blockIdx.x);
  const int tid = threadIdx.x, ty = tid >> 5, tx = tid & 31, q0 = g.blk * BH, dh = a.head_dim;
  const int kvh = g.head / (a.n_heads / a.n_kv_heads);
  const int64_t tok0 = (int64_t)g.b * a.seq;
  const float* q = (const float*)a.q_dev + tok0 * a.q_stride + g.head * dh;
  const float* k = (const float*)a.k_dev + tok0 * a.k_stride + kvh * dh;
  const float* v = (const float*)a.v_dev + tok0 * a.v_stride + kvh * dh;
  float o[4][DH / 32], m[4], l[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    m[i] = -INFINITY;
    l[i] = 0.f;
#pragma unroll
    for (int c = 0; c < DH / 32; ++c) o[i][c] = 0.f;
  }
  const float sl2 = a.scale * kLog2e;
  if (q0 < g.len) {
    load_rows<DH, BH>(Q, q, a.q_stride, q0, g.len, dh);
    const KeyBlocks kb = key_blocks(q0, q0 + BH - 1 < g.len ? q0 + BH - 1 : g.len - 1, W, a.sinks);
    auto fetch = [&](int n) {
      if (n < kb.n) {
        float* to = KV + (n & 1) * 2 * P::TILE;
        load_rows<DH, BT>(to, k, a.k_stride, kb.at(n) * BT, g.len, dh);
        load_rows<DH, BT>(to + P::TILE, v, a.v_stride, kb.at(n) * BT, g.len, dh);
      }
      loads_commit();
    };
    fetch(0);
    for (int n = 0; n < kb.n; ++n) {
      const int k0 = kb.at(n) * BT;
      const float *K = KV + (n & 1) * 2 * P::TILE, *V = K + P::TILE;
      fetch(n + 1);
      loads_before_newest();
      __syncthreads();
      float s[4][2];
      dot_rows<DH>(s, Q, K, ty, tx);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int qi = q0 + 4 * ty + i;
        float bm = -INFINITY;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          s[i][j] = sees(qi, k0 + tx + 32 * j, W, a.sinks, g.len) ? s[i][j] * sl2 : -INFINITY;
          bm = fmaxf(bm, s[i][j]);
        }
        bm = warp_max(bm);
        const float mn = fmaxf(m[i], bm), ms = mn == -INFINITY ? 0.f : mn, f = exp2f(m[i] - ms);
        m[i] = mn;
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float p = exp2f(s[i][j] - ms);
          sum += p;
          X[(4 * ty + i) * PP + tx + 32 * j] = p;
        }
        l[i] = l[i] * f + sum;  // (a lane's own share; the lanes are summed at the end)
#pragma unroll
        for (int c = 0; c < DH / 32; ++c) o[i][c] *= f;
      }
      __syncthreads();
      times_rows<DH>(o, X, V, ty, tx);
      __syncthreads();  // the buffer and X are free again
    }
  }
  loads_done();
  float f[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    l[i] = warp_sum(l[i]);
    f[i] = l[i] > 0.f ? 1.f / l[i] : l[i] == 0.f ? 0.f : l[i];
    const int qi = q0 + 4 * ty + i;
    if (a.lse_dev && tx == 0 && qi < a.seq)  // (the maximum of NaN scores stays -inf, their sum does not stay 0)
      a.lse_dev[((int64_t)g.b * a.n_heads + g.head) * a.seq + qi] =
          m[i] == -INFINITY && l[i] == 0.f ? -INFINITY : (m[i] + log2f(l[i])) * 0.69314718055994531f;
  }
  store_rows<DH>((float*)a.out_dev + tok0 * a.out_stride + g.head * dh, a.out_stride, o, f, q0, a.seq, dh, ty, tx);
}

// ---- backward ------------------------------------------------------------------------------
// D = dO . o of every row and head, eight threads each
__global__ void __launch_bounds__(256) window_d_simt_kernel(const __grid_constant__ ra_attention_window_args a, float* Dv) {
  pdl_wait();
  pdl_trigger();
  const int64_t row = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> 3;  // (token of the batch, head)
  const int64_t tok = row / a.n_heads;
  const int h = (int)(row - tok * a.n_heads), part = threadIdx.x & 7;
  const int64_t b = tok / a.seq;
  if (b >= a.batch) return;  // (the eight of a row together)
  const int q = (int)(tok - b * a.seq), len = clamp_len(a.lens_dev ? a.lens_dev[b] : a.seq, a.seq, a.err_dev);
  float d = 0.f;
  if (q < len) {
    const float* o = (const float*)a.out_dev + tok * a.out_stride + h * a.head_dim;
    const float* g = (const float*)a.dout_dev + tok * a.dout_stride + h * a.head_dim;
    for (int c = 4 * part; c < a.head_dim; c += 32) {
      const float4 x = *reinterpret_cast<const float4*>(o + c), y = *reinterpret_cast<const float4*>(g + c);
      d = fmaf(x.x, y.x, fmaf(x.y, y.y, fmaf(x.z, y.z, fmaf(x.w, y.w, d))));
    }
  }
#pragma unroll
  for (int m = 1; m < 8; m <<= 1) d += __shfl_xor_sync(0xffu << (threadIdx.x & 24), d, m);
  if (part == 0) Dv[(b * a.n_heads + h) * a.seq + q] = d;
}

// KEYS: the held rows are keys (dK, dV), the streamed ones queries; else queries (dQ) and keys
template <int DH, bool KEYS>
__device__ __forceinline__ void bwd_pass(const ra_attention_window_args& a, const float* Dv, float* parts, int W, int n_blk, int split, int chunks,
                                         int64_t cta) {
  extern __shared__ __align__(16) float sm[];
  using P = Plan<DH>;
  float *T0 = sm, *T1 = T0 + P::HELD, *BUF = T1 + P::HELD, *X = BUF + 4 * P::TILE, *STAT = X + BH * PP;  // (two buffers of the streamed pair, and of lse and D)
  const int G = a.n_heads / a.n_kv_heads, items = n_blk - split + split * chunks;
  Geometry g = geometry(a, KEYS ? a.n_kv_heads : a.n_heads, items, cta);
  int chunk = 0, n_chunks = 1;
  if (KEYS) {  // (g.blk counts down: the first blocks, which most queries see, come first)
    const int it = items - 1 - g.blk;
    const bool shared = it < split * chunks;
    g.blk = shared ? it / chunks : it - split * chunks + split;
    chunk = shared ? it - g.blk * chunks : 0;
    n_chunks = shared ? chunks : 1;
  }
  const int tid = threadIdx.x, ty = tid >> 5, tx = tid & 31, r0 = g.blk * BH, dh = a.head_dim;
  const int kvh = KEYS ? g.head : g.head / G;
  const int64_t tok0 = (int64_t)g.b * a.seq;
  const float* k = (const float*)a.k_dev + tok0 * a.k_stride + kvh * dh;
  const float* v = (const float*)a.v_dev + tok0 * a.v_stride + kvh * dh;
  float u[4][DH / 32], w[4][DH / 32];  // KEYS: dK, dV; else dQ
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int c = 0; c < DH / 32; ++c) u[i][c] = w[i][c] = 0.f;
  const float sl2 = a.scale * kLog2e;
  // X = P (or P^T), then dS in s
  auto probabilities = [&](float (&s)[4][2], int c0, const float* L) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int row = 4 * ty + i, col = tx + 32 * j;
        const int qi = KEYS ? c0 + col : r0 + row, ki = KEYS ? r0 + row : c0 + col;
        s[i][j] = sees(qi, ki, W, a.sinks, g.len) ? exp2f(s[i][j] * sl2 - L[KEYS ? col : row] * kLog2e) : 0.f;
      }
  };
  auto put = [&](const float (&s)[4][2]) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) X[(4 * ty + i) * PP + tx + 32 * j] = s[i][j];
  };
  if (r0 < g.len) {
    const int last = r0 + BH - 1 < g.len ? r0 + BH - 1 : g.len - 1;
    if (KEYS) {
      load_rows<DH, BH>(T0, k, a.k_stride, r0, g.len, dh);
      load_rows<DH, BH>(T1, v, a.v_stride, r0, g.len, dh);
      const int64_t far = r0 < a.sinks ? g.len - 1 : (int64_t)last + W - 1;
      const int first = r0 / BT, per_head = (int)(far < g.len ? far : g.len - 1) / BT - first + 1;
      const int64_t total = (int64_t)per_head * G;
      const int n1 = (int)(total * (chunk + 1) / n_chunks);
      const int n0 = (int)(total * chunk / n_chunks);
      auto fetch = [&](int n) {
        if (n < n1) {
          const int h = kvh * G + n / per_head, q0 = (first + n % per_head) * BT, buf = (n - n0) & 1;
          float* to = BUF + buf * 2 * P::TILE;
          load_rows<DH, BT>(to, (const float*)a.q_dev + tok0 * a.q_stride + h * dh, a.q_stride, q0, g.len, dh);
          load_rows<DH, BT>(to + P::TILE, (const float*)a.dout_dev + tok0 * a.dout_stride + h * dh, a.dout_stride, q0, g.len, dh);
          const int64_t at = ((int64_t)g.b * a.n_heads + h) * a.seq;
          load_stats(STAT + buf * 2 * BT, a.lse_dev + at, q0, g.len);
          load_stats(STAT + buf * 2 * BT + BT, Dv + at, q0, g.len);
        }
        loads_commit();
      };
      fetch(n0);
      for (int n = n0; n < n1; ++n) {
        const int q0 = (first + n % per_head) * BT, buf = (n - n0) & 1;
        const float *T2 = BUF + buf * 2 * P::TILE, *T3 = T2 + P::TILE, *L = STAT + buf * 2 * BT, *D = L + BT;
        fetch(n + 1);
        loads_before_newest();
        __syncthreads();
        float s[4][2], dp[4][2];
        dot_rows<DH>(s, T0, T2, ty, tx);
        probabilities(s, q0, L);
        put(s);
        dot_rows<DH>(dp, T1, T3, ty, tx);
        __syncthreads();
        times_rows<DH>(w, X, T3, ty, tx);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) s[i][j] *= dp[i][j] - D[tx + 32 * j];
        __syncthreads();
        put(s);
        __syncthreads();
        times_rows<DH>(u, X, T2, ty, tx);
        __syncthreads();  // the buffer and X are free again
      }
    } else {
      load_rows<DH, BH>(T0, (const float*)a.q_dev + tok0 * a.q_stride + g.head * dh, a.q_stride, r0, g.len, dh);
      load_rows<DH, BH>(T1, (const float*)a.dout_dev + tok0 * a.dout_stride + g.head * dh, a.dout_stride, r0, g.len, dh);
      const int64_t at = ((int64_t)g.b * a.n_heads + g.head) * a.seq + r0;
      float *L = STAT, *D = L + BT;
      if (tid < BH) {
        L[tid] = r0 + tid < g.len ? a.lse_dev[at + tid] : 0.f;
        D[tid] = r0 + tid < g.len ? Dv[at + tid] : 0.f;
      }
      const KeyBlocks kb = key_blocks(r0, last, W, a.sinks);
      auto fetch = [&](int n) {
        if (n < kb.n) {
          float* to = BUF + (n & 1) * 2 * P::TILE;
          load_rows<DH, BT>(to, k, a.k_stride, kb.at(n) * BT, g.len, dh);
          load_rows<DH, BT>(to + P::TILE, v, a.v_stride, kb.at(n) * BT, g.len, dh);
        }
        loads_commit();
      };
      fetch(0);
      for (int n = 0; n < kb.n; ++n) {
        const int k0 = kb.at(n) * BT;
        const float *T2 = BUF + (n & 1) * 2 * P::TILE, *T3 = T2 + P::TILE;
        fetch(n + 1);
        loads_before_newest();
        __syncthreads();
        float s[4][2], dp[4][2];
        dot_rows<DH>(s, T0, T2, ty, tx);
        probabilities(s, k0, L);
        dot_rows<DH>(dp, T1, T3, ty, tx);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) s[i][j] *= dp[i][j] - D[4 * ty + i];
        put(s);
        __syncthreads();
        times_rows<DH>(u, X, T2, ty, tx);
        __syncthreads();  // the buffer and X are free again
      }
    }
  }
  loads_done();
  const float fs[4] = {a.scale, a.scale, a.scale, a.scale}, f1[4] = {1.f, 1.f, 1.f, 1.f};
  if (KEYS && n_chunks > 1) {
    float* part = parts + (((int64_t)(g.b * a.n_kv_heads + g.head) * split + g.blk) * chunks + chunk) * (2 * BH * DH);
    store_rows<DH>(part, DH, u, fs, 0, BH, DH, ty, tx);
    store_rows<DH>(part + BH * DH, DH, w, f1, 0, BH, DH, ty, tx);
  } else if (KEYS) {
    store_rows<DH>((float*)a.dk_dev + tok0 * a.dk_stride + kvh * dh, a.dk_stride, u, fs, r0, a.seq, dh, ty, tx);
    store_rows<DH>((float*)a.dv_dev + tok0 * a.dv_stride + kvh * dh, a.dv_stride, w, f1, r0, a.seq, dh, ty, tx);
  } else {
    store_rows<DH>((float*)a.dq_dev + tok0 * a.dq_stride + g.head * dh, a.dq_stride, u, fs, r0, a.seq, dh, ty, tx);
  }
}

// Both passes in one launch, the keys' CTAs (the longer ones) first: where there are few of either they run at once
template <int DH>
__global__ void __launch_bounds__(NT) window_bwd_simt_kernel(const __grid_constant__ ra_attention_window_args a, const float* Dv, float* parts, int W,
                                                             int n_blk, int split, int chunks, int64_t key_ctas) {
  pdl_wait();
  pdl_trigger();
  if (blockIdx.x < key_ctas)
    bwd_pass<DH, true>(a, Dv, parts, W, n_blk, split, chunks, blockIdx.x);
  else
    bwd_pass<DH, false>(a, Dv, parts, W, n_blk, 0, 1, blockIdx.x - key_ctas);
}

// dK and dV of the shared key blocks: the parts in order, four values a thread
template <int DH>
__global__ void __launch_bounds__(256) window_bwd_simt_parts_kernel(const __grid_constant__ ra_attention_window_args a, const float* parts,
                                                                    int split, int chunks) {
  pdl_wait();
  pdl_trigger();
  constexpr int PER = BH * DH / 4;
  const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x, blk = e / (2 * PER);
  if (blk >= (int64_t)a.batch * a.n_kv_heads * split) return;
  const int x = (int)(e - blk * (2 * PER)), o = x / PER, y = x - o * PER, row = y / (DH / 4), c = (y - row * (DH / 4)) * 4;
  const int64_t unit = blk / split;
  const int r = (int)(blk - unit * split) * BH + row, head = (int)(unit % a.n_kv_heads), b = (int)(unit / a.n_kv_heads);
  if (r >= a.seq || c >= a.head_dim) return;
  const float* p = parts + blk * chunks * (2 * BH * DH) + (o * BH + row) * DH + c;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int i = 0; i < chunks; ++i) {
    const float4 v = *reinterpret_cast<const float4*>(p + (int64_t)i * (2 * BH * DH));
    s.x += v.x;
    s.y += v.y;
    s.z += v.z;
    s.w += v.w;
  }
  float* d = o == 0 ? (float*)a.dk_dev + ((int64_t)b * a.seq + r) * a.dk_stride : (float*)a.dv_dev + ((int64_t)b * a.seq + r) * a.dv_stride;
  *reinterpret_cast<float4*>(d + head * a.head_dim + c) = s;
}

int window_of(const ra_attention_window_args& a) { return a.window == 0 || a.window > a.seq ? a.seq : a.window; }

int dims_of(const ra_attention_window_args& a) { return a.head_dim <= 32 ? 32 : a.head_dim <= 64 ? 64 : a.head_dim <= 96 ? 96 : 128; }

// How many CTAs share each of the first `split` key blocks.  An ordinary block is seen from W + 32 queries, one with sinks
// from all: up to 128 sinks and where that is twice as long, as many CTAs as bring those blocks back to an ordinary one's
// length, at most 32.  Where the key blocks are fewer than 152 (the SMs, as a constant: the order of the sums is the shape's),
// all are shared, so that the SMs have two CTAs each beside those of the queries, at most 8 a block (63 blocks of 2000 tokens,
// 2 heads of 32 over 1: one CTA an SM 136 us, two 88; 66 blocks of the case above: 57 and 55 us; 176 blocks: 62 us, shared 66).
void split_of(const ra_attention_window_args& a, int& split, int& chunks) {
  const int64_t ordinary = (int64_t)window_of(a) + BH;
  split = 0;
  chunks = 1;
  const int n_blk = (a.seq + BH - 1) / BH;
  const int64_t all = (int64_t)n_blk * a.batch * a.n_kv_heads;
  if (all == 0) return;
  if (all < 152) {
    split = n_blk;
    chunks = (int)((2 * 152 + all - 1) / all);
    if (chunks > 8) chunks = 8;
    return;
  }
  if (a.sinks < 1 || a.sinks > 128 || a.seq < 2 * ordinary) return;
  const int blocks = (a.sinks + BH - 1) / BH;
  split = blocks < n_blk ? blocks : n_blk;
  const int64_t n = (a.seq + ordinary - 1) / ordinary;
  chunks = n < 32 ? (int)n : 32;
}
size_t d_bytes(const ra_attention_window_args& a) { return ((size_t)a.batch * a.seq * a.n_heads * 4 + 255) / 256 * 256; }

template <int DH>
cudaError_t fwd_simt(const ra_attention_window_args& a, cudaStream_t st) {
  const int n_blk = (a.seq + BH - 1) / BH;
  const int64_t grid = (int64_t)n_blk * a.batch * a.n_heads;
  if (grid > INT32_MAX) return cudaErrorNotSupported;
  cudaError_t e = allow_smem(window_fwd_simt_kernel<DH>, Plan<DH>::FWD_BYTES);
  if (e != cudaSuccess) return e;
  e = launch_pdl(window_fwd_simt_kernel<DH>, dim3((unsigned)grid), dim3(NT), Plan<DH>::FWD_BYTES, st, a, window_of(a), n_blk);
  note_launch(1);
  return e;
}
template <int DH>
cudaError_t bwd_simt(const ra_attention_window_args& a, cudaStream_t st) {
  int split, chunks;
  split_of(a, split, chunks);
  const int n_blk = (a.seq + BH - 1) / BH;
  const int64_t gq = (int64_t)n_blk * a.batch * a.n_heads, gk = (int64_t)(n_blk - split + split * chunks) * a.batch * a.n_kv_heads;
  const int64_t d_ctas = ((int64_t)a.batch * a.seq * a.n_heads + 31) / 32;
  if (gq + gk > INT32_MAX || d_ctas > INT32_MAX) return cudaErrorNotSupported;
  float* D = (float*)((char*)a.workspace_dev + WS_ZERO);
  float* parts = (float*)((char*)D + d_bytes(a));
  cudaError_t e = allow_smem(window_bwd_simt_kernel<DH>, Plan<DH>::BWD_BYTES);
  if (e == cudaSuccess) e = launch_pdl(window_d_simt_kernel, dim3((unsigned)d_ctas), dim3(256), 0, st, a, D);
  if (e == cudaSuccess)
    e = launch_pdl(window_bwd_simt_kernel<DH>, dim3((unsigned)(gq + gk)), dim3(NT), Plan<DH>::BWD_BYTES, st, a, (const float*)D, parts, window_of(a),
                   n_blk, split, chunks, gk);
  note_launch(2);
  if (e == cudaSuccess && split > 0) {
    const int64_t threads = (int64_t)a.batch * a.n_kv_heads * split * 2 * BH * DH / 4;
    e = launch_pdl(window_bwd_simt_parts_kernel<DH>, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, st, a, (const float*)parts, split, chunks);
    note_launch(1);
  }
  return e;
}

}  // namespace

size_t attention_window_workspace(const ra_attention_window_args& a) {
  if (a.dtype == RA_BF16) return attention_window_workspace_tc(a);
  int split, chunks;
  split_of(a, split, chunks);
  return WS_ZERO + d_bytes(a) + (size_t)a.batch * a.n_kv_heads * split * chunks * 2 * BH * dims_of(a) * 4;
}

cudaError_t attention_window_fwd_simt(const ra_attention_window_args& a, cudaStream_t st) {
  if (a.dtype != RA_F32) return cudaErrorNotSupported;
  const int d = dims_of(a);
  return d == 32 ? fwd_simt<32>(a, st) : d == 64 ? fwd_simt<64>(a, st) : d == 96 ? fwd_simt<96>(a, st) : fwd_simt<128>(a, st);
}
cudaError_t attention_window_bwd_simt(const ra_attention_window_args& a, cudaStream_t st) {
  if (a.dtype != RA_F32) return cudaErrorNotSupported;
  const int d = dims_of(a);
  return d == 32 ? bwd_simt<32>(a, st) : d == 64 ? bwd_simt<64>(a, st) : d == 96 ? bwd_simt<96>(a, st) : bwd_simt<128>(a, st);
}

}  // namespace ra
