// k_kv_cache.cu -- the paged key-value cache: putting new tokens in (with RoPE) and evicting those of little
// accumulated weight.
#include <type_traits>

#include "common.cuh"
#include "operators.h"
#include "paged.cuh"

namespace ra {
namespace {

// ---------------------------------------------------------------------------------------
// Append.  A thread turns VE pairs (i, i + head_dim / 2) of one row (a head's query, key or value) of TOK tokens: a row
// of q goes to q_out, one of k or v to its page.  Bound by memory: every value is read once and written once, the
// table's row by all heads of its token (from L1).  The values of all TOK tokens are requested before the tokens' slots
// are known, which one thread a token looks up.
// ---------------------------------------------------------------------------------------
constexpr int TOK = 4;
template <typename T, int VE>
__device__ __forceinline__ void load_pack(T* dst, const T* src) {
  typedef typename std::conditional<sizeof(T) * VE == 16, uint4, uint2>::type V;
  *reinterpret_cast<V*>(dst) = *reinterpret_cast<const V*>(src);
}
template <typename T, int VE>
__device__ __forceinline__ void store_pack(T* dst, const T* src) {
  typedef typename std::conditional<sizeof(T) * VE == 16, uint4, uint2>::type V;
  *reinterpret_cast<V*>(dst) = *reinterpret_cast<const V*>(src);
}

template <typename T, int VE>
__global__ void __launch_bounds__(256) kv_append_kernel(const __grid_constant__ ra_kv_append_args a) {
  struct Token {
    int64_t row;  // of key-value head 0 in the pools; the heads are page_size rows apart
    int pos;
    bool live, stored;
  };
  __shared__ Token info[TOK];
  pdl_wait();
  pdl_trigger();
  const ra_kv_cache& c = a.cache;
  const int half = c.head_dim / 2, chunks = half / VE, hq = a.q_dev ? a.n_heads : 0;
  const int items = (hq + 2 * c.n_kv_heads) * chunks, t0 = blockIdx.x * TOK;
  const int n = a.n_new - t0 < TOK ? a.n_new - t0 : TOK;
  for (int b = blockIdx.y; b < a.batch; b += gridDim.y) {
    const int64_t tok0 = (int64_t)b * a.n_new + t0;
    bool known = false;
    for (int item = threadIdx.x; item < items || !known; item += 256) {
      const bool mine = item < items;
      const int row = item / chunks, i = (item - row * chunks) * VE;
      const bool is_q = row < hq, is_k = !is_q && row < hq + c.n_kv_heads;
      const int head = is_q ? row : is_k ? row - hq : row - hq - c.n_kv_heads;
      const int64_t stride = is_q ? a.q_stride : is_k ? a.k_stride : a.v_stride;
      const T* src = (const T*)(is_q ? a.q_dev : is_k ? a.k_dev : a.v_dev) + tok0 * stride + (int64_t)head * c.head_dim + i;
      __align__(16) T lo[TOK][VE], hi[TOK][VE];
#pragma unroll
      for (int t = 0; t < TOK; ++t)
        if (mine && t < n) {
          load_pack<T, VE>(lo[t], src + t * stride);
          load_pack<T, VE>(hi[t], src + t * stride + half);
        }
      if (!known) {
        known = true;
        __syncthreads();  // (the sequence before is done with info)
        if ((int)threadIdx.x < n) {
          const int cap = (int)((int64_t)c.max_pages * c.page_size), len = clamp_len(a.lens_dev[b], cap, c.err_dev);
          const int slot = len - a.n_new + t0 + (int)threadIdx.x;
          Token x;
          x.live = slot >= 0;
          x.row = x.live ? slot_row(c, b, slot, 0) : -1;
          x.stored = x.row >= 0;
          x.pos = (a.pos_dev ? a.pos_dev[b] : len) - a.n_new + t0 + (int)threadIdx.x;
          if (a.rope_dev && (x.pos < 0 || x.pos >= a.rope_len)) {
            if (x.live) set_dev_error(c.err_dev, RA_DEVERR_BOUNDS);
            x.pos = x.pos < 0 ? 0 : a.rope_len - 1;
          }
          info[threadIdx.x] = x;
        }
        __syncthreads();
      }
      if (!mine) break;
#pragma unroll
      for (int t = 0; t < TOK; ++t) {
        if (t >= n) break;
        const Token x = info[t];
        if (a.rope_dev && (is_q || is_k)) {
          const float* w = a.rope_dev + (int64_t)x.pos * c.head_dim + i;
          __align__(16) float cs[VE], sn[VE];
#pragma unroll
          for (int e = 0; e < VE; e += VE < 4 ? VE : 4) {
            load_pack<float, VE < 4 ? VE : 4>(cs + e, w + e);
            load_pack<float, VE < 4 ? VE : 4>(sn + e, w + half + e);
          }
#pragma unroll
          for (int e = 0; e < VE; ++e) {
            const float u = to_f(lo[t][e]), v = to_f(hi[t][e]);
            lo[t][e] = from_f<T>(u * cs[e] - v * sn[e]);
            hi[t][e] = from_f<T>(v * cs[e] + u * sn[e]);
          }
        }
        T* dst;
        if (is_q) {
          dst = (T*)a.q_out_dev + (tok0 + t) * a.q_out_stride + (int64_t)head * c.head_dim + i;
          if (!x.live) {
#pragma unroll
            for (int e = 0; e < VE; ++e) lo[t][e] = hi[t][e] = from_f<T>(0.f);
          }
        } else {
          if (!x.stored) continue;
          dst = (T*)(is_k ? c.k_dev : c.v_dev) + (x.row + (int64_t)head * c.page_size) * c.head_dim + i;
        }
        store_pack<T, VE>(dst, lo[t]);
        store_pack<T, VE>(dst + half, hi[t]);
      }
    }
  }
}

template <typename T, int VE>
cudaError_t launch_append(const ra_kv_append_args& a, cudaStream_t st) {
  const dim3 grid((unsigned)((a.n_new + TOK - 1) / TOK), (unsigned)(a.batch < 65535 ? a.batch : 65535));
  cudaError_t e = launch_pdl(kv_append_kernel<T, VE>, grid, dim3(256), 0, st, a);
  note_launch(1);
  return e;
}

// ---------------------------------------------------------------------------------------
// Eviction, first kernel: which slots stay.  A CTA takes one key-value head of one sequence.  The weights
// become 32-bit keys that rise with them (in shared memory where they fit); the budget-th largest key of the
// middle is found by its digits, 11, 11 and 10 bits from the top, each by a histogram of the keys that share
// the digits found so far; then every warp counts its part of the slots, and writes what stays in order behind
// what the warps before it count.  Counts are integers: no order of atomics changes a result.
// ---------------------------------------------------------------------------------------
constexpr int SEL_THREADS = 1024, SEL_WARPS = SEL_THREADS / 32, SEL_BINS = 2048;
constexpr int SEL_KEYS = 48 * 1024;  // keys held in shared memory; longer sequences read their weights again

__device__ __forceinline__ uint32_t weight_key(float w) {
  if (w != w) return 0xffffffffu;
  const uint32_t u = __float_as_uint(w == 0.f ? 0.f : w);  // -0 and 0 are equal
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

template <bool IN_SMEM>
__global__ void __launch_bounds__(SEL_THREADS) evict_select_kernel(const __grid_constant__ ra_kv_evict_args a, int max_len) {
  extern __shared__ uint32_t keys[];
  __shared__ uint32_t hist[SEL_BINS];
  __shared__ uint32_t warp_sum[SEL_WARPS], warp_eq[SEL_WARPS];
  __shared__ uint32_t found_digit, found_left;
  pdl_wait();
  pdl_trigger();
  const int kv = a.src.n_kv_heads, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int64_t unit = blockIdx.x;
  const int b = (int)(unit / kv), head = (int)(unit - (int64_t)b * kv);
  const int n = clamp_len(a.lens_dev[b], max_len, a.src.err_dev);
  const float* w = a.weights_dev + unit * a.weights_stride;
  int32_t* kept = a.kept_dev + unit * a.budget;
  float* wout = a.weights_out_dev ? a.weights_out_dev + unit * a.weights_out_stride : nullptr;
  const int stay = n < a.budget ? n : a.budget;
  if (head == 0 && tid == 0) a.lens_out_dev[b] = stay;
  for (int i = stay + tid; i < a.budget; i += SEL_THREADS) {
    kept[i] = -1;
    if (wout) wout[i] = 0.f;
  }
  if (n <= a.budget) {
    for (int i = tid; i < n; i += SEL_THREADS) {
      kept[i] = i;
      if (wout) wout[i] = w[i];
    }
    return;
  }
  const int m0 = a.first, m1 = n - a.recent;  // the middle
  if (IN_SMEM) {
#pragma unroll 8
    for (int i = tid; i < n; i += SEL_THREADS) keys[i] = weight_key(w[i]);
  }
  auto key_at = [&](int i) { return IN_SMEM ? keys[i] : weight_key(w[i]); };
  uint32_t left = (uint32_t)(a.budget - a.first - a.recent);  // how many of the middle stay
  uint32_t prefix = 0xffffffffu;  // (left == 0: nothing is larger)
  if (left > 0) {
    prefix = 0;
    uint32_t mask = 0;
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bins = pass == 2 ? 1024 : 2048;
      for (int i = tid; i < SEL_BINS; i += SEL_THREADS) hist[i] = 0;
      __syncthreads();
#pragma unroll 4
      for (int i = m0 + tid; i < m1; i += SEL_THREADS) {
        const uint32_t k = key_at(i);
        if ((k & mask) == prefix) atomicAdd(&hist[(k >> shift) & (bins - 1)], 1u);
      }
      __syncthreads();
      // the digit at which the count from the top reaches `left`: thread t has bins 2 r and 2 r + 1, r from the top
      const int r = SEL_THREADS - 1 - tid;
      const uint32_t hi = hist[2 * r + 1], lo = hist[2 * r];
      uint32_t incl = hi + lo;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t v = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += v;
      }
      if (lane == 31) warp_sum[warp] = incl;
      __syncthreads();
      uint32_t before = 0;
      for (int i = 0; i < warp; ++i) before += warp_sum[i];
      const uint32_t above = before + incl - hi - lo;  // keys with a larger digit than this thread's
      if (above < left && left <= above + hi + lo) {
        const bool in_hi = left <= above + hi;
        found_digit = (uint32_t)(2 * r + (in_hi ? 1 : 0));
        found_left = left - above - (in_hi ? 0 : hi);
      }
      __syncthreads();
      prefix |= found_digit << shift;
      mask |= (uint32_t)(bins - 1) << shift;
      left = found_left;  // how many of the keys with this digit (at last: of the keys equal to it) stay
    }
  } else if (IN_SMEM) {
    __syncthreads();
  }
  const uint32_t edge = prefix, equal_stay = left;
  const int seg = ((n + SEL_WARPS - 1) / SEL_WARPS + 31) / 32 * 32, s0 = warp * seg, s1 = s0 + seg < n ? s0 + seg : n;
  uint32_t gt = 0, eq = 0;
#pragma unroll 4
  for (int i = s0 + lane; i < s1; i += 32) {
    const bool always = i < m0 || i >= m1;
    const uint32_t k = key_at(i);
    gt += always || k > edge;
    eq += !always && k == edge;
  }
  gt = __reduce_add_sync(0xffffffffu, gt);
  eq = __reduce_add_sync(0xffffffffu, eq);
  if (lane == 0) {
    warp_sum[warp] = gt;
    warp_eq[warp] = eq;
  }
  __syncthreads();
  uint32_t gt0 = 0, eq0 = 0;  // of the slots before the ones at hand
  for (int i = 0; i < warp; ++i) {
    gt0 += warp_sum[i];
    eq0 += warp_eq[i];
  }
#pragma unroll 4
  for (int base = s0; base < s1; base += 32) {
    const int i = base + lane;
    const bool live = i < s1, always = live && (i < m0 || i >= m1);
    const uint32_t k = live ? key_at(i) : 0;
    const bool is_gt = always || (live && k > edge), is_eq = live && !always && k == edge;
    const uint32_t bg = __ballot_sync(0xffffffffu, is_gt), be = __ballot_sync(0xffffffffu, is_eq);
    const uint32_t below = (1u << lane) - 1u;
    const uint32_t g = gt0 + __popc(bg & below), q = eq0 + __popc(be & below);
    if (is_gt || (is_eq && q < equal_stay)) {
      const uint32_t at = g + (q < equal_stay ? q : equal_stay);
      kept[at] = i;
      if (wout) wout[at] = w[i];
    }
    gt0 += __popc(bg);
    eq0 += __popc(be);
  }
}

// Second kernel: the rows that stay, K and V, 16 bytes a thread and load, MOVE rows of a thread in flight.
constexpr int MOVE = 4;
__global__ void __launch_bounds__(256) evict_move_kernel(const __grid_constant__ ra_kv_evict_args a, int cpr, int rows_per_block,
                                                         int blocks_per_unit, int64_t n_blocks) {
  pdl_wait();
  pdl_trigger();
  const int kv = a.src.n_kv_heads, per = 256 / cpr, r0 = threadIdx.x / cpr, col = threadIdx.x - r0 * cpr;
  if (r0 >= per) return;
  for (int64_t blk = blockIdx.x; blk < n_blocks; blk += gridDim.x) {
    const int64_t unit = blk / blocks_per_unit;
    const int b = (int)(unit / kv), head = (int)(unit - (int64_t)b * kv);
    const int row0 = (int)(blk - unit * blocks_per_unit) * rows_per_block + r0;
    uint4 kx[MOVE], vx[MOVE];
    int from[MOVE];
#pragma unroll
    for (int i = 0; i < MOVE; ++i) {
      const int row = row0 + i * per;
      from[i] = row < a.budget ? a.kept_dev[unit * a.budget + row] : -1;
    }
#pragma unroll
    for (int i = 0; i < MOVE; ++i) {
      kx[i] = vx[i] = make_uint4(0, 0, 0, 0);
      if (from[i] >= 0) {
        const int64_t at = slot_row(a.src, b, from[i], head);
        if (at >= 0) {
          kx[i] = reinterpret_cast<const uint4*>(a.src.k_dev)[at * cpr + col];
          vx[i] = reinterpret_cast<const uint4*>(a.src.v_dev)[at * cpr + col];
        }
      }
    }
#pragma unroll
    for (int i = 0; i < MOVE; ++i) {
      if (from[i] < 0) continue;
      const int64_t at = slot_row(a.dst, b, row0 + i * per, head);
      if (at < 0) continue;
      reinterpret_cast<uint4*>(a.dst.k_dev)[at * cpr + col] = kx[i];
      reinterpret_cast<uint4*>(a.dst.v_dev)[at * cpr + col] = vx[i];
    }
  }
}

}  // namespace

cudaError_t kv_append(const ra_kv_append_args& a, cudaStream_t st) {
  const int half = a.cache.head_dim / 2;
  if (a.cache.dtype == RA_BF16) return half % 8 ? launch_append<bf16, 4>(a, st) : launch_append<bf16, 8>(a, st);
  return half % 4 ? launch_append<float, 2>(a, st) : launch_append<float, 4>(a, st);
}

cudaError_t kv_evict(const ra_kv_evict_args& a, cudaStream_t st) {
  const int max_len = call_max_len(a.src, a.max_len);
  const int64_t units = (int64_t)a.batch * a.src.n_kv_heads;
  // (the keys' space goes by the longest sequence that can come, so that short ones leave room for more CTAs)
  cudaError_t e;
  if (max_len <= SEL_KEYS) {
    e = allow_smem(evict_select_kernel<true>, SEL_KEYS * 4);
    if (e == cudaSuccess)
      e = launch_pdl(evict_select_kernel<true>, dim3((unsigned)units), dim3(SEL_THREADS), 4 * (size_t)max_len, st, a, max_len);
  } else {
    e = launch_pdl(evict_select_kernel<false>, dim3((unsigned)units), dim3(SEL_THREADS), 0, st, a, max_len);
  }
  if (e != cudaSuccess) return e;
  const int cpr = a.src.head_dim * (a.src.dtype == RA_BF16 ? 2 : 4) / 16, rows = 256 / cpr * MOVE;
  const int per_unit = (a.budget + rows - 1) / rows;
  const int64_t n_blocks = units * per_unit, most = 8LL * 8 * device_sm_count();
  e = launch_pdl(evict_move_kernel, dim3((unsigned)(n_blocks < most ? n_blocks : most)), dim3(256), 0, st, a, cpr, rows, per_unit,
                 n_blocks);
  note_launch(2);
  return e;
}

}  // namespace ra
