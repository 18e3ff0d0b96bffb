// k_kv_cache.cu -- the paged key-value cache: putting new tokens in (with RoPE) and evicting those of little
// accumulated weight.
#include <type_traits>

#include "common.cuh"
#include "operators.h"
#include "paged.cuh"

namespace ra {
namespace {

// ---------------------------------------------------------------------------------------
// Append.  A thread turns VE pairs (i, i + head_dim / 2) of up to four rows at a time (heads' queries, keys and values) of
// one token: a row of q goes to q_out, one of k or v to its page.  Bound by memory: every value is read once and written
// once; the table's values serve a thread's rows from registers and the token's other threads from L1.  The rows are
// requested before the token's place is looked up.  8 x 1024 bf16 tokens, 16 heads of 128 over 4: 20.3 us, 5.2 TB/s; one fp32
// token: 2.6 us, a launch and its dependent loads.
// ---------------------------------------------------------------------------------------
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
__global__ void __launch_bounds__(256, 3) kv_append_kernel(const __grid_constant__ ra_kv_append_args a, int row_lanes, int tokens_per_block) {
  pdl_wait();
  pdl_trigger();
  const ra_kv_cache& c = a.cache;
  const int half = c.head_dim / 2, chunks = half / VE, hq = a.q_dev ? a.n_heads : 0, rows = hq + 2 * c.n_kv_heads;
  const int sub = threadIdx.x / (chunks * row_lanes), rest = threadIdx.x - sub * (chunks * row_lanes);
  const unsigned tok = blockIdx.x * (unsigned)tokens_per_block + sub, tokens = (unsigned)a.batch * (unsigned)a.n_new;
  if (sub >= tokens_per_block || tok >= tokens) return;
  const int row0 = rest / chunks, i = (rest - row0 * chunks) * VE;
  const int b = (int)(tok / (unsigned)a.n_new), t = (int)(tok - (unsigned)b * (unsigned)a.n_new);
  bool known = false, live = false;
  int64_t at = -1;  // of key-value head 0 in the pools; the heads are page_size rows apart
  __align__(16) float cs[VE], sn[VE];
  for (int base = row0; base < rows; base += 4 * row_lanes) {
    __align__(16) T lo[4][VE], hi[4][VE];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int row = base + u * row_lanes;
      if (row >= rows) break;
      const bool is_q = row < hq, is_k = !is_q && row < hq + c.n_kv_heads;
      const int head = is_q ? row : is_k ? row - hq : row - hq - c.n_kv_heads;
      const T* src = (const T*)(is_q ? a.q_dev : is_k ? a.k_dev : a.v_dev) +
                     (int64_t)tok * (is_q ? a.q_stride : is_k ? a.k_stride : a.v_stride) + (int64_t)head * c.head_dim + i;
      load_pack<T, VE>(lo[u], src);
      load_pack<T, VE>(hi[u], src + half);
    }
    if (!known) {
      known = true;
      const int cap = (int)((int64_t)c.max_pages * c.page_size), len = clamp_len(__ldg(a.lens_dev + b), cap, c.err_dev);
      const int slot = len - a.n_new + t;
      live = slot >= 0;
      if (a.rope_dev) {
        int pos = (a.pos_dev ? a.pos_dev[b] : len) - a.n_new + t;
        if (pos < 0 || pos >= a.rope_len) {
          if (live) set_dev_error(c.err_dev, RA_DEVERR_BOUNDS);
          pos = pos < 0 ? 0 : a.rope_len - 1;
        }
        const float* w = a.rope_dev + (int64_t)pos * c.head_dim + i;
#pragma unroll
        for (int e = 0; e < VE; e += VE < 4 ? VE : 4) {
          load_pack<float, VE < 4 ? VE : 4>(cs + e, w + e);
          load_pack<float, VE < 4 ? VE : 4>(sn + e, w + half + e);
        }
      }
      if (live) at = slot_row(c, b, slot, 0);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int row = base + u * row_lanes;
      if (row >= rows) break;
      const bool is_q = row < hq, is_k = !is_q && row < hq + c.n_kv_heads;
      const int head = is_q ? row : is_k ? row - hq : row - hq - c.n_kv_heads;
      if (a.rope_dev && (is_q || is_k)) {
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          const float x = to_f(lo[u][e]), y = to_f(hi[u][e]);
          lo[u][e] = from_f<T>(x * cs[e] - y * sn[e]);
          hi[u][e] = from_f<T>(y * cs[e] + x * sn[e]);
        }
      }
      T* dst;
      if (is_q) {
        dst = (T*)a.q_out_dev + (int64_t)tok * a.q_out_stride + (int64_t)head * c.head_dim + i;
        if (!live) {
#pragma unroll
          for (int e = 0; e < VE; ++e) lo[u][e] = hi[u][e] = from_f<T>(0.f);
        }
      } else {
        if (at < 0) continue;
        dst = (T*)(is_k ? c.k_dev : c.v_dev) + (at + (int64_t)head * c.page_size) * c.head_dim + i;
      }
      store_pack<T, VE>(dst, lo[u]);
      store_pack<T, VE>(dst + half, hi[u]);
    }
  }
}

template <typename T, int VE>
cudaError_t launch_append(const ra_kv_append_args& a, cudaStream_t st) {
  const int rows = (a.q_dev ? a.n_heads : 0) + 2 * a.cache.n_kv_heads, chunks = a.cache.head_dim / 2 / VE;  // (at most 63 chunks: f32, head dim 252)
  int lanes = (rows + 3) / 4;  // four rows a thread, more where a token would not fit a block
  if (lanes * chunks > 256) lanes = 256 / chunks;
  const int per = 256 / (lanes * chunks);
  const int64_t tokens = (int64_t)a.batch * a.n_new;
  cudaError_t e = launch_pdl(kv_append_kernel<T, VE>, dim3((unsigned)((tokens + per - 1) / per)), dim3(256), 0, st, a, lanes, per);
  note_launch(1);
  return e;
}

// ---------------------------------------------------------------------------------------
// Eviction, first kernel: which slots stay.  A CTA takes one key-value head of one sequence, a warp a part of its slots in
// a row.  The weights become 32-bit keys that rise with them (in registers up to 16384 slots, in shared memory up to
// 49152, else read again); the budget-th largest key of the
// middle is found by its digits, 11, 11 and 10 bits from the top, each by a histogram of the keys that share
// the digits found so far; then every warp counts its part of the slots, and writes what stays in order behind
// what the warps before it count.  Counts are integers: no order of atomics changes a result.  Bound by the latency of its
// passes, one CTA's: 17 us for 16384 slots (16 sequences of 4 heads); a sequence of 700 with its rows' move 7.8 us, one
// more with the keys in shared memory.
// ---------------------------------------------------------------------------------------
constexpr int SEL_BINS = 2048;
constexpr int SEL_KEYS = 48 * 1024;  // keys held in shared memory; longer sequences read their weights again

__device__ __forceinline__ uint32_t weight_key(float w) {
  const uint32_t u = __float_as_uint(w == 0.f ? 0.f : w);  // -0 and 0 are equal
  const uint32_t k = u ^ (u & 0x80000000u ? 0xffffffffu : 0x80000000u);
  return w != w ? 0xffffffffu : k;
}

// KPT: keys a thread holds (0: in shared memory; -1: nowhere)
template <int SEL_THREADS, int KPT>
__global__ void __launch_bounds__(SEL_THREADS) evict_select_kernel(const __grid_constant__ ra_kv_evict_args a, int max_len) {
  constexpr int SEL_WARPS = SEL_THREADS / 32, OWN = SEL_BINS / SEL_THREADS;  // bins a thread adds up
  extern __shared__ uint32_t keys[];
  __shared__ uint32_t hist[SEL_BINS];
  __shared__ uint32_t warp_sum[SEL_WARPS], warp_eq[SEL_WARPS];
  __shared__ uint32_t found_digit, found_left;
  pdl_wait();
  pdl_trigger();
  const int kv = a.src.n_kv_heads, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int64_t unit = blockIdx.x;
  const int b = (int)(unit / kv);
  const int n = clamp_len(a.lens_dev[b], max_len, a.src.err_dev);
  const float* w = a.weights_dev + unit * a.weights_stride;
  int32_t* kept = a.kept_dev + unit * a.budget;
  float* wout = a.weights_out_dev ? a.weights_out_dev + unit * a.weights_out_stride : nullptr;
  const int stay = n < a.budget ? n : a.budget;
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
  const int seg = ((n + SEL_WARPS - 1) / SEL_WARPS + 31) / 32 * 32, s0 = warp * seg, s1 = s0 + seg < n ? s0 + seg : n;
  uint32_t mine[KPT > 0 ? KPT : 1];
  if constexpr (KPT > 0) {
    float x[KPT > 0 ? KPT : 1];
#pragma unroll
    for (int k = 0; k < KPT; ++k) {
      const int i = s0 + 32 * k + lane;
      x[k] = w[i < s1 ? i : 0];  // (slot 0 is there: n > budget)
    }
#pragma unroll
    for (int k = 0; k < KPT; ++k) mine[k] = weight_key(x[k]);
  } else if constexpr (KPT == 0) {
#pragma unroll 8
    for (int i = s0 + lane; i < s1; i += 32) keys[i] = weight_key(w[i]);
  }
  // f(slot, key) for each of this thread's slots, rising
  auto each = [&](auto f) {
    if constexpr (KPT > 0) {
#pragma unroll
      for (int k = 0; k < KPT; ++k) {
        const int i = s0 + 32 * k + lane;
        if (i < s1) f(i, mine[k]);
      }
    } else {
#pragma unroll 4
      for (int i = s0 + lane; i < s1; i += 32) f(i, KPT == 0 ? keys[i] : weight_key(w[i]));
    }
  };
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
      each([&](int i, uint32_t k) {
        if (i >= m0 && i < m1 && (k & mask) == prefix) atomicAdd(&hist[(k >> shift) & (bins - 1)], 1u);
      });
      __syncthreads();
      // the digit at which the count from the top reaches `left`: thread t has bins OWN r ... from the top, r = threads - 1 - t
      const int r = SEL_THREADS - 1 - tid;
      uint32_t own[OWN], sum = 0;
#pragma unroll
      for (int k = 0; k < OWN; ++k) sum += own[k] = hist[OWN * r + OWN - 1 - k];
      uint32_t incl = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t v = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += v;
      }
      if (lane == 31) warp_sum[warp] = incl;
      __syncthreads();
      uint32_t above = incl - sum;  // keys with a larger digit than the one at hand
      for (int i = 0; i < warp; ++i) above += warp_sum[i];
#pragma unroll
      for (int k = 0; k < OWN; ++k) {
        if (above < left && left <= above + own[k]) {
          found_digit = (uint32_t)(OWN * r + OWN - 1 - k);
          found_left = left - above;
        }
        above += own[k];
      }
      __syncthreads();
      prefix |= found_digit << shift;
      mask |= (uint32_t)(bins - 1) << shift;
      left = found_left;  // how many of the keys with this digit (at last: of the keys equal to it) stay
    }
  }
  const uint32_t edge = prefix, equal_stay = left;
  uint32_t gt = 0, eq = 0;
  each([&](int i, uint32_t k) {
    const bool always = i < m0 || i >= m1;
    gt += always || k > edge;
    eq += !always && k == edge;
  });
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
  auto place = [&](int i, uint32_t k) {
    const bool live = i < s1, always = live && (i < m0 || i >= m1);
    const bool is_gt = always || (live && k > edge), is_eq = live && !always && k == edge;
    const uint32_t bg = __ballot_sync(0xffffffffu, is_gt), be = __ballot_sync(0xffffffffu, is_eq);
    const uint32_t below = (1u << lane) - 1u;
    const uint32_t g = gt0 + __popc(bg & below), q = eq0 + __popc(be & below);
    if (is_gt || (is_eq && q < equal_stay)) {
      const uint32_t at = g + (q < equal_stay ? q : equal_stay);
      kept[at] = i;
      // (the key is the weight but for zeros, of which it knows one, and NaN)
      if (wout) wout[at] = k == 0x80000000u || k == 0xffffffffu ? w[i] : __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
    }
    gt0 += __popc(bg);
    eq0 += __popc(be);
  };
  if constexpr (KPT > 0) {
#pragma unroll
    for (int k = 0; k < KPT; ++k)
      if (s0 + 32 * k < s1) place(s0 + 32 * k + lane, mine[k]);
  } else {
    for (int base = s0; base < s1; base += 32) {
      const int i = base + lane;
      place(i, i < s1 ? (KPT == 0 ? keys[i] : weight_key(w[i])) : 0);
    }
  }
}

// Second kernel: the rows that stay, K and V, 16 bytes of each a thread.  Bound by memory: 268 MB read and written (4096 rows of 64
// heads, K and V) in 43 us, 6.2 TB/s, by as many CTAs as the SMs hold at once (eight times as many: 45 us; with four rows of a
// thread in flight: 46 us, and a sequence of 700, with its selection, in 8.6 us instead of 7.8).  The last CTA writes the new
// lengths, which may lie where the old ones do: all of the first kernel's threads have read those (in a CTA of the rows: 60.4 us
// for the call above where this takes 59.2).
__global__ void __launch_bounds__(256) evict_move_kernel(const __grid_constant__ ra_kv_evict_args a, int max_len, int cpr, int blocks_per_unit, int64_t n_blocks) {
  pdl_wait();
  pdl_trigger();
  if (blockIdx.x == gridDim.x - 1) {
    for (int b = threadIdx.x; b < a.batch; b += 256) {
      const int n = clamp_len(a.lens_dev[b], max_len, a.src.err_dev);
      a.lens_out_dev[b] = n < a.budget ? n : a.budget;
    }
    return;
  }
  const int kv = a.src.n_kv_heads, per = 256 / cpr, r0 = threadIdx.x / cpr, col = threadIdx.x - r0 * cpr;
  if (r0 >= per) return;
  for (int64_t blk = blockIdx.x; blk < n_blocks; blk += gridDim.x - 1) {
    const int64_t unit = blk / blocks_per_unit;
    const int b = (int)(unit / kv), head = (int)(unit - (int64_t)b * kv);
    const int row = (int)(blk - unit * blocks_per_unit) * per + r0;
    const int from = row < a.budget ? a.kept_dev[unit * a.budget + row] : -1;
    if (from < 0) continue;
    const int64_t at = slot_row(a.src, b, from, head), to = slot_row(a.dst, b, row, head);
    uint4 kx = make_uint4(0, 0, 0, 0), vx = kx;
    if (at >= 0) {
      kx = reinterpret_cast<const uint4*>(a.src.k_dev)[at * cpr + col];
      vx = reinterpret_cast<const uint4*>(a.src.v_dev)[at * cpr + col];
    }
    if (to >= 0) {
      reinterpret_cast<uint4*>(a.dst.k_dev)[to * cpr + col] = kx;
      reinterpret_cast<uint4*>(a.dst.v_dev)[to * cpr + col] = vx;
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
  auto select = [&](auto kernel, int threads, size_t smem) { return launch_pdl(kernel, dim3((unsigned)units), dim3(threads), smem, st, a, max_len); };
  cudaError_t e;
  if (max_len <= 1024) {
    e = select(evict_select_kernel<256, 4>, 256, 0);
  } else if (max_len <= 4096) {
    e = select(evict_select_kernel<1024, 4>, 1024, 0);
  } else if (max_len <= 16384) {
    e = select(evict_select_kernel<1024, 16>, 1024, 0);
  } else if (max_len <= SEL_KEYS) {
    e = allow_smem(evict_select_kernel<1024, 0>, SEL_KEYS * 4);
    if (e == cudaSuccess) e = select(evict_select_kernel<1024, 0>, 1024, 4 * (size_t)max_len);
  } else {
    e = select(evict_select_kernel<1024, -1>, 1024, 0);
  }
  if (e != cudaSuccess) return e;
  const int cpr = a.src.head_dim * (a.src.dtype == RA_BF16 ? 2 : 4) / 16, rows = 256 / cpr, per_unit = (a.budget + rows - 1) / rows;
  const int64_t n_blocks = units * per_unit, most = 8LL * device_sm_count();  // what the SMs hold
  e = launch_pdl(evict_move_kernel, dim3((unsigned)(n_blocks + 1 < most ? n_blocks + 1 : most)), dim3(256), 0, st, a, max_len, cpr, per_unit, n_blocks);
  note_launch(2);
  return e;
}

}  // namespace ra
