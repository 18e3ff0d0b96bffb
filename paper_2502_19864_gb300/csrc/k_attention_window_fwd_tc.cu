// k_attention_window_fwd_tc.cu -- causal attention with a sliding window and sinks over whole bf16 sequences, forward,
// on the 5th-generation tensor cores.
//
// One pass over the keys with a running maximum m and sum l per row:
//   S = q K_j^T;  p = 2^(S scale log2 e - m);  O += p V_j;  l += sum p;   at the end o = O / l, lse = m + log l.
// A CTA takes two tiles of 128 queries that walk the same key blocks of 128: the same rows of two heads that share their
// keys, or (heads of their own) two consecutive row blocks of one head.  Ten warps:
//   warps 0-3 and 4-7   the softmax of tile 0 and 1, a thread a row: its 128 scores come from TMEM in one load, its p go back
//                       to TMEM as bf16 over the scores, where the next product reads them as its A operand;
//   warp 8              issues the products: O0 += P0 V, S0 = Q0 K', O1 += P1 V, S1 = Q1 K', ...: while one tile's softmax
//                       runs the tensor cores have the other's products;
//   warp 9              loads Q, then K and V blocks by TMA into a ring.
// O stays in TMEM.  It is rescaled only when a row's maximum has grown by more than 2^8 since the scale in use (p then stays
// below 2^8 and sums in fp32 lose nothing): the first block sets the scale and almost none after it changes it.
// Key blocks that no row of a tile sees are not loaded: a tile walks the blocks that hold sinks, then its window.  Rows past a
// sequence's end are zero in V's last block before it is read (p = 0 there, but 0 times NaN would not be 0).
#include "common.cuh"
#include "operators.h"
#include "window_tc.cuh"

namespace ra {
namespace {

using namespace tc;

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.69314718055994531f;
constexpr int BR = 128, THREADS = 320;
constexpr float RESCALE = 8.f;  // powers of two

struct WindowFwdArgs {
  const int32_t* lens;
  float* lse;
  uint32_t* err;
  int batch, seq, n_heads, n_kv_heads, W, sinks;
  int pair_heads;  // the two tiles are two heads of a group; else two row blocks
  int n_work;      // row blocks (or pairs of them) a (sequence, head or pair of heads)
  float sl2;
};

template <int DH>
struct FwdPlan {
  static constexpr int BLK = BR * DH * 2, SLOTS = DH == 128 ? 4 : 6;
  static constexpr int Q = 0, RING = 2 * BLK, BYTES = RING + SLOTS * BLK;
  static constexpr uint32_t C_S = 0, C_O = 256;  // scores of tile t at 128 t; outputs at 256 + DH t
};

// The key blocks of a CTA: those with sinks, [0, ns), then [lo, hi], ns <= lo; and each tile's part of them
struct Blocks {
  int ns, lo, hi, n;
  int tlo[2], thi[2];
  __device__ __forceinline__ int at(int i) const { return i < ns ? i : i - ns + lo; }
  __device__ __forceinline__ bool active(int t, int j) const { return j <= thi[t] && (j >= tlo[t] || j < ns); }
};

template <int DH>
__global__ void __launch_bounds__(THREADS, 1) window_fwd_tc_kernel(const __grid_constant__ CUtensorMap tmQ,
    const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CUtensorMap tmO,
    const __grid_constant__ WindowFwdArgs a) {
  using Pl = FwdPlan<DH>;
  constexpr int SLOTS = Pl::SLOTS, BLK = Pl::BLK;
  extern __shared__ __align__(1024) uint8_t smem[];
  __shared__ __align__(8) uint64_t full[SLOTS], empty[SLOTS], q_full, s_full[2], p_full[2], o_full[2], staged[2], drain;
  __shared__ uint32_t tmem_sh;
  __shared__ volatile int abort_sh;
  const uint32_t sb = smem_u32(smem);
  if (sb & 1023u) {  // the swizzled operand tiles need 1024-byte alignment
    if (threadIdx.x == 0) set_dev_error(a.err, RA_DEVERR_BOUNDS);
    return;
  }
  const int tid = threadIdx.x, warp = warp_index(), lane = tid & 31;

  // ---- this CTA's tiles; the row blocks with the most keys first
  const int G = a.n_heads / a.n_kv_heads, units = a.pair_heads ? a.n_heads / 2 : a.n_heads;
  const int work = a.n_work - 1 - (int)(blockIdx.x % a.n_work), bu = (int)(blockIdx.x / a.n_work);
  const int b = bu / units, unit = bu - b * units;
  int head[2], q0[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    head[t] = a.pair_heads ? 2 * unit + t : unit;
    q0[t] = a.pair_heads ? work * BR : (2 * work + t) * BR;
  }
  const int kvh = head[0] / G;

  if (warp == 9) {
    if (elect_one()) {
#pragma unroll
      for (int i = 0; i < SLOTS; ++i) {
        mbar_init(&full[i], 1);
        mbar_init(&empty[i], 1);
      }
      mbar_init(&q_full, 1);
      mbar_init(&drain, 1);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        mbar_init(&s_full[t], 1);
        mbar_init(&p_full[t], 4);
        mbar_init(&o_full[t], 1);
        mbar_init(&staged[t], 4);
      }
      abort_sh = 0;
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    __syncwarp();
  }
  if (warp == 8) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&tmem_sh)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  pdl_wait();
  pdl_trigger();
  int len = a.lens ? a.lens[b] : a.seq;
  if (len < 0 || len > a.seq) {
    if (tid == 0) set_dev_error(a.err, RA_DEVERR_BOUNDS);
    len = len < 0 ? 0 : a.seq;
  }
  Blocks kb;
  kb.lo = 1 << 30;
  kb.hi = -1;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const bool any = q0[t] < len;
    const int last = q0[t] + BR - 1 < len ? q0[t] + BR - 1 : len - 1, first = q0[t] - a.W + 1;
    kb.thi[t] = any ? last / BR : -1;
    kb.tlo[t] = any && first > 0 ? first / BR : 0;
    if (any && kb.tlo[t] < kb.lo) kb.lo = kb.tlo[t];
    if (kb.thi[t] > kb.hi) kb.hi = kb.thi[t];
  }
  const int sink_blocks = a.sinks / BR + (a.sinks % BR != 0);
  kb.ns = sink_blocks < kb.hi + 1 ? sink_blocks : kb.hi + 1;
  if (kb.lo < kb.ns) kb.lo = kb.ns;
  kb.n = kb.hi < 0 ? 0 : kb.ns + (kb.hi >= kb.lo ? kb.hi - kb.lo + 1 : 0);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_sh;

  if (warp == 9) {
    // ------------------------------------------------------------ copies
    if (kb.n > 0 && elect_one()) {
      auto load = [&](const CUtensorMap* tm, uint32_t dst, uint64_t* bar, int col, int row) {
        mbar_expect_tx(bar, BLK);
#pragma unroll
        for (int n = 0; n < DH / 64; ++n) tma_load3(tm, dst + n * (BR * 128), bar, col + 64 * n, row, b);
      };
      mbar_expect_tx(&q_full, 2 * BLK);
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int n = 0; n < DH / 64; ++n)
          tma_load3(&tmQ, sb + Pl::Q + t * BLK + n * (BR * 128), &q_full, head[t] * DH + 64 * n, q0[t], b);
      int i = 0;  // block of the ring: keys and values in turn
      bool ok = true;
      for (; i < 2 * kb.n && ok; ++i) {
        const int s = i % SLOTS;
        if (i >= SLOTS) ok = mbar_wait(&empty[s], ((i / SLOTS) - 1) & 1, &abort_sh, a.err);
        if (ok) load(i & 1 ? &tmV : &tmK, sb + Pl::RING + s * BLK, &full[s], kvh * DH, kb.at(i >> 1) * BR);
      }
      if (!ok) {
        // a wait gave up: let the copies on their way land before shared memory is released
        volatile int no_abort = 0;
        const int issued = i - 1;  // (the block whose slot did not come free was not)
        mbar_wait(&q_full, 0, &no_abort, nullptr);
        for (int k = issued > SLOTS ? issued - SLOTS : 0; k < issued; ++k)
          mbar_wait(&full[k % SLOTS], (k / SLOTS) & 1, &no_abort, nullptr);
      }
    }
    __syncwarp();
  } else if (warp == 8) {
    // ------------------------------------------------------------ products
    constexpr uint32_t IDS = idesc_bf16(BR, BR), IDO = idesc_bf16_bmn(BR, DH);
    bool ok = kb.n == 0 || mbar_wait_warp(&q_full, 0, &abort_sh, a.err);
    uint32_t p_phase[2] = {0, 0};
    bool started[2] = {false, false}, pend[2] = {false, false};
    int prev = 0;
    for (int i = 0; i <= kb.n && ok; ++i) {
      const int j = i < kb.n ? kb.at(i) : -1;
      const int ks = (2 * i) % SLOTS, vs = (2 * i - 1 + SLOTS) % SLOTS;  // this block's keys, the last one's values
      if (i > 0) {
        ok = mbar_wait_warp(&full[vs], ((2 * i - 1) / SLOTS) & 1, &abort_sh, a.err);
        if (!ok) break;
        const int dead = len - prev * BR;  // rows from here on are past the sequence's end
        if (dead < BR) zero_rows<DH>(smem + Pl::RING + vs * BLK, dead, lane);
      }
      if (i < kb.n) {
        ok = mbar_wait_warp(&full[ks], ((2 * i) / SLOTS) & 1, &abort_sh, a.err);
        if (!ok) break;
      }
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        if (pend[t]) {
          ok = mbar_wait_warp(&p_full[t], p_phase[t], &abort_sh, a.err);
          if (!ok) break;
          p_phase[t] ^= 1u;
          tc_fence_after();
          if (elect_one()) {
            const uint32_t v = sb + Pl::RING + vs * BLK;
#pragma unroll
            for (int kk = 0; kk < BR / 16; ++kk)
              umma_bf16_ts(tmem + Pl::C_O + t * DH, tmem + Pl::C_S + t * BR + kk * 8, sdesc_mn_sw128_lbo(v + kk * 2048, BR * 128), IDO,
                           started[t] || kk > 0 ? 1u : 0u);
            if (prev == kb.thi[t]) umma_commit(&o_full[t]);
          }
          __syncwarp();
          started[t] = true;
          pend[t] = false;
        }
        if (i < kb.n && kb.active(t, j)) {
          if (elect_one()) {
            const uint32_t q = sb + Pl::Q + t * BLK, k = sb + Pl::RING + ks * BLK;
#pragma unroll
            for (int kk = 0; kk < DH / 16; ++kk) {
              const uint32_t o = (kk >> 2) * (BR * 128) + (kk & 3) * 32;
              umma_bf16(tmem + Pl::C_S + t * BR, sdesc_sw128(q + o), sdesc_sw128(k + o), IDS, kk > 0 ? 1u : 0u);
            }
            umma_commit(&s_full[t]);
          }
          __syncwarp();
          pend[t] = true;
        }
      }
      if (!ok) break;
      if (elect_one()) {
        if (i > 0) umma_commit(&empty[vs]);
        if (i < kb.n) umma_commit(&empty[ks]);
      }
      __syncwarp();
      prev = j;
    }
    // what was issued ends before shared memory and TMEM are released
    if (elect_one()) {
      volatile int no_abort = 0;
      umma_commit(&drain);
      mbar_wait(&drain, 0, &no_abort, nullptr);
    }
    __syncwarp();
  } else {
    // ------------------------------------------------------------ softmax: warps 4 t .. 4 t + 3, thread = row
    const int t = warp >> 2, row = tid & 127, q = q0[t] + row;
    const uint32_t tS = tmem + ((uint32_t)(32 * (warp & 3)) << 16) + Pl::C_S + t * BR;
    const uint32_t tO = tmem + ((uint32_t)(32 * (warp & 3)) << 16) + Pl::C_O + t * DH;
    float m = -INFINITY, l = 0.f;  // m: the scale in use (powers of two); l: this row's sum under it
    uint32_t s_phase = 0;
    bool ok = true, first = true;
    for (int i = 0; i < kb.n && ok; ++i) {
      const int j = kb.at(i);
      if (!kb.active(t, j)) continue;
      ok = mbar_wait_warp(&s_full[t], s_phase, &abort_sh, a.err);
      if (!ok) break;
      s_phase ^= 1u;
      tc_fence_after();
      float s[128];
      uint32_t* su = reinterpret_cast<uint32_t*>(s);
#pragma unroll
      for (int c = 0; c < 4; ++c) tmem_ld32_issue(tS + 32 * c, su + 32 * c);
#pragma unroll
      for (int c = 0; c < 4; ++c) tmem_wait32(su + 32 * c);
      const int j0 = j * BR;
      // a block that all rows of the tile see whole has no test a key
      const bool whole = j0 + BR - 1 <= q0[t] && (q0[t] + BR - 1 - j0 < a.W || j0 + BR <= a.sinks);
      if (!whole) {
        const int hi = q < len ? q - j0 : -1, lo = hi - a.W + 1, sk = a.sinks - j0;
#pragma unroll
        for (int c = 0; c < 128; ++c)
          if (!(c <= hi && (c >= lo || c < sk))) s[c] = -INFINITY;
      }
      float bm[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
      for (int c = 4; c < 128; c += 4)
#pragma unroll
        for (int u = 0; u < 4; ++u) bm[u] = fmaxf(bm[u], s[c + u]);
      const float top = fmaxf(fmaxf(bm[0], bm[1]), fmaxf(bm[2], bm[3])) * a.sl2;  // (scale is positive)
      const bool grew = top > m + RESCALE;  // (-inf: nothing seen before)
      if (__any_sync(0xffffffffu, grew)) {
        const float mn = fmaxf(m, top), ms = mn == -INFINITY ? 0.f : mn, f = ex2_fast(m - ms);
        l *= f;
        m = mn;
        if (!first) {
          float o[32];
          uint32_t* ou = reinterpret_cast<uint32_t*>(o);
#pragma unroll 1
          for (int c = 0; c < DH; c += 32) {
            tmem_ld32(tO + c, o);
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] *= f;
            tmem_st16(tO + c, ou);
            tmem_st16(tO + c + 16, ou + 16);
          }
        }
      }
      first = false;
      const float ms = m == -INFINITY ? 0.f : m;
      float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        uint32_t w[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float p0 = ex2_fast(fmaf(s[32 * c + 2 * e], a.sl2, -ms)), p1 = ex2_fast(fmaf(s[32 * c + 2 * e + 1], a.sl2, -ms));
          sum[(2 * e) & 3] += p0;
          sum[(2 * e + 1) & 3] += p1;
          w[e] = pk2(p0, p1);
        }
        tmem_st16(tS + 16 * c, w);
      }
      l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
      tmem_st_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&p_full[t]);
    }
    // ---- outputs: staged over this tile's queries (whose last product is done), stored by TMA, which leaves out rows past seq
    const bool any = kb.thi[t] >= 0;
    if (ok && kb.n > 0) {
      // (a tile without a key still has its queries on their way to where zeros go now)
      ok = mbar_wait_warp(any ? &o_full[t] : &q_full, 0, &abort_sh, a.err);
      tc_fence_after();
    }
    if (ok && q0[t] < a.seq) {
      const float f = q < len && m != -INFINITY ? 1.f / l : 0.f;
      uint8_t* stage = smem + Pl::Q + t * BLK;
#pragma unroll 1
      for (int c = 0; c < DH; c += 32) {
        float o[32];
        if (any) tmem_ld32(tO + c, o);
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          uint32_t w[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) w[e] = q < len ? pk2(o[8 * g + 2 * e] * f, o[8 * g + 2 * e + 1] * f) : 0u;
          *reinterpret_cast<uint4*>(stage + (c >> 6) * (BR * 128) + swz(row, ((c & 63) >> 3) + g)) = make_uint4(w[0], w[1], w[2], w[3]);
        }
      }
      if (a.lse && q < a.seq)
        a.lse[((int64_t)b * a.n_heads + head[t]) * a.seq + q] = q < len && m != -INFINITY ? (m + log2f(l)) * kLn2 : -INFINITY;
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(&staged[t]);
      if (row == 0 && mbar_wait(&staged[t], 0, &abort_sh, a.err)) {
#pragma unroll
        for (int n = 0; n < DH / 64; ++n) tma_store3(&tmO, smem_u32(stage) + n * (BR * 128), head[t] * DH + 64 * n, q0[t], b);
        tma_store_done();
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 8) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
}

template <int DH>
cudaError_t launch(const ra_attention_window_args& p, cudaStream_t st) {
  WindowFwdArgs a;
  a.lens = p.lens_dev;
  a.lse = p.lse_dev;
  a.err = p.err_dev;
  a.batch = p.batch;
  a.seq = p.seq;
  a.n_heads = p.n_heads;
  a.n_kv_heads = p.n_kv_heads;
  a.W = p.window == 0 || p.window > p.seq ? p.seq : p.window;
  a.sinks = p.sinks;
  a.pair_heads = (p.n_heads / p.n_kv_heads) % 2 == 0;
  const int n_blk = (p.seq + BR - 1) / BR;
  a.n_work = a.pair_heads ? n_blk : (n_blk + 1) / 2;
  a.sl2 = p.scale * kLog2e;
  const int64_t grid = (int64_t)a.n_work * p.batch * (a.pair_heads ? p.n_heads / 2 : p.n_heads);
  if (grid > INT32_MAX) return cudaErrorNotSupported;
  CUtensorMap q, k, v, o;
  if (!tma_map_bf16_batch(&q, p.q_dev, p.batch, p.seq, (int64_t)p.n_heads * DH, p.q_stride, 64, BR) ||
      !tma_map_bf16_batch(&k, p.k_dev, p.batch, p.seq, (int64_t)p.n_kv_heads * DH, p.k_stride, 64, BR) ||
      !tma_map_bf16_batch(&v, p.v_dev, p.batch, p.seq, (int64_t)p.n_kv_heads * DH, p.v_stride, 64, BR) ||
      !tma_map_bf16_batch(&o, p.out_dev, p.batch, p.seq, (int64_t)p.n_heads * DH, p.out_stride, 64, BR))
    return cudaErrorNotSupported;
  cudaError_t e = allow_smem(window_fwd_tc_kernel<DH>, FwdPlan<DH>::BYTES);
  if (e == cudaSuccess) e = launch_pdl(window_fwd_tc_kernel<DH>, dim3((unsigned)grid), dim3(THREADS), (size_t)FwdPlan<DH>::BYTES, st, q, k, v, o, a);
  note_launch(1);
  return e;
}

}  // namespace

cudaError_t attention_window_fwd_tc(const ra_attention_window_args& a, cudaStream_t st) {
  return a.head_dim == 64 ? launch<64>(a, st) : a.head_dim == 128 ? launch<128>(a, st) : cudaErrorNotSupported;
}

}  // namespace ra
