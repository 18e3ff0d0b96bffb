// k_attention_window_bwd_tc.cu -- backward of the windowed attention in bf16 on the 5th-generation tensor cores.
//
//   P = 2^(scale log2 e q k^T - lse log2 e);  dV = P^T dO;  dP = dO V^T;  dS = P (dP - D), D_i = dO_i . o_i;
//   dQ = scale dS K;  dK = scale dS^T Q, dV and dK summed over the query heads that share the key.
// Two kernels of one form, so that every gradient is one accumulator's sum in a fixed order (no atomics):
//   queries  a CTA holds Q_i, dO_i and streams the key blocks that the rows see: S, dP, dQ += dS K_j.  It computes D first
//            and leaves it for
//   keys     a CTA holds K_j, V_j and streams the query blocks that see the rows, head by head of the group: S^T, dP^T,
//            dV += P^T dO_i, dK += dS^T Q_i.
// The scores are computed in both: seven products a pair of blocks where atomics would do with five.
// Ten warps: eight of arithmetic (a thread a row of the held block and half of the columns), one that issues the products,
// one that loads by TMA.  P (in fp32, in registers) and dS are the owner's of the row; as bf16 they go back to TMEM, over the
// scores they came from, and are the A operand of the next product there.
//   keys:    dV(n), S(n+1) run while the warps turn dP(n) into dS(n); dK(n), dP(n+1) while they turn S(n+1) into P(n+1).
//   queries: the scores have two buffers: dP(n+1), dQ(n), S(n+2) run while the warps turn S(n+1) into P(n+1).
// The first key blocks may hold sinks, which every later query sees: where that makes them much longer than a block of the
// window, several CTAs share such a block's queries and a last kernel adds their fp32 parts in order.
// Rows past a sequence's end are set to zero in operands that a product sums over.
#include "common.cuh"
#include "operators.h"
#include "window_tc.cuh"

namespace ra {
namespace {

using namespace tc;

constexpr float kLog2e = 1.4426950408889634f;
constexpr int BR = 128, THREADS = 320, NA = 3, NB = 2;  // ring slots of the two streams

struct WindowBwdArgs {
  const int32_t* lens;
  const float* lse;
  const bf16* out;
  int64_t out_stride;
  float* D;        // [batch, n_heads, seq]
  float* part;     // [batch, n_kv_heads, split blocks, chunks][dK | dV][128][DH], in order
  uint32_t* err;
  int batch, seq, n_heads, n_kv_heads, W, sinks, n_blk;
  int split, chunks;  // the first `split` key blocks are shared by `chunks` CTAs each
  float scale, sl2;
};

template <int DH>
struct BwdPlan {
  static constexpr int BLK = BR * DH * 2;
  static constexpr int F0 = 0, F1 = BLK, A = 2 * BLK, B = A + NA * BLK, BYTES = B + NB * BLK;
  static constexpr uint32_t C_S = 0, C_DP = 128, C_A0 = 256, C_A1 = 256 + DH, C_S1 = 384;
};

// D[128 x 128] = A B^T over DH, both K-major blocks (a, b: the low words of their descriptors)
template <int DH>
__device__ __forceinline__ void mma_nt(uint32_t d, uint32_t a, uint32_t b) {
  constexpr uint32_t ID = idesc_bf16(BR, BR);
#pragma unroll
  for (int kk = 0; kk < DH / 16; ++kk) {
    const uint32_t o = ((kk >> 2) * (BR * 128) + (kk & 3) * 32) >> 4;
    umma_bf16(d, desc_of(a + o), desc_of(b + o), ID, kk > 0 ? 1u : 0u);
  }
}
// D[128 x DH] (+)= X[128 x 128, bf16 in TMEM: columns 0-63 packed at x, 64-127 at x + 64] B[128 x DH]
template <int DH>
__device__ __forceinline__ void mma_tn(uint32_t d, uint32_t x, uint32_t b, uint32_t acc) {
  constexpr uint32_t ID = idesc_bf16_bmn(BR, DH);
#pragma unroll
  for (int kk = 0; kk < BR / 16; ++kk)
    umma_bf16_ts(d, x + 64 * (kk >> 2) + 8 * (kk & 3), desc_of(b + kk * (2048 >> 4)), ID, kk > 0 ? 1u : acc);
}

template <int DH, bool KEYS>
__global__ void __launch_bounds__(THREADS, 1) window_bwd_tc_kernel(const __grid_constant__ CUtensorMap tmQ,
    const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CUtensorMap tmDO,
    const __grid_constant__ CUtensorMap tmG0, const __grid_constant__ CUtensorMap tmG1, const __grid_constant__ WindowBwdArgs a) {
  using Pl = BwdPlan<DH>;
  constexpr int BLK = Pl::BLK;
  extern __shared__ __align__(1024) uint8_t smem[];
  __shared__ __align__(8) uint64_t fixed_full, a_full[NA], a_empty[NA], b_full[NB], b_empty[NB], s_full[2], dp_full, p_full, ds_full, stat_full, staged, done, drain;
  __shared__ uint32_t tmem_sh;
  __shared__ volatile int abort_sh;
  __shared__ __align__(16) float stat[2][2][BR];  // keys: log-sum-exps and D of the query block, two steps; queries: [0][0]: D's halves
  const uint32_t sb = smem_u32(smem);
  if (sb & 1023u) {  // the swizzled operand tiles need 1024-byte alignment
    if (threadIdx.x == 0) set_dev_error(a.err, RA_DEVERR_BOUNDS);
    return;
  }
  const int tid = threadIdx.x, warp = warp_index(), lane = tid & 31;
  const int G = a.n_heads / a.n_kv_heads;

  // ---- this CTA's block: the ones with the most steps first
  int blk, b, head, chunk = 0, chunks = 1;  // head: keys: key-value head
  if (KEYS) {
    const int units = a.batch * a.n_kv_heads, it = (int)(blockIdx.x / units), u = (int)(blockIdx.x % units);
    if (it < a.split * a.chunks) {
      blk = it / a.chunks;
      chunk = it - blk * a.chunks;
      chunks = a.chunks;
    } else {
      blk = a.split + it - a.split * a.chunks;
    }
    b = u / a.n_kv_heads;
    head = u - b * a.n_kv_heads;
  } else {
    const int units = a.batch * a.n_heads, u = (int)(blockIdx.x % units);
    blk = a.n_blk - 1 - (int)(blockIdx.x / units);
    b = u / a.n_heads;
    head = u - b * a.n_heads;
  }
  const int kvh = KEYS ? head : head / G, r0 = blk * BR;

  if (warp == 9) {
    if (elect_one()) {
      mbar_init(&fixed_full, 1);
#pragma unroll
      for (int i = 0; i < NA; ++i) {
        mbar_init(&a_full[i], 1);
        mbar_init(&a_empty[i], 1);
      }
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        mbar_init(&b_full[i], 1);
        mbar_init(&b_empty[i], 1);
      }
      mbar_init(&s_full[0], 1);
      mbar_init(&s_full[1], 1);
      mbar_init(&dp_full, 1);
      mbar_init(&p_full, 8);
      mbar_init(&ds_full, 8);
      mbar_init(&stat_full, 8);
      mbar_init(&staged, 8);
      mbar_init(&done, 1);
      mbar_init(&drain, 1);
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
  // ---- the steps: keys: (head of the group, query block); queries: key blocks [0, ns), then [lo, hi]
  int n_steps = 0, s0 = 0, per_head = 1, ns = 0, lo = 0;
  const int last = r0 + BR - 1 < len ? r0 + BR - 1 : len - 1;  // the last live row
  if (r0 < len) {
    if (KEYS) {
      const int64_t far = r0 < a.sinks ? len - 1 : (int64_t)last + a.W - 1;
      per_head = (int)(far < len ? far : len - 1) / BR - blk + 1;
      const int64_t total = (int64_t)per_head * G;
      s0 = (int)(total * chunk / chunks);
      n_steps = (int)(total * (chunk + 1) / chunks) - s0;
    } else {
      const int first = r0 - a.W + 1, sink_blocks = a.sinks / BR + (a.sinks % BR != 0);
      lo = first > 0 ? first / BR : 0;
      ns = sink_blocks < blk + 1 ? sink_blocks : blk + 1;
      if (lo < ns) lo = ns;
      n_steps = ns + (blk >= lo ? blk - lo + 1 : 0);
    }
  }
  // the streamed block of step n, and (keys) its head
  auto step_head = [&](int n) { return KEYS ? kvh * G + (s0 + n) / per_head : kvh; };
  auto step_blk = [&](int n) { return KEYS ? blk + (s0 + n) % per_head : n < ns ? n : n - ns + lo; };
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_sh;

  if (warp == 9) {
    // ------------------------------------------------------------ copies
    if (n_steps > 0 && elect_one()) {
      auto load = [&](const CUtensorMap* tm, uint32_t dst, uint64_t* bar, int h, int row) {
#pragma unroll
        for (int n = 0; n < DH / 64; ++n) tma_load3(tm, dst + n * (BR * 128), bar, h * DH + 64 * n, row, b);
      };
      mbar_expect_tx(&fixed_full, 2 * BLK);
      load(KEYS ? &tmK : &tmQ, sb + Pl::F0, &fixed_full, head, r0);
      load(KEYS ? &tmV : &tmDO, sb + Pl::F1, &fixed_full, head, r0);
      bool ok = true;
      int na = 0, nb = 0;
      for (int n = 0; n < n_steps && ok; ++n) {
        const int sa = n % NA, sl = n % NB, h = step_head(n), row = step_blk(n) * BR;
        if (n >= NA) ok = mbar_wait(&a_empty[sa], ((n / NA) - 1) & 1, &abort_sh, a.err);
        if (!ok) break;
        mbar_expect_tx(&a_full[sa], BLK);
        load(KEYS ? &tmQ : &tmK, sb + Pl::A + sa * BLK, &a_full[sa], h, row);
        na = n + 1;
        if (n >= NB) ok = mbar_wait(&b_empty[sl], ((n / NB) - 1) & 1, &abort_sh, a.err);
        if (!ok) break;
        mbar_expect_tx(&b_full[sl], BLK);
        load(KEYS ? &tmDO : &tmV, sb + Pl::B + sl * BLK, &b_full[sl], h, row);
        nb = n + 1;
      }
      if (!ok) {
        // a wait gave up: let the copies on their way land before shared memory is released
        volatile int no_abort = 0;
        mbar_wait(&fixed_full, 0, &no_abort, nullptr);
        for (int n = na > NA ? na - NA : 0; n < na; ++n) mbar_wait(&a_full[n % NA], (n / NA) & 1, &no_abort, nullptr);
        for (int n = nb > NB ? nb - NB : 0; n < nb; ++n) mbar_wait(&b_full[n % NB], (n / NB) & 1, &no_abort, nullptr);
      }
    }
    __syncwarp();
  } else if (warp == 8) {
    // ------------------------------------------------------------ products
    bool ok = n_steps == 0 || mbar_wait_warp(&fixed_full, 0, &abort_sh, a.err);
    const uint32_t utmem = uniform(tmem), f0 = desc_lo_k(sb + Pl::F0), f1 = desc_lo_k(sb + Pl::F1);
    // S(n), into buffer n & 1 (queries)
    auto scores = [&](int n) {
      const int s = n % NA;
      ok = ok && mbar_wait_warp(&a_full[s], (n / NA) & 1, &abort_sh, a.err);
      if (!ok) return;
      const int dead = len - step_blk(n) * BR;
      if (dead < BR) zero_rows<DH>(smem + Pl::A + s * BLK, dead, lane);
      const uint32_t d = uniform(tmem + (!KEYS && (n & 1) ? Pl::C_S1 : Pl::C_S)), x = desc_lo_k(sb + Pl::A + s * BLK);
      if (elect_one()) {
        mma_nt<DH>(d, f0, x);
        umma_commit(&s_full[KEYS ? 0 : n & 1]);
      }
      __syncwarp();
    };
    auto dprobs = [&](int n) {
      const int s = n % NB;
      ok = ok && mbar_wait_warp(&b_full[s], (n / NB) & 1, &abort_sh, a.err);
      if (!ok) return;
      const int dead = len - step_blk(n) * BR;
      if (KEYS && dead < BR) zero_rows<DH>(smem + Pl::B + s * BLK, dead, lane);
      const uint32_t x = desc_lo_k(sb + Pl::B + s * BLK);
      if (elect_one()) {
        mma_nt<DH>(utmem + Pl::C_DP, f1, x);
        umma_commit(&dp_full);
        if (!KEYS) umma_commit(&b_empty[s]);
      }
      __syncwarp();
    };
    if (n_steps > 0) {
      scores(0);
      dprobs(0);
      if (!KEYS && n_steps > 1) scores(1);
    }
    for (int n = 0; n < n_steps && ok; ++n) {
      if (KEYS) {
        ok = mbar_wait_warp(&p_full, n & 1, &abort_sh, a.err);
        if (!ok) break;
        tc_fence_after();
        const uint32_t acc = uniform(n > 0), g = desc_lo_mn(sb + Pl::B + (n % NB) * BLK, BR * 128);
        const uint32_t q = desc_lo_mn(sb + Pl::A + (n % NA) * BLK, BR * 128);
        if (elect_one()) {  // dV += P^T dO
          mma_tn<DH>(utmem + Pl::C_A1, utmem + Pl::C_S, g, acc);
          umma_commit(&b_empty[n % NB]);
        }
        __syncwarp();
        if (n + 1 < n_steps) scores(n + 1);
        ok = ok && mbar_wait_warp(&ds_full, n & 1, &abort_sh, a.err);
        if (!ok) break;
        tc_fence_after();
        if (elect_one()) {  // dK += dS^T Q
          mma_tn<DH>(utmem + Pl::C_A0, utmem + Pl::C_DP, q, acc);
          umma_commit(&a_empty[n % NA]);
          if (n + 1 == n_steps) umma_commit(&done);
        }
        __syncwarp();
        if (n + 1 < n_steps) dprobs(n + 1);
      } else {
        ok = mbar_wait_warp(&ds_full, n & 1, &abort_sh, a.err);
        if (!ok) break;
        tc_fence_after();
        if (n + 1 < n_steps) dprobs(n + 1);
        if (!ok) break;
        const uint32_t acc = uniform(n > 0), x = uniform(tmem + (n & 1 ? Pl::C_S1 : Pl::C_S)), k = desc_lo_mn(sb + Pl::A + (n % NA) * BLK, BR * 128);
        if (elect_one()) {  // dQ += dS K
          mma_tn<DH>(utmem + Pl::C_A0, x, k, acc);
          umma_commit(&a_empty[n % NA]);
          if (n + 1 == n_steps) umma_commit(&done);
        }
        __syncwarp();
        if (n + 2 < n_steps) scores(n + 2);
      }
    }
    // what was issued ends before shared memory and TMEM are released
    if (elect_one()) {
      volatile int no_abort = 0;
      umma_commit(&drain);
      mbar_wait(&drain, 0, &no_abort, nullptr);
    }
    __syncwarp();
  } else {
    // ------------------------------------------------------------ P and dS: thread = row, half of the columns
    const int half = warp >> 2, row = 32 * (warp & 3) + lane, r = r0 + row, c0 = 64 * half;
    const uint32_t trow = tmem + ((uint32_t)(32 * (warp & 3)) << 16);
    bool ok = true;
    float my_lse = 0.f, my_d = 0.f;  // queries: of this row, in powers of two
    float next_stat = 0.f;           // keys: this thread's value of the next step's statistics
    auto fetch = [&](int n) {
      const int q = step_blk(n) * BR + (tid & 127);
      const int64_t at = ((int64_t)b * a.n_heads + step_head(n)) * a.seq + q;
      next_stat = q >= len ? 0.f : tid < BR ? a.lse[at] * kLog2e : a.D[at];
    };
    if (KEYS) {
      if (n_steps > 0) fetch(0);
    } else {
      // D = dO . o: each thread half a row
      const int64_t at = ((int64_t)b * a.n_heads + head) * a.seq + r;
      if (n_steps > 0) {
        float d = 0.f;
        ok = mbar_wait_warp(&fixed_full, 0, &abort_sh, a.err);
        if (ok && r < len) {
          my_lse = a.lse[at] * kLog2e;
          const bf16* o = a.out + ((int64_t)b * a.seq + r) * a.out_stride + head * DH + (DH / 2) * half;
#pragma unroll
          for (int g = 0; g < DH / 16; ++g) {
            const int c = (DH / 16) * half + g;  // 16-byte chunk of the row
            const uint4 x = *reinterpret_cast<const uint4*>(o + 8 * g);
            const uint4 y = *reinterpret_cast<const uint4*>(smem + Pl::F1 + (c >> 3) * (BR * 128) + swz(row, c & 7));
            const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float2 u = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&xs[e]));
              const float2 v = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&ys[e]));
              d = fmaf(u.x, v.x, fmaf(u.y, v.y, d));
            }
          }
        }
        stat[0][half][row] = d;
        named_sync(1, 256);
        my_d = stat[0][0][row] + stat[0][1][row];
      }
      if (half == 0 && r < a.seq) a.D[at] = my_d;
    }
    for (int n = 0; n < n_steps && ok; ++n) {
      const int st0 = step_blk(n) * BR;
      if (KEYS) {
        stat[n & 1][tid >> 7][tid & 127] = next_stat;
        if (n + 1 < n_steps) fetch(n + 1);
        __syncwarp();
        if (lane == 0) mbar_arrive(&stat_full);
        ok = mbar_wait_warp(&stat_full, n & 1, &abort_sh, a.err);
        if (!ok) break;
      }
      ok = mbar_wait_warp(&s_full[KEYS ? 0 : n & 1], (KEYS ? n : n >> 1) & 1, &abort_sh, a.err);
      if (!ok) break;
      tc_fence_after();
      const uint32_t tS = trow + (!KEYS && (n & 1) ? Pl::C_S1 : Pl::C_S) + c0, tDP = trow + Pl::C_DP + c0;
      const float* L = &stat[n & 1][0][c0];
      const float* Dc = &stat[n & 1][1][c0];
      float p[64];
      uint32_t* pu = reinterpret_cast<uint32_t*>(p);
      tmem_ld32_issue(tS, pu);
      tmem_ld32_issue(tS + 32, pu + 32);
      tmem_wait32(pu);
      tmem_wait32(pu + 32);
#pragma unroll
      for (int c = 0; c < 64; c += 4) {
        float4 x = make_float4(my_lse, my_lse, my_lse, my_lse);
        if (KEYS) x = *reinterpret_cast<const float4*>(L + c);
        p[c] = ex2_fast(fmaf(p[c], a.sl2, -x.x));
        p[c + 1] = ex2_fast(fmaf(p[c + 1], a.sl2, -x.y));
        p[c + 2] = ex2_fast(fmaf(p[c + 2], a.sl2, -x.z));
        p[c + 3] = ex2_fast(fmaf(p[c + 3], a.sl2, -x.w));
      }
      // the columns that this row's pairs are: [from, to), and (queries) those below `sk`
      const int k_first = KEYS ? r0 : st0, q_first = KEYS ? st0 : r0;
      const bool whole = k_first + BR - 1 <= q_first && (q_first + BR - 1 - k_first < a.W || k_first + BR <= a.sinks) &&
                         q_first + BR <= len;
      if (!whole) {
        int from, to, sk = 0;
        if (KEYS) {  // queries from the key itself to its window's end, or the sequence's
          from = r - st0;
          const int64_t end = r < a.sinks ? len : (int64_t)r + a.W;
          to = (int)(end < len ? end : len) - st0;
          if (r >= len) to = from = 0;
        } else {     // keys to the query itself, inside the window or among the sinks
          to = r < len ? r + 1 - st0 : 0;
          from = r + 1 - a.W - st0;
          sk = r < len ? a.sinks - st0 : 0;
        }
#pragma unroll
        for (int c = 0; c < 64; ++c)
          if (!(c0 + c < to && (c0 + c >= from || c0 + c < sk))) p[c] = 0.f;
      }
      if (KEYS) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          uint32_t w[16];
#pragma unroll
          for (int e = 0; e < 16; ++e) w[e] = pk2(p[32 * c + 2 * e], p[32 * c + 2 * e + 1]);
          tmem_st16(tS + 16 * c, w);
        }
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&p_full);
      }
      ok = mbar_wait_warp(&dp_full, n & 1, &abort_sh, a.err);
      if (!ok) break;
      tc_fence_after();
      float dp[64];
      uint32_t* du = reinterpret_cast<uint32_t*>(dp);
      tmem_ld32_issue(tDP, du);
      tmem_ld32_issue(tDP + 32, du + 32);
      tmem_wait32(du);
      tmem_wait32(du + 32);
#pragma unroll
      for (int c = 0; c < 64; c += 4) {
        float4 x = make_float4(my_d, my_d, my_d, my_d);
        if (KEYS) x = *reinterpret_cast<const float4*>(Dc + c);
        // (a pair that is not one stays zero, whatever its dP is)
        p[c] = p[c] == 0.f ? 0.f : p[c] * (dp[c] - x.x);
        p[c + 1] = p[c + 1] == 0.f ? 0.f : p[c + 1] * (dp[c + 1] - x.y);
        p[c + 2] = p[c + 2] == 0.f ? 0.f : p[c + 2] * (dp[c + 2] - x.z);
        p[c + 3] = p[c + 3] == 0.f ? 0.f : p[c + 3] * (dp[c + 3] - x.w);
      }
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        uint32_t w[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) w[e] = pk2(p[32 * c + 2 * e], p[32 * c + 2 * e + 1]);
        tmem_st16((KEYS ? tDP : tS) + 16 * c, w);
      }
      tmem_st_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&ds_full);
    }
    // ---- gradients: staged over the held blocks (the last product is done), stored by TMA, which leaves out rows past seq
    if (ok && n_steps > 0) {
      ok = mbar_wait_warp(&done, 0, &abort_sh, a.err);
      tc_fence_after();
    }
    if (ok) {
      const bool live = r < len;
#pragma unroll
      for (int o = 0; o < (KEYS ? 2 : 1); ++o) {
        const float f = o == 0 ? a.scale : 1.f;
        float* part = nullptr;
        if (KEYS && chunks > 1)
          part = a.part + ((((int64_t)(b * a.n_kv_heads + head) * a.split + blk) * a.chunks + chunk) * 2 + o) * (BR * DH) + row * DH;
#pragma unroll 1
        for (int c = (DH / 2) * half; c < (DH / 2) * (half + 1); c += 32) {
          float x[32];
          if (n_steps > 0) tmem_ld32(trow + (o == 0 ? Pl::C_A0 : Pl::C_A1) + c, x);
#pragma unroll
          for (int e = 0; e < 32; ++e) x[e] = live && n_steps > 0 ? x[e] * f : 0.f;
          if (part) {
#pragma unroll
            for (int e = 0; e < 32; e += 4) *reinterpret_cast<float4*>(part + c + e) = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
          } else {
#pragma unroll
            for (int g = 0; g < 4; ++g)
              *reinterpret_cast<uint4*>(smem + (o == 0 ? Pl::F0 : Pl::F1) + (c >> 6) * (BR * 128) + swz(row, ((c & 63) >> 3) + g)) =
                  make_uint4(pk2(x[8 * g], x[8 * g + 1]), pk2(x[8 * g + 2], x[8 * g + 3]), pk2(x[8 * g + 4], x[8 * g + 5]),
                             pk2(x[8 * g + 6], x[8 * g + 7]));
          }
        }
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(&staged);
      if (tid == 0 && !(KEYS && chunks > 1) && mbar_wait(&staged, 0, &abort_sh, a.err)) {
#pragma unroll
        for (int o = 0; o < (KEYS ? 2 : 1); ++o)
#pragma unroll
          for (int n = 0; n < DH / 64; ++n)
            tma_store3(o == 0 ? &tmG0 : &tmG1, sb + (o == 0 ? Pl::F0 : Pl::F1) + n * (BR * 128), head * DH + 64 * n, r0, b);
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

// dK and dV of the shared key blocks: the parts in order, four values a thread
template <int DH>
__global__ void __launch_bounds__(256) window_bwd_parts_kernel(const __grid_constant__ WindowBwdArgs a, bf16* dk, int64_t dk_stride,
                                                               bf16* dv, int64_t dv_stride) {
  pdl_wait();
  pdl_trigger();
  const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
  constexpr int PER = BR * DH / 4;  // of one output of one block
  const int64_t blkid = e / (2 * PER);
  const int64_t blocks = (int64_t)a.batch * a.n_kv_heads * a.split;
  if (blkid >= blocks) return;
  const int w = (int)(e - blkid * (2 * PER)), o = w / PER, v = w - o * PER, row = v / (DH / 4), c = (v - row * (DH / 4)) * 4;
  const int j = (int)(blkid % a.split);
  const int64_t u = blkid / a.split;
  const int head = (int)(u % a.n_kv_heads), b = (int)(u / a.n_kv_heads), r = j * BR + row;
  if (r >= a.seq) return;
  const float* p = a.part + (blkid * a.chunks * 2 + o) * (BR * DH) + row * DH + c;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int i = 0; i < a.chunks; ++i) {
    const float4 x = *reinterpret_cast<const float4*>(p + (int64_t)i * 2 * BR * DH);
    s.x += x.x;
    s.y += x.y;
    s.z += x.z;
    s.w += x.w;
  }
  bf16* d = (o == 0 ? dk + ((int64_t)b * a.seq + r) * dk_stride : dv + ((int64_t)b * a.seq + r) * dv_stride) + head * DH + c;
  *reinterpret_cast<uint2*>(d) = make_uint2(pk2(s.x, s.y), pk2(s.z, s.w));
}

// How many CTAs share each of the key blocks that hold sinks.  An ordinary key block has (W / 128 + 2) G steps at most and
// one with sinks up to n_blk G: with up to two such blocks, as many CTAs as bring them back to an ordinary one's length, at
// most 32.  (With more sinks than that most blocks are long, and the CTAs have even work without it.)
void split_of(const ra_attention_window_args& p, int& split, int& chunks) {
  const int n_blk = (p.seq + BR - 1) / BR;
  const int64_t W = p.window == 0 || p.window > p.seq ? p.seq : p.window;
  const int64_t ordinary = W / BR + 2;
  split = 0;
  chunks = 1;
  const int sink_blocks = p.sinks / BR + (p.sinks % BR != 0);
  if (p.dtype != RA_BF16 || sink_blocks < 1 || sink_blocks > 2 || n_blk < 2 * ordinary) return;
  split = sink_blocks < n_blk ? sink_blocks : n_blk;
  chunks = (int)((n_blk + ordinary - 1) / ordinary);
  if (chunks > 32) chunks = 32;
}
size_t d_bytes(const ra_attention_window_args& p) { return ((size_t)p.batch * p.seq * p.n_heads * 4 + 255) / 256 * 256; }

template <int DH>
cudaError_t launch(const ra_attention_window_args& p, cudaStream_t st) {
  WindowBwdArgs a;
  a.lens = p.lens_dev;
  a.lse = p.lse_dev;
  a.out = (const bf16*)p.out_dev;
  a.out_stride = p.out_stride;
  a.D = (float*)p.workspace_dev;
  a.part = (float*)((char*)p.workspace_dev + d_bytes(p));
  a.err = p.err_dev;
  a.batch = p.batch;
  a.seq = p.seq;
  a.n_heads = p.n_heads;
  a.n_kv_heads = p.n_kv_heads;
  a.W = p.window == 0 || p.window > p.seq ? p.seq : p.window;
  a.sinks = p.sinks;
  a.n_blk = (p.seq + BR - 1) / BR;
  split_of(p, a.split, a.chunks);
  a.scale = p.scale;
  a.sl2 = p.scale * kLog2e;
  const int64_t gq = (int64_t)a.n_blk * p.batch * p.n_heads;
  const int64_t gk = (int64_t)(a.n_blk - a.split + a.split * a.chunks) * p.batch * p.n_kv_heads;
  if (gq > INT32_MAX || gk > INT32_MAX) return cudaErrorNotSupported;
  CUtensorMap q, k, v, g, dq, dk, dv;
  const int64_t hq = (int64_t)p.n_heads * DH, hk = (int64_t)p.n_kv_heads * DH;
  if (!tma_map_bf16_batch(&q, p.q_dev, p.batch, p.seq, hq, p.q_stride, 64, BR) ||
      !tma_map_bf16_batch(&k, p.k_dev, p.batch, p.seq, hk, p.k_stride, 64, BR) ||
      !tma_map_bf16_batch(&v, p.v_dev, p.batch, p.seq, hk, p.v_stride, 64, BR) ||
      !tma_map_bf16_batch(&g, p.dout_dev, p.batch, p.seq, hq, p.dout_stride, 64, BR) ||
      !tma_map_bf16_batch(&dq, p.dq_dev, p.batch, p.seq, hq, p.dq_stride, 64, BR) ||
      !tma_map_bf16_batch(&dk, p.dk_dev, p.batch, p.seq, hk, p.dk_stride, 64, BR) ||
      !tma_map_bf16_batch(&dv, p.dv_dev, p.batch, p.seq, hk, p.dv_stride, 64, BR))
    return cudaErrorNotSupported;
  cudaError_t e = allow_smem(window_bwd_tc_kernel<DH, false>, BwdPlan<DH>::BYTES);
  if (e == cudaSuccess) e = allow_smem(window_bwd_tc_kernel<DH, true>, BwdPlan<DH>::BYTES);
  if (e == cudaSuccess)
    e = launch_pdl(window_bwd_tc_kernel<DH, false>, dim3((unsigned)gq), dim3(THREADS), (size_t)BwdPlan<DH>::BYTES, st, q, k, v, g, dq, dq, a);
  if (e == cudaSuccess)
    e = launch_pdl(window_bwd_tc_kernel<DH, true>, dim3((unsigned)gk), dim3(THREADS), (size_t)BwdPlan<DH>::BYTES, st, q, k, v, g, dk, dv, a);
  note_launch(2);
  if (e == cudaSuccess && a.split > 0) {
    const int64_t threads = (int64_t)p.batch * p.n_kv_heads * a.split * 2 * BR * DH / 4;
    e = launch_pdl(window_bwd_parts_kernel<DH>, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, st, a, (bf16*)p.dk_dev, p.dk_stride,
                   (bf16*)p.dv_dev, p.dv_stride);
    note_launch(1);
  }
  return e;
}

}  // namespace

size_t attention_window_workspace_tc(const ra_attention_window_args& p) {
  int split, chunks;
  split_of(p, split, chunks);
  return d_bytes(p) + (size_t)p.batch * p.n_kv_heads * split * chunks * 2 * BR * p.head_dim * 4;
}

cudaError_t attention_window_bwd_tc(const ra_attention_window_args& a, cudaStream_t st) {
  return a.head_dim == 64 ? launch<64>(a, st) : a.head_dim == 128 ? launch<128>(a, st) : cudaErrorNotSupported;
}

}  // namespace ra
