// k_attention_window_bwd_tc.cu -- backward of the windowed attention in bf16 on the 5th-generation tensor cores.
//
//   P = 2^(scale log2 e q k^T - lse log2 e);  dV = P^T dO;  dP = dO V^T;  dS = P (dP - D), D_i = dO_i . o_i;
//   dQ = scale dS K;  dK = scale dS^T Q, dV and dK summed over the query heads that share the key.
// Two kernels of one form, so that every gradient is one accumulator's sum in a fixed order (no atomics):
//   queries  a CTA holds Q_i, dO_i and streams the key blocks that the rows see: S, dP, dQ += dS K_j.  It computes D first
//            and leaves it for
//   keys     a CTA holds K_j, V_j and streams the query blocks that see the rows, head by head of the group: S^T, dP^T,
//            dV += P^T dO_i, dK += dS^T Q_i.
// The scores are computed in both, and dQ in two terms: eight products a pair of blocks where atomics and one term would do with
// five.
// Eleven warps: eight of arithmetic (a thread a row of the held block and half of the columns), two that issue products, one
// that loads by TMA.  P (in fp32, in registers) and dS are the owner's of the row; as bf16 they go back to TMEM, over the
// values they came from, and are the A operand of the next product there.  A warp that issues has a place in TMEM and all that
// goes through it, so that its products are in order by themselves:
//   keys:    dV(n), S(n+1) while the warps turn dP(n) into dS(n); dK(n), dP(n+1) while they turn S(n+1) into P(n+1).
//   queries: dQ(n) in two terms, S(n+2) in two buffers of scores; dP(n+1).
// (One warp for all of a pass's products: 3000 and 4150 cycles a step of long sequences, of which it issued 2700 and 3900;
// two: 2500 and 3500, which the warps of arithmetic take, 1100 for P (64 exponentials a thread on a pipe that two warps
// share) and 1000 for dS, and their waits.)
// The CTAs are persistent: a CTA's next block is loaded when the last products with this one are done, and its first scores
// are computed while gradients leave.  Steps are masked by bits, and 32 columns that no row of a warp sees are left out: of a
// window of 256 two blocks of three are masked.  8 x 1024 tokens, 16 heads of 128, window 256, 4 sinks: 65 us the queries, 76 the
// keys (a CTA a block, one warp of products, a compare a column, dS in one term: 94 and 109); what it reads and writes takes 30
// us each.  2 x 4096 tokens without a window: 503 us, 1093 TFLOP/s over eight products.
// The first key blocks may hold sinks, which every later query sees: where that makes them much longer than a block of the
// window, several CTAs share such a block's queries and a last kernel adds their fp32 parts in order.
// Rows past a sequence's end are set to zero in operands that a product sums over.
// What is rounded: P to bf16 before dV.  dS goes into dQ in two bf16 terms (its first product is followed by one with what the
// first left over) and into dK in one; D, of the rounded output, is good enough for dQ then, and leaves the query pass as
// sum_j P_ij dP_ij for dK.  dQ and dK are 0.0023 from 64 bits, where their own rounding is 0.0017; with dS in one term and D of
// the rounded output in both, 0.0027 to 0.0029 (and 203 us where this takes 211: 8 x 1024 tokens below, both directions).
#include "common.cuh"
#include "operators.h"
#include "window_tc.cuh"

namespace ra {
namespace {

using namespace tc;

constexpr float kLog2e = 1.4426950408889634f;
constexpr int BR = 128, THREADS = 352, NA = 3, NB = 2;  // ring slots of the two streams

struct WindowBwdArgs {
  const int32_t* lens;
  const float* lse;
  float* D;        // [batch, n_heads, seq]
  float* part;     // [batch, n_kv_heads, split blocks, chunks][dK | dV][128][DH], in order
  uint32_t* err;
  int batch, seq, n_heads, n_kv_heads, W, sinks, n_blk;
  int split, chunks;  // the first `split` key blocks are shared by `chunks` CTAs each
  float scale, sl2;
  int items;
  bf16* grad[2];  // queries: dQ; keys: dK, dV
  int64_t grad_stride[2];
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

// A CTA's block and its steps.  keys: (head of the group, query block); queries: key blocks [0, ns), then [lo, blk]
struct Item {
  int blk, b, head, chunk, chunks;  // head: keys: key-value head
  int len, n_steps, s0, per_head, ns, lo;
};
// the ones with the most steps first
template <bool KEYS>
__device__ __forceinline__ Item item_of(const WindowBwdArgs& a, int id) {
  Item x;
  x.chunk = 0;
  x.chunks = 1;
  if (KEYS) {
    const int units = a.batch * a.n_kv_heads, it = id / units, u = id % units;
    if (it < a.split * a.chunks) {
      x.blk = it / a.chunks;
      x.chunk = it - x.blk * a.chunks;
      x.chunks = a.chunks;
    } else {
      x.blk = a.split + it - a.split * a.chunks;
    }
    x.b = u / a.n_kv_heads;
    x.head = u - x.b * a.n_kv_heads;
  } else {
    const int units = a.batch * a.n_heads, u = id % units;
    x.blk = a.n_blk - 1 - id / units;
    x.b = u / a.n_heads;
    x.head = u - x.b * a.n_heads;
  }
  int len = a.lens ? __ldg(a.lens + x.b) : a.seq;
  if (len < 0 || len > a.seq) {
    set_dev_error(a.err, RA_DEVERR_BOUNDS);
    len = len < 0 ? 0 : a.seq;
  }
  x.len = len;
  x.n_steps = x.s0 = x.ns = x.lo = 0;
  x.per_head = 1;
  const int r0 = x.blk * BR, last = r0 + BR - 1 < len ? r0 + BR - 1 : len - 1;  // the last live row
  if (r0 < len) {
    if (KEYS) {
      const int64_t far = r0 < a.sinks ? len - 1 : (int64_t)last + a.W - 1;
      x.per_head = (int)(far < len ? far : len - 1) / BR - x.blk + 1;
      const int64_t total = (int64_t)x.per_head * (a.n_heads / a.n_kv_heads);
      x.s0 = (int)(total * x.chunk / x.chunks);
      x.n_steps = (int)(total * (x.chunk + 1) / x.chunks) - x.s0;
    } else {
      const int first = r0 - a.W + 1, sink_blocks = a.sinks / BR + (a.sinks % BR != 0);
      x.lo = first > 0 ? first / BR : 0;
      x.ns = sink_blocks < x.blk + 1 ? sink_blocks : x.blk + 1;
      if (x.lo < x.ns) x.lo = x.ns;
      x.n_steps = x.ns + (x.blk >= x.lo ? x.blk - x.lo + 1 : 0);
    }
  }
  return x;
}
// A step of an item: the streamed block and its head (stepped from one to the next: a division costs as much as a handshake)
template <bool KEYS>
struct Step {
  int head, blk;
  __device__ __forceinline__ Step(const WindowBwdArgs& a, const volatile Item& x) {
    if (KEYS) {
      const int h = x.s0 / x.per_head;
      head = x.head * (a.n_heads / a.n_kv_heads) + h;
      blk = x.blk + x.s0 - h * x.per_head;
    } else {
      head = x.head / (a.n_heads / a.n_kv_heads);
      blk = x.ns > 0 ? 0 : x.lo;
    }
  }
  __device__ __forceinline__ void next(const volatile Item& x) {
    ++blk;
    if (KEYS) {
      if (blk == x.blk + x.per_head) {
        blk = x.blk;
        ++head;
      }
    } else if (blk == x.ns) {
      blk = x.lo;
    }
  }
};

template <int DH, bool KEYS>
__global__ void __launch_bounds__(THREADS, 1) window_bwd_tc_kernel(const __grid_constant__ CUtensorMap tmQ,
    const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CUtensorMap tmDO,
    const __grid_constant__ CUtensorMap tmO, const __grid_constant__ WindowBwdArgs a) {
  using Pl = BwdPlan<DH>;
  constexpr int BLK = Pl::BLK;
  extern __shared__ __align__(1024) uint8_t smem[];
  // f_free: the held blocks were read for the last time; zeroed: (keys) rows past the end in a dO slot; done: an item's gradients
  // are complete; o_read: they have left TMEM
  __shared__ __align__(8) uint64_t fixed_full, f_free, a_full[NA], a_empty[NA], b_full[NB], b_empty[NB], zeroed[NB];
  __shared__ __align__(8) uint64_t s_full[2], dp_full, p_full, ds_full[2], stat_full, sum_full, done, o_read, drain[2];
  __shared__ uint32_t tmem_sh;
  __shared__ Item info[8][2];
  __shared__ volatile int abort_sh;
  __shared__ __align__(16) float stat[2][2][BR];  // keys: log-sum-exps and D of the query block, two steps; queries: halves of D, of the sums of dS
  const uint32_t sb = smem_u32(smem);
  if (sb & 1023u) {  // the swizzled operand tiles need 1024-byte alignment
    if (threadIdx.x == 0) set_dev_error(a.err, RA_DEVERR_BOUNDS);
    return;
  }
  const int tid = threadIdx.x, warp = warp_index(), lane = tid & 31;

  if (warp == 10) {
    if (elect_one()) {
      mbar_init(&fixed_full, 1);
      mbar_init(&f_free, KEYS ? 2 : 10);
#pragma unroll
      for (int i = 0; i < NA; ++i) {
        mbar_init(&a_full[i], 1);
        mbar_init(&a_empty[i], 1);
      }
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        mbar_init(&b_full[i], 1);
        mbar_init(&b_empty[i], KEYS ? 2 : 1);
        mbar_init(&zeroed[i], 1);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        mbar_init(&s_full[i], 1);
        mbar_init(&ds_full[i], 8);
        mbar_init(&drain[i], 1);
      }
      mbar_init(&dp_full, 1);
      mbar_init(&p_full, 8);
      mbar_init(&stat_full, 8);
      mbar_init(&sum_full, 8);
      mbar_init(&done, KEYS ? 2 : 1);
      mbar_init(&o_read, 8);
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
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  pdl_trigger();  // (TMEM is allocated: the next kernel's CTAs cannot come before this one)
  const uint32_t tmem = tmem_sh;
  // Every role counts its steps over all items (g): ring slots, buffers and the barriers' phases go by that.

  if (warp == 10) {
    // ------------------------------------------------------------ copies
    if (elect_one()) {
      bool ok = true;
      int na = 0, nb = 0, ni = 0;  // blocks of the two rings and items that were started
      for (int id = blockIdx.x; id < a.items && ok; id += gridDim.x) {
        const Item x = item_of<KEYS>(a, id);
        if (x.n_steps == 0) continue;
        auto load = [&](const CUtensorMap* tm, uint32_t dst, uint64_t* bar, int h, int row) {
#pragma unroll
          for (int n = 0; n < DH / 64; ++n) tma_load3(tm, dst + n * (BR * 128), bar, h * DH + 64 * n, row, x.b);
        };
        if (ni > 0) ok = mbar_wait(&f_free, (ni - 1) & 1, &abort_sh, a.err);
        if (!ok) break;
        mbar_expect_tx(&fixed_full, 2 * BLK);
        load(KEYS ? &tmK : &tmQ, sb + Pl::F0, &fixed_full, x.head, x.blk * BR);
        load(KEYS ? &tmV : &tmDO, sb + Pl::F1, &fixed_full, x.head, x.blk * BR);
        ++ni;
        if (!KEYS) {  // o, for D, in a slot of the keys' ring
          const int s = na % NA;
          if (na >= NA) ok = mbar_wait(&a_empty[s], ((na / NA) - 1) & 1, &abort_sh, a.err);
          if (!ok) break;
          mbar_expect_tx(&a_full[s], BLK);
          load(&tmO, sb + Pl::A + s * BLK, &a_full[s], x.head, x.blk * BR);
          ++na;
        }
        Step<KEYS> at(a, x);
        for (int n = 0; n < x.n_steps; ++n, at.next(x)) {
          const int sa = na % NA, sl = nb % NB, h = at.head, row = at.blk * BR;
          if (na >= NA) ok = mbar_wait(&a_empty[sa], ((na / NA) - 1) & 1, &abort_sh, a.err);
          if (!ok) break;
          mbar_expect_tx(&a_full[sa], BLK);
          load(KEYS ? &tmQ : &tmK, sb + Pl::A + sa * BLK, &a_full[sa], h, row);
          ++na;
          if (nb >= NB) ok = mbar_wait(&b_empty[sl], ((nb / NB) - 1) & 1, &abort_sh, a.err);
          if (!ok) break;
          mbar_expect_tx(&b_full[sl], BLK);
          load(KEYS ? &tmDO : &tmV, sb + Pl::B + sl * BLK, &b_full[sl], h, row);
          ++nb;
        }
      }
      if (!ok) {
        // a wait gave up: let the copies on their way land before shared memory is released
        volatile int no_abort = 0;
        if (ni > 0) mbar_wait(&fixed_full, (ni - 1) & 1, &no_abort, nullptr);
        for (int n = na > NA ? na - NA : 0; n < na; ++n) mbar_wait(&a_full[n % NA], (n / NA) & 1, &no_abort, nullptr);
        for (int n = nb > NB ? nb - NB : 0; n < nb; ++n) mbar_wait(&b_full[n % NB], (n / NB) & 1, &no_abort, nullptr);
      }
    }
    __syncwarp();
  } else if (warp == 8) {
    // ------------------------------------------------------------ products: scores, and what follows from them in their place
    const uint32_t utmem = uniform(tmem), f0 = desc_lo_k(sb + Pl::F0);
    bool ok = true;
    uint32_t z_phase = 0;  // a bit a slot, which is zeroed again only when this warp has let it go
    int g0 = 0, ni = 0;
    for (int id = blockIdx.x; id < a.items && ok; id += gridDim.x) {
      const Item x = item_of<KEYS>(a, id);
      if (x.n_steps == 0) continue;
      ok = mbar_wait_warp(&fixed_full, ni & 1, &abort_sh, a.err);
      // S(n); queries: into buffer g & 1
      Step<KEYS> at(a, x), to(a, x);  // of S and of what follows from it
      auto scores = [&](int n) {
        const int g = g0 + n, ga = KEYS ? g : g + ni + 1, s = ga % NA;
        ok = ok && mbar_wait_warp(&a_full[s], (ga / NA) & 1, &abort_sh, a.err);
        if (!ok) return;
        const int dead = x.len - at.blk * BR;
        at.next(x);
        if (dead < BR) zero_rows<DH>(smem + Pl::A + s * BLK, dead, lane);
        const uint32_t d = uniform(tmem + (!KEYS && (g & 1) ? Pl::C_S1 : Pl::C_S)), k = desc_lo_k(sb + Pl::A + s * BLK);
        if (elect_one()) {
          mma_nt<DH>(d, f0, k);
          umma_commit(&s_full[KEYS ? 0 : g & 1]);
          if (n + 1 == x.n_steps) umma_commit(&f_free);
        }
        __syncwarp();
      };
      if (ok) scores(0);
      if (ok && !KEYS && x.n_steps > 1) scores(1);
      if (ok && !KEYS) {  // o has been read: the slot before this item's first keys is free
        ok = mbar_wait_warp(&stat_full, ni & 1, &abort_sh, a.err);
        if (ok && lane == 0) mbar_arrive(&a_empty[(g0 + ni) % NA]);
      }
      for (int n = 0; n < x.n_steps && ok; ++n, to.next(x)) {
        const int g = g0 + n;
        const uint32_t acc = uniform(n > 0);
        if (n == 0 && ni > 0) ok = mbar_wait_warp(&o_read, (ni - 1) & 1, &abort_sh, a.err);
        if (!ok) break;
        if (KEYS) {
          const int s = g % NB;
          const uint32_t y = desc_lo_mn(sb + Pl::B + s * BLK, BR * 128);
          ok = mbar_wait_warp(&b_full[s], (g / NB) & 1, &abort_sh, a.err);
          if (ok && x.len - to.blk * BR < BR) {
            ok = mbar_wait_warp(&zeroed[s], (z_phase >> s) & 1u, &abort_sh, a.err);
            z_phase ^= 1u << s;
          }
          ok = ok && mbar_wait_warp(&p_full, g & 1, &abort_sh, a.err);
          if (!ok) break;
          tc_fence_after();
          if (elect_one()) {  // dV += P^T dO
            mma_tn<DH>(utmem + Pl::C_A1, utmem + Pl::C_S, y, acc);
            umma_commit(&b_empty[s]);
            if (n + 1 == x.n_steps) umma_commit(&done);
          }
          __syncwarp();
          if (n + 1 < x.n_steps) scores(n + 1);
        } else {
          const int s = (g + ni + 1) % NA;
          const uint32_t d = uniform(tmem + (g & 1 ? Pl::C_S1 : Pl::C_S)), k = desc_lo_mn(sb + Pl::A + s * BLK, BR * 128);
          ok = mbar_wait_warp(&ds_full[g & 1], (g >> 1) & 1, &abort_sh, a.err);
          if (!ok) break;
          tc_fence_after();
          if (elect_one()) {  // dQ += dS K
            mma_tn<DH>(utmem + Pl::C_A0, d, k, acc);
            mma_tn<DH>(utmem + Pl::C_A0, d + 32, k, 1u);
            umma_commit(&a_empty[s]);
            if (n + 1 == x.n_steps) umma_commit(&done);
          }
          __syncwarp();
          if (n + 2 < x.n_steps) scores(n + 2);
        }
      }
      g0 += x.n_steps;
      ++ni;
    }
    // what was issued ends before shared memory and TMEM are released
    if (elect_one()) {
      volatile int no_abort = 0;
      umma_commit(&drain[0]);
      mbar_wait(&drain[0], 0, &no_abort, nullptr);
    }
    __syncwarp();
  } else if (warp == 9) {
    // ------------------------------------------------------------ products: dP, and (keys) dK from dS in its place
    const uint32_t utmem = uniform(tmem), f1 = desc_lo_k(sb + Pl::F1);
    bool ok = true;
    int g0 = 0, ni = 0;
    for (int id = blockIdx.x; id < a.items && ok; id += gridDim.x) {
      const Item x = item_of<KEYS>(a, id);
      if (x.n_steps == 0) continue;
      ok = mbar_wait_warp(&fixed_full, ni & 1, &abort_sh, a.err);
      Step<KEYS> at(a, x);
      for (int n = 0; n <= x.n_steps && ok; ++n, at.next(x)) {
        const int g = g0 + n, s = g % NB;
        const uint32_t v = desc_lo_k(sb + Pl::B + s * BLK), q = desc_lo_mn(sb + Pl::A + ((g + NA - 1) % NA) * BLK, BR * 128);
        const uint32_t acc = uniform(n > 1);
        if (n < x.n_steps) {
          ok = mbar_wait_warp(&b_full[s], (g / NB) & 1, &abort_sh, a.err);
          if (!ok) break;
          const int dead = x.len - at.blk * BR;
          if (KEYS && dead < BR) {
            zero_rows<DH>(smem + Pl::B + s * BLK, dead, lane);
            if (lane == 0) mbar_arrive(&zeroed[s]);
          }
        } else if (!KEYS) {
          break;
        }
        if (KEYS && n == 1 && ni > 0) ok = mbar_wait_warp(&o_read, (ni - 1) & 1, &abort_sh, a.err);
        // the last step's dP has been read; (keys) its dS is there
        if (KEYS ? n > 0 : g > 0) ok = ok && mbar_wait_warp(&ds_full[(g - 1) & 1], ((g - 1) >> 1) & 1, &abort_sh, a.err);
        if (!ok) break;
        tc_fence_after();
        if (elect_one()) {
          if (KEYS && n > 0) {  // dK += dS^T Q
            mma_tn<DH>(utmem + Pl::C_A0, utmem + Pl::C_DP, q, acc);
            umma_commit(&a_empty[(g + NA - 1) % NA]);
            if (n == x.n_steps) umma_commit(&done);
          }
          if (n < x.n_steps) {
            mma_nt<DH>(utmem + Pl::C_DP, f1, v);
            umma_commit(&dp_full);
            umma_commit(&b_empty[s]);
            if (n + 1 == x.n_steps) umma_commit(&f_free);
          }
        }
        __syncwarp();
      }
      g0 += x.n_steps;
      ++ni;
    }
    if (elect_one()) {
      volatile int no_abort = 0;
      umma_commit(&drain[1]);
      mbar_wait(&drain[1], 0, &no_abort, nullptr);
    }
    __syncwarp();
  } else {
    // ------------------------------------------------------------ P and dS: thread = row, half of the columns
    const int half = warp >> 2, row = 32 * (warp & 3) + lane, c0 = 64 * half;
    const uint32_t trow = tmem + ((uint32_t)(32 * (warp & 3)) << 16);
    bool ok = true;
    // the next item and what of it comes by plain loads are on their way before this one's end: keys: this thread's value of the
    // next step's statistics; queries: its row's log-sum-exp
    // (what an item is, is kept in shared memory: P and dP take most of a thread's registers)
    float next = 0.f;
    auto fetch = [&](const volatile Item& x, const Step<KEYS>& s) {
      const int q = s.blk * BR + (tid & 127);
      const float* from = tid < BR ? a.lse : a.D;
      next = 0.f;
      if (q < x.len) next = from[((int64_t)x.b * a.n_heads + s.head) * a.seq + q];
    };
    auto ahead = [&](int id, int slot) {
      if (id >= a.items) return;
      const Item x = item_of<KEYS>(a, id);
      __syncwarp();
      if (lane == 0) info[warp][slot] = x;
      if (x.n_steps > 0) {
        if (KEYS) {
          fetch(x, Step<KEYS>(a, x));
        } else {
          const int r = x.blk * BR + row;
          next = 0.f;
          if (r < x.len) next = a.lse[((int64_t)x.b * a.n_heads + x.head) * a.seq + r];
        }
      }
      __syncwarp();
    };
    ahead(blockIdx.x, 0);
    int g0 = 0, ni = 0, slot = 0;
    for (int id = blockIdx.x; id < a.items && ok; id += gridDim.x, slot ^= 1) {
      const volatile Item& x = info[warp][slot];
      const int r0 = x.blk * BR, r = r0 + row, len = x.len;
      float my_lse = 0.f, my_d = 0.f;  // queries: of this row, in powers of two
      if (!KEYS) {
        if (x.n_steps > 0) {
          // D = dO . o: each thread half a row
          float d = 0.f;
          my_lse = next * kLog2e;
          const int ga = g0 + ni, s = ga % NA;
          ok = mbar_wait_warp(&fixed_full, ni & 1, &abort_sh, a.err) && mbar_wait_warp(&a_full[s], (ga / NA) & 1, &abort_sh, a.err);
          if (!ok) break;
          if (r < len) {
#pragma unroll
            for (int i = 0; i < DH / 16; ++i) {
              const int c = (DH / 16) * half + i, at = (c >> 3) * (BR * 128) + swz(row, c & 7);  // 16-byte chunk of the row
              const uint4 o = *reinterpret_cast<const uint4*>(smem + Pl::A + s * BLK + at);
              const uint4 y = *reinterpret_cast<const uint4*>(smem + Pl::F1 + at);
              const uint32_t xs[4] = {o.x, o.y, o.z, o.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float2 u = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&xs[e]));
                const float2 v = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&ys[e]));
                d = fmaf(u.x, v.x, fmaf(u.y, v.y, d));
              }
            }
          }
          stat[0][half][row] = d;
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(&f_free);
            mbar_arrive(&stat_full);
          }
          ok = mbar_wait_warp(&stat_full, ni & 1, &abort_sh, a.err);
          if (!ok) break;
          my_d = stat[0][0][row] + stat[0][1][row];
        }
      }
      float sum = 0.f;  // queries: of the row's dS
      Step<KEYS> at(a, x);
      for (int n = 0; n < x.n_steps; ++n) {
        const int st0 = at.blk * BR, g = g0 + n;
        at.next(x);
        if (KEYS) {
          stat[g & 1][tid >> 7][tid & 127] = tid < BR ? next * kLog2e : next;
          if (n + 1 < x.n_steps) fetch(x, at);
          __syncwarp();
          if (lane == 0) mbar_arrive(&stat_full);
          ok = mbar_wait_warp(&stat_full, g & 1, &abort_sh, a.err);
          if (!ok) break;
        }
        ok = mbar_wait_warp(&s_full[KEYS ? 0 : g & 1], (KEYS ? g : g >> 1) & 1, &abort_sh, a.err);
        if (!ok) break;
        tc_fence_after();
        const uint32_t tS = trow + (!KEYS && (g & 1) ? Pl::C_S1 : Pl::C_S) + c0, tDP = trow + Pl::C_DP + c0;
        const float* L = &stat[g & 1][0][c0];
        const float* Dc = &stat[g & 1][1][c0];
        // the columns that this row's pairs are, a bit each: [from, to), and (queries) those below `sk`
        uint32_t live[2] = {~0u, ~0u};
        bool some[2] = {true, true};  // a row of this warp has pairs among these 32 columns
        const int k_first = KEYS ? r0 : st0, q_first = KEYS ? st0 : r0;
        const bool whole = k_first + BR - 1 <= q_first && (q_first + BR - 1 - k_first < a.W || k_first + BR <= a.sinks) &&
                           q_first + BR <= len;
        if (!whole) {
          int from, to, sk = 0;
          if (KEYS) {  // queries from the key itself to its window's end, or the sequence's
            const int64_t end = r < a.sinks ? len : (int64_t)r + a.W;
            from = r - st0;
            to = r < len ? (int)(end < len ? end : len) - st0 : 0;
          } else {     // keys to the query itself, inside the window or among the sinks
            to = r < len ? r + 1 - st0 : 0;
            from = r + 1 - a.W - st0;
            sk = a.sinks - st0;
          }
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const int at = c0 + 32 * c;
            live[c] = below(to - at) & (~below(from - at) | below(sk - at));
            some[c] = __any_sync(0xffffffffu, live[c] != 0);
          }
        }
        float p[64];
        tmem_ld32_issue(tS, reinterpret_cast<uint32_t*>(p));
        tmem_ld32_issue(tS + 32, reinterpret_cast<uint32_t*>(p + 32));
        tmem_wait32(reinterpret_cast<uint32_t*>(p));
        tmem_wait32(reinterpret_cast<uint32_t*>(p + 32));
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          float* pc = p + 32 * c;
          if (some[c]) {
#pragma unroll
            for (int e = 0; e < 32; e += 4) {
              float4 x = make_float4(my_lse, my_lse, my_lse, my_lse);
              if (KEYS) x = *reinterpret_cast<const float4*>(L + 32 * c + e);
              pc[e] = ex2_fast(fmaf(pc[e], a.sl2, -x.x));
              pc[e + 1] = ex2_fast(fmaf(pc[e + 1], a.sl2, -x.y));
              pc[e + 2] = ex2_fast(fmaf(pc[e + 2], a.sl2, -x.z));
              pc[e + 3] = ex2_fast(fmaf(pc[e + 3], a.sl2, -x.w));
            }
            if (!whole) {
#pragma unroll
              for (int e = 0; e < 32; ++e) pc[e] = (live[c] >> e) & 1u ? pc[e] : 0.f;
            }
          } else {
#pragma unroll
            for (int e = 0; e < 32; ++e) pc[e] = 0.f;
          }
          if (KEYS) {
            uint32_t w[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) w[e] = pk2(pc[2 * e], pc[2 * e + 1]);
            tmem_st16(tS + 16 * c, w);  // over columns that have been read
          }
        }
        if (KEYS) {
          tmem_st_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&p_full);
        }
        ok = mbar_wait_warp(&dp_full, g & 1, &abort_sh, a.err);
        if (!ok) break;
        tc_fence_after();
#pragma unroll
        for (int c = 0; c < 4; ++c) {  // (16 columns at a time: more would leave too few registers)
          uint32_t w[8], rest[8];
          if (some[c >> 1]) {
            float dp[16];
            tmem_ld16(tDP + 16 * c, dp);
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
              float4 y = make_float4(my_d, my_d, my_d, my_d);
              if (KEYS) y = *reinterpret_cast<const float4*>(Dc + 16 * c + e);
              // (a pair that is not one stays zero, whatever its dP is)
              const float* pe = p + 16 * c + e;
              const float ds[4] = {pe[0] == 0.f ? 0.f : pe[0] * (dp[e] - y.x), pe[1] == 0.f ? 0.f : pe[1] * (dp[e + 1] - y.y),
                                   pe[2] == 0.f ? 0.f : pe[2] * (dp[e + 2] - y.z), pe[3] == 0.f ? 0.f : pe[3] * (dp[e + 3] - y.w)};
              if (!KEYS) sum += (ds[0] + ds[1]) + (ds[2] + ds[3]);
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const uint32_t x2 = pk2(ds[2 * h], ds[2 * h + 1]);
                w[(e >> 1) + h] = x2;
                if (!KEYS) {
                  const float2 hi = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&x2));
                  rest[(e >> 1) + h] = pk2(ds[2 * h] - hi.x, ds[2 * h + 1] - hi.y);
                }
              }
            }
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = rest[e] = 0u;
          }
          tmem_st8((KEYS ? tDP : tS) + 8 * c, w);  // (keys: over columns that have been read)
          if (!KEYS) tmem_st8(tS + 32 + 8 * c, rest);
        }
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&ds_full[g & 1]);
      }
      if (!ok) break;
      if (!KEYS) {
        // D of the rounded output is off by what the row's dS add up to (with sum P dP for D they add up to 0)
        if (x.n_steps > 0) {
          stat[1][half][row] = sum;
          __syncwarp();
          if (lane == 0) mbar_arrive(&sum_full);
          ok = mbar_wait_warp(&sum_full, ni & 1, &abort_sh, a.err);
          if (!ok) break;
          my_d += stat[1][0][row] + stat[1][1][row];
        }
        if (half == 0 && r < a.seq) a.D[((int64_t)x.b * a.n_heads + x.head) * a.seq + r] = my_d;
      }
      // ---- gradients
      ahead(id + gridDim.x, slot ^ 1);
      if (x.n_steps > 0) {
        ok = mbar_wait_warp(&done, ni & 1, &abort_sh, a.err);
        if (!ok) break;
        tc_fence_after();
      }
      const bool any = x.n_steps > 0, split = KEYS && x.chunks > 1;
      const int quad = r & ~3;
      const int64_t quad_row = (int64_t)x.b * a.seq + quad, col = x.head * DH + 8 * (lane & 3);
      float* part = nullptr;
      if (split)
        part = a.part + (((int64_t)(x.b * a.n_kv_heads + x.head) * a.split + x.blk) * a.chunks + x.chunk) * (2 * BR * DH) +
               (row & ~3) * DH + 4 * (lane & 3);
      constexpr int PIECES = DH / 64, ALL = (KEYS ? 2 : 1) * PIECES;  // 32 columns each
#pragma unroll 1
      for (int it = 0; it < ALL; ++it) {
        const int o = it / PIECES, c = (DH / 2) * half + 32 * (it % PIECES);
        const float f = r >= len ? 0.f : o == 0 ? a.scale : 1.f;
        float v[32];
        if (any) {
          tmem_ld32(trow + (o == 0 ? Pl::C_A0 : Pl::C_A1) + c, v);
          if (it + 1 == ALL) {  // the accumulators are free for the next item's products
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&o_read);
          }
        }
#pragma unroll
        for (int e = 0; e < 32; ++e) v[e] = any && r < len ? v[e] * f : 0.f;
        uint32_t w[16];
        if (split) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int e = 0; e < 16; ++e) w[e] = __float_as_uint(v[16 * h + e]);
            transpose4(w, lane);
#pragma unroll
            for (int i = 0; i < 4; ++i)
              *reinterpret_cast<uint4*>(part + o * (BR * DH) + i * DH + c + 16 * h) = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
          }
        } else {
          bf16* out = a.grad[o] + quad_row * a.grad_stride[o] + col + c;
#pragma unroll
          for (int e = 0; e < 16; ++e) w[e] = pk2(v[2 * e], v[2 * e + 1]);
          transpose4(w, lane);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (quad + i < a.seq)
              *reinterpret_cast<uint4*>(out + i * a.grad_stride[o]) = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
        }
      }
      g0 += x.n_steps;
      if (x.n_steps > 0) ++ni;
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
// one with sinks up to n_blk G: with up to two such blocks, as many CTAs as bring them back to an ordinary one's length, or to
// half of what each of the 152 SMs has to do in all, at most 32.  (With more sinks than that most blocks are long, and the CTAs
// have even work without it.  1 x 8192 tokens, 16 heads over 4, window 1024, forward and backward: shared
// 336 us, else 748; 8 x 1024 tokens of 16 heads, window 256, where an SM has 24 steps and the longest block 8: 217 us, else 203.
// With dS in two terms, which came later, the first takes 359 us as it is, shared, and the second 212, not shared.)
void split_of(const ra_attention_window_args& p, int& split, int& chunks) {
  const int64_t n_blk = (p.seq + BR - 1) / BR, G = p.n_heads / p.n_kv_heads, units = (int64_t)p.batch * p.n_kv_heads;
  const int64_t W = p.window == 0 || p.window > p.seq ? p.seq : p.window;
  const int64_t ordinary = (W / BR + 2) * G;
  split = 0;
  chunks = 1;
  const int sink_blocks = p.sinks / BR + (p.sinks % BR != 0);
  if (p.dtype != RA_BF16 || sink_blocks < 1 || sink_blocks > 2 || sink_blocks >= n_blk) return;
  const int64_t total = units * (sink_blocks * n_blk * G + (n_blk - sink_blocks) * ordinary), half = total / (2 * 152);
  const int64_t most = ordinary > half ? ordinary : half;
  if (n_blk * G < 2 * most) return;
  split = sink_blocks;
  chunks = (int)((n_blk * G + most - 1) / most);
  if (chunks > 32) chunks = 32;
}
size_t d_bytes(const ra_attention_window_args& p) { return ((size_t)p.batch * p.seq * p.n_heads * 4 + 255) / 256 * 256; }

template <int DH>
cudaError_t launch(const ra_attention_window_args& p, cudaStream_t st) {
  WindowBwdArgs a;
  a.lens = p.lens_dev;
  a.lse = p.lse_dev;
  a.D = (float*)((char*)p.workspace_dev + WS_ZERO);
  a.part = (float*)((char*)a.D + d_bytes(p));
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
  if (gq > INT32_MAX - 1024 || gk > INT32_MAX - 1024) return cudaErrorNotSupported;
  CUtensorMap q, k, v, g, o;
  const int64_t hq = (int64_t)p.n_heads * DH, hk = (int64_t)p.n_kv_heads * DH;
  if (!tma_map_bf16_batch(&q, p.q_dev, p.batch, p.seq, hq, p.q_stride, 64, BR) ||
      !tma_map_bf16_batch(&k, p.k_dev, p.batch, p.seq, hk, p.k_stride, 64, BR) ||
      !tma_map_bf16_batch(&v, p.v_dev, p.batch, p.seq, hk, p.v_stride, 64, BR) ||
      !tma_map_bf16_batch(&g, p.dout_dev, p.batch, p.seq, hq, p.dout_stride, 64, BR) ||
      !tma_map_bf16_batch(&o, p.out_dev, p.batch, p.seq, hq, p.out_stride, 64, BR))
    return cudaErrorNotSupported;
  cudaError_t e = allow_smem(window_bwd_tc_kernel<DH, false>, BwdPlan<DH>::BYTES);
  if (e == cudaSuccess) e = allow_smem(window_bwd_tc_kernel<DH, true>, BwdPlan<DH>::BYTES);
  const int sms = device_sm_count();
  a.items = (int)gq;
  a.grad[0] = (bf16*)p.dq_dev;
  a.grad_stride[0] = p.dq_stride;
  a.grad[1] = nullptr;
  a.grad_stride[1] = 0;
  if (e == cudaSuccess)
    e = launch_pdl(window_bwd_tc_kernel<DH, false>, dim3(a.items < sms ? a.items : sms), dim3(THREADS), (size_t)BwdPlan<DH>::BYTES, st, q, k, v, g, o, a);
  a.items = (int)gk;
  a.grad[0] = (bf16*)p.dk_dev;
  a.grad_stride[0] = p.dk_stride;
  a.grad[1] = (bf16*)p.dv_dev;
  a.grad_stride[1] = p.dv_stride;
  if (e == cudaSuccess)
    e = launch_pdl(window_bwd_tc_kernel<DH, true>, dim3(a.items < sms ? a.items : sms), dim3(THREADS), (size_t)BwdPlan<DH>::BYTES, st, q, k, v, g, o, a);
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
  return WS_ZERO + d_bytes(p) + (size_t)p.batch * p.n_kv_heads * split * chunks * 2 * BR * p.head_dim * 4;
}

cudaError_t attention_window_bwd_tc(const ra_attention_window_args& a, cudaStream_t st) {
  return a.head_dim == 64 ? launch<64>(a, st) : a.head_dim == 128 ? launch<128>(a, st) : cudaErrorNotSupported;
}

}  // namespace ra
