// k_attention_window_fwd_tc.cu -- causal attention with a sliding window and sinks over whole bf16 sequences, forward,
// on the 5th-generation tensor cores.
//
// One pass over the keys with a running maximum m and sum l per row:
//   S = q K_j^T;  p = 2^(S scale log2 e - m);  O += p V_j;  l += sum p;   at the end o = O / l, lse = m + log l.
// A CTA takes two tiles of 128 queries that walk the same key blocks of 128: the same rows of two heads that share their
// keys, or (heads of their own) two consecutive row blocks of one head.  Eleven warps:
//   warps 0-3 and 4-7   the softmax of tile 0 and 1, a thread a row: its scores come from TMEM 32 at a time, its p go back to
//                       TMEM as bf16 over the scores, where the next product reads them as its A operand;
//   warps 8 and 9       issue the products of tile 0 and 1, in turns: O0 += P0 V, S0 = Q0 K', O1 += P1 V, S1 = Q1 K', ...:
//                       while one tile's softmax runs the tensor cores have the other's products;
//   warp 10             loads Q, then K and V blocks by TMA into a ring.
// What bounds it is each tile's round of softmax (1900 cycles a block of 128 keys: 500 for the maximum, 1000 for the
// exponentials, 400 until its p are seen) and products (1230).  One warp for both tiles' products had its waits and
// commits in that round: 406 us for 16384 tokens of 16 heads over 4, window 4096, against 360 on the same GPU.  Two warps without
// turns interleave their products, so that each tile waits for both: 488 us.  On other GPUs of the kind this takes 374 to 380 us,
// 1290 to 1270 TFLOP/s.
// The CTAs are persistent: the copies and first products of a CTA's next pair of tiles run while the last outputs of this one
// leave (one pair of tiles a CTA: 60 us for 8 x 1024 tokens of 16 heads and window 256, this: 50 us; a pair takes as
// little as three blocks, and its start and end as long).
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
constexpr int BR = 128, THREADS = 352;
constexpr float RESCALE = 8.f;  // powers of two

struct WindowFwdArgs {
  const int32_t* lens;
  float* lse;
  uint32_t* err;
  int batch, seq, n_heads, n_kv_heads, W, sinks;
  int pair_heads;  // the two tiles are two heads of a group; else two row blocks
  int n_work;      // row blocks (or pairs of them) a (sequence, head or pair of heads)
  int units, items;  // (sequence, head or pair of heads)s; pairs of tiles
  bf16* out;
  int64_t out_stride;
  float sl2;
};

template <int DH>
struct FwdPlan {
  static constexpr int BLK = BR * DH * 2, SLOTS = DH == 128 ? 4 : 6;
  static constexpr int Q = 0, RING = 2 * BLK, BYTES = RING + SLOTS * BLK;
  static constexpr uint32_t C_S = 0, C_O = 256;  // scores of tile t at 128 t; outputs at 256 + DH t
};

// the columns of a key block that products and softmax go through, where its sinks alone are seen: in sixteens
__device__ __forceinline__ int sink_columns(bool alone, int j, int sinks) {
  const int n = sinks - j * BR;
  return alone && n < BR ? (n + 15) & ~15 : BR;
}
// The key blocks of a CTA: those with sinks, [0, ns), then [lo, hi], ns <= lo; and each tile's part of them
struct Blocks {
  int ns, lo, hi, n;
  int tlo[2], thi[2];
  __device__ __forceinline__ int at(int i) const { return i < ns ? i : i - ns + lo; }
};

// A pair of tiles, and what its rows see; the row blocks with the most keys come first
struct Item {
  int b, len, head[2], q0[2], kvh;
  Blocks kb;
};
__device__ __forceinline__ Item item_of(const WindowFwdArgs& a, int id) {
  Item x;
  const int work = a.n_work - 1 - id / a.units, u = id % a.units;
  const int per = a.pair_heads ? a.n_heads / 2 : a.n_heads;
  x.b = u / per;
  const int unit = u - x.b * per;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    x.head[t] = a.pair_heads ? 2 * unit + t : unit;
    x.q0[t] = a.pair_heads ? work * BR : (2 * work + t) * BR;
  }
  x.kvh = x.head[0] / (a.n_heads / a.n_kv_heads);
  int len = a.lens ? __ldg(a.lens + x.b) : a.seq;
  if (len < 0 || len > a.seq) {
    set_dev_error(a.err, RA_DEVERR_BOUNDS);
    len = len < 0 ? 0 : a.seq;
  }
  x.len = len;
  Blocks& kb = x.kb;
  kb.lo = 1 << 30;
  kb.hi = -1;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const bool any = x.q0[t] < len;
    const int last = x.q0[t] + BR - 1 < len ? x.q0[t] + BR - 1 : len - 1, first = x.q0[t] - a.W + 1;
    kb.thi[t] = any ? last / BR : -1;
    kb.tlo[t] = any && first > 0 ? first / BR : 0;
    if (any && kb.tlo[t] < kb.lo) kb.lo = kb.tlo[t];
    if (kb.thi[t] > kb.hi) kb.hi = kb.thi[t];
  }
  const int sink_blocks = a.sinks / BR + (a.sinks % BR != 0);
  kb.ns = sink_blocks < kb.hi + 1 ? sink_blocks : kb.hi + 1;
  if (kb.lo < kb.ns) kb.lo = kb.ns;
  kb.n = kb.hi < 0 ? 0 : kb.ns + (kb.hi >= kb.lo ? kb.hi - kb.lo + 1 : 0);
  return x;
}

template <int DH>
__global__ void __launch_bounds__(THREADS, 1) window_fwd_tc_kernel(const __grid_constant__ CUtensorMap tmQ,
    const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const __grid_constant__ WindowFwdArgs a) {
  using Pl = FwdPlan<DH>;
  constexpr int SLOTS = Pl::SLOTS, BLK = Pl::BLK;
  extern __shared__ __align__(1024) uint8_t smem[];
  // q_read: the last product with this pair's queries is done; o_full: a tile's outputs are complete; o_read: they have left TMEM
  __shared__ __align__(8) uint64_t full[SLOTS], empty[SLOTS], zeroed[SLOTS], q_full, q_read, s_full[2], p_full[2], o_full[2], o_read[2], turn[2], drain[2];
  __shared__ uint32_t tmem_sh;
  __shared__ volatile int abort_sh;
  __shared__ int info[8][8];
  const uint32_t sb = smem_u32(smem);
  if (sb & 1023u) {  // the swizzled operand tiles need 1024-byte alignment
    if (threadIdx.x == 0) set_dev_error(a.err, RA_DEVERR_BOUNDS);
    return;
  }
  const int tid = threadIdx.x, warp = warp_index(), lane = tid & 31;
  if (warp == 10) {
    if (elect_one()) {
#pragma unroll
      for (int i = 0; i < SLOTS; ++i) {
        mbar_init(&full[i], 1);
        mbar_init(&empty[i], 2);
        mbar_init(&zeroed[i], 1);
      }
      mbar_init(&q_full, 1);
      mbar_init(&q_read, 2);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        mbar_init(&s_full[t], 1);
        mbar_init(&p_full[t], 4);
        mbar_init(&o_full[t], 1);
        mbar_init(&o_read[t], 4);
        mbar_init(&turn[t], 1);
        mbar_init(&drain[t], 1);
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
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  pdl_trigger();  // (TMEM is allocated: the next kernel's CTAs cannot come before this one)
  const uint32_t tmem = tmem_sh;

  if (warp == 10) {
    // ------------------------------------------------------------ copies
    if (elect_one()) {
      auto load = [&](const CUtensorMap* tm, uint32_t dst, uint64_t* bar, int col, int row, int b) {
#pragma unroll
        for (int n = 0; n < DH / 64; ++n) tma_load3(tm, dst + n * (BR * 128), bar, col + 64 * n, row, b);
      };
      int i = 0, nq = 0;  // blocks of the ring (keys and values in turn) and pairs of query tiles that were started
      bool ok = true;
      for (int id = blockIdx.x; id < a.items && ok; id += gridDim.x) {
        const Item x = item_of(a, id);
        if (x.kb.n == 0) continue;
        if (nq > 0) ok = mbar_wait(&q_read, (nq - 1) & 1, &abort_sh, a.err);
        if (!ok) break;
        mbar_expect_tx(&q_full, 2 * BLK);
#pragma unroll
        for (int t = 0; t < 2; ++t) load(&tmQ, sb + Pl::Q + t * BLK, &q_full, x.head[t] * DH, x.q0[t], x.b);
        ++nq;
        for (int k = 0; k < 2 * x.kb.n; ++k) {
          const int s = i % SLOTS;
          if (i >= SLOTS) ok = mbar_wait(&empty[s], ((i / SLOTS) - 1) & 1, &abort_sh, a.err);
          if (!ok) break;
          mbar_expect_tx(&full[s], BLK);
          load(k & 1 ? &tmV : &tmK, sb + Pl::RING + s * BLK, &full[s], x.kvh * DH, x.kb.at(k >> 1) * BR, x.b);
          ++i;
        }
      }
      if (!ok) {
        // a wait gave up: let the copies on their way land before shared memory is released
        volatile int no_abort = 0;
        if (nq > 0) mbar_wait(&q_full, (nq - 1) & 1, &no_abort, nullptr);
        for (int k = i > SLOTS ? i - SLOTS : 0; k < i; ++k) mbar_wait(&full[k % SLOTS], (k / SLOTS) & 1, &no_abort, nullptr);
      }
    }
    __syncwarp();
  } else if (warp >= 8) {
    // ------------------------------------------------------------ products, of tile 0 and of tile 1
    // A block of the ring is free, and the queries are, when both tiles are done with them; a tile that does not see a block
    // says so as soon as that has landed (not before: its word would count for what the slot held earlier).
    constexpr uint32_t IDS = idesc_bf16(BR, 0), IDO = idesc_bf16_bmn(BR, DH);  // (the scores' columns come with the block)
    const int t = warp - 8;
    const uint32_t tS = uniform(tmem + Pl::C_S + t * BR), tO = uniform(tmem + Pl::C_O + t * DH);
    const uint32_t q = desc_lo_k(sb + Pl::Q + t * BLK);
    bool ok = true;
    uint32_t turns = 0;  // each warp has one a block and one after the last, with or without products
    uint32_t p_phase = 0, z_phase = 0;  // (z_phase: a bit a slot, which tile 0 zeroes again only when tile 1 has let it go)
    int nq = 0, no = 0, ring = 0;  // pairs of tiles; tiles with outputs; blocks of the ring before this pair's
    for (int id = blockIdx.x; id < a.items && ok; id += gridDim.x) {
      const Item x = item_of(a, id);
      const Blocks& kb = x.kb;
      if (kb.n == 0) continue;
      ok = mbar_wait_warp(&q_full, nq & 1, &abort_sh, a.err);
      ++nq;
      const int thi = t ? kb.thi[1] : kb.thi[0], tlo = t ? kb.tlo[1] : kb.tlo[0];
      bool started = false, pend = false;
      int prev = 0, prev_n = 0;
      for (int i = 0; i <= kb.n && ok; ++i) {
        const int kn = ring + 2 * i, vn = kn - 1, ks = kn % SLOTS, vs = (vn + SLOTS) % SLOTS;  // this block's keys, the last one's values
        if (i > 0) {
          ok = mbar_wait_warp(&full[vs], (vn / SLOTS) & 1, &abort_sh, a.err);
          if (!ok) break;
          const int dead = x.len - prev * BR;  // rows from here on are past the sequence's end
          if (dead < BR) {
            if (t == 0) {
              zero_rows<DH>(smem + Pl::RING + vs * BLK, dead, lane);
              if (lane == 0) mbar_arrive(&zeroed[vs]);
            } else {
              ok = mbar_wait_warp(&zeroed[vs], (z_phase >> vs) & 1u, &abort_sh, a.err);
              if (!ok) break;
              z_phase ^= 1u << vs;
            }
          }
          if (pend && !started) {  // the outputs of this tile's last pair have left TMEM
            if (no > 0) ok = mbar_wait_warp(&o_read[t], (no - 1) & 1, &abort_sh, a.err);
            ++no;
            if (!ok) break;
          }
        }
        const int j = i < kb.n ? kb.at(i) : 0;
        bool next = false;
        int next_n = 0;
        if (i < kb.n) {
          ok = mbar_wait_warp(&full[ks], (kn / SLOTS) & 1, &abort_sh, a.err);
          if (!ok) break;
          next = j <= thi && (j >= tlo || j < kb.ns);
          next_n = sink_columns(j < tlo, j, a.sinks);
        }
        const uint32_t v = desc_lo_mn(sb + Pl::RING + vs * BLK, BR * 128), acc = uniform(started ? 1u : 0u);
        const uint32_t k = desc_lo_k(sb + Pl::RING + ks * BLK);
        const uint32_t ids = uniform(IDS | ((uint32_t)(next_n >> 3) << 17));
        const int n = (int)uniform(prev_n);
        if (t == 1 || turns > 0) ok = mbar_wait_warp(&turn[t], (turns - (t == 0)) & 1, &abort_sh, a.err);
        if (!ok) break;
        ++turns;
        if (pend) {
          ok = mbar_wait_warp(&p_full[t], p_phase, &abort_sh, a.err);
          if (!ok) break;
          p_phase ^= 1u;
        }
        tc_fence_after();
        if (elect_one()) {
          if (pend) {
#pragma unroll
            for (int kk = 0; kk < BR / 16; ++kk)
              if (16 * kk < n) umma_bf16_ts(tO, tS + kk * 8, desc_of(v + kk * (2048 >> 4)), IDO, kk > 0 ? 1u : acc);
          }
          if (next) {
#pragma unroll
            for (int kk = 0; kk < DH / 16; ++kk) {
              const uint32_t o = ((kk >> 2) * (BR * 128) + (kk & 3) * 32) >> 4;
              umma_bf16(tS, desc_of(q + o), desc_of(k + o), ids, kk > 0 ? 1u : 0u);
            }
            umma_commit(&s_full[t]);
          }
          mbar_arrive(&turn[t ^ 1]);
          if (pend && prev == thi) umma_commit(&o_full[t]);
          if (i > 0) {
            if (pend) umma_commit(&empty[vs]);
            else mbar_arrive(&empty[vs]);
          }
          if (i < kb.n) {
            if (next) umma_commit(&empty[ks]);
            else mbar_arrive(&empty[ks]);
            if (i == kb.n - 1) umma_commit(&q_read);
          }
        }
        __syncwarp();
        if (pend) started = true;
        pend = next;
        prev = j;
        prev_n = next_n;
      }
      ring += 2 * kb.n;
    }
    // what was issued ends before shared memory and TMEM are released
    if (elect_one()) {
      volatile int no_abort = 0;
      umma_commit(&drain[t]);
      mbar_wait(&drain[t], 0, &no_abort, nullptr);
    }
    __syncwarp();
  } else {
    // ------------------------------------------------------------ softmax: warps 4 t .. 4 t + 3, thread = row
    const int t = warp >> 2, row = tid & 127;
    const uint32_t tS = tmem + ((uint32_t)(32 * (warp & 3)) << 16) + Pl::C_S + t * BR;
    const uint32_t tO = tmem + ((uint32_t)(32 * (warp & 3)) << 16) + Pl::C_O + t * DH;
    uint32_t s_phase = 0, o_phase = 0;
    bool ok = true;
    for (int id = blockIdx.x; id < a.items && ok; id += gridDim.x) {
      // (what a pair is, is kept in shared memory: the scores of a row take most of a thread's registers)
      {
        const Item x = item_of(a, id);
        __syncwarp();
        if (lane == 0) {
          info[warp][0] = x.kb.ns;
          info[warp][1] = x.kb.lo;
          info[warp][2] = t ? x.kb.tlo[1] : x.kb.tlo[0];
          info[warp][3] = t ? x.kb.thi[1] : x.kb.thi[0];
          info[warp][4] = x.len;
          info[warp][5] = t ? x.q0[1] : x.q0[0];
          info[warp][6] = x.b;
          info[warp][7] = t ? x.head[1] : x.head[0];
        }
        __syncwarp();
      }
      const volatile int* I = info[warp];
      float m = -INFINITY, l = 0.f;  // m: the scale in use (powers of two); l: this row's sum under it
      bool first = true;
      for (int i = 0;; ++i) {
        int j = i;
        if (i >= I[0]) j = i - I[0] + I[1];
        if (j > I[3]) break;  // (the other tile may have a block more)
        if (j < I[2] && j >= I[0]) continue;
        ok = mbar_wait_warp(&s_full[t], s_phase, &abort_sh, a.err);
        if (!ok) break;
        s_phase ^= 1u;
        tc_fence_after();
        const int j0 = j * BR, q0 = I[5];
        // a block that all rows of the tile see whole has no test a key; else a bit a key
        const bool whole = j0 + BR - 1 <= q0 && (q0 + BR - 1 - j0 < a.W || j0 + BR <= a.sinks);
        const int chunks = (sink_columns(j < I[2], j, a.sinks) + 31) >> 5;  // of 32 columns
        uint32_t live[4] = {~0u, ~0u, ~0u, ~0u};
        uint32_t some = 0xfu;  // chunks that a row of this warp sees something of
        if (!whole) {
          const int q = q0 + row, hi = q < I[4] ? q - j0 + 1 : 0, lo = q - a.W + 1 - j0, sk = a.sinks - j0;
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            live[c] = below(hi - 32 * c) & (~below(lo - 32 * c) | below(sk - 32 * c));
            if (!__any_sync(0xffffffffu, live[c] != 0)) some &= ~(1u << c);
          }
        }
        // the scores are read twice, 32 at a time, for the maximum and for the exponentials: held in registers all along they
        // leave too few for the rest
        float s[2][32];
        float bm[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
        if (whole) {
          tmem_ld32_issue(tS, reinterpret_cast<uint32_t*>(s[0]));
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            float* x = s[c & 1];
            tmem_wait32(reinterpret_cast<uint32_t*>(x));
            if (c < 3) tmem_ld32_issue(tS + 32 * (c + 1), reinterpret_cast<uint32_t*>(s[(c + 1) & 1]));
#pragma unroll
            for (int e = 0; e < 32; ++e) bm[e & 3] = fmaxf(bm[e & 3], x[e]);
          }
        } else {
#pragma unroll
          for (int c = 0; c < 4; ++c)
            if ((some >> c) & 1u) {
              tmem_ld32(tS + 32 * c, s[0]);
#pragma unroll
              for (int e = 0; e < 32; ++e) bm[e & 3] = fmaxf(bm[e & 3], (live[c] >> e) & 1u ? s[0][e] : -INFINITY);
            }
        }
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
        float2 sum[2] = {f2(0.f), f2(0.f)};
        auto exponentials = [&](int c, const float* x) {
          uint32_t w[16];
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float2 z = __ffma2_rn(make_float2(x[2 * e], x[2 * e + 1]), f2(a.sl2), f2(-ms));
            const float2 p = make_float2(ex2_fast(z.x), ex2_fast(z.y));
            sum[e & 1] = __fadd2_rn(sum[e & 1], p);
            w[e] = pk2(p.x, p.y);
          }
          tmem_st16(tS + 16 * c, w);  // over scores that have been read
        };
        if (whole) {
          tmem_ld32_issue(tS, reinterpret_cast<uint32_t*>(s[0]));
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            float* x = s[c & 1];
            tmem_wait32(reinterpret_cast<uint32_t*>(x));
            if (c < 3) tmem_ld32_issue(tS + 32 * (c + 1), reinterpret_cast<uint32_t*>(s[(c + 1) & 1]));
            exponentials(c, x);
          }
        } else {
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            if (c >= chunks) break;
            if ((some >> c) & 1u) {
              tmem_ld32(tS + 32 * c, s[0]);
#pragma unroll
              for (int e = 0; e < 32; ++e) s[0][e] = (live[c] >> e) & 1u ? s[0][e] : -INFINITY;
              exponentials(c, s[0]);
            } else {
              const uint32_t none[16] = {};
              tmem_st16(tS + 16 * c, none);
            }
          }
        }
        l += (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&p_full[t]);
      }
      // ---- outputs
      const bool any = I[3] >= 0;
      if (ok && any) {
        ok = mbar_wait_warp(&o_full[t], o_phase, &abort_sh, a.err);
        o_phase ^= 1u;
        tc_fence_after();
      }
      if (!ok) break;
      const int len = I[4], q = I[5] + row, head = I[7], b = I[6];
      const bool seen = q < len && !(m == -INFINITY && l == 0.f);  // (the maximum of NaN scores stays -inf, their sum does not stay 0)
      const float f = seen ? 1.f / l : 0.f;
      bf16* out = a.out + ((int64_t)b * a.seq + (q < a.seq ? q : 0)) * a.out_stride + head * DH;
#pragma unroll 1
      for (int c = 0; c < DH; c += 32) {
        float o[32];
        if (any) tmem_ld32(tO + c, o);
        if (any && c + 32 == DH) {  // the accumulator is free for the next pair's products
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&o_read[t]);
        }
        if (q < a.seq) {
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = q < len ? pk2(o[8 * g + 2 * e] * f, o[8 * g + 2 * e + 1] * f) : 0u;
            *reinterpret_cast<uint4*>(out + c + 8 * g) = make_uint4(w[0], w[1], w[2], w[3]);
          }
        }
      }
      if (a.lse && q < a.seq) a.lse[((int64_t)b * a.n_heads + head) * a.seq + q] = seen ? (m + log2f(l)) * kLn2 : -INFINITY;
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
  const int64_t units = (int64_t)p.batch * (a.pair_heads ? p.n_heads / 2 : p.n_heads), items = units * a.n_work;
  if (items > INT32_MAX - 1024) return cudaErrorNotSupported;
  a.units = (int)units;
  a.items = (int)items;
  a.out = (bf16*)p.out_dev;
  a.out_stride = p.out_stride;
  CUtensorMap q, k, v;
  if (!tma_map_bf16_batch(&q, p.q_dev, p.batch, p.seq, (int64_t)p.n_heads * DH, p.q_stride, 64, BR) ||
      !tma_map_bf16_batch(&k, p.k_dev, p.batch, p.seq, (int64_t)p.n_kv_heads * DH, p.k_stride, 64, BR) ||
      !tma_map_bf16_batch(&v, p.v_dev, p.batch, p.seq, (int64_t)p.n_kv_heads * DH, p.v_stride, 64, BR))
    return cudaErrorNotSupported;
  const int sms = device_sm_count();
  cudaError_t e = allow_smem(window_fwd_tc_kernel<DH>, FwdPlan<DH>::BYTES);
  if (e == cudaSuccess)
    e = launch_pdl(window_fwd_tc_kernel<DH>, dim3(a.items < sms ? a.items : sms), dim3(THREADS), (size_t)FwdPlan<DH>::BYTES, st, q, k, v, a);
  note_launch(1);
  return e;
}

}  // namespace

cudaError_t attention_window_fwd_tc(const ra_attention_window_args& a, cudaStream_t st) {
  return a.head_dim == 64 ? launch<64>(a, st) : a.head_dim == 128 ? launch<128>(a, st) : cudaErrorNotSupported;
}

}  // namespace ra
