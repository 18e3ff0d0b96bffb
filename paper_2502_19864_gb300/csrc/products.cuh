// products.cuh -- products of bf16 operands, or of fp32 ones in bf16 planes, on the tensor cores, for operators that differ in
// where tiles come from and what becomes of them.
//
// A unit of work is a tile C[m0.., n0..] of 128 CG x BN (BN <= 256) over a range of k-blocks of 64.  Each operand is
// K-major or MN-major, read by TMA through a map of (inner, rows, z).  An fp32 operand is given as planes of bf16 that lie
// at consecutive z, each holding the next 8 bits: of the planes' products those that matter are added up, the smallest
// first.  The tensor cores truncate what they add to an accumulator: a sum of K products of one sign loses about 4.3e-10 K of
// itself (measured: 9e-7 at K = 2048, 3.5e-5 at 32768).  So an accumulator takes `chunk` k-blocks, and the epilogue's threads
// add up the chunks' accumulators in fp32 registers, rounded to nearest; and of three planes' products all but the largest
// have an accumulator of their own, so that their five steps a k-block are not truncated at the largest's size (two of 777 x 777 x
// 1000 orthogonalised: 1.5e-5 from 64 bits with one accumulator, 3e-6 with two).
//
// One persistent CTA an SM (or, CG = 2, a pair on two): warp 0 keeps a ring of operand stages filled by TMA, warp 1
// issues the products into one of two accumulators in TMEM, warps 2..9 take the finished one into registers, 128 values a thread,
// and hand the tile to the operator.  Waits are bounded; on expiry the kernel records it, lets its copies land and returns.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

#include "common.cuh"
#include "kernels.h"
#include "tcgen05.cuh"
#include "window_tc.cuh"

namespace ra {
namespace prod {

using namespace tc;

constexpr int BM = 128, BK = 64, MAX_BN = 256, MAX_STAGES = 8;
constexpr int THREADS = 320, EPI_WARPS = 8;
constexpr int A_BYTES = BM * BK * 2;
constexpr int STAGING = 4096;  // of an epilogue warp: two boxes of 2 KB
constexpr int RING = 192 * 1024;
constexpr int SMEM = RING + EPI_WARPS * STAGING + 1024;

// The planes of a product's terms, the smallest first: 2 bits each of A's and of B's plane a term
struct Terms {
  int n;
  uint32_t a, b;
};
// Of operands of pa and pb planes: all pairs (i, j) with i + j less than the larger number; what is left out is below 2^-8 of
// the last plane's part (three planes: (0, 2) (1, 1) (2, 0) (0, 1) (1, 0) (0, 0), 2^-24 of the whole)
__host__ __device__ constexpr Terms terms_of(int pa, int pb) {
  Terms t = {0, 0u, 0u};
  for (int sum = (pa > pb ? pa : pb) - 1; sum >= 0; --sum)
    for (int i = 0; i <= sum; ++i)
      if (i < pa && sum - i < pb) {
        t.a |= (uint32_t)i << (2 * t.n);
        t.b |= (uint32_t)(sum - i) << (2 * t.n);
        ++t.n;
      }
  return t;
}

// A stage of the ring has a k-block of all planes of both operands: each comes once, for all the terms it is in (2 x 777 x 1000
// orthogonalised in fp32: 500 us with a stage a term, which loads twice as much, 400 so)
struct Shape {
  int bn;       // columns of a tile: a multiple of 32, of 64 CG for an MN-major B
  int chunk;    // k-blocks of an accumulator
  int b_bytes, stages, stage_bytes;
};
inline int stages_of(int bn, int cg, int pa, int pb) {
  const int stage = pa * A_BYTES + pb * ((bn / cg + 63) / 64 * 64 * BK * 2);
  return RING / stage < MAX_STAGES ? RING / stage : MAX_STAGES;
}
inline Shape shape_of(int bn, int cg, int pa, int pb, int chunk) {
  Shape s;
  s.bn = bn;
  s.chunk = chunk;
  s.b_bytes = (bn / cg + 63) / 64 * 64 * BK * 2;
  s.stage_bytes = pa * A_BYTES + pb * s.b_bytes;
  s.stages = stages_of(bn, cg, pa, pb);
  return s;
}

// Which tiles: CTAs to a tile, and its columns
struct Pick {
  int cg, bn;
};
constexpr int SMS = 152;  // a plan is the same on every device
inline int parts_of(int64_t a, int b) { return (int)((a + b - 1) / b); }
inline int up(int64_t a, int b) { return (int)((a + b - 1) / b * b); }
// microseconds of a k-block of a tile (measured on long products; the issue of products and copies paces the narrow ones, power the widest:
// by the share of SMs that have one)
inline double block_time(Pick k, double share = 1.) {
  if (k.cg == 2) return 0.24 + 0.105 * (share < 1. ? share : 1.);  // (256 columns: of 128 a pair takes longer than its CTAs apart, 0.25)
  return k.bn <= 64 ? 0.2 : k.bn <= 128 ? 0.222 : k.bn <= 192 ? 0.31 : 0.365;
}
// ... of `tiles` tiles of `blocks` k-blocks, terms counted, in rounds, each with about 1 us for its start and end, and a tile's epilogue,
// `out` microseconds for 128 columns, beside the next one's products
inline double time_of_tiles(Pick k, int64_t tiles, int blocks, double out) {
  const double in = blocks * block_time(k, (double)tiles * k.cg / SMS) + 1., end = out * k.bn / 128.;
  return in + (parts_of(tiles, SMS / k.cg) - 1) * (in > end ? in : end) + end + (k.cg == 2 ? 1. : 0.);
}
// ... of `batch` products m x n
inline double time_of(Pick k, int64_t m, int64_t n, int64_t batch, int blocks, double out = 0.) {
  return time_of_tiles(k, batch * parts_of(m, BM * k.cg) * parts_of(n, k.bn), blocks, out);
}
// whether a tile's ring has two stages, and TMEM room for two accumulators, of three planes twice
inline bool takes(Pick k, int pa, int pb) { return stages_of(k.bn, k.cg, pa, pb) >= 2 && (pa < 3 && pb < 3 ? k.bn <= MAX_BN : k.bn <= MAX_BN / 2); }
// the fastest
inline Pick pick(int64_t m, int64_t n, int64_t batch, int blocks, int pa, int pb, double out = 0.) {
  Pick best = {1, n <= 64 ? 64 : 128};
  for (Pick k : {Pick{1, 64}, Pick{1, 256}, Pick{2, 256}})
    if ((k.cg == 1 || m > BM) && n > k.bn / 2 && takes(k, pa, pb) &&
        time_of(k, m, n, batch, blocks, out) < time_of(best, m, n, batch, blocks, out))
      best = k;
  return best;
}

struct Unit {
  const CUtensorMap *a, *b;
  int ar, br;        // the tile's first row of A and of B (of C's columns)
  int ak, bk;        // where K begins in each
  int az, bz;
  int kb0, kb1;      // k-blocks
  bool a_mn, b_mn;   // MN-major: K runs along the map's rows
  int job, m0, n0, z;  // the operator's own
};

// tiles in groups of eight rows of tiles swept across the columns: those that run at the same time share operands in L2
__device__ __forceinline__ void tile_of(int tile, int m_tiles, int n_tiles, int& mt, int& nt) {
  const int per = 8 * n_tiles, grp = tile / per, in = tile % per, rows = min(8, m_tiles - grp * 8);
  mt = grp * 8 + in % rows;
  nt = in / rows;
}

template <int CG>
__device__ __forceinline__ void load(const CUtensorMap* tm, uint32_t dst, uint32_t bar, int c0, int c1, int c2) {
  if (CG == 2)
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(tm)), "r"(c0), "r"(c1), "r"(c2), "r"(bar)
        : "memory");
  else
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(tm)), "r"(c0), "r"(c1), "r"(c2), "r"(bar)
        : "memory");
}

// The next 8 bits of x's significand and what is left, exactly (truncated, so that no plane overflows and all have x's sign).
// What is not finite leaves NaN.
__device__ __forceinline__ float plane_trunc(float& x) {
  const float h = __uint_as_float(__float_as_uint(x) & 0xffff0000u);
  x = __fsub_rn(x, h);
  return h;
}
// Two values' planes, a word of two bf16 each: three truncated ones (exact: the words are the upper halves), or two rounded
template <int PLANES>
__device__ __forceinline__ void planes_of(float x, float y, uint32_t (&w)[PLANES]) {
  if constexpr (PLANES == 3) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      w[k] = __byte_perm(__float_as_uint(x), __float_as_uint(y), 0x7632);
      plane_trunc(x);
      plane_trunc(y);
    }
    w[2] = __byte_perm(__float_as_uint(x), __float_as_uint(y), 0x7632);
  } else {
    const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
    w[0] = *reinterpret_cast<const uint32_t*>(&h);
    const __nv_bfloat162 l = __floats2bfloat162_rn(__fsub_rn(x, __uint_as_float(w[0] << 16)), __fsub_rn(y, __uint_as_float(w[0] & 0xffff0000u)));
    w[1] = *reinterpret_cast<const uint32_t*>(&l);
  }
}
// Plane K of two values, a word
template <int PLANES, int K>
__device__ __forceinline__ uint32_t plane_of(float x, float y) {
  uint32_t w[PLANES];
  planes_of<PLANES>(x, y, w);
  return w[K];
}
// What an epilogue warp stores through: boxes of 32 rows x 64 bytes (32 bf16 or 16 fp32 columns), 64-byte swizzled, by TMA
struct Store {
  uint8_t* staging;
  int lane, turn;
  __device__ __forceinline__ uint8_t* slot() {
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(1) : "memory");
    __syncwarp();
    return staging + (turn++ & 1) * 2048;
  }
  __device__ __forceinline__ void send(const CUtensorMap* tm, uint8_t* s, int c0, int c1, int c2, bool add) {
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (lane == 0) {
      if (add)
        asm volatile("cp.reduce.async.bulk.tensor.3d.global.shared::cta.add.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(
                         reinterpret_cast<uint64_t>(tm)),
                     "r"(c0), "r"(c1), "r"(c2), "r"(smem_u32(s))
                     : "memory");
      else
        asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(
                         reinterpret_cast<uint64_t>(tm)),
                     "r"(c0), "r"(c1), "r"(c2), "r"(smem_u32(s))
                     : "memory");
      asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
  }
  // this thread's row of 32 columns f(0), f(1), .., rounded to bf16
  template <typename F>
  __device__ __forceinline__ void bf16_row(const CUtensorMap* tm, F f, int col, int row, int z) {
    uint8_t* s = slot();
    const int sw = (lane >> 1) & 3;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      uint4 x;
      __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&x);
#pragma unroll
      for (int i = 0; i < 4; ++i) h[i] = __floats2bfloat162_rn(f(8 * q + 2 * i), f(8 * q + 2 * i + 1));
      *reinterpret_cast<uint4*>(s + lane * 64 + ((q ^ sw) << 4)) = x;
    }
    send(tm, s, col, row, z, false);
  }
  // ... its planes, which are z0, z0 + 1, .. of the map (straight from registers, 64 bytes of eight rows a store, 2 x 777 x 1000 in fp32
  // orthogonalised takes 370 us, so 352).  TURNED: the warp's 32 x 32 transposed, with `row` and `col` as they are then
  template <int PLANES, bool TURNED, int K = 0, typename F>
  __device__ __forceinline__ void planes(const CUtensorMap* tm, F f, int col, int row, int z0) {
    if constexpr (K < PLANES) {
      uint32_t w[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) w[i] = plane_of<PLANES, K>(f(2 * i), f(2 * i + 1));
      uint8_t* s = slot();
      if (TURNED) {  // this lane's values are a column: two bytes of each row
#pragma unroll
        for (int j = 0; j < 32; ++j)
          *reinterpret_cast<uint16_t*>(s + j * 64 + ((((lane >> 3) ^ (j >> 1)) & 3) << 4) + (lane & 7) * 2) = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
      } else {
        const int sw = (lane >> 1) & 3;
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *reinterpret_cast<uint4*>(s + lane * 64 + ((q ^ sw) << 4)) = make_uint4(w[4 * q], w[4 * q + 1], w[4 * q + 2], w[4 * q + 3]);
      }
      send(tm, s, col, row, z0 + K, false);
      planes<PLANES, TURNED, K + 1>(tm, f, col, row, z0);
    }
  }
  // ... not by TMA: g(r, value) for this lane's column of the warp's rows r, so that a row's 32 values leave side by side
  template <typename G>
  __device__ __forceinline__ void by_columns(const float (&v)[32], G g) {
    float* s = reinterpret_cast<float*>(staging);
#pragma unroll
    for (int j = 0; j < 32; ++j) s[lane * 32 + (j ^ lane)] = v[j];
    __syncwarp();
#pragma unroll 8
    for (int r = 0; r < 32; ++r) g(r, s[r * 32 + (lane ^ r)]);
    __syncwarp();
  }
  // ... in fp32, stored or added to what is there; columns from `cols` on are not the map's
  __device__ __forceinline__ void f32_row(const CUtensorMap* tm, const float* v, int col, int row, int z, bool add, int cols) {
    const int sw = (lane >> 1) & 3;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (col + 16 * h >= cols) break;
      uint8_t* s = slot();
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<float4*>(s + lane * 64 + ((q ^ sw) << 4)) =
            make_float4(v[16 * h + 4 * q], v[16 * h + 4 * q + 1], v[16 * h + 4 * q + 2], v[16 * h + 4 * q + 3]);
      send(tm, s, col + 16 * h, row, z, add);
    }
  }
};

struct Tile {
  int quad, lane, half;  // TMEM lanes 32 quad.. ; columns 32 (half + 2 i)..
  int rank;              // of the CTA in its pair
  int chunks;            // of 32 columns that this warp holds
};

__device__ __forceinline__ void prefetch_map(const CUtensorMap* tm) {
  asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(tm)) : "memory");
}
// P: the operands' planes PA and PB, Args (with `Shape shape`, `unsigned* err`), static void prefetch(const Args&) (of the operands'
// maps), static int count(const Args&), static void unit(const Args&, int, Unit&) and
// PARTS (ONE: a unit has k-blocks, and one accumulator takes them all) and static void part(const Args&, const Unit&, const Tile&,
// Store&, int i, float (&v)[32]) for this warp's i-th 32 columns, or
// static void finish(const Args&, const Unit&, const Tile&, Store&, float (&v)[CH][32]) for all of them.
template <class P, int CG>
__global__ void __launch_bounds__(THREADS, 1) products_kernel(const __grid_constant__ typename P::Args p) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t full_bar[MAX_STAGES], empty_bar[MAX_STAGES], tfull_bar[2], tempty_bar[2], drain_bar;
  __shared__ uint32_t tmem_base_sh;
  __shared__ volatile int abort_sh;
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  const uint32_t smem_base = smem_u32(smem);
  const int warp = warp_index(), lane = threadIdx.x & 31;
  const int rank = CG == 2 ? (int)cluster_rank() : 0;
  const int worker = (int)blockIdx.x / CG, workers = (int)gridDim.x / CG;
  const int stages = p.shape.stages, bn = p.shape.bn, bnc = bn / CG;

  if (threadIdx.x == 0) {
    for (int s = 0; s < MAX_STAGES; ++s) {
      mbar_init(&full_bar[s], 1);
      mbar_init(&empty_bar[s], 1);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(&tfull_bar[a], 1);
      mbar_init(&tempty_bar[a], EPI_WARPS * CG);
    }
    mbar_init(&drain_bar, 1);
    abort_sh = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (threadIdx.x == 32) P::prefetch(p);
  if (CG == 2) {  // the barriers of both CTAs are there before either signals the other's
    __syncthreads();
    cluster_arrive();
    cluster_wait();
  }
  if (warp == 1) {
    if (CG == 2) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base_sh)), "r"(512u) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base_sh)), "r"(512u) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = tmem_base_sh;
  pdl_wait();
  pdl_trigger();
  const int units = P::count(p);
  constexpr bool TWO = P::PA == 3 && P::PB == 3;  // accumulators: the largest term's, and 128 columns on the others'
  const int chunk = p.shape.chunk;

  if (warp == 0) {
    // ---- operand stages by TMA
    if (elect_one()) {
      int stage = 0, issued = 0;
      uint32_t phase = 0;
      bool ok = true;
      const int boxes = (bnc + 63) / 64;
      for (int u = worker; ok && u < units; u += workers) {
        Unit w;
        P::unit(p, u, w);
        const int ar = w.ar + rank * BM, br = w.br + rank * bnc;
        const uint32_t all = CG * (uint32_t)(P::PA * A_BYTES + P::PB * (w.b_mn ? boxes * 64 : bnc) * BK * 2);
        for (int c0 = w.kb0; ok && c0 < w.kb1; c0 += chunk) {
          const int c1 = min(c0 + chunk, w.kb1);
          for (int kb = c0; kb < c1; ++kb) {
            if (!mbar_wait(&empty_bar[stage], phase ^ 1u, &abort_sh, p.err)) { ok = false; break; }
            if (rank == 0) mbar_expect_tx(&full_bar[stage], all);
            const uint32_t full = CG == 2 ? peer_addr(smem_u32(&full_bar[stage]), 0) : smem_u32(&full_bar[stage]);
            const int ka = w.ak + kb * BK, kbb = w.bk + kb * BK;
            uint32_t to = smem_base + stage * p.shape.stage_bytes;
#pragma unroll
            for (int z = 0; z < P::PA; ++z, to += A_BYTES) {
              if (w.a_mn) {
                load<CG>(w.a, to, full, ar, ka, w.az + z);
                load<CG>(w.a, to + 8192, full, ar + 64, ka, w.az + z);
              } else {
                load<CG>(w.a, to, full, ka, ar, w.az + z);
              }
            }
#pragma unroll
            for (int z = 0; z < P::PB; ++z, to += p.shape.b_bytes) {
              if (w.b_mn) {
                for (int x = 0; x < boxes; ++x) load<CG>(w.b, to + x * 8192, full, br + 64 * x, kbb, w.bz + z);
              } else {
                load<CG>(w.b, to, full, kbb, br, w.bz + z);
              }
            }
            ++issued;
            if (++stage == stages) { stage = 0; phase ^= 1u; }
          }
        }
      }
      // copies land before the CTA goes away; a pair's last signals to this CTA's barriers, too
      if (!ok && rank == 0) {
        volatile int no_abort = 0;
        for (int i = max(0, issued - stages); i < issued; ++i)
          mbar_wait(&full_bar[i % stages], (uint32_t)(i / stages) & 1u, &no_abort, nullptr);
      }
      if (CG == 2 && ok)
        for (int i = max(0, issued - stages); i < issued; ++i)
          mbar_wait(&empty_bar[i % stages], (uint32_t)(i / stages) & 1u, &abort_sh, p.err);
    }
    __syncwarp();
  } else if (warp == 1) {
    // ---- products
    if (rank == 0 && elect_one()) {
      const uint64_t kmaj = sdesc_sw128(smem_base), mnmaj = sdesc_mn_sw128_lbo(smem_base, 8192);
      int stage = 0, acc = 0;
      uint32_t phase = 0, acc_phase = 0;
      bool ok = true;
      for (int u = worker; ok && u < units; u += workers) {
        Unit w;
        P::unit(p, u, w);
        const uint32_t idesc = idesc_bf16(CG * BM, bn) | (w.a_mn ? 1u << 15 : 0u) | (w.b_mn ? 1u << 16 : 0u);
        // 16 values of K on: 32 bytes inside the swizzle's atom, or 16 rows of 128 bytes
        const uint64_t ad = w.a_mn ? mnmaj : kmaj, bd = (w.b_mn ? mnmaj : kmaj) + (uint64_t)(P::PA * A_BYTES / 16);
        const uint32_t bplane = (uint32_t)p.shape.b_bytes / 16;
        const uint64_t as = w.a_mn ? 128u : 2u, bs = w.b_mn ? 128u : 2u;
        for (int c0 = w.kb0; ok && c0 < w.kb1; c0 += chunk) {
          const int steps = min(c0 + chunk, w.kb1) - c0;
          if (!mbar_wait(&tempty_bar[acc], acc_phase ^ 1u, &abort_sh, p.err)) { ok = false; break; }
          tc_fence_after();
          const uint32_t d = tmem_base + (uint32_t)(acc * MAX_BN);
          for (int i = 0; i < steps; ++i) {
            if (!mbar_wait(&full_bar[stage], phase, &abort_sh, p.err)) { ok = false; break; }
            tc_fence_after();
            const uint64_t off = (uint64_t)(stage * (p.shape.stage_bytes / 16));
            constexpr Terms terms = terms_of(P::PA, P::PB);
#pragma unroll
            for (int t = 0; t < terms.n; ++t) {
              const uint32_t dt = TWO && t < terms.n - 1 ? d + MAX_BN / 2 : d;
              const uint64_t at = ad + off + (uint64_t)((terms.a >> (2 * t) & 3u) * (A_BYTES / 16)), bt = bd + off + (uint64_t)((terms.b >> (2 * t) & 3u) * bplane);
#pragma unroll
              for (int k = 0; k < BK / 16; ++k) {
                const uint64_t x = at + as * (uint64_t)k, y = bt + bs * (uint64_t)k;
                const uint32_t more = TWO && t == terms.n - 1 ? i | k : i | t | k;
                if (CG == 2) umma_bf16_pair(dt, x, y, idesc, more);
                else umma_bf16(dt, x, y, idesc, more);
              }
            }
            if (CG == 2) umma_commit_pair(&empty_bar[stage]);
            else umma_commit(&empty_bar[stage]);
            if (++stage == stages) { stage = 0; phase ^= 1u; }
          }
          if (!ok) break;
          if (CG == 2) umma_commit_pair(&tfull_bar[acc]);
          else umma_commit(&tfull_bar[acc]);
          if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
        }
      }
      // all products are complete before TMEM and shared memory are given back
      if (CG == 2) umma_commit_pair_own(&drain_bar);
      else umma_commit(&drain_bar);
      volatile int no_abort = 0;
      mbar_wait(&drain_bar, 0, &no_abort, nullptr);
    }
    __syncwarp();
  } else {
    // ---- finished tiles
    Tile t;
    t.quad = warp & 3;
    t.lane = lane;
    t.half = (warp - 2) >> 2;
    t.rank = rank;
    t.chunks = (bn / 32 - t.half + 1) / 2;
    Store st{smem + RING + (warp - 2) * STAGING, lane, 0};
    int acc = 0;
    uint32_t acc_phase = 0;
    bool ok = true;
    for (int u = worker; ok && u < units; u += workers) {
      Unit w;
      P::unit(p, u, w);
      constexpr int CH = TWO ? 2 : 4;
      const uint32_t mine = tmem_base + ((uint32_t)(t.quad * 32) << 16) + (uint32_t)(32 * t.half);
      // this warp's i-th 32 columns of the accumulator
      auto read = [&](int i, float* x) {
        tmem_ld32(mine + (uint32_t)(acc * MAX_BN + 64 * i), x);
        if (TWO) {
          float y[32];
          tmem_ld32(mine + (uint32_t)(acc * MAX_BN + MAX_BN / 2 + 64 * i), y);
#pragma unroll
          for (int j = 0; j < 32; j += 2) {
            const float2 s = __fadd2_rn(make_float2(x[j], x[j + 1]), make_float2(y[j], y[j + 1]));
            x[j] = s.x;
            x[j + 1] = s.y;
          }
        }
      };
      auto release = [&]() {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          if (CG == 2) mbar_arrive_cluster(peer_addr(smem_u32(&tempty_bar[acc]), 0));
          else mbar_arrive(&tempty_bar[acc]);
        }
        if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
      };
      if constexpr (P::PARTS) {
        // one accumulator has it all: straight from there, 32 columns at a time (the operator's code once: where it runs once or twice
        // a launch, it takes the time in which its instructions come; 2048 x 2048 in bf16 orthogonalised 475 us unrolled, 428 so)
        if (P::ONE || (w.kb0 < w.kb1 && w.kb0 + chunk >= w.kb1)) {
          if (!mbar_wait_warp(&tfull_bar[acc], acc_phase, &abort_sh, p.err)) break;
          tc_fence_after();
#pragma unroll 1
          for (int i = 0; i < t.chunks; ++i) {
            float x[32];
            __syncwarp();
            read(i, x);
            P::part(p, w, t, st, i, x);
          }
          release();
          continue;
        }
      }
      if constexpr (!P::ONE) {
      float v[CH][32];
#pragma unroll
      for (int i = 0; i < CH; ++i)
#pragma unroll
        for (int j = 0; j < 32; ++j) v[i][j] = 0.f;
      for (int c0 = w.kb0; c0 < w.kb1; c0 += chunk) {
        if (!mbar_wait_warp(&tfull_bar[acc], acc_phase, &abort_sh, p.err)) { ok = false; break; }
        tc_fence_after();
#pragma unroll
        for (int i = 0; i < CH; ++i)
          if (i < t.chunks) {
            float x[32];
            read(i, x);
#pragma unroll
            for (int j = 0; j < 32; j += 2) {
              const float2 s = __fadd2_rn(make_float2(v[i][j], v[i][j + 1]), make_float2(x[j], x[j + 1]));
              v[i][j] = s.x;
              v[i][j + 1] = s.y;
            }
          }
        release();
      }
      if (!ok) break;
      if constexpr (P::PARTS) {
#pragma unroll
        for (int i = 0; i < CH; ++i)
          if (i < t.chunks) P::part(p, w, t, st, i, v[i]);
      } else {
        P::finish(p, w, t, st, v);
      }
      }
    }
    if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");  // this warp's stores are complete
  }

  tc_fence_before();
  __syncthreads();
  if (CG == 2) {  // neither CTA leaves while the other may read its operands or signal its barriers
    cluster_arrive();
    cluster_wait();
  }
  if (warp == 1) {
    tc_fence_after();
    if (CG == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512u) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512u) : "memory");
  }
}

// (tiles of three planes have at most 128 columns, and are one CTA's)
template <class P>
constexpr bool has_pairs() { return P::PA < 3 && P::PB < 3; }

template <class P, int CG>
cudaError_t launch(const typename P::Args& p, int units, cudaStream_t st) {
  auto k = products_kernel<P, CG>;
  static const cudaError_t attr = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM);
  if (attr != cudaSuccess) return attr;
  const int most = device_sm_count() / CG;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = CG;
  at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  cfg.gridDim = dim3((unsigned)((units < most ? units : most) * CG));
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = SMEM;
  cfg.stream = st;
  cfg.attrs = at;
  cfg.numAttrs = CG == 2 ? 2 : 1;
  note_launch(1);
  return cudaLaunchKernelEx(&cfg, k, p);
}
template <class P>
cudaError_t launch(const typename P::Args& p, int cg, int units, cudaStream_t st) {
  if constexpr (has_pairs<P>())
    if (cg == 2) return launch<P, 2>(p, units, st);
  return launch<P, 1>(p, units, st);
}

}  // namespace prod
}  // namespace ra
