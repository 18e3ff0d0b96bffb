// k_attention_decode.cu -- attention of a sequence's newest tokens over its paged key-value cache.
//
//   o = sum_j p_j v_j, p = softmax(scale q K^T) over the slots that the token sees.
//
// The query rows of a key-value head are its group's heads times the new tokens (R rows, a few to a few dozen); K and
// V are read once for all of them, 4 R head_dim flops for every 2 head_dim values: bound by memory.  The slots that
// any row sees (all, or the sinks and the windows) are numbered 0, 1, ... and cut into tiles of TK; the tiles of all
// sequences and heads, one after the other, are dealt to the CTAs in equal runs, whatever the lengths are.  A CTA
// walks its run with a ring of tiles on their way (cp.async, so that a page may end anywhere), keeping the running
// maximum m, sum l and outputs of the (sequence, head) at hand; where a run ends inside one, (m, l, o) go to the
// workspace and a second kernel joins the parts in the order of their slots.
//   bf16: the products are mma.sync m16n8k16: sixteen rows take the tensor instruction of one, and the rate asked of
//         it, 16 flops a byte of K and V, is a tenth of what it gives, so nothing is won by tcgen05's 128 rows.
//   f32:  FFMA, a warp's lanes on 32 tokens for q k and a thread a column for p v.
#include "common.cuh"
#include "operators.h"
#include "paged.cuh"

namespace ra {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.69314718055994531f;

struct DecodeArgs {
  ra_kv_cache c;
  const int32_t* lens;
  const void* q;
  void* out;
  int64_t q_stride, out_stride;
  float* lse;                    // user's, nullable
  const float* w_in;
  float* w_out;
  int64_t w_stride;
  float* part_o;                 // [2 grid][rows of a tile][DHT]
  float2* part_ml;               // [2 grid][rows of a tile]
  float* lse2;                   // [batch, kv heads, R] (powers of two), where weights are wanted
  float* scores;                 // [batch, kv heads, R, x_stride], scaled, in powers of two
  int64_t x_stride;
  int batch, n_new, n_heads, G, R, groups, max_len, window, sinks, grid;
  float sl2;                     // scale log2 e
};

// The slots that a call's new tokens see of a sequence: [0, n_sink) and [w0, len), as n numbers
struct Seen {
  int len, w0, n_sink, n;
};
__device__ __forceinline__ Seen seen_of(const DecodeArgs& a, int b) {
  Seen s;
  s.len = clamp_len(a.lens[b], a.max_len, a.c.err_dev);
  s.w0 = 0;
  if (a.window > 0) {
    const int64_t w0 = (int64_t)s.len - a.n_new - a.window + 1;  // the first new token's window
    s.w0 = w0 > 0 ? (int)w0 : 0;
  }
  s.n_sink = a.sinks < s.w0 ? a.sinks : s.w0;
  s.n = s.n_sink + s.len - s.w0;
  return s;
}
__device__ __forceinline__ int slot_of(const Seen& s, int x) { return x < s.n_sink ? x : x - s.n_sink + s.w0; }
// whether the query at slot i sees slot j <= its sequence's last
__device__ __forceinline__ bool sees(const DecodeArgs& a, int i, int j) {
  return j <= i && (a.window == 0 || i - j < a.window || j < a.sinks);
}
__device__ __forceinline__ int64_t warp_sum64(int64_t v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// How the tiles are dealt: unit (b, u), u = kv head * groups + row group, has tiles(b) tiles; units in order.
// One warp computes; `total` tiles go to min(grid, total) CTAs.
template <int TK>
struct Deal {
  int64_t total;
  int workers;
  __device__ __forceinline__ int tiles(const DecodeArgs& a, int b) const { return (seen_of(a, b).n + TK - 1) / TK; }
  __device__ void count(const DecodeArgs& a, int lane) {
    const int units = a.c.n_kv_heads * a.groups;
    int64_t t = 0;
    for (int b = lane; b < a.batch; b += 32) t += (int64_t)tiles(a, b) * units;
    total = warp_sum64(t);
    workers = total < a.grid ? (int)total : a.grid;
  }
  __device__ __forceinline__ int64_t start(int cta) const { return total * cta / workers; }
  __device__ __forceinline__ int owner(int64_t tile) const { return (int)(((tile + 1) * workers - 1) / total); }
  // the sequence that tile `at` belongs to, and its first tile (lane-wide, same in all lanes)
  __device__ void find(const DecodeArgs& a, int64_t at, int lane, int& b, int64_t& first) const {
    const int units = a.c.n_kv_heads * a.groups;
    int64_t acc = 0;
    for (int base = 0;; base += 32) {
      const int64_t t = base + lane < a.batch ? (int64_t)tiles(a, base + lane) * units : 0;
      int64_t incl = t;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int64_t v = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += v;
      }
      const uint32_t past = __ballot_sync(0xffffffffu, acc + incl > at);
      if (past) {
        const int l = __ffs(past) - 1;
        b = base + l;
        first = acc + __shfl_sync(0xffffffffu, incl - t, l);
        return;
      }
      acc += __shfl_sync(0xffffffffu, incl, 31);
    }
  }
  // the first tile of sequence b's unit u
  __device__ int64_t first_of(const DecodeArgs& a, int b, int u, int lane) const {
    const int units = a.c.n_kv_heads * a.groups;
    int64_t t = 0;
    for (int i = lane; i < b; i += 32) t += (int64_t)tiles(a, i) * units;
    return warp_sum64(t) + (int64_t)u * tiles(a, b);
  }
};

// Where a CTA is in its run: a tile of a unit
template <int TK>
struct Cursor {
  int b, u, tile, tiles;
  Seen s;
  __device__ __forceinline__ void enter(const DecodeArgs& a) {
    s = seen_of(a, b);
    tiles = (s.n + TK - 1) / TK;
  }
  __device__ __forceinline__ void next(const DecodeArgs& a) {
    if (++tile < tiles) return;
    tile = 0;
    if (++u < a.c.n_kv_heads * a.groups) return;
    u = 0;
    do {
      if (++b >= a.batch) return;  // (the run ends before)
      enter(a);
    } while (tiles == 0);
  }
};

__device__ __forceinline__ void cp16(uint32_t dst, const void* src, bool live) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(live ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ uint32_t pack2(float x, float y) {
  __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
  return *reinterpret_cast<uint32_t*>(&h);
}
__device__ __forceinline__ void ldsm4(uint32_t* r, uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void ldsm4t(uint32_t* r, uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void mma16816(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// The start of a CTA's run, for all its threads; false where it has none
template <int TK>
__device__ bool begin_run(const DecodeArgs& a, Cursor<TK>& cur, int64_t& n_tiles) {
  __shared__ int64_t run_n, run_first;
  __shared__ int run_b;
  if (threadIdx.x < 32) {
    Deal<TK> d;
    d.count(a, threadIdx.x);
    int b = 0;
    int64_t first = 0, n = 0;
    if ((int)blockIdx.x < d.workers) {
      const int64_t s = d.start(blockIdx.x);
      n = d.start(blockIdx.x + 1) - s;
      d.find(a, s, threadIdx.x, b, first);
      first = s - first;  // of its sequence's tiles
    }
    if (threadIdx.x == 0) {
      run_n = n;
      run_b = b;
      run_first = first;
    }
  }
  __syncthreads();
  n_tiles = run_n;
  if (n_tiles == 0) return false;
  cur.b = run_b;
  cur.enter(a);
  cur.u = (int)(run_first / cur.tiles);
  cur.tile = (int)(run_first - (int64_t)cur.u * cur.tiles);
  return true;
}

// A tile's rows: their places in the pools (-1: none), by the threads below TK; the pages' numbers are requested a
// tile ahead.
template <int TK>
struct RowPlan {
  int page, off;  // page number read from the table; row of the page
  __device__ __forceinline__ void request(const DecodeArgs& a, const Cursor<TK>& c, bool live) {
    page = -1;
    const int x = c.tile * TK + (int)threadIdx.x;
    if (live && x < c.s.n) {
      const int slot = slot_of(c.s, x), p = slot / a.c.page_size;
      off = slot - p * a.c.page_size;
      page = a.c.block_table_dev[(int64_t)c.b * a.c.max_pages + p];
      if ((uint32_t)page >= (uint32_t)a.c.n_pages) {
        set_dev_error(a.c.err_dev, RA_DEVERR_BOUNDS);
        page = -1;
      }
    }
  }
  __device__ __forceinline__ int64_t row(const DecodeArgs& a, int head) const {
    return page < 0 ? -1 : ((int64_t)page * a.c.n_kv_heads + head) * a.c.page_size + off;
  }
};

// ---------------------------------------------------------------------------------------
// bf16.  Tiles of 64 tokens; 4 WM warps: warp (w, g) takes 16 of the tokens for rows 16 g .. 16 g + 15, with
// its own m, l and outputs; the four warps of a row group are added up where the CTA leaves a unit.
// ---------------------------------------------------------------------------------------
constexpr int TKB = 64;
template <int DHT, int WM>
struct MmaPlan {
  static constexpr int THREADS = 128 * WM, STAGES = DHT == 64 ? 6 : 3, ROWS = 16 * WM;
  static constexpr int TILE = TKB * DHT * 2, STAGE = 2 * TILE;
  // two sets of outputs are added up in the stage of the tile just done, which nothing is copied into before the
  // next tile's barrier; four row groups have more than it holds and a space of their own
  static constexpr bool IN_STAGE = 2 * ROWS * DHT * 4 <= STAGE;
  static constexpr int STATS = STAGES * STAGE + (IN_STAGE ? 0 : 2 * ROWS * DHT * 4), ROWOFF = STATS + 4 * ROWS * 8,
                       MASK = ROWOFF + 2 * TKB * 8, BYTES = MASK + (STAGES + 1) * 8;
  // float `col` of a row of the sum: eight rows' pairs fall in distinct banks
  static __device__ __forceinline__ int at(int buf, int row, int col) { return (buf * ROWS + row) * DHT + (col ^ ((row & 7) << 3)); }
};

template <int DHT, int WM>
__global__ void __launch_bounds__(128 * WM) decode_mma_kernel(const __grid_constant__ DecodeArgs a) {
  using P = MmaPlan<DHT, WM>;
  constexpr int TK = TKB, S = P::STAGES, CH = DHT / 8;
  extern __shared__ __align__(128) uint8_t sm[];
  pdl_wait();
  pdl_trigger();
  Cursor<TK> cur;
  int64_t n_tiles;
  if (!begin_run<TK>(a, cur, n_tiles)) return;
  Cursor<TK> ahead = cur;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, wt = warp & 3, wg = warp >> 2;
  const int g = lane >> 2, t2 = (lane & 3) * 2, dh = a.c.head_dim;
  float2* stats = reinterpret_cast<float2*>(sm + P::STATS);  // [4][ROWS]
  int64_t* rowoff = reinterpret_cast<int64_t*>(sm + P::ROWOFF);
  // [STAGES + 1][2]: one more than there are stages, as a tile's is written before the barrier that its stage waits for
  uint32_t* mask = reinterpret_cast<uint32_t*>(sm + P::MASK);
  const uint32_t ring = smem_addr(sm);
  const bf16 *Kp = (const bf16*)a.c.k_dev, *Vp = (const bf16*)a.c.v_dev;
  const int col = tid % CH, r_first = tid / CH;  // this thread's 16-byte column of the rows it copies

  RowPlan<TK> plan;
  int64_t asked = 0;  // tiles whose pages were requested
  if (tid < TK) plan.request(a, ahead, true);
  asked = 1;
  // the requested tile's rows -> rowoff and mask; the next tile's pages are requested
  auto place = [&](int64_t tile, int head) {
    if (tid < TK) {
      const int64_t r = plan.row(a, head);
      rowoff[(tile & 1) * TK + tid] = r;
      const uint32_t m = __ballot_sync(0xffffffffu, r >= 0);
      if (lane == 0) mask[2 * (int)(tile % (S + 1)) + warp] = m;
    }
  };
  auto copy = [&](int64_t tile) {
    const uint32_t st = ring + (uint32_t)(tile % S) * P::STAGE;
    const bool in = col * 8 < dh;
#pragma unroll 4
    for (int r = r_first; r < TK; r += P::THREADS / CH) {
      const int64_t at = rowoff[(tile & 1) * TK + r];
      const bool live = in && at >= 0;
      const int64_t e = live ? at * dh + col * 8 : 0;
      const uint32_t d = st + r * (DHT * 2) + ((col ^ (r & 7)) << 4);
      cp16(d, Kp + e, live);
      cp16(d + P::TILE, Vp + e, live);
    }
  };
  auto step_ahead = [&]() {  // after place(): on to the next tile's pages
    ahead.next(a);
    if (tid < TK) plan.request(a, ahead, asked < n_tiles);
    ++asked;
  };
#pragma unroll 1
  for (int i = 0; i < S - 1; ++i) {
    if (i < n_tiles) {
      place(i, ahead.u / a.groups);
      __syncthreads();
      copy(i);
      if (asked < n_tiles) step_ahead();
    }
    cp_commit();
  }

  uint32_t qf[DHT / 16][4];
  float o[DHT / 8][4], m[2], l[2];
  int qslot[2];
  bool first_tile_of_unit = true, first_segment = true;
  int seg_start = cur.tile;
  for (int64_t i = 0; i < n_tiles; ++i) {
    if (first_tile_of_unit) {
      first_tile_of_unit = false;
      seg_start = cur.tile;
      const int hk = cur.u / a.groups, r0 = (cur.u - hk * a.groups) * P::ROWS + 16 * wg;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int r = r0 + g + 8 * h, t = r / a.G;
        const bool live = r < a.R;
        qslot[h] = live ? cur.s.len - a.n_new + t : -1;
        const bf16* q = (const bf16*)a.q + ((int64_t)cur.b * a.n_new + t) * a.q_stride + (hk * a.G + r - t * a.G) * dh;
#pragma unroll
        for (int ks = 0; ks < DHT / 16; ++ks)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int k = 16 * ks + 8 * e + t2;
            qf[ks][h + 2 * e] = live && k < dh ? *reinterpret_cast<const uint32_t*>(q + k) : 0u;
          }
        m[h] = -INFINITY;
        l[h] = 0.f;
      }
#pragma unroll
      for (int n = 0; n < DHT / 8; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[n][e] = 0.f;
    }
    cp_wait<S - 2>();
    const int64_t nt = i + S - 1;  // the tile whose copies start now
    if (nt < n_tiles) place(nt, ahead.u / a.groups);
    __syncthreads();  // tile i is there for all; all are done with tile i - 1; rowoff is written
    if (nt < n_tiles) {
      copy(nt);
      if (asked < n_tiles) step_ahead();
    }
    cp_commit();

    // ---- scores of this warp's 16 tokens
    const uint32_t st = ring + (uint32_t)(i % S) * P::STAGE;
    float s[2][4] = {};
    {
      const int row = 16 * wt + ((lane >> 4) << 3) + (lane & 7), half = (lane >> 3) & 1;
      const uint32_t base = st + row * (DHT * 2);
#pragma unroll
      for (int ks = 0; ks < DHT / 16; ++ks) {
        uint32_t kf[4];
        ldsm4(kf, base + (((2 * ks + half) ^ (row & 7)) << 4));
        mma16816(s[0], qf[ks], kf[0], kf[1]);
        mma16816(s[1], qf[ks], kf[2], kf[3]);
      }
    }
    const uint32_t live = mask[2 * (int)(i % (S + 1)) + (wt >> 1)] >> (16 * (wt & 1)) & 0xffffu;
    const int x0 = cur.tile * TK + 16 * wt;
    // every row sees all sixteen: no test a token
    const int j0 = slot_of(cur.s, x0), j1 = slot_of(cur.s, x0 + 15), qmin = cur.s.len - a.n_new;
    const bool all = live == 0xffffu && j1 <= qmin && (a.window == 0 || j1 < a.sinks || (x0 >= cur.s.n_sink && cur.s.len - 1 - j0 < a.window));
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[n][e] *= a.sl2;
        if (!all) {
          const int k = 8 * n + t2 + (e & 1);
          if (!((live >> k) & 1u) || !sees(a, qslot[e >> 1], slot_of(cur.s, x0 + k))) s[n][e] = -INFINITY;
        }
      }
    if (a.scores) {
      const int hk = cur.u / a.groups, r0 = (cur.u - hk * a.groups) * P::ROWS + 16 * wg;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int r = r0 + g + 8 * h;
        if (r < a.R) {
          float* d = a.scores + (((int64_t)cur.b * a.c.n_kv_heads + hk) * a.R + r) * a.x_stride + x0 + t2;
          *reinterpret_cast<float2*>(d) = make_float2(s[0][2 * h], s[0][2 * h + 1]);
          *reinterpret_cast<float2*>(d + 8) = make_float2(s[1][2 * h], s[1][2 * h + 1]);
        }
      }
    }
    // ---- running maximum and sum
    float ms[2];
    bool grew = false;
    float mn[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float bm = fmaxf(fmaxf(s[0][2 * h], s[0][2 * h + 1]), fmaxf(s[1][2 * h], s[1][2 * h + 1]));
      bm = fmaxf(bm, __shfl_xor_sync(0xffffffffu, bm, 1));
      bm = fmaxf(bm, __shfl_xor_sync(0xffffffffu, bm, 2));
      mn[h] = fmaxf(m[h], bm);
      grew = grew || mn[h] > m[h];
      ms[h] = mn[h] == -INFINITY ? 0.f : mn[h];
    }
    if (__any_sync(0xffffffffu, grew)) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float f = ex2_fast(m[h] - ms[h]);
        l[h] *= f;
        m[h] = mn[h];
#pragma unroll
        for (int n = 0; n < DHT / 8; ++n) {
          o[n][2 * h] *= f;
          o[n][2 * h + 1] *= f;
        }
      }
    }
    // P as an A operand (rows g, g + 8; tokens 2 t and 8 + 2 t), in two bf16 terms: rounded to one it would add as much to
    // the error as the output's own rounding does
    uint32_t pf[4], pl[4];
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float p0 = ex2_fast(s[n][2 * h] - ms[h]), p1 = ex2_fast(s[n][2 * h + 1] - ms[h]);
        l[h] += p0 + p1;
        pf[2 * n + h] = pack2(p0, p1);
        const float2 hi = __bfloat1622float2(*reinterpret_cast<__nv_bfloat162*>(&pf[2 * n + h]));
        pl[2 * n + h] = pack2(p0 - hi.x, p1 - hi.y);
      }
    // ---- outputs
    {
      const int row = 16 * wt + (((lane >> 3) & 1) << 3) + (lane & 7), half = lane >> 4;
      const uint32_t base = st + P::TILE + row * (DHT * 2);
#pragma unroll
      for (int nb = 0; nb < DHT / 16; ++nb) {
        uint32_t vf[4];
        ldsm4t(vf, base + (((2 * nb + half) ^ (row & 7)) << 4));
        mma16816(o[2 * nb], pf, vf[0], vf[1]);
        mma16816(o[2 * nb + 1], pf, vf[2], vf[3]);
        mma16816(o[2 * nb], pl, vf[0], vf[1]);
        mma16816(o[2 * nb + 1], pl, vf[2], vf[3]);
      }
    }

    const bool unit_ends = cur.tile + 1 == cur.tiles;
    if (unit_ends || i + 1 == n_tiles) {
      // ---- the four warps of a row group together, in the order ((0 + 2) + (1 + 3))
      float* merge = reinterpret_cast<float*>(sm + (P::IN_STAGE ? (int)(i % S) : S) * P::STAGE);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
        l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
        if ((lane & 3) == 0) stats[wt * P::ROWS + 16 * wg + g + 8 * h] = make_float2(m[h], l[h]);
      }
      __syncthreads();
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float M = -INFINITY;
#pragma unroll
        for (int w = 0; w < 4; ++w) M = fmaxf(M, stats[w * P::ROWS + 16 * wg + g + 8 * h].x);
        const float f = M == -INFINITY ? 0.f : ex2_fast(m[h] - M);
#pragma unroll
        for (int n = 0; n < DHT / 8; ++n) {
          o[n][2 * h] *= f;
          o[n][2 * h + 1] *= f;
        }
      }
      auto put = [&](int buf) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int n = 0; n < DHT / 8; ++n)
            *reinterpret_cast<float2*>(merge + P::at(buf, 16 * wg + g + 8 * h, 8 * n + t2)) =
                make_float2(o[n][2 * h], o[n][2 * h + 1]);
      };
      auto add = [&](int buf) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int n = 0; n < DHT / 8; ++n) {
            const float2 x = *reinterpret_cast<const float2*>(merge + P::at(buf, 16 * wg + g + 8 * h, 8 * n + t2));
            o[n][2 * h] += x.x;
            o[n][2 * h + 1] += x.y;
          }
      };
      if (wt >= 2) put(wt - 2);
      __syncthreads();
      if (wt < 2) add(wt);
      if (wt == 1) put(1);
      __syncthreads();
      if (wt == 0) {
        add(1);
        put(0);
      }
      __syncthreads();
      const int hk = cur.u / a.groups, r0 = (cur.u - hk * a.groups) * P::ROWS;
      const bool whole = seg_start == 0 && unit_ends;
      const int64_t slot = 2 * (int64_t)blockIdx.x + (first_segment ? 0 : 1);
      for (int e = tid; e < P::ROWS * (DHT / 4); e += P::THREADS) {
        const int r = e / (DHT / 4), d = (e - r * (DHT / 4)) * 4;
        if (r0 + r >= a.R || d >= dh) continue;
        float M = -INFINITY, L = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) M = fmaxf(M, stats[w * P::ROWS + r].x);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const float2 x = stats[w * P::ROWS + r];
          if (x.x != -INFINITY) L += x.y * ex2_fast(x.x - M);
        }
        float4 v = *reinterpret_cast<const float4*>(merge + P::at(0, r, d));
        if (whole) {
          const float f = M == -INFINITY ? 0.f : 1.f / L;
          const int t = (r0 + r) / a.G, head = hk * a.G + r0 + r - t * a.G;
          bf16* out = (bf16*)a.out + ((int64_t)cur.b * a.n_new + t) * a.out_stride + head * dh + d;
          *reinterpret_cast<uint2*>(out) = make_uint2(pack2(v.x * f, v.y * f), pack2(v.z * f, v.w * f));
          if (d == 0) {
            const float lse2 = M == -INFINITY ? -INFINITY : M + log2f(L);
            if (a.lse) a.lse[((int64_t)cur.b * a.n_new + t) * a.n_heads + head] = lse2 * kLn2;
            if (a.scores) a.lse2[((int64_t)cur.b * a.c.n_kv_heads + hk) * a.R + r0 + r] = lse2;
          }
        } else {
          *reinterpret_cast<float4*>(a.part_o + (slot * P::ROWS + r) * DHT + d) = v;
          if (d == 0) a.part_ml[slot * P::ROWS + r] = make_float2(M, L);
        }
      }
      __syncthreads();  // the merge space and the statistics are free again
      first_segment = false;
      first_tile_of_unit = true;
    }
    cur.next(a);
  }
  cp_wait<0>();
}

// ---------------------------------------------------------------------------------------
// f32.  Tiles of 32 tokens, 128 threads, RM rows.  Scores: warp w's lanes on the tokens, rows w, w + 4, ...; outputs:
// a thread a column (two at head dims above 128, half the rows each at 64).
// ---------------------------------------------------------------------------------------
constexpr int TKF = 32;
template <int DHT, int RM>
struct SimtPlan {
  static constexpr int STAGES = DHT == 64 ? 6 : 3, DP = DHT + 4;  // (padded rows: lanes on tokens without conflicts)
  static constexpr int TILE = TKF * DP * 4, STAGE = 2 * TILE, Q = STAGES * STAGE, X = Q + RM * DHT * 4,
                       XP = TKF + 4, FAC = X + RM * XP * 4, STATS = FAC + RM * 4, ROWOFF = STATS + RM * 8 + 8,
                       MASK = ROWOFF + 2 * TKF * 8, BYTES = MASK + (STAGES + 1) * 4;
  static constexpr int CT = DHT > 128 ? DHT / 128 : 1, RG = DHT < 128 ? 128 / DHT : 1, RT = RM / RG;
};

template <int DHT, int RM>
__global__ void __launch_bounds__(128) decode_simt_kernel(const __grid_constant__ DecodeArgs a) {
  using P = SimtPlan<DHT, RM>;
  constexpr int TK = TKF, S = P::STAGES, CH = DHT / 4, RW = RM / 4;
  extern __shared__ __align__(128) uint8_t sm[];
  pdl_wait();
  pdl_trigger();
  Cursor<TK> cur;
  int64_t n_tiles;
  if (!begin_run<TK>(a, cur, n_tiles)) return;
  Cursor<TK> ahead = cur;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, dh = a.c.head_dim;
  float *Q = reinterpret_cast<float*>(sm + P::Q), *X = reinterpret_cast<float*>(sm + P::X), *fac = reinterpret_cast<float*>(sm + P::FAC);
  float2* stats = reinterpret_cast<float2*>(sm + P::STATS);
  int64_t* rowoff = reinterpret_cast<int64_t*>(sm + P::ROWOFF);
  uint32_t* mask = reinterpret_cast<uint32_t*>(sm + P::MASK);
  const uint32_t ring = smem_addr(sm);
  const float *Kp = (const float*)a.c.k_dev, *Vp = (const float*)a.c.v_dev;

  RowPlan<TK> plan;
  int64_t asked = 1;
  if (tid < TK) plan.request(a, ahead, true);
  auto place = [&](int64_t tile, int head) {
    if (tid < TK) {
      const int64_t r = plan.row(a, head);
      rowoff[(tile & 1) * TK + tid] = r;
      const uint32_t m = __ballot_sync(0xffffffffu, r >= 0);
      if (lane == 0) mask[tile % (S + 1)] = m;
    }
  };
  auto copy = [&](int64_t tile) {
    const uint32_t st = ring + (uint32_t)(tile % S) * P::STAGE;
#pragma unroll 4
    for (int e = tid; e < TK * CH; e += 128) {
      const int r = e / CH, col = e - r * CH;
      const int64_t at = rowoff[(tile & 1) * TK + r];
      const bool live = at >= 0 && col * 4 < dh;
      const int64_t src = live ? at * dh + col * 4 : 0;
      const uint32_t d = st + (r * P::DP + col * 4) * 4;
      cp16(d, Kp + src, live);
      cp16(d + P::TILE, Vp + src, live);
    }
  };
  auto step_ahead = [&]() {
    ahead.next(a);
    if (tid < TK) plan.request(a, ahead, asked < n_tiles);
    ++asked;
  };
#pragma unroll 1
  for (int i = 0; i < S - 1; ++i) {
    if (i < n_tiles) {
      place(i, ahead.u / a.groups);
      __syncthreads();
      copy(i);
      if (asked < n_tiles) step_ahead();
    }
    cp_commit();
  }
  const int c0 = DHT < 128 ? tid % DHT : tid, rg = DHT < 128 ? tid / DHT : 0;  // output columns c0 (+ 128), rows rg RT ...
  float o[P::RT][P::CT], m[RW], l[RW];
  bool first_tile_of_unit = true, first_segment = true;
  int seg_start = cur.tile;
  for (int64_t i = 0; i < n_tiles; ++i) {
    const int hk = cur.u / a.groups, r0 = (cur.u - hk * a.groups) * RM;
    if (first_tile_of_unit) {
      first_tile_of_unit = false;
      seg_start = cur.tile;
      for (int e = tid; e < RM * DHT; e += 128) {
        const int r = e / DHT, d = e - r * DHT, t = (r0 + r) / a.G;
        Q[e] = r0 + r < a.R && d < dh
                   ? ((const float*)a.q)[((int64_t)cur.b * a.n_new + t) * a.q_stride + (hk * a.G + r0 + r - t * a.G) * dh + d] : 0.f;
      }
#pragma unroll
      for (int r = 0; r < P::RT; ++r)
#pragma unroll
        for (int c = 0; c < P::CT; ++c) o[r][c] = 0.f;
#pragma unroll
      for (int r = 0; r < RW; ++r) {
        m[r] = -INFINITY;
        l[r] = 0.f;
      }
    }
    cp_wait<S - 2>();
    const int64_t nt = i + S - 1;
    if (nt < n_tiles) place(nt, ahead.u / a.groups);
    __syncthreads();
    if (nt < n_tiles) {
      copy(nt);
      if (asked < n_tiles) step_ahead();
    }
    cp_commit();
    const float* K = reinterpret_cast<const float*>(sm + (i % S) * P::STAGE);
    const float* V = reinterpret_cast<const float*>(sm + (i % S) * P::STAGE + P::TILE);
    float s[RW] = {};
#pragma unroll 4
    for (int d = 0; d < DHT; d += 4) {
      const float4 k = *reinterpret_cast<const float4*>(K + lane * P::DP + d);
#pragma unroll
      for (int r = 0; r < RW; ++r) {
        const float4 q = *reinterpret_cast<const float4*>(Q + (warp + 4 * r) * DHT + d);
        s[r] = fmaf(q.x, k.x, s[r]);
        s[r] = fmaf(q.y, k.y, s[r]);
        s[r] = fmaf(q.z, k.z, s[r]);
        s[r] = fmaf(q.w, k.w, s[r]);
      }
    }
    const int x = cur.tile * TK + lane, slot = slot_of(cur.s, x);
    const bool live = mask[i % (S + 1)] >> lane & 1u;
#pragma unroll
    for (int r = 0; r < RW; ++r) {
      const int row = r0 + warp + 4 * r, qs = row < a.R ? cur.s.len - a.n_new + row / a.G : -1;
      s[r] = live && sees(a, qs, slot) ? s[r] * a.sl2 : -INFINITY;
      if (a.scores && row < a.R) a.scores[(((int64_t)cur.b * a.c.n_kv_heads + hk) * a.R + row) * a.x_stride + x] = s[r];
      const float mn = fmaxf(m[r], warp_max(s[r])), ms = mn == -INFINITY ? 0.f : mn;
      const float p = exp2f(s[r] - ms), f = exp2f(m[r] - ms);
      m[r] = mn;
      l[r] = l[r] * f + p;  // a lane's share
      X[(warp + 4 * r) * P::XP + lane] = p;
      if (lane == 0) fac[warp + 4 * r] = f;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < P::RT; ++r) {
      const float f = fac[rg * P::RT + r];
#pragma unroll
      for (int c = 0; c < P::CT; ++c) o[r][c] *= f;
    }
#pragma unroll 2
    for (int k = 0; k < TK; k += 4) {
      float v[4][P::CT];
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int c = 0; c < P::CT; ++c) v[u][c] = V[(k + u) * P::DP + c0 + 128 * c];
#pragma unroll
      for (int r = 0; r < P::RT; ++r) {
        const float4 p = *reinterpret_cast<const float4*>(X + (rg * P::RT + r) * P::XP + k);
#pragma unroll
        for (int c = 0; c < P::CT; ++c) {
          o[r][c] = fmaf(p.x, v[0][c], o[r][c]);
          o[r][c] = fmaf(p.y, v[1][c], o[r][c]);
          o[r][c] = fmaf(p.z, v[2][c], o[r][c]);
          o[r][c] = fmaf(p.w, v[3][c], o[r][c]);
        }
      }
    }
    const bool unit_ends = cur.tile + 1 == cur.tiles;
    if (unit_ends || i + 1 == n_tiles) {
#pragma unroll
      for (int r = 0; r < RW; ++r) {
        const float sum = warp_sum(l[r]);
        if (lane == 0) stats[warp + 4 * r] = make_float2(m[r], sum);
      }
      __syncthreads();
      const bool whole = seg_start == 0 && unit_ends;
      const int64_t slot_ = 2 * (int64_t)blockIdx.x + (first_segment ? 0 : 1);
#pragma unroll
      for (int r = 0; r < P::RT; ++r) {
        const int row = rg * P::RT + r;
        if (r0 + row >= a.R) continue;
        const float2 ml = stats[row];
        const int t = (r0 + row) / a.G, head = hk * a.G + r0 + row - t * a.G;
#pragma unroll
        for (int c = 0; c < P::CT; ++c) {
          const int d = c0 + 128 * c;
          if (d >= dh) continue;
          if (whole) {
            ((float*)a.out)[((int64_t)cur.b * a.n_new + t) * a.out_stride + head * dh + d] = ml.x == -INFINITY ? 0.f : o[r][c] / ml.y;
            if (d == 0) {
              const float lse2 = ml.x == -INFINITY ? -INFINITY : ml.x + log2f(ml.y);
              if (a.lse) a.lse[((int64_t)cur.b * a.n_new + t) * a.n_heads + head] = lse2 * kLn2;
              if (a.scores) a.lse2[((int64_t)cur.b * a.c.n_kv_heads + hk) * a.R + r0 + row] = lse2;
            }
          } else {
            a.part_o[(slot_ * RM + row) * DHT + d] = o[r][c];
            if (d == 0) a.part_ml[slot_ * RM + row] = ml;
          }
        }
      }
      __syncthreads();
      first_segment = false;
      first_tile_of_unit = true;
    }
    cur.next(a);
  }
  cp_wait<0>();
}

// ---------------------------------------------------------------------------------------
// Joins the parts of one query row: a CTA a row; its 256 threads take the parts in turns of 1024 / DHT, each four
// columns, and are added in a fixed order.  Rows of one part were written by the first kernel; sequences without a
// token get their zeros here.
// ---------------------------------------------------------------------------------------
template <typename T, int DHT, int TK, int ROWS>
__global__ void __launch_bounds__(256) decode_join_kernel(const __grid_constant__ DecodeArgs a) {
  constexpr int TPP = DHT / 4, TURNS = 256 / TPP;
  __shared__ float4 red[256];
  __shared__ float L_part[TURNS];
  __shared__ int64_t sh_first;
  __shared__ int sh_c0, sh_c1, sh_tiles;
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x;
  const int64_t id = blockIdx.x;
  const int per_b = a.c.n_kv_heads * a.R, b = (int)(id / per_b), hk = (int)(id - (int64_t)b * per_b) / a.R, row = (int)(id % a.R);
  const int grp = row / ROWS, lr = row - grp * ROWS;
  if (tid < 32) {
    Deal<TK> d;
    d.count(a, tid);
    const int tiles = d.tiles(a, b);
    if (tiles > 0) {
      const int64_t first = d.first_of(a, b, hk * a.groups + grp, tid);
      if (tid == 0) {
        sh_c0 = d.owner(first);
        sh_c1 = d.owner(first + tiles - 1);
        sh_first = first - d.start(sh_c0);
      }
    }
    if (tid == 0) sh_tiles = tiles;
  }
  __syncthreads();
  const int t = row / a.G, head = hk * a.G + row - t * a.G, dh = a.c.head_dim;
  T* out = (T*)a.out + ((int64_t)b * a.n_new + t) * a.out_stride + head * dh;
  if (sh_tiles == 0) {
    for (int d = tid; d < dh; d += 256) out[d] = from_f<T>(0.f);
    if (tid == 0) {
      if (a.lse) a.lse[((int64_t)b * a.n_new + t) * a.n_heads + head] = -INFINITY;
      if (a.scores) a.lse2[((int64_t)b * a.c.n_kv_heads + hk) * a.R + row] = -INFINITY;
    }
    return;
  }
  const int c0 = sh_c0, parts = sh_c1 - c0 + 1;
  if (parts == 1) return;
  // the first part is its CTA's last segment, unless the unit starts that CTA's run
  auto slot = [&](int p) { return 2 * (int64_t)(c0 + p) + (p == 0 && sh_first != 0 ? 1 : 0); };
  float M = -INFINITY;
  for (int p = tid & 31; p < parts; p += 32) M = fmaxf(M, a.part_ml[slot(p) * ROWS + lr].x);
  M = warp_max(M);
  const int turn = tid / TPP, d = (tid - turn * TPP) * 4;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  float L = 0.f;
  if (M != -INFINITY) {
#pragma unroll 4
    for (int p = turn; p < parts; p += TURNS) {
      const float2 ml = a.part_ml[slot(p) * ROWS + lr];
      const float4 x = d < dh ? *reinterpret_cast<const float4*>(a.part_o + (slot(p) * ROWS + lr) * DHT + d) : s;
      const float f = ml.x == -INFINITY ? 0.f : exp2f(ml.x - M);
      if (f > 0.f) {
        s.x = fmaf(x.x, f, s.x);
        s.y = fmaf(x.y, f, s.y);
        s.z = fmaf(x.z, f, s.z);
        s.w = fmaf(x.w, f, s.w);
        L = fmaf(ml.y, f, L);
      }
    }
  }
  red[tid] = s;
  if (d == 0) L_part[turn] = L;
  __syncthreads();
  if (tid >= TPP || d >= dh) return;
  L = 0.f;
#pragma unroll
  for (int i = 0; i < TURNS; ++i) L += L_part[i];
#pragma unroll
  for (int i = 1; i < TURNS; ++i) {
    const float4 x = red[i * TPP + tid];
    s.x += x.x;
    s.y += x.y;
    s.z += x.z;
    s.w += x.w;
  }
  const float f = M == -INFINITY ? 0.f : 1.f / L;
  out[d] = from_f<T>(s.x * f);
  out[d + 1] = from_f<T>(s.y * f);
  out[d + 2] = from_f<T>(s.z * f);
  out[d + 3] = from_f<T>(s.w * f);
  if (d == 0) {
    const float lse2 = M == -INFINITY ? -INFINITY : M + log2f(L);
    if (a.lse) a.lse[((int64_t)b * a.n_new + t) * a.n_heads + head] = lse2 * kLn2;
    if (a.scores) a.lse2[((int64_t)b * a.c.n_kv_heads + hk) * a.R + row] = lse2;
  }
}

// weights_out = weights_in + the rows' softmax weights, in row order: a thread a slot
__global__ void __launch_bounds__(256) decode_weights_kernel(const __grid_constant__ DecodeArgs a, int chunks) {
  pdl_wait();
  pdl_trigger();
  const int64_t unit = blockIdx.x / chunks;  // b * kv heads + head
  const int b = (int)(unit / a.c.n_kv_heads);
  const Seen s = seen_of(a, b);
  const float* lse2 = a.lse2 + unit * a.R;
  const float* sc = a.scores + unit * a.R * a.x_stride;
  const int j0 = (int)(blockIdx.x - unit * chunks) * 1024;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int j = j0 + 256 * i + (int)threadIdx.x;
    if (j >= s.len) return;
    float w = a.w_in ? a.w_in[unit * a.w_stride + j] : 0.f;
    const int x = j < s.n_sink ? j : j >= s.w0 ? j - s.w0 + s.n_sink : -1;
    if (x >= 0)
      for (int r = 0; r < a.R; ++r) {
        const float z = lse2[r];
        if (z != -INFINITY) w += exp2f(sc[(int64_t)r * a.x_stride + x] - z);
      }
    a.w_out[unit * a.w_stride + j] = w;
  }
}

// ---- host ------------------------------------------------------------------------------
struct DecodeLayout {
  int rows, groups, dht, tk, grid, R;
  int64_t x_stride;
  size_t ml, o, lse2, scores, bytes;
};
DecodeLayout layout_of(const ra_attention_decode_args& p) {
  DecodeLayout L;
  const int G = p.n_heads / p.cache.n_kv_heads;
  const bool b16 = p.cache.dtype == RA_BF16;
  L.R = G * p.n_new;
  L.dht = p.cache.head_dim <= 64 ? 64 : p.cache.head_dim <= 128 ? 128 : 256;
  // rows that one pass over K and V serves: 16, 32 or 64 (bf16; 16 at head dims above 128, whose outputs fill the
  // registers), 4 or 16 (f32)
  L.rows = b16 ? (L.R <= 16 || L.dht == 256 ? 16 : L.R <= 32 ? 32 : 64) : (L.R <= 4 ? 4 : 16);
  L.groups = (L.R + L.rows - 1) / L.rows;
  L.tk = b16 ? TKB : TKF;
  // CTAs that the SMs hold at once: by shared memory two of a plan up to 112 KB, one of a larger
  L.grid = (L.dht == 256 || (b16 && L.rows == 64) ? 1 : 2) * device_sm_count();
  L.x_stride = ((int64_t)call_max_len(p.cache, p.max_len) + 63) / 64 * 64;
  size_t at = 0;
  auto take = [&](size_t n) {
    const size_t o = at;
    at += (n + 255) / 256 * 256;
    return o;
  };
  L.ml = take((size_t)2 * L.grid * L.rows * 8);
  L.o = take((size_t)2 * L.grid * L.rows * L.dht * 4);
  L.lse2 = L.scores = 0;
  if (p.weights_out_dev) {
    const size_t rows = (size_t)p.batch * p.cache.n_kv_heads * L.R;
    L.lse2 = take(rows * 4);
    L.scores = take(rows * L.x_stride * 4);
  }
  L.bytes = at;
  return L;
}

template <typename K>
cudaError_t start(K* kernel, int smem, int threads, const DecodeArgs& a, cudaStream_t st) {
  cudaError_t e = allow_smem(kernel, smem);
  return e == cudaSuccess ? launch_pdl(kernel, dim3(a.grid), dim3(threads), (size_t)smem, st, a) : e;
}
template <int DHT>
cudaError_t run_mma(const DecodeArgs& a, int rows, cudaStream_t st) {
  const dim3 joins((unsigned)((int64_t)a.batch * a.c.n_kv_heads * a.R));
  cudaError_t e;
  if constexpr (DHT < 256) {
    if (rows == 32) {
      e = start(decode_mma_kernel<DHT, 2>, MmaPlan<DHT, 2>::BYTES, 256, a, st);
      return e == cudaSuccess ? launch_pdl(decode_join_kernel<bf16, DHT, TKB, 32>, joins, dim3(256), 0, st, a) : e;
    }
    if (rows == 64) {
      e = start(decode_mma_kernel<DHT, 4>, MmaPlan<DHT, 4>::BYTES, 512, a, st);
      return e == cudaSuccess ? launch_pdl(decode_join_kernel<bf16, DHT, TKB, 64>, joins, dim3(256), 0, st, a) : e;
    }
  }
  e = start(decode_mma_kernel<DHT, 1>, MmaPlan<DHT, 1>::BYTES, 128, a, st);
  return e == cudaSuccess ? launch_pdl(decode_join_kernel<bf16, DHT, TKB, 16>, joins, dim3(256), 0, st, a) : e;
}
template <int DHT>
cudaError_t run_simt(const DecodeArgs& a, int rows, cudaStream_t st) {
  const dim3 joins((unsigned)((int64_t)a.batch * a.c.n_kv_heads * a.R));
  cudaError_t e;
  if (rows == 4) {
    e = start(decode_simt_kernel<DHT, 4>, SimtPlan<DHT, 4>::BYTES, 128, a, st);
    return e == cudaSuccess ? launch_pdl(decode_join_kernel<float, DHT, TKF, 4>, joins, dim3(256), 0, st, a) : e;
  }
  e = start(decode_simt_kernel<DHT, 16>, SimtPlan<DHT, 16>::BYTES, 128, a, st);
  return e == cudaSuccess ? launch_pdl(decode_join_kernel<float, DHT, TKF, 16>, joins, dim3(256), 0, st, a) : e;
}

}  // namespace

size_t attention_decode_workspace(const ra_attention_decode_args& p) { return layout_of(p).bytes; }

cudaError_t attention_decode(const ra_attention_decode_args& p, cudaStream_t st) {
  const DecodeLayout L = layout_of(p);
  char* ws = (char*)p.workspace_dev;
  DecodeArgs a;
  a.c = p.cache;
  a.lens = p.lens_dev;
  a.q = p.q_dev;
  a.q_stride = p.q_stride;
  a.out = p.out_dev;
  a.out_stride = p.out_stride;
  a.lse = p.lse_dev;
  a.w_in = p.weights_in_dev;
  a.w_out = p.weights_out_dev;
  a.w_stride = p.weights_stride;
  a.part_ml = (float2*)(ws + L.ml);
  a.part_o = (float*)(ws + L.o);
  a.lse2 = p.weights_out_dev ? (float*)(ws + L.lse2) : nullptr;
  a.scores = p.weights_out_dev ? (float*)(ws + L.scores) : nullptr;
  a.x_stride = L.x_stride;
  a.batch = p.batch;
  a.n_new = p.n_new;
  a.n_heads = p.n_heads;
  a.G = p.n_heads / p.cache.n_kv_heads;
  a.R = L.R;
  a.groups = L.groups;
  a.max_len = call_max_len(p.cache, p.max_len);
  a.window = p.window;
  a.sinks = p.sinks;
  a.grid = L.grid;
  a.sl2 = p.scale * kLog2e;
  cudaError_t e;
  if (p.cache.dtype == RA_BF16)
    e = L.dht == 64 ? run_mma<64>(a, L.rows, st) : L.dht == 128 ? run_mma<128>(a, L.rows, st) : run_mma<256>(a, L.rows, st);
  else
    e = L.dht == 64 ? run_simt<64>(a, L.rows, st) : L.dht == 128 ? run_simt<128>(a, L.rows, st) : run_simt<256>(a, L.rows, st);
  note_launch(2);
  if (e != cudaSuccess || !a.scores) return e;
  const int chunks = (a.max_len + 1023) / 1024;
  const int64_t n = (int64_t)chunks * a.batch * a.c.n_kv_heads;
  if (n > INT32_MAX) return cudaErrorNotSupported;
  e = launch_pdl(decode_weights_kernel, dim3((unsigned)n), dim3(256), 0, st, a, chunks);
  note_launch(1);
  return e;
}

}  // namespace ra
