// k_attention_decode.cu -- attention of a sequence's newest tokens over its paged key-value cache.
//
//   o = sum_j p_j v_j, p = softmax(scale q K^T) over the slots that the token sees.
//
// The query rows of a key-value head are its group's heads times the new tokens (R rows, a few to a few dozen); K and
// V are read once for up to 64 of them (bf16; 16 at head dims above 128) or 16 (f32), and again for the next as many, 4 R
// head_dim flops for every 2 head_dim values: bound by memory where the rows are few.  The slots that
// any row sees (all, or the sinks and the windows) are numbered 0, 1, ... and cut into tiles of TK; the tiles of all
// sequences and heads, one after the other, are dealt to the CTAs in equal runs, whatever the lengths are.  Two warps of a
// CTA look up pages and copy tiles, in turn, into a ring; the others (or groups of 2 or 4 that split more than sixteen rows) take
// the tiles in turn, each with its own running maximum m, sum l and outputs; nothing but the end of a (sequence, head)
// makes them wait for one another.  There the CTA adds them up; where its run covers a part of the head's tiles only,
// (m, l, o) go to the workspace, and the last CTA to leave its part (a counter; the order of the sum is the parts', not
// theirs) joins them.  The counter is that of the CTA with the head's first tile: a head that is cut ends the run it starts
// in, so that a CTA starts one at most, and the counters, all that has to be zero between calls, have their place whatever
// the call's shape is.
//   bf16: the products are mma.sync m16n8k16: sixteen rows take the tensor instruction of one, and the rate asked of
//         it, 16 flops a byte of K and V, is a tenth of what it gives, so nothing is won by tcgen05's 128 rows.
//   f32:  FFMA on packed pairs of rows, for the rows that there are (4, 8 or 16).  Shared memory paces it: 128 bytes a cycle
//         reach the registers, whether lanes read different values or the same one.  So a lane takes four tokens by an eighth
//         of the dims for q K^T (a key is read once, a query once for four tokens), and 16 lanes all dims of every other token
//         for p V.  (With a lane a token, queries read by every lane: 2.4 times the reads, 224 us where this takes 175 for
//         10 rows of 453 MB; tf32 products of operands split in two terms, sixteen rows always: 217 us for 671 MB.)
// 16 bf16 sequences of up to 32768 tokens, 16 heads of 128 over 4: 107 us, 6.3 TB/s of the 6.8 that a copy has (125 us with
// the weights for an eviction, which read the scores again); fp32, 16 sequences of 16384 tokens, 4 heads of 128: 161 us with up to
// four rows a head, 6.7 TB/s, 197 with eight, 5.5 TB/s.  One sequence of 1000 tokens: 10 us, the
// latency of a launch, a page, a tile, the joining of parts.
#include <cstring>

#include "common.cuh"
#include "operators.h"
#include "paged.cuh"
#include "window_tc.cuh"

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
  unsigned* done;                // [grid]: CTAs that have left their part of the unit that starts in CTA i; zero between calls
  float* part_o;                 // [2 grid][rows of a unit][head dim]
  float2* part_ml;               // [2 grid][rows of a unit]
  float* lse2;                   // [batch, kv heads, R] (powers of two), where weights are wanted
  float* scores;                 // [batch, kv heads, R, x_stride], scaled, in powers of two
  int64_t x_stride;
  int batch, n_new, n_heads, G, R, groups, max_len, window, sinks, grid;
  int page_shift;                // pages of 2^page_shift tokens, or -1
  int brs, whole_rows;           // the tensor maps' boxes: 2^brs rows; whole rows of the head, or 128 bytes of them
  int join;                      // the last CTA of a unit joins its parts (else a kernel of its own)
  float sl2;                     // scale log2 e
};

// What a call's new tokens see of a sequence: slots [0, n_sink) and [w0, len), in tiles of TK slots: sink_tiles from the
// first, the others from tile w_tile on
struct Seen {
  int len, w0, n_sink, sink_tiles, w_tile, tiles;
};
template <int TK>
__device__ __forceinline__ Seen seen_of(const DecodeArgs& a, int b) {
  Seen s;
  s.len = clamp_len(__ldg(a.lens + b), a.max_len, a.c.err_dev);
  s.w0 = 0;
  if (a.window > 0) {
    const int64_t w0 = (int64_t)s.len - a.n_new - a.window + 1;  // the first new token's window
    s.w0 = w0 > 0 ? (int)w0 : 0;
  }
  s.n_sink = a.sinks < s.w0 ? a.sinks : s.w0;
  s.w_tile = s.w0 / TK;
  s.sink_tiles = (s.n_sink + TK - 1) / TK;
  if (s.sink_tiles > s.w_tile) s.sink_tiles = s.w_tile;
  s.tiles = s.len > 0 ? s.sink_tiles + (s.len + TK - 1) / TK - s.w_tile : 0;
  return s;
}
template <int TK>
__device__ __forceinline__ int first_slot(const Seen& s, int tile) {
  return (tile < s.sink_tiles ? tile : tile - s.sink_tiles + s.w_tile) * TK;
}
// whether the query at slot i sees slot j <= its sequence's last
__device__ __forceinline__ bool sees(const DecodeArgs& a, int i, int j) {
  return j <= i && (a.window == 0 || i - j < a.window || j < a.sinks);
}
// How the tiles are dealt: unit (b, u), u = kv head * groups + row group, has tiles(b) tiles; units in order.
// One warp computes; `total` tiles go to as many CTAs as have LEAST tiles each, or one a unit, at most the grid: the
// first `extra` of them take base + 1 tiles, the others base.  (The host has checked that 32 bits hold the total.)
__device__ __forceinline__ int warp_sum_int(int v) { return (int)__reduce_add_sync(0xffffffffu, (unsigned)v); }
template <int TK, int LEAST>
struct Deal {
  int total, workers, base, extra;
  __device__ __forceinline__ int tiles(const DecodeArgs& a, int b) const { return seen_of<TK>(a, b).tiles; }
  __device__ void count(const DecodeArgs& a, int lane) {
    const int units = a.c.n_kv_heads * a.groups;
    int t = 0, live = 0;
    for (int b = lane; b < a.batch; b += 32) {
      const int n = tiles(a, b);
      t += n * units;
      live += n > 0 ? units : 0;
    }
    total = warp_sum_int(t);
    live = warp_sum_int(live);
    int w = (total + LEAST - 1) / LEAST;
    if (w < live) w = live;  // (short sequences: a CTA a unit)
    workers = w < a.grid ? w : a.grid;
    base = workers ? (int)((unsigned)total / (unsigned)workers) : 0;
    extra = total - base * workers;
  }
  __device__ __forceinline__ int start(int cta) const { return cta * base + (cta < extra ? cta : extra); }
  __device__ __forceinline__ int owner(int tile) const {
    const int more = extra * (base + 1);
    return tile < more ? (int)((unsigned)tile / (unsigned)(base + 1)) : extra + (int)((unsigned)(tile - more) / (unsigned)base);
  }
  // the sequence that tile `at` belongs to, and its first tile (same in all lanes)
  __device__ void find(const DecodeArgs& a, int at, int lane, int& b, int& first) const {
    const int units = a.c.n_kv_heads * a.groups;
    int acc = 0;
    for (int base_b = 0;; base_b += 32) {
      const int t = base_b + lane < a.batch ? tiles(a, base_b + lane) * units : 0;
      int incl = t;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += v;
      }
      const uint32_t past = __ballot_sync(0xffffffffu, acc + incl > at);
      if (past) {
        const int l = __ffs(past) - 1;
        b = base_b + l;
        first = acc + __shfl_sync(0xffffffffu, incl - t, l);
        return;
      }
      acc += __shfl_sync(0xffffffffu, incl, 31);
    }
  }
  // the first tile of sequence b's unit u
  __device__ int first_of(const DecodeArgs& a, int b, int u, int lane) const {
    const int units = a.c.n_kv_heads * a.groups;
    int t = 0;
    for (int i = lane; i < b; i += 32) t += tiles(a, i) * units;
    return warp_sum_int(t) + u * tiles(a, b);
  }
};

// Where in its run a CTA is: a tile of a unit
template <int TK>
struct Cursor {
  int b, u, tile, tiles;
  Seen s;
  __device__ __forceinline__ void enter(const DecodeArgs& a) {
    s = seen_of<TK>(a, b);
    tiles = s.tiles;
  }
  // on to the next unit's tile 0 (past the last sequence: b == batch)
  __device__ __forceinline__ void next_unit(const DecodeArgs& a) {
    if (++u < a.c.n_kv_heads * a.groups) return;
    u = 0;
    do {
      if (++b >= a.batch) {
        tiles = 1 << 30;
        return;
      }
      enter(a);
    } while (tiles == 0);
  }
  __device__ __forceinline__ void skip(const DecodeArgs& a, int n) {
    tile += n;
    while (tile >= tiles) {
      tile -= tiles;
      next_unit(a);
    }
  }
};

__device__ __forceinline__ void cp16(uint32_t dst, const void* src, bool live) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(live ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp4(uint32_t dst, const void* src, bool live) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(live ? 4 : 0) : "memory");
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
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t* r, uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma16816(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// ---------------------------------------------------------------------------------------
// WM warps a group, each on RM of the unit's rows (bf16: sixteen).  NG groups and two copying warps a CTA, one CTA an SM.  A
// stage holds K and V of TK tokens, rows of DHT values (zeros past head_dim) whose 16-byte chunks are permuted so that the
// reads below meet no bank twice.
//   TMA   pages of a multiple of 8 tokens: boxes of BR slots of a page, BR the largest of 32, 16 and 8 that divides a page and
//         a tile: 8 instructions a tile of 32 tokens in pages of 16;
//   else  cp.async, 16 bytes a lane.
// ---------------------------------------------------------------------------------------
template <typename T, int DHT, int WM, int RM>
struct Plan {
  static constexpr bool B16 = sizeof(T) == 2;
  static constexpr int TK = (DHT == 256 ? 16 : WM == 4 || DHT == 64 ? 64 : 32) / (B16 ? 1 : 2);
  // bf16: six warps and the two that copy may have 255 registers each (four row groups: eight and two, 168); f32: eight
  // (eight rows) with 168, twelve (four rows) with 128
  static constexpr int F32_WARPS = RM == 8 ? 8 : DHT == 256 ? 10 : 12, NG = B16 ? (WM == 4 ? 2 : 6 / WM) : F32_WARPS / WM, WORKERS = 32 * WM * NG, THREADS = WORKERS + 64, ROWS = RM * WM;
  static constexpr int TILE = TK * DHT * (int)sizeof(T), STAGE = 2 * TILE, STAGES = B16 ? 192 * 1024 / STAGE : F32_WARPS;
  static constexpr int Q = STAGES * STAGE, QB = ROWS * DHT * (int)sizeof(T), STATS = Q + 2 * QB, MASK = STATS + NG * ROWS * 8;
  static_assert(ROWS * DHT * 4 <= STAGE, "a group's outputs are put into the stage of its last tile");
  // float `col` of row `row` of a group's outputs in its stage: eight rows' pairs fall in distinct banks
  static __device__ __forceinline__ int sum_at(int row, int col) { return row * DHT + (col ^ ((row & 7) << 3)); }
  // K or V of a stage: boxes of 2^brs rows, of each box the atoms of 128 bytes of every row, whose chunks the 128-byte
  // swizzle of TMA permutes.  A row's place, an atom's distance, and a 16-byte chunk's place in a row of its atom:
  static __device__ __forceinline__ int row_at(int r, int brs) { return ((r >> brs) * ATOMS << (brs + 7)) + ((r & ((1 << brs) - 1)) << 7); }
  static __device__ __forceinline__ int chunk_at(int r, int c) { return ((c & 7) ^ (r & 7)) << 4; }
  static __device__ __forceinline__ int at(int r, int c, int brs) { return row_at(r, brs) + ((c >> 3) << (brs + 7)) + chunk_at(r, c); }
  static constexpr int ATOMS = DHT * (int)sizeof(T) / 128, MBAR = MASK + STAGES * 8, PLACES = MBAR + 2 * STAGES * 8,
                       X = (PLACES + 2 * 32 * 8 + 15) / 16 * 16, BYTES = X + (B16 ? 0 : NG * TK * ROWS * 4);
  // a stage is filled by the same warp and read by the same group every time round, so that each has seen every phase of
  // its barriers: a wait by parity for a phase that is two ahead would return at once
  static_assert(STAGES % 2 == 0 && STAGES % NG == 0, "stages belong to copying warps and to groups");
  static_assert(STATS % 16 == 0 && MBAR % 8 == 0 && X % 16 == 0 && BYTES <= 226 * 1024, "shared memory");
};

template <typename T>
__device__ __forceinline__ void store4(T* dst, float4 v);
template <>
__device__ __forceinline__ void store4<bf16>(bf16* dst, float4 v) {
  *reinterpret_cast<uint2*>(dst) = make_uint2(pack2(v.x, v.y), pack2(v.z, v.w));
}
template <>
__device__ __forceinline__ void store4<float>(float* dst, float4 v) {
  *reinterpret_cast<float4*>(dst) = v;
}
// f a + s
__device__ __forceinline__ float4 fma4(float4 a, float f, float4 s) {
  return make_float4(fmaf(a.x, f, s.x), fmaf(a.y, f, s.y), fmaf(a.z, f, s.z), fmaf(a.w, f, s.w));
}
// the factor of a part with statistics (m, l) under the common maximum M; what has seen nothing takes no part
__device__ __forceinline__ bool counts(float2 ml) { return !(ml.x == -INFINITY && ml.y == 0.f); }
// a finished row: output (four columns from d) and, with column 0, its log-sum-exp
template <typename T>
__device__ __forceinline__ void finish(const DecodeArgs& a, int b, int hk, int row, int d, float4 o, float M, float L, bool any) {
  const int t = row / a.G, head = hk * a.G + row - t * a.G;
  const float f = any ? 1.f / L : 0.f;
  store4<T>((T*)a.out + ((int64_t)b * a.n_new + t) * a.out_stride + head * a.c.head_dim + d, make_float4(o.x * f, o.y * f, o.z * f, o.w * f));
  if (d == 0) {
    const float lse2 = any ? M + log2f(L) : -INFINITY;
    if (a.lse) a.lse[((int64_t)b * a.n_new + t) * a.n_heads + head] = lse2 * kLn2;
    if (a.scores) a.lse2[((int64_t)b * a.c.n_kv_heads + hk) * a.R + row] = lse2;
  }
}

// shares of a call with few tiles: a CTA has at least this many (fewer CTAs would leave SMs without copies, more make joins)
constexpr int SHARE = 4;

template <typename T, int DHT, int WM, int RM, bool TMA>
__global__ void __launch_bounds__(Plan<T, DHT, WM, RM>::THREADS, 1) decode_kernel(const __grid_constant__ CUtensorMap tmK,
    const __grid_constant__ CUtensorMap tmV, const __grid_constant__ DecodeArgs a) {
  using P = Plan<T, DHT, WM, RM>;
  constexpr bool B16 = P::B16;
  constexpr int TK = P::TK, S = P::STAGES, NG = P::NG, ROWS = P::ROWS, VE = 16 / (int)sizeof(T), CH = DHT / VE, NT = TK / 8;
  constexpr uint64_t FULL = TK == 64 ? ~0ull : (1ull << (TK & 63)) - 1;
  extern __shared__ __align__(1024) uint8_t sm[];
  __shared__ Deal<TK, SHARE> deal;
  __shared__ int run_start, run_in, run_n, run_b, joins;
  __shared__ int last_stage[NG];
  __shared__ volatile int abort_sh;
  uint64_t* full = reinterpret_cast<uint64_t*>(sm + P::MBAR);  // [S]: a stage's copies have landed
  uint64_t* empty = full + S;                                  // [S]: its group has read it
  uint64_t* mask = reinterpret_cast<uint64_t*>(sm + P::MASK);  // [S]: tokens of the tile that are there and seen by a row
  if (smem_addr(sm) & 1023u) {  // the swizzle goes by the address
    if (threadIdx.x == 0) set_dev_error(a.c.err_dev, RA_DEVERR_BOUNDS);
    return;
  }
  const int tid = threadIdx.x, warp = tc::warp_index(), lane = tid & 31, grp = warp / WM, wm = warp - grp * WM;
  if (tid < S) {
    tc::mbar_init(&full[tid], TMA ? 1 : 33);
    tc::mbar_init(&empty[tid], WM);
  }
  if (tid == 0) {
    abort_sh = 0;
    if (TMA) {
      asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmK)) : "memory");
      asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmV)) : "memory");
    }
  }
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  pdl_wait();
  pdl_trigger();
  if (warp == 0) {
    Deal<TK, SHARE> d;
    d.count(a, lane);
    int b = 0, first = 0, n = 0, s = 0;
    if ((int)blockIdx.x < d.workers) {
      s = d.start(blockIdx.x);
      n = d.start(blockIdx.x + 1) - s;
      d.find(a, s, lane, b, first);
    }
    if (lane == 0) {
      run_n = n;
      run_b = b;
      run_in = s - first;  // of its sequence's tiles
      run_start = s;
      deal = d;
    }
  }
  __syncthreads();
  // sequences without a token: zeros (dealt in turn to all CTAs)
  for (int b = blockIdx.x; b < a.batch; b += gridDim.x)
    if (seen_of<TK>(a, b).tiles == 0)
      for (int e = tid; e < a.c.n_kv_heads * a.R * (a.c.head_dim / 4); e += P::THREADS) {
        const int row = e / (a.c.head_dim / 4), d = (e - row * (a.c.head_dim / 4)) * 4;
        finish<T>(a, b, row / a.R, row % a.R, d, make_float4(0.f, 0.f, 0.f, 0.f), 0.f, 0.f, false);
      }
  const int n_tiles = run_n;
  if (n_tiles == 0) return;
  const int g = lane >> 2, t4 = lane & 3, dh = a.c.head_dim;
  Cursor<TK> cur;
  cur.b = run_b;
  cur.enter(a);
  cur.u = run_in / cur.tiles;
  cur.tile = run_in - cur.u * cur.tiles;

  if (warp >= P::WORKERS / 32) {
    // ------------------------------------------------------------ copies: the two warps take the tiles in turn
    const int odd = warp - P::WORKERS / 32;
    const T *Kp = (const T*)a.c.k_dev, *Vp = (const T*)a.c.v_dev;
    int2* boxes_at = reinterpret_cast<int2*>(sm + P::PLACES) + 32 * odd;  // of the batch: page and kv head, row of the page
    const int box = TMA ? 1 << a.brs : 1, nb = TK / box;  // slots a box, boxes a tile
    constexpr int HALVES = TMA ? 1 : (TK + 31) / 32;      // boxes a lane looks up
    const int batch = TMA ? 32 / nb : 1;                  // tiles looked up at once, of one unit
    int64_t place[HALVES], next_place[HALVES];            // TMA: page and kv head; else the row of the pools; -1: not there
    int off = 0, next_off = 0;                            // TMA: row of the page
    auto look_up = [&](const Cursor<TK>& c, int tiles, int64_t (&pl)[HALVES], int& po) {
#pragma unroll
      for (int h = 0; h < HALVES; ++h) {
        const int i = 32 * h + lane, t = i / nb, slot = first_slot<TK>(c.s, c.tile + t) + (i - t * nb) * box;
        pl[h] = -1;
        if (t < tiles && slot < c.s.len && (TMA || slot < c.s.n_sink || slot >= c.s.w0)) {
          const int p = a.page_shift >= 0 ? slot >> a.page_shift : slot / a.c.page_size;
          const int page = a.c.block_table_dev[(int64_t)c.b * a.c.max_pages + p];
          if ((uint32_t)page < (uint32_t)a.c.n_pages) {
            const int64_t ph = (int64_t)page * a.c.n_kv_heads + c.u / a.groups;
            po = slot - p * a.c.page_size;
            pl[h] = TMA ? ph : ph * a.c.page_size + po;
          } else {
            set_dev_error(a.c.err_dev, RA_DEVERR_BOUNDS);
          }
        }
      }
    };
    auto batch_of = [&](const Cursor<TK>& c, int left) {
      const int n = c.tiles - c.tile < left ? c.tiles - c.tile : left;
      return n < batch ? n : batch;
    };
    const uint32_t all_boxes = TMA ? (uint32_t)((1ull << (nb & 63)) - 1) : 0;
    int done = 0, st = -1, round = 0, tile = -1, many = batch_of(cur, n_tiles);
    bool ok = true;
    look_up(cur, many, next_place, next_off);
    while (done < n_tiles && ok) {
      // this batch's places; the next one's are requested
      const Cursor<TK> at = cur;
      const int now = many;
#pragma unroll
      for (int h = 0; h < HALVES; ++h) place[h] = next_place[h];
      off = next_off;
      const uint32_t there = TMA ? __ballot_sync(0xffffffffu, place[0] >= 0) : 0;
      if (TMA) {
        __syncwarp();
        boxes_at[lane] = make_int2((int)place[0], off);
        __syncwarp();
      }
      done += now;
      if (done < n_tiles) {
        cur.skip(a, now);
        many = batch_of(cur, n_tiles - done);
        look_up(cur, many, next_place, next_off);
      }
      for (int t = 0; t < now; ++t) {
        ++tile;
        if (++st == S) {
          st = 0;
          ++round;
        }
        if ((tile & 1) != odd) continue;
        const int slot0 = first_slot<TK>(at.s, at.tile + t);
        const uint32_t boxes = TMA ? (there >> (t * nb)) & all_boxes : 0;
        uint64_t live = FULL;
        if (!TMA || boxes != all_boxes || slot0 + TK > at.s.len || (slot0 < at.s.w0 && slot0 + TK > at.s.n_sink)) {
          live = 0;
#pragma unroll
          for (int h = 0; h < (TK + 31) / 32; ++h) {
            const int i = 32 * h + lane, slot = slot0 + i;
            const bool on = TMA ? i < TK && slot < at.s.len && (slot < at.s.n_sink || slot >= at.s.w0) && ((boxes >> (i / box)) & 1u)
                                : place[TMA ? 0 : h] >= 0;
            live |= (uint64_t)__ballot_sync(0xffffffffu, on) << (32 * h);
          }
        }
        if (round > 0) ok = __all_sync(0xffffffffu, tc::mbar_wait(&empty[st], (round - 1) & 1, &abort_sh, a.c.err_dev)) != 0;
        if (!ok) break;
        const uint32_t dst = smem_addr(sm + st * P::STAGE);
        if constexpr (TMA) {
          if (tc::elect_one()) {
            mask[st] = live;
            tc::mbar_expect_tx(&full[st], (uint32_t)__popc(boxes) * (uint32_t)box * (2 * 128 * P::ATOMS));
#pragma unroll
            for (int i = 0; i < TK / 8; ++i)
              if ((boxes >> i) & 1u) {
                const int2 at_ = boxes_at[t * nb + i];
                const uint32_t d = dst + i * box * (128 * P::ATOMS);
                if (a.whole_rows) {
                  tc::tma_load4(&tmK, d, &full[st], 0, at_.y, 0, at_.x);
                  tc::tma_load4(&tmV, d + P::TILE, &full[st], 0, at_.y, 0, at_.x);
                } else {
#pragma unroll
                  for (int n = 0; n < P::ATOMS; ++n) {
                    tc::tma_load3(&tmK, d + n * box * 128, &full[st], n * (128 / (int)sizeof(T)), at_.y, at_.x);
                    tc::tma_load3(&tmV, d + P::TILE + n * box * 128, &full[st], n * (128 / (int)sizeof(T)), at_.y, at_.x);
                  }
                }
              }
          }
          __syncwarp();
        } else {
          if (lane == 0) mask[st] = live;
          constexpr int PER = CH < 32 ? 32 / CH : 1;  // rows copied at once
          const int rsub = CH < 32 ? lane / CH : 0;
#pragma unroll 4
          for (int r0 = 0; r0 < TK; r0 += PER) {
            const int r = r0 + rsub;
            const int64_t row = __shfl_sync(0xffffffffu, (TK > 32 && r0 >= 32) ? place[HALVES - 1] : place[0], r & 31);
#pragma unroll
            for (int c = CH < 32 ? lane % CH : lane; c < CH; c += 32) {
              const bool on = row >= 0 && c * VE < dh;
              const int64_t e = on ? row * dh + c * VE : 0;
              cp16(dst + P::at(r, c, a.brs), Kp + e, on);
              cp16(dst + P::TILE + P::at(r, c, a.brs), Vp + e, on);
            }
          }
          asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_addr(&full[st])) : "memory");
          if (lane == 0) tc::mbar_arrive(&full[st]);
        }
      }
    }
    if (!TMA) cp_wait<0>();
    if (TMA && !ok) {
      // a wait gave up: let the copies on their way land before shared memory is released (those of tiles below `tile`)
      volatile int no_abort = 0;
      for (int i = tile > S ? tile - S : 0; i < tile; ++i)
        if ((i & 1) == odd) tc::mbar_wait(&full[i % S], (i / S) & 1, &no_abort, nullptr);
    }
    return;
  }

  // ------------------------------------------------------------ arithmetic
  float2* stats = reinterpret_cast<float2*>(sm + P::STATS);  // [NG][ROWS]
  auto group_sync = [&]() {
    if (WM == 1)
      __syncwarp();
    else
      tc::named_sync(2 + grp, 32 * WM);
  };
  int n = 0;                     // run-relative number of the segment's first tile
  int mine = grp;                // of this group's next tile
  int st = grp % S, round = 0;   // its stage
  bool first_segment = true;
  // a unit's queries into one of two buffers, the next unit's while this one's tiles are done
  auto load_queries = [&](const Cursor<TK>& c, int buf) {
    const int hk = c.u / a.groups, r0 = (c.u - hk * a.groups) * ROWS;
    for (int e = tid; e < ROWS * (B16 ? CH : DHT); e += P::WORKERS) {
      constexpr int PER = B16 ? CH : DHT, V = B16 ? VE : 1;
      const int r = e / PER, k = e - r * PER, t = (r0 + r) / a.G;
      const bool live = r0 + r < a.R && k * V < dh;
      const T* src = live ? (const T*)a.q + ((int64_t)c.b * a.n_new + t) * a.q_stride + (hk * a.G + r0 + r - t * a.G) * dh + k * V : (const T*)a.q;
      const uint32_t to = smem_addr(sm + P::Q + buf * P::QB);
      if (B16)
        cp16(to + r * (DHT * 2) + ((k ^ (r & 7)) << 4), src, live);
      else  // pairs of rows side by side: [pair][half of a chunk of four dims][chunk][two dims of two rows]
        cp4(to + ((((r >> 1) * 2 + ((k >> 1) & 1)) * CH + (k >> 2)) * 4 + (k & 1) * 2 + (r & 1)) * 4, src, live);
    }
    cp_commit();
  };
  Cursor<TK> nxt = cur;
  int qbuf = 0;
  load_queries(cur, 0);
  while (n < n_tiles) {
    // ---- a segment: the tiles of one unit in this run
    const int seg = cur.tiles - cur.tile < n_tiles - n ? cur.tiles - cur.tile : n_tiles - n;
    const int hk = cur.u / a.groups, r0 = (cur.u - hk * a.groups) * ROWS;
    cp_wait<0>();
    tc::named_sync(1, P::WORKERS);  // this unit's queries are there
    T* Qs = reinterpret_cast<T*>(sm + P::Q + qbuf * P::QB);
    qbuf ^= 1;
    if (n + seg < n_tiles) {
      nxt = cur;
      nxt.tile = 0;
      nxt.next_unit(a);
      load_queries(nxt, qbuf);
    }
    // bf16: the sixteen rows of this warp as A operands, outputs and statistics in the layout of the products: rows g and
    // g + 8.  f32: a lane has the statistics of row lane % RM and, of the outputs of all rows (in pairs), its dims
    uint32_t qf[B16 ? DHT / 16 : 1][4];
    if constexpr (B16) {
#pragma unroll
      for (int ks = 0; ks < DHT / 16; ++ks) {
        const int row = 16 * wm + (lane & 15), c = 2 * ks + (lane >> 4);
        ldsm4(qf[ks], smem_addr(Qs + row * DHT + ((c ^ (row & 7)) * VE)));
      }
    }
    constexpr int MR = B16 ? 2 : 1;
    int qslot[MR];
    float m[MR], l[MR];
#pragma unroll
    for (int h = 0; h < MR; ++h) {
      const int r = r0 + RM * wm + (B16 ? g + 8 * h : lane % RM);
      qslot[h] = r < a.R ? cur.s.len - a.n_new + r / a.G : -1;
      m[h] = -INFINITY;
      l[h] = 0.f;
    }
    constexpr int HS = !B16 && DHT <= 128 ? 2 : 1, OC = DHT * HS / 128 > 0 ? DHT * HS / 128 : 1;  // f32: token halves; chunks a lane
    float o[B16 ? DHT / 8 : 1][4];
    float2 o2[B16 ? 1 : RM / 2][4 * OC];
#pragma unroll
    for (int d = 0; d < (B16 ? DHT / 8 : 1); ++d)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[d][e] = 0.f;
#pragma unroll
    for (int r = 0; r < (B16 ? 1 : RM / 2); ++r)
#pragma unroll
      for (int e = 0; e < 4 * OC; ++e) o2[r][e] = f2(0.f);
    int held = -1;  // the stage of this group's last tile, kept until its outputs have been in it
    for (; mine < n + seg; mine += NG) {
      const uint32_t base = smem_addr(sm + st * P::STAGE);
      const uint8_t* stage = sm + st * P::STAGE;
      const int x0 = (cur.tile + mine - n) * TK, j0 = first_slot<TK>(cur.s, cur.tile + mine - n);
      tc::mbar_wait(&full[st], round & 1, &abort_sh, a.c.err_dev);
      __syncwarp();
      const uint64_t live = mask[st];
      if (TMA && live != FULL) {
        // what was copied beside the tokens (or was not: a bad page's place) may be anything, and 0 times NaN is not 0
        for (int r = wm; r < TK; r += WM)
          if (!((live >> r) & 1ull))
            for (int c = lane; c < CH; c += 32) *reinterpret_cast<uint4*>(sm + st * P::STAGE + P::TILE + P::at(r, c, a.brs)) = make_uint4(0, 0, 0, 0);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        group_sync();
      }

      // every row sees every token of the tile: no test a token
      const bool all = live == FULL && j0 + TK - 1 <= cur.s.len - a.n_new &&
                       (a.window == 0 || j0 + TK <= a.sinks || cur.s.len - 1 - j0 < a.window);
      if constexpr (B16) {
      // ---- scores
      float s[NT][4] = {};
      {
        const int rr = ((lane >> 4) << 3) + (lane & 7), half = (lane >> 3) & 1;
        int krow[NT / 2];
#pragma unroll
        for (int n2 = 0; n2 < NT / 2; ++n2) krow[n2] = P::row_at(16 * n2 + rr, a.brs);
#pragma unroll
        for (int ks = 0; ks < DHT / 16; ++ks)
#pragma unroll
          for (int n2 = 0; n2 < NT / 2; ++n2) {
            uint32_t kf[4];
            const int row = 16 * n2 + rr;
            ldsm4(kf, base + krow[n2] + ((ks >> 2) << (a.brs + 7)) + P::chunk_at(row, 2 * ks + half));
            mma16816(s[2 * n2], qf[ks], kf[0], kf[1]);
            mma16816(s[2 * n2 + 1], qf[ks], kf[2], kf[3]);
          }
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[nt][e] *= a.sl2;
      if (!all) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int k = 8 * nt + 2 * t4 + (e & 1);
            if (!((live >> k) & 1ull) || !sees(a, qslot[e >> 1], j0 + k)) s[nt][e] = -INFINITY;
          }
      }
      if (a.scores) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int r = r0 + 16 * wm + g + 8 * h;
          if (r < a.R) {
            float* d = a.scores + (((int64_t)cur.b * a.c.n_kv_heads + hk) * a.R + r) * a.x_stride + x0 + 2 * t4;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) *reinterpret_cast<float2*>(d + 8 * nt) = make_float2(s[nt][2 * h], s[nt][2 * h + 1]);
          }
        }
      }
      // ---- running maximum and sum
      float ms[2], mn[2];
      bool grew = false;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float bm = fmaxf(s[0][2 * h], s[0][2 * h + 1]);
#pragma unroll
        for (int nt = 1; nt < NT; ++nt) bm = fmaxf(bm, fmaxf(s[nt][2 * h], s[nt][2 * h + 1]));
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
          for (int d = 0; d < DHT / 8; ++d) {
            o[d][2 * h] *= f;
            o[d][2 * h + 1] *= f;
          }
        }
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s[nt][e] = ex2_fast(s[nt][e] - ms[e >> 1]);
          l[e >> 1] += s[nt][e];
        }
      // ---- outputs
      {
        // P as an A operand, in two bf16 terms: rounded to one it would add as much to the error as the output's own
        // rounding does
        const int rr = (((lane >> 3) & 1) << 3) + (lane & 7), half = lane >> 4;
#pragma unroll
        for (int n2 = 0; n2 < NT / 2; ++n2) {
          uint32_t pf[4], pl[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float p0 = s[2 * n2 + (k >> 1)][2 * (k & 1)], p1 = s[2 * n2 + (k >> 1)][2 * (k & 1) + 1];
            pf[k] = pack2(p0, p1);
            const float2 hi = __bfloat1622float2(*reinterpret_cast<__nv_bfloat162*>(&pf[k]));
            pl[k] = pack2(p0 - hi.x, p1 - hi.y);
          }
          const int row = 16 * n2 + rr, vrow = P::row_at(row, a.brs);
#pragma unroll
          for (int nb = 0; nb < DHT / 16; ++nb) {
            uint32_t vf[4];
            ldsm4t(vf, base + P::TILE + vrow + ((nb >> 2) << (a.brs + 7)) + P::chunk_at(row, 2 * nb + half));
            mma16816(o[2 * nb], pf, vf[0], vf[1]);
            mma16816(o[2 * nb + 1], pf, vf[2], vf[3]);
            mma16816(o[2 * nb], pl, vf[0], vf[1]);
            mma16816(o[2 * nb + 1], pl, vf[2], vf[3]);
          }
        }
      }
      } else {
      // ---- scores: lane (tg, part) takes four tokens (TK 8: two) by every eighth chunk of their dims, then the eight parts are
      // added so that each lane is left with a part of the sums: row lane % RM and, of its tokens, all (RM 8) or half (RM 4)
      constexpr int TPL = TK < 16 ? TK / 4 : 4, PASS = TK / (4 * TPL), NV = TPL * RM / 8;
      const int tg = lane >> 3, part = lane & 7;
      float s[PASS * NV];
#pragma unroll
      for (int ps = 0; ps < PASS; ++ps) {
        float2 acc[RM / 2][TPL];
#pragma unroll
        for (int r = 0; r < RM / 2; ++r)
#pragma unroll
          for (int i = 0; i < TPL; ++i) acc[r][i] = f2(0.f);
#pragma unroll 2
        for (int c8 = 0; c8 < CH; c8 += 8) {
          const int c = c8 + part;
          float4 k[TPL];
#pragma unroll
          for (int i = 0; i < TPL; ++i) k[i] = *reinterpret_cast<const float4*>(stage + P::at((ps * 4 + tg) * TPL + i, c, a.brs));
#pragma unroll
          for (int r = 0; r < RM / 2; ++r) {
            const float* q = reinterpret_cast<const float*>(Qs) + ((RM / 2 * wm + r) * 2 * CH + c) * 4;
            const float4 q0 = *reinterpret_cast<const float4*>(q), q1 = *reinterpret_cast<const float4*>(q + CH * 4);
#pragma unroll
            for (int i = 0; i < TPL; ++i) {
              acc[r][i] = __ffma2_rn(make_float2(q0.x, q0.y), f2(k[i].x), acc[r][i]);
              acc[r][i] = __ffma2_rn(make_float2(q0.z, q0.w), f2(k[i].y), acc[r][i]);
              acc[r][i] = __ffma2_rn(make_float2(q1.x, q1.y), f2(k[i].z), acc[r][i]);
              acc[r][i] = __ffma2_rn(make_float2(q1.z, q1.w), f2(k[i].w), acc[r][i]);
            }
          }
        }
        const bool b2 = lane & 4, b1 = lane & 2, b0 = lane & 1;
        float2 h4[RM / 2 * TPL / 2];  // after lanes 4 apart: RM 8: pairs of rows 0, 1 or 2, 3; RM 4: half of the tokens
#pragma unroll
        for (int i = 0; i < RM / 2 * TPL / 2; ++i) {
          const float2 lo = RM == 8 ? acc[i / TPL][i % TPL] : acc[i / (TPL / 2)][i % (TPL / 2)];
          const float2 hi = RM == 8 ? acc[(i / TPL + 2) % (RM / 2)][i % TPL] : acc[i / (TPL / 2)][i % (TPL / 2) + TPL / 2];
          const float2 give = b2 ? lo : hi, keep = b2 ? hi : lo;
          h4[i] = make_float2(keep.x + __shfl_xor_sync(0xffffffffu, give.x, 4), keep.y + __shfl_xor_sync(0xffffffffu, give.y, 4));
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          const float2 give = b1 ? h4[i] : h4[i + NV], keep = b1 ? h4[i + NV] : h4[i];
          const float2 h2 = make_float2(keep.x + __shfl_xor_sync(0xffffffffu, give.x, 2), keep.y + __shfl_xor_sync(0xffffffffu, give.y, 2));
          s[ps * NV + i] = (b0 ? h2.y : h2.x) + __shfl_xor_sync(0xffffffffu, b0 ? h2.x : h2.y, 1);
        }
      }
      auto token = [&](int i) { return ((i / NV) * 4 + tg) * TPL + (RM == 8 ? 0 : ((lane >> 2) & 1) * (TPL / 2)) + i % NV; };
      const int row = r0 + RM * wm + lane % RM;
      float top = -INFINITY;
#pragma unroll
      for (int i = 0; i < PASS * NV; ++i) {
        const int k = token(i);
        s[i] = ((live >> k) & 1ull) && (all || sees(a, qslot[0], j0 + k)) ? s[i] * a.sl2 : -INFINITY;
        if (a.scores && row < a.R) a.scores[(((int64_t)cur.b * a.c.n_kv_heads + hk) * a.R + row) * a.x_stride + x0 + k] = s[i];
        top = fmaxf(top, s[i]);
      }
#pragma unroll
      for (int x = RM; x < 32; x <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
      const float mn = fmaxf(m[0], top), ms = mn == -INFINITY ? 0.f : mn;
      if (__any_sync(0xffffffffu, mn > m[0])) {
        const float f = exp2f(m[0] - ms);
        l[0] *= f;
        m[0] = mn;
#pragma unroll
        for (int r = 0; r < RM / 2; ++r) {
          const float2 fr = make_float2(__shfl_sync(0xffffffffu, f, 2 * r), __shfl_sync(0xffffffffu, f, 2 * r + 1));
#pragma unroll
          for (int e = 0; e < 4 * OC; ++e) o2[r][e] = __fmul2_rn(o2[r][e], fr);
        }
      }
      float* X = reinterpret_cast<float*>(sm + P::X) + warp * (TK * RM);  // p, [token][row]
#pragma unroll
      for (int i = 0; i < PASS * NV; ++i) {
        const float x = exp2f(s[i] - ms);
        l[0] += x;  // a lane's share
        X[token(i) * RM + lane % RM] = x;
      }
      __syncwarp();
      // ---- outputs: a half of the lanes every other token (head dims above 128: all lanes every token), a lane chunks
      // li + 16 j (32 j) of the dims
      const int hw = HS == 2 ? lane >> 4 : 0, li = HS == 2 ? lane & 15 : lane;
#pragma unroll 2
      for (int k = hw; k < TK; k += HS) {
        float2 pp[RM / 2];
#pragma unroll
        for (int r = 0; r < RM / 2; r += 2) {
          const float4 x = *reinterpret_cast<const float4*>(X + k * RM + 2 * r);
          pp[r] = make_float2(x.x, x.y);
          pp[r + 1] = make_float2(x.z, x.w);
        }
#pragma unroll
        for (int j = 0; j < OC; ++j) {
          const float4 v = *reinterpret_cast<const float4*>(stage + P::TILE + P::at(k, li + 32 / HS * j, a.brs));
          const float vs[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int r = 0; r < RM / 2; ++r) o2[r][4 * j + e] = __ffma2_rn(pp[r], f2(vs[e]), o2[r][4 * j + e]);
        }
      }
      __syncwarp();
      }
      // the stage is free again, but for the last one's
      if (mine + NG < n + seg) {
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&empty[st]);
      } else {
        held = st;
      }
      st += NG;
      if (st >= S) {
        st -= S;
        ++round;
      }
    }

    // ---- the groups' outputs together: each puts its own into its last tile's stage
    group_sync();
    float* to = reinterpret_cast<float*>(sm + (held >= 0 ? held : 0) * P::STAGE);
    if constexpr (B16) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
        l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
        const int row = 16 * wm + g + 8 * h;
        if (t4 == 0) stats[grp * ROWS + row] = make_float2(m[h], l[h]);
        if (held >= 0) {
#pragma unroll
          for (int d = 0; d < DHT / 8; ++d) *reinterpret_cast<float2*>(to + P::sum_at(row, 8 * d + 2 * t4)) = make_float2(o[d][2 * h], o[d][2 * h + 1]);
        }
      }
    } else {
#pragma unroll
      for (int x = RM; x < 32; x <<= 1) l[0] += __shfl_xor_sync(0xffffffffu, l[0], x);
      if (lane < RM) stats[grp * ROWS + RM * wm + lane] = make_float2(m[0], l[0]);
      if (held >= 0) {
#pragma unroll
        for (int r = 0; r < RM / 2; ++r) {
          if (HS == 2) {
#pragma unroll
            for (int e = 0; e < 4 * OC; ++e)
              o2[r][e] = make_float2(o2[r][e].x + __shfl_xor_sync(0xffffffffu, o2[r][e].x, 16), o2[r][e].y + __shfl_xor_sync(0xffffffffu, o2[r][e].y, 16));
          }
          const int row = RM * wm + 2 * r, li = HS == 2 ? lane & 15 : lane;
          if (HS == 1 || lane < 16) {
#pragma unroll
            for (int j = 0; j < OC; ++j) {
              const int d = 4 * (li + 32 / HS * j);
              *reinterpret_cast<float4*>(to + P::sum_at(row, d)) = make_float4(o2[r][4 * j].x, o2[r][4 * j + 1].x, o2[r][4 * j + 2].x, o2[r][4 * j + 3].x);
              *reinterpret_cast<float4*>(to + P::sum_at(row + 1, d)) = make_float4(o2[r][4 * j].y, o2[r][4 * j + 1].y, o2[r][4 * j + 2].y, o2[r][4 * j + 3].y);
            }
          }
        }
      }
    }
    if (lane == 0 && wm == 0) last_stage[grp] = held;
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    tc::named_sync(1, P::WORKERS);
    const bool whole = seg == cur.tiles;
    const int64_t slot = 2 * (int64_t)blockIdx.x + (first_segment ? 0 : 1);
    for (int e = tid; e < ROWS * (DHT / 4); e += P::WORKERS) {
      const int r = e / (DHT / 4), d = (e - r * (DHT / 4)) * 4;
      if (r0 + r >= a.R || d >= dh) continue;
      float M = -INFINITY, L = 0.f;
      bool any = false;
#pragma unroll
      for (int k = 0; k < NG; ++k) M = fmaxf(M, stats[k * ROWS + r].x);
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k = 0; k < NG; ++k) {
        const float2 ml = stats[k * ROWS + r];
        if (counts(ml)) {
          const float f = ex2_fast(ml.x - M);
          any = true;
          L = fmaf(ml.y, f, L);
          v = fma4(*reinterpret_cast<const float4*>(reinterpret_cast<const float*>(sm + last_stage[k] * P::STAGE) + P::sum_at(r, d)), f, v);
        }
      }
      if (whole) {
        finish<T>(a, cur.b, hk, r0 + r, d, v, M, L, any);
      } else {
        *reinterpret_cast<float4*>(a.part_o + (slot * ROWS + r) * DHT + d) = v;
        if (d == 0) a.part_ml[slot * ROWS + r] = make_float2(M, any ? L : 0.f);
      }
    }
    if (!whole && a.join) {
      // the last CTA to come here has all parts
      tc::named_sync(1, P::WORKERS);
      const int first = run_start + n - cur.tile;  // the unit's first tile
      const int c0 = deal.owner(first);
      if (tid == 0) {
        const int c1 = deal.owner(first + cur.tiles - 1);
        unsigned* count = a.done + c0;
        __threadfence();  // (of all threads' parts: the barrier came before)
        const unsigned before = atomicAdd(count, 1u);
        joins = before == (unsigned)(c1 - c0) ? c1 - c0 + 1 : 0;
        if (joins) *count = 0;
        __threadfence();
      }
      tc::named_sync(1, P::WORKERS);
      const int parts = joins;
      if (parts) {
        // part p's slot: the first is its CTA's last segment, unless the unit starts that CTA's run
        const bool starts = deal.start(c0) == first;
        const int rows = a.R - r0 < ROWS ? a.R - r0 : ROWS, per = dh / 4;
        for (int e = tid; e < rows * per; e += P::WORKERS) {
          const int r = e / per, d = (e - r * per) * 4;
          float M = -INFINITY, L = 0.f;
          bool any = false;
          float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
          for (int p0 = 0; p0 < parts; p0 += 8) {  // eight parts on their way at once
            float2 ml[8];
            float4 x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const int p = p0 + i, at = (2 * (c0 + p) + (p == 0 && !starts ? 1 : 0)) * ROWS + r;
              ml[i] = make_float2(-INFINITY, 0.f);
              if (p < parts) {
                ml[i] = __ldcg(&a.part_ml[at]);
                x[i] = __ldcg(reinterpret_cast<const float4*>(a.part_o + (int64_t)at * DHT + d));
              }
            }
            float Mn = M;
#pragma unroll
            for (int i = 0; i < 8; ++i) Mn = fmaxf(Mn, ml[i].x);
            if (any) {
              const float f = ex2_fast(M - Mn);
              L *= f;
              v = make_float4(v.x * f, v.y * f, v.z * f, v.w * f);
            }
            M = Mn;
#pragma unroll
            for (int i = 0; i < 8; ++i)
              if (counts(ml[i])) {
                const float f = ex2_fast(ml[i].x - M);
                any = true;
                L = fmaf(ml[i].y, f, L);
                v = fma4(x[i], f, v);
              }
          }
          finish<T>(a, cur.b, hk, r0 + r, d, v, M, L, any);
        }
      }
    }
    tc::named_sync(1, P::WORKERS);  // the held stages, the statistics and Q's space are free again
    if (held >= 0 && lane == 0) tc::mbar_arrive(&empty[held]);
    first_segment = false;
    n += seg;
    cur = nxt;
  }
}

// ---------------------------------------------------------------------------------------
// Joins the parts of one query row where there may be many: a CTA a row; its 256 threads take the parts in turns of
// 1024 / DHT, four columns each, and are added in a fixed order.  What one CTA finished is left alone.
// ---------------------------------------------------------------------------------------
template <typename T, int DHT, int TK, int ROWS>
__global__ void __launch_bounds__(256) decode_join_kernel(const __grid_constant__ DecodeArgs a) {
  constexpr int TPP = DHT / 4, TURNS = 256 / TPP;
  __shared__ float4 red[256];
  __shared__ float L_part[TURNS];
  __shared__ int any_part[TURNS];
  __shared__ int sh_starts, sh_c0, sh_parts;
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x;
  const int64_t id = blockIdx.x;
  const int per_b = a.c.n_kv_heads * a.R, b = (int)(id / per_b), hk = (int)(id - (int64_t)b * per_b) / a.R, row = (int)(id % a.R);
  const int grp = row / ROWS, lr = row - grp * ROWS;
  if (tid < 32) {
    Deal<TK, SHARE> d;
    d.count(a, tid);
    const int tiles = d.tiles(a, b);
    if (tid == 0) sh_parts = 0;
    if (tiles > 0) {
      const int first = d.first_of(a, b, hk * a.groups + grp, tid);
      if (tid == 0) {
        sh_c0 = d.owner(first);
        sh_parts = d.owner(first + tiles - 1) - sh_c0 + 1;
        sh_starts = first == d.start(sh_c0);
      }
    }
  }
  __syncthreads();
  const int c0 = sh_c0, parts = sh_parts, dh = a.c.head_dim;
  if (parts < 2) return;
  auto slot = [&](int p) { return 2 * (int64_t)(c0 + p) + (p == 0 && !sh_starts ? 1 : 0); };
  float M = -INFINITY;
  for (int p = tid & 31; p < parts; p += 32) M = fmaxf(M, a.part_ml[slot(p) * ROWS + lr].x);
  M = warp_max(M);
  const int turn = tid / TPP, d = (tid - turn * TPP) * 4;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  float L = 0.f;
  int any = 0;
#pragma unroll 4
  for (int p = turn; p < parts; p += TURNS) {
    const float2 ml = a.part_ml[slot(p) * ROWS + lr];
    const float4 x = d < dh ? *reinterpret_cast<const float4*>(a.part_o + (slot(p) * ROWS + lr) * DHT + d) : make_float4(0.f, 0.f, 0.f, 0.f);
    if (counts(ml)) {
      const float f = ex2_fast(ml.x - M);
      any = 1;
      L = fmaf(ml.y, f, L);
      s = fma4(x, f, s);
    }
  }
  red[tid] = s;
  if (d == 0) {
    L_part[turn] = L;
    any_part[turn] = any;
  }
  __syncthreads();
  if (tid >= TPP || d >= dh) return;
  L = 0.f;
  any = 0;
#pragma unroll
  for (int i = 0; i < TURNS; ++i) {
    L += L_part[i];
    any |= any_part[i];
  }
#pragma unroll
  for (int i = 1; i < TURNS; ++i) s = fma4(red[i * TPP + tid], 1.f, s);
  finish<T>(a, b, hk, row, d, s, M, L, any != 0);
}

// weights_out = weights_in + the rows' softmax weights, in row order: a thread four slots, four rows on their way at once
template <int TK>
__global__ void __launch_bounds__(256) decode_weights_kernel(const __grid_constant__ DecodeArgs a, int chunks) {
  pdl_wait();
  pdl_trigger();
  const int64_t unit = blockIdx.x / chunks;  // b * kv heads + head
  const int b = (int)(unit / a.c.n_kv_heads);
  const Seen s = seen_of<TK>(a, b);
  const int j = (int)(blockIdx.x - unit * chunks) * 1024 + 4 * (int)threadIdx.x, n = s.len - j < 4 ? s.len - j : 4;
  if (n <= 0) return;
  const float* lse2 = a.lse2 + unit * a.R;
  const int tile = j / TK;
  const int x = tile < s.sink_tiles ? j : tile >= s.w_tile ? j + (s.sink_tiles - s.w_tile) * TK : -1;
  float w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = i < n && a.w_in ? a.w_in[unit * a.w_stride + j + i] : 0.f;
  if (x >= 0) {
    const float* sc = a.scores + unit * a.R * a.x_stride + x;
#pragma unroll 4
    for (int r = 0; r < a.R; ++r) {
      const float4 v = *reinterpret_cast<const float4*>(sc + (int64_t)r * a.x_stride);
      const float z = lse2[r];
      if (z != -INFINITY) {
        w[0] += ex2_fast(v.x - z);
        w[1] += ex2_fast(v.y - z);
        w[2] += ex2_fast(v.z - z);
        w[3] += ex2_fast(v.w - z);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < n) a.w_out[unit * a.w_stride + j + i] = w[i];
}

// ---- host ------------------------------------------------------------------------------
struct DecodeLayout {
  int rows, groups, dht, grid, R, join;
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
  // registers), 4, 8 or 16 (f32)
  L.rows = !b16 ? (L.R <= 4 ? 4 : L.R <= 8 ? 8 : 16) : L.R <= 16 || L.dht == 256 ? 16 : L.R <= 32 ? 32 : 64;
  L.groups = (L.R + L.rows - 1) / L.rows;
  L.grid = device_sm_count();
  if (L.grid > WS_COUNTERS) L.grid = WS_COUNTERS;
  // A unit has about grid / units parts if the lengths are near to one another, which the host does not know; the last CTA
  // reads them all, alone on its SM (about 20 us a MB), while a kernel of its own takes about 3 us and has the GPU.  (Of
  // one sequence of 65536 tokens beside 31 of 200, with 16 heads over one, it reads some 150 where this counts on 6: 44 us.)
  const int64_t units = (int64_t)p.batch * p.cache.n_kv_heads * L.groups;
  const int64_t parts = units > 0 ? L.grid / units + 2 : 0;
  L.join = parts * (L.R < L.rows ? L.R : L.rows) * p.cache.head_dim * 4 <= 128 * 1024;
  L.x_stride = ((int64_t)call_max_len(p.cache, p.max_len) + 63) / 64 * 64;
  size_t at = WS_ZERO;
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

template <typename T, int DHT, int WM, int RM, bool TMA>
cudaError_t launch_kernel(const CUtensorMap& k, const CUtensorMap& v, const DecodeArgs& a, cudaStream_t st) {
  using P = Plan<T, DHT, WM, RM>;
  cudaError_t e = allow_smem(decode_kernel<T, DHT, WM, RM, TMA>, P::BYTES);
  return e == cudaSuccess ? launch_pdl(decode_kernel<T, DHT, WM, RM, TMA>, dim3(a.grid), dim3(P::THREADS), (size_t)P::BYTES, st, k, v, a) : e;
}
template <typename T, int DHT, int WM, int RM>
cudaError_t launch(DecodeArgs& a, cudaStream_t st) {
  using P = Plan<T, DHT, WM, RM>;
  const ra_kv_cache& c = a.c;
  // boxes of 2^brs slots of a page: a pool is [pages x kv heads][page_size][head_dim]
  a.brs = c.page_size % 32 == 0 && P::TK >= 32 ? 5 : c.page_size % 16 == 0 && P::TK >= 16 ? 4 : 3;
  a.whole_rows = c.head_dim == DHT;
  CUtensorMap k, v;
  memset(&k, 0, sizeof k);
  memset(&v, 0, sizeof v);
  const int64_t planes = (int64_t)c.n_pages * c.n_kv_heads;
  auto map = [&](CUtensorMap* m, const void* p) {
    return tma_map_planes(m, p, sizeof(T) == 2 ? DT_BF16 : DT_F32, (int)planes, c.page_size, c.head_dim, 128 / (int)sizeof(T), 1 << a.brs,
                          a.whole_rows != 0);
  };
  // tiles are counted in 32 bits
  if ((int64_t)a.batch * c.n_kv_heads * a.groups * ((a.max_len + P::TK - 1) / P::TK) > INT32_MAX) return cudaErrorNotSupported;
  const bool tma = c.page_size % 8 == 0 && planes <= INT32_MAX && map(&k, c.k_dev) && map(&v, c.v_dev);
  cudaError_t e = tma ? launch_kernel<T, DHT, WM, RM, true>(k, v, a, st) : launch_kernel<T, DHT, WM, RM, false>(k, v, a, st);
  note_launch(1);
  if (e == cudaSuccess && !a.join) {
    e = launch_pdl(decode_join_kernel<T, DHT, P::TK, P::ROWS>, dim3((unsigned)((int64_t)a.batch * c.n_kv_heads * a.R)), dim3(256), 0, st, a);
    note_launch(1);
  }
  if (e != cudaSuccess || !a.scores) return e;
  const int chunks = (a.max_len + 1023) / 1024;
  const int64_t n = (int64_t)chunks * a.batch * c.n_kv_heads;
  if (n > INT32_MAX) return cudaErrorNotSupported;
  note_launch(1);
  return launch_pdl(decode_weights_kernel<P::TK>, dim3((unsigned)n), dim3(256), 0, st, a, chunks);
}

template <int DHT>
cudaError_t launch_f32(DecodeArgs& a, int rows, cudaStream_t st) {
  return rows == 4 ? launch<float, DHT, 1, 4>(a, st) : rows == 8 ? launch<float, DHT, 1, 8>(a, st) : launch<float, DHT, 2, 8>(a, st);
}
template <int DHT>
cudaError_t launch_bf16(DecodeArgs& a, int rows, cudaStream_t st) {
  return rows == 16 ? launch<bf16, DHT, 1, 16>(a, st) : rows == 32 ? launch<bf16, DHT, 2, 16>(a, st) : launch<bf16, DHT, 4, 16>(a, st);
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
  a.done = (unsigned*)ws;
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
  a.join = L.join;
  a.page_shift = -1;
  for (int i = 0; i < 31; ++i)
    if (p.cache.page_size == 1 << i) a.page_shift = i;
  a.sl2 = p.scale * kLog2e;
  if (p.cache.dtype == RA_F32) return L.dht == 64 ? launch_f32<64>(a, L.rows, st) : L.dht == 128 ? launch_f32<128>(a, L.rows, st) : launch_f32<256>(a, L.rows, st);
  return L.dht == 64 ? launch_bf16<64>(a, L.rows, st) : L.dht == 128 ? launch_bf16<128>(a, L.rows, st) : launch<bf16, 256, 1, 16>(a, st);
}

}  // namespace ra
