// k_vocab_loss.cu -- cross-entropy over a vocabulary from hidden states, without keeping logits.
//
// First the tokens that are counted are found and numbered (a CTA counts those before its own), and where not all are, their
// hidden states are gathered, so that what is not counted costs nothing and is never read.  (But for the forward of up to 128 bf16 tokens,
// which are one row of tiles in any case: it takes them as they are, reads all of W, and drops the results of those that are not counted.)
// Forward: tiles of logits z = x W^T; of each tile's rows the maximum and the sum of exp(z - maximum) go to the workspace,
// with the label's logit; a second kernel joins them: lse = m + log(sum), loss = lse - z[label].
// Backward, piece by piece of the vocabulary: the piece's logits again and dz = dloss (exp(z - lse) - onehot) into the
// workspace (rounded, in bf16, relative to the largest |dloss|; of up to 128 tokens in two terms); then, in one launch, dw of the piece = dz^T x and the sums of dx += dz W, the latter in fp32 and, where its tiles are
// few, in parts of the vocabulary, which a last kernel adds up and puts where the tokens were.
// fp32 operands are cut into three planes of bf16 (products.cuh), dz too; bf16 ones are read where they are.
//
// Bound: the products, four of tokens x vocab x hidden with the logits computed again (keeping them would be three, and 2 tokens x
// vocab bytes).  8192 x 32000 x 2048 in bf16, one pass after the other: forward 0.55 ms (2.0 PFLOP/s), backward 2.0 ms (1.6 PFLOP/s), 2.65 ms
// in all, at the clock that the power leaves.  One launch at a time, with pauses, the logits take 0.53 ms, the backward's 0.59 and its
// gradients 1.18 (1.8 PFLOP/s).  Few tokens: W's bytes; 16 of 32000 x 2048 in 33 us (3.9 TB/s).
#include <algorithm>

#include "common.cuh"
#include "operators.h"
#include "products.cuh"

namespace ra {
namespace {

using prod::parts_of;
using prod::Pick;
using prod::Shape;
using prod::SMS;
using prod::Store;
using prod::Tile;
using prod::Unit;
using prod::up;

constexpr float LOG2E = 1.44269504088896341f;
constexpr int ROWS = 256;  // rows of tokens in the workspace: whole tiles of a pair

// ---- which tokens are counted -------------------------------------------------------------
struct Prep {
  int *count, *index, *label;  // of the counted tokens: how many; each one's place among all, its label,
  float *scale, *lse, *ref;    // ... dloss over the largest of them, lse, and that largest (backward)
  void* x;                     // ... and hidden states: [planes][rows][pitch]
  int rows, width, pitch, planes;  // (zeros from hidden to width)
};
__device__ __forceinline__ bool counted(const ra_vocab_loss_args& a, int label) { return (uint32_t)label < (uint32_t)a.vocab; }

// sums of two counts over the CTA's 256 threads
__device__ __forceinline__ int2 sum2(int2 v, int2* sh) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
    v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
  }
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
  __syncthreads();
  int2 r = make_int2(0, 0);
#pragma unroll
  for (int i = 0; i < 8; ++i) r.x += sh[i].x, r.y += sh[i].y;
  return r;
}
// A row of hidden states (src NULL: zeros) into row r of the gathered ones, by a warp
__device__ __forceinline__ void put_row(const Prep& p, const bf16* src, int r, int H, int lane) {
  bf16* d = static_cast<bf16*>(p.x) + (int64_t)r * p.pitch;
  for (int c = lane * 8; c < H; c += 256)
    *reinterpret_cast<uint4*>(d + c) = src ? *reinterpret_cast<const uint4*>(src + c) : make_uint4(0, 0, 0, 0);
}
__device__ __forceinline__ void split4(float4 v, bf16* d, int64_t plane) {
  uint32_t x[3], y[3];
  prod::planes_of<3>(v.x, v.y, x);
  prod::planes_of<3>(v.z, v.w, y);
#pragma unroll
  for (int k = 0; k < 3; ++k) *reinterpret_cast<uint2*>(d + k * plane) = make_uint2(x[k], y[k]);
}
__device__ __forceinline__ void put_row(const Prep& p, const float* src, int r, int H, int lane) {
  bf16* d = static_cast<bf16*>(p.x) + (int64_t)r * p.pitch;
  for (int c = lane * 4; c < p.width; c += 128)
    split4(src && c < H ? *reinterpret_cast<const float4*>(src + c) : make_float4(0.f, 0.f, 0.f, 0.f), d + c, (int64_t)p.rows * p.pitch);
}

// rows of W into planes (fp32)
struct Split {
  const float* w;
  int64_t stride;
  bf16* out;
  int rows, hidden, width, pitch;
};
__device__ __forceinline__ void split_rows(const Split& s, int cta, int ctas) {
  const int per = s.width / 4;
  for (int64_t i = (int64_t)cta * 256 + threadIdx.x; i < (int64_t)s.rows * per; i += (int64_t)ctas * 256) {
    const int r = (int)(i / per), c = (int)(i % per) * 4;
    split4(c < s.hidden ? *reinterpret_cast<const float4*>(s.w + r * s.stride + c) : make_float4(0.f, 0.f, 0.f, 0.f), s.out + (int64_t)r * s.pitch + c,
           (int64_t)s.rows * s.pitch);
  }
}
__global__ void __launch_bounds__(256) vocab_split_kernel(const Split s) {
  pdl_wait();
  pdl_trigger();
  split_rows(s, blockIdx.x, gridDim.x);
}

// The first `ctas` CTAs number and gather the tokens; those behind them take the vocabulary's first piece apart
template <typename T>
__global__ void __launch_bounds__(256) vocab_prep_kernel(const ra_vocab_loss_args a, const Prep p, int backward, int ctas, const Split split) {
  __shared__ int2 sh[8];
  __shared__ int list[256], warp_n[8];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, T_ = a.tokens;
  pdl_wait();
  pdl_trigger();
  if ((int)blockIdx.x >= ctas) {
    split_rows(split, blockIdx.x - ctas, gridDim.x - ctas);
    return;
  }
  const int per = (T_ + ctas - 1) / ctas;
  const int start = min(T_, (int)blockIdx.x * per), end = min(T_, start + per);
  int2 n = make_int2(0, 0);
  float top = 0.f;
  const bool want_top = backward && p.planes == 1;
  for (int t0 = tid; t0 < T_; t0 += 2048) {  // eight at once on their way
    int l[8];
    float d[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int t = t0 + 256 * i;
      l[i] = t < T_ ? a.labels_dev[t] : -1;
      d[i] = want_top && t < T_ ? a.dloss_dev[t] : 0.f;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const bool c = counted(a, l[i]);
      n.x += c && t0 + 256 * i < start;
      n.y += c;
      if (c) top = fmaxf(top, fabsf(d[i]));
    }
  }
  n = sum2(n, sh);
  // dz is rounded to bf16 relative to the largest |dloss|: where all are equal, as in a mean, -onehot stays exact, whose
  // rounding, the same in every row, would be that of the whole gradient (2^-9 at worst)
  __shared__ float sh_top[8];
  top = warp_max(top);
  if (lane == 0) sh_top[warp] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 8; ++i) top = fmaxf(top, sh_top[i]);
  if (!(top > 0.f) || !isfinite(top)) top = 1.f;
  int base = n.x;
  const int total = n.y;
  const bool gather = p.planes > 1 || total < T_;
  const T* x = static_cast<const T*>(a.x_dev);
  for (int s = start; s < end; s += 256) {
    const int t = s + tid;
    const int l = t < end ? a.labels_dev[t] : -1;
    const bool c = counted(a, l);
    const uint32_t ballot = __ballot_sync(0xffffffffu, c);
    if (lane == 0) warp_n[warp] = __popc(ballot);
    __syncthreads();
    int at = __popc(ballot & ((1u << lane) - 1u)), here = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      at += i < warp ? warp_n[i] : 0;
      here += warp_n[i];
    }
    if (t < end) {
      if (c) {
        list[at] = t;
        p.index[base + at] = t;
        p.label[base + at] = l;
        p.scale[base + at] = backward ? a.dloss_dev[t] / top : 0.f;
        p.lse[base + at] = backward ? a.lse_dev[t] : 0.f;
      } else {
        if (l >= a.vocab) set_dev_error(a.err_dev, RA_DEVERR_BOUNDS);
        if (!backward) {
          a.loss_dev[t] = 0.f;
          if (a.lse_dev) a.lse_dev[t] = 0.f;
        }
        list[255 - (tid - at)] = t;  // those that are not, from the other end
      }
    }
    __syncthreads();
    if (gather)
      for (int i = warp; i < here; i += 8) put_row(p, x + list[i] * a.x_stride, base + i, a.hidden, lane);
    if (backward && a.dx_dev)
      for (int i = warp; i < min(256, end - s) - here; i += 8) {
        T* d = static_cast<T*>(a.dx_dev) + list[255 - i] * a.dx_stride;
        for (int k = lane * (16 / (int)sizeof(T)); k < a.hidden; k += 512 / (int)sizeof(T))
          *reinterpret_cast<uint4*>(d + k) = make_uint4(0, 0, 0, 0);
      }
    base += here;
    __syncthreads();
  }
  // the rows up to whole tiles
  const int up = (total + ROWS - 1) / ROWS * ROWS;
  if (gather)
    for (int r = total + blockIdx.x * 8 + warp; r < up; r += ctas * 8) put_row(p, (const T*)nullptr, r, a.hidden, lane);
  for (int r = total + blockIdx.x * 256 + tid; r < up; r += ctas * 256) {
    p.label[r] = -1;
    p.scale[r] = p.lse[r] = 0.f;
  }
  if (blockIdx.x == 0 && tid == 0) {
    *p.count = total;
    *p.ref = top;
  }
}

// ---- products -----------------------------------------------------------------------------
struct VocabArgs {
  CUtensorMap x, xc, w;         // logits: K-major operands (x as given, gathered)
  CUtensorMap dzk, dzm, wm, xm, xcm;  // gradients: dz K-major and MN-major, W and x MN-major
  CUtensorMap dz, dw, dxs;      // stores
  Shape shape;
  unsigned* err;
  const int *count, *label;
  const float *scale, *lse, *ref;
  float2* stats;
  float* zlab;
  int tokens, hidden, rows, planes;
  int v0, width;                // the piece: words v0 .. v0 + width
  int wrow;                     // where it begins in the map of W
  int stat0;                    // its first part of the statistics
  int cg, splits_x, splits_w, want_x, want_w;
  int dtype;
};

__device__ __forceinline__ int ceil_div(int a, int b) { return (a + b - 1) / b; }
__device__ __forceinline__ const CUtensorMap* hidden_map(const VocabArgs& p, int count, const CUtensorMap* given, const CUtensorMap* gathered) {
  return p.planes == 1 && count == p.tokens ? given : gathered;
}

// tiles of logits; BACK: into dz, else into statistics; PLANES: of the operands; DZ: of dz
template <bool BACK, int PLANES, int DZ>
struct Logits {
  static constexpr int PA = PLANES, PB = PLANES;
  static constexpr bool PARTS = BACK, ONE = false;
  using Args = VocabArgs;
  static __device__ __forceinline__ int count(const Args& p) {
    return ceil_div(tokens(p), prod::BM * p.cg) * ceil_div(p.width, p.shape.bn);
  }
  static __device__ __forceinline__ void prefetch(const Args& p) {
    prod::prefetch_map(&p.xc);
    prod::prefetch_map(&p.w);
  }
  // (count NULL: all, as they are)
  static __device__ __forceinline__ int tokens(const Args& p) { return p.count ? *p.count : p.tokens; }
  static __device__ __forceinline__ void unit(const Args& p, int u, Unit& w) {
    const int n = tokens(p), mt_n = ceil_div(n, prod::BM * p.cg), nt_n = ceil_div(p.width, p.shape.bn);
    int mt, nt;
    prod::tile_of(u, mt_n, nt_n, mt, nt);
    w.a = hidden_map(p, n, &p.x, &p.xc);
    w.b = &p.w;
    w.m0 = w.ar = mt * prod::BM * p.cg;
    w.n0 = nt * p.shape.bn;
    w.br = p.wrow + w.n0;
    w.ak = w.bk = w.az = w.bz = w.kb0 = 0;
    w.kb1 = ceil_div(p.hidden, prod::BK);
    w.a_mn = w.b_mn = false;
    w.job = 0;
    w.z = nt;
  }
  // this lane's row of the tile, and where its label is among the tile's columns
  static __device__ __forceinline__ int row_of(const Unit& w, const Tile& t) { return w.m0 + t.rank * prod::BM + t.quad * 32 + t.lane; }
  static __device__ __forceinline__ int label_of(const Args& p, const Unit& w, int row) {
    return (p.count || row < p.tokens ? p.label[row] : -1) - p.v0 - w.n0;
  }
  // dz = scale (exp(z - lse) - onehot)
  static __device__ __forceinline__ void part(const Args& p, const Unit& w, const Tile& t, Store& st, int i, float (&v)[32]) {
    const int row = row_of(w, t), row0 = row - t.lane, label = label_of(p, w, row);
    const float scale = p.scale[row], lse = p.lse[row];
    const int c = 32 * (t.half + 2 * i), left = p.width - w.n0 - c;  // (zeros up to a whole k-block of the sums that follow)
    if (w.n0 + c >= (p.width + 63) / 64 * 64) return;
#pragma unroll
    for (int j = 0; j < 32; ++j) {
      const float e = ex2_fast(__fmul_rn(__fsub_rn(v[j], lse), LOG2E));
      v[j] = j < left ? __fmul_rn(scale, c + j == label ? __fsub_rn(e, 1.f) : e) : 0.f;
    }
    auto at = [&](int j) { return v[j]; };
    if constexpr (DZ == 1) st.bf16_row(&p.dz, at, w.n0 + c, row0, 0);
    else st.planes<DZ, false>(&p.dz, at, w.n0 + c, row0, 0);
  }
  template <int CH>
  static __device__ __forceinline__ void finish(const Args& p, const Unit& w, const Tile& t, Store& st, float (&v)[CH][32]) {
    const int row = row_of(w, t), label = label_of(p, w, row);
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int c = 32 * (t.half + 2 * i);
      if (i >= t.chunks) break;
      if (w.n0 + c + 32 > p.width)
#pragma unroll
        for (int j = 0; j < 32; ++j)
          if (w.n0 + c + j >= p.width) v[i][j] = -INFINITY;
      if ((uint32_t)(label - c) < 32u)
#pragma unroll
        for (int j = 0; j < 32; ++j)
          if (c + j == label) p.zlab[row] = v[i][j];
#pragma unroll
      for (int j = 0; j < 32; ++j) m = fmaxf(m, v[i][j]);
    }
    float l = 0.f;
    const float from = m > -INFINITY ? m : 0.f;  // (nothing but NaN, or no words at all)
#pragma unroll
    for (int i = 0; i < CH; ++i)
      if (i < t.chunks)
#pragma unroll
        for (int j = 0; j < 32; ++j) l += ex2_fast(__fmul_rn(__fsub_rn(v[i][j], from), LOG2E));
    p.stats[(int64_t)(p.stat0 + 2 * w.z + t.half) * p.rows + row] = make_float2(m, l);
  }
};

// dx sums (job 0) and dw (job 1) of a piece, the longer ones first
template <int PLANES, int DZ>
struct Grads {
  static constexpr int PA = DZ, PB = PLANES;
  static constexpr bool PARTS = true, ONE = false;
  using Args = VocabArgs;
  struct Count {
    int n, mx, mw, nt, kx, kw, ux, uw;
    bool x_first;
    __device__ __forceinline__ explicit Count(const Args& p) {
      n = *p.count;
      mx = ceil_div(n, prod::BM * p.cg);
      mw = ceil_div(p.width, prod::BM * p.cg);
      nt = ceil_div(p.hidden, p.shape.bn);
      kx = ceil_div(ceil_div(p.width, prod::BK), p.splits_x);
      kw = ceil_div(ceil_div(n, prod::BK), p.splits_w);
      ux = p.want_x ? mx * nt * p.splits_x : 0;
      uw = p.want_w ? mw * nt * p.splits_w : 0;
      x_first = kx >= kw;
    }
  };
  static __device__ __forceinline__ void prefetch(const Args& p) {
    prod::prefetch_map(&p.dzk);
    prod::prefetch_map(&p.dzm);
    prod::prefetch_map(&p.wm);
    prod::prefetch_map(&p.xcm);
  }
  static __device__ __forceinline__ int count(const Args& p) {
    const Count c(p);
    return c.ux + c.uw;
  }
  static __device__ __forceinline__ void unit(const Args& p, int u, Unit& w) {
    const Count c(p);
    bool x = u < (c.x_first ? c.ux : c.uw);
    if (!x) u -= c.x_first ? c.ux : c.uw;
    x = x == c.x_first;
    const int m_n = x ? c.mx : c.mw, tiles = m_n * c.nt;
    int mt, nt;
    prod::tile_of(u % tiles, m_n, c.nt, mt, nt);
    w.z = u / tiles;
    w.job = x ? 0 : 1;
    w.m0 = w.ar = mt * prod::BM * p.cg;
    w.n0 = w.br = nt * p.shape.bn;
    w.ak = 0;
    w.az = w.bz = 0;
    w.b_mn = true;
    if (x) {
      w.a = &p.dzk;
      w.b = &p.wm;
      w.bk = p.wrow;
      w.a_mn = false;
      w.kb0 = w.z * c.kx;
      w.kb1 = min(w.kb0 + c.kx, ceil_div(p.width, prod::BK));
    } else {
      w.a = &p.dzm;
      w.b = hidden_map(p, c.n, &p.xm, &p.xcm);
      w.bk = 0;
      w.a_mn = true;
      w.kb0 = w.z * c.kw;
      w.kb1 = min(w.kb0 + c.kw, ceil_div(c.n, prod::BK));
    }
  }
  static __device__ __forceinline__ void part(const Args& p, const Unit& w, const Tile& t, Store& st, int i, float (&v)[32]) {
    const int row0 = w.m0 + t.rank * prod::BM + t.quad * 32, c = w.n0 + 32 * (t.half + 2 * i);
    if ((w.job == 1 && row0 >= p.width) || c >= p.hidden) return;
    const float ref = *p.ref;
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] *= ref;
    if (w.job == 0) st.f32_row(&p.dxs, v, c, row0, w.z, p.v0 > 0, p.hidden);
    else if (p.splits_w > 1) st.f32_row(&p.dw, v, c, row0, w.z, false, p.hidden);
    else if (p.dtype == RA_BF16) st.bf16_row(&p.dw, [&](int j) { return v[j]; }, c, p.v0 + row0, 0);
    else st.f32_row(&p.dw, v, c, p.v0 + row0, 0, false, p.hidden);
  }
};

// ---- what is joined at the end ------------------------------------------------------------
// eight tokens a CTA, 64 threads on each one's parts
__global__ void __launch_bounds__(512) vocab_join_kernel(const ra_vocab_loss_args a, const Prep p, const float2* stats, const float* zlab, int parts, int direct) {
  __shared__ float2 sh[16][8];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, k = tid & 7, r = blockIdx.x * 8 + k;
  pdl_wait();
  pdl_trigger();
  const int n = direct ? a.tokens : *p.count;
  if ((int)blockIdx.x * 8 >= n) return;
  // maximum and sum of two parts (-inf and 0, or NaN, where there is nothing, or nothing but NaN)
  auto join = [](float2 x, float2 y) {
    const float top = fmaxf(x.x, y.x);
    if (!(top > -INFINITY)) return make_float2(top, x.y + y.y);
    return make_float2(top, x.y * ex2_fast((x.x - top) * LOG2E) + y.y * ex2_fast((y.x - top) * LOG2E));
  };
  float2 s = make_float2(-INFINITY, 0.f);
  if (r < n)
    for (int i0 = tid >> 3; i0 < parts; i0 += 256) {  // four at once on their way
      float2 v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int part = i0 + 64 * i;
        v[i] = part < parts ? stats[(int64_t)part * p.rows + r] : make_float2(-INFINITY, 0.f);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) s = join(s, v[i]);
    }
#pragma unroll
  for (int o = 8; o < 32; o <<= 1) s = join(s, make_float2(__shfl_xor_sync(0xffffffffu, s.x, o), __shfl_xor_sync(0xffffffffu, s.y, o)));
  if (lane < 8) sh[warp][lane] = s;
  __syncthreads();
  if (tid >= 8 || r >= n) return;
  s = sh[0][k];
#pragma unroll
  for (int i = 1; i < 16; ++i) s = join(s, sh[i][k]);
  const float lse = s.x + logf(s.y);
  if (direct) {
    const int l = a.labels_dev[r];
    if (l >= a.vocab) set_dev_error(a.err_dev, RA_DEVERR_BOUNDS);
    a.loss_dev[r] = counted(a, l) ? lse - zlab[r] : 0.f;
    if (a.lse_dev) a.lse_dev[r] = counted(a, l) ? lse : 0.f;
    return;
  }
  const int t = p.index[r];
  a.loss_dev[t] = lse - zlab[r];
  if (a.lse_dev) a.lse_dev[t] = lse;
}

// rows of sums, added up over their parts and rounded, to where they belong
template <typename T>
__global__ void __launch_bounds__(128) vocab_sum_kernel(const float* sums, int splits, int64_t part, int pitch, int H, const int* count,
                                                        int rows, const int* index, T* out, int64_t stride) {
  pdl_wait();
  pdl_trigger();
  const int n = count ? *count : rows;
  for (int r = blockIdx.x; r < n; r += gridDim.x) {
    T* o = out + (index ? index[r] : r) * stride;
    for (int c = threadIdx.x * 4; c < H; c += 512) {
      float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int i0 = 0; i0 < splits; i0 += 8) {  // eight at once on their way
        float4 v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
          v[i] = i0 + i < splits ? *reinterpret_cast<const float4*>(sums + (i0 + i) * part + (int64_t)r * pitch + c) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          s.x += v[i].x;
          s.y += v[i].y;
          s.z += v[i].z;
          s.w += v[i].w;
        }
      }
      if (sizeof(T) == 4) {
        *reinterpret_cast<float4*>(o + c) = s;
      } else {
        __nv_bfloat162 h[2] = {__floats2bfloat162_rn(s.x, s.y), __floats2bfloat162_rn(s.z, s.w)};
        *reinterpret_cast<uint2*>(o + c) = *reinterpret_cast<uint2*>(h);
      }
    }
  }
}

// ---- few fp32 tokens ----------------------------------------------------------------------
// Up to 32 tokens in fp32 are bound by W's bytes, which its planes would be four times over (a word of 100000 x 1024 is read in
// 61 us in all; 16 tokens through planes 330 us, trained 915; here 128 and 438).  So on the CUDA cores, with the hidden states in
// shared memory, a warp four words at a time.  W is read once by the forward, and by the backward once for dz and dw and once
// for dx.  From 16 tokens on the multiply-adds bound, four to a value of shared memory (32 tokens 203 and 708 us).
constexpr int FEW = 32, FEW_WORDS = 4, FEW_THREADS = 256, FEW_SMEM = 128 * 1024;

// The sums over the warp of N (a multiple of 32) values; lane l is left with the N / 32 from l N / 32 on, in v[0], v[1], ..
template <int N>
__device__ __forceinline__ void scatter_sum(float (&v)[N], int lane) {
  int o = 16;
#pragma unroll
  for (int k = N / 2; k >= N / 32; k >>= 1, o >>= 1) {
    const bool high = lane & o;
#pragma unroll
    for (int i = 0; i < k; ++i) {
      const float give = high ? v[i] : v[i + k], keep = high ? v[i + k] : v[i];
      v[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
    }
  }
}

// Logits of words in fours; forward: each warp's maxima and sums to stats [warps][TT]; BACK: dz [vocab][TT] and dw
template <int TT, bool BACK>
__global__ void __launch_bounds__(FEW_THREADS, TT <= 16 ? 2 : 1)
    vocab_few_kernel(const __grid_constant__ ra_vocab_loss_args a, float2* stats, float* zlab, float* dz) {
  extern __shared__ __align__(16) float xs[];  // [TT][H]
  __shared__ float4 dzs[FEW_THREADS / 32][TT];
  constexpr int EACH = FEW_WORDS * TT / 32;  // logits of a lane: of tokens t0.., of word k of the four
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, H = a.hidden;
  const float* x = static_cast<const float*>(a.x_dev);
  const float* w = static_cast<const float*>(a.w_dev);
  pdl_wait();
  pdl_trigger();
  for (int i = tid; i < TT * (H / 4); i += FEW_THREADS) {
    const int t = i / (H / 4), c = i % (H / 4) * 4;
    const bool in = t < a.tokens && counted(a, a.labels_dev[t]);
    *reinterpret_cast<float4*>(xs + t * H + c) = in ? *reinterpret_cast<const float4*>(x + t * a.x_stride + c) : make_float4(0.f, 0.f, 0.f, 0.f);
  }
  __syncthreads();
  if (blockIdx.x == 0 && tid < a.tokens && a.labels_dev[tid] >= a.vocab) set_dev_error(a.err_dev, RA_DEVERR_BOUNDS);
  const int k = lane * EACH / TT, t0 = lane * EACH % TT;
  int label[EACH];
  float scale[EACH], lse[EACH], m[EACH], l[EACH];
#pragma unroll
  for (int e = 0; e < EACH; ++e) {
    const int t = t0 + e;
    label[e] = t < a.tokens ? a.labels_dev[t] : -1;
    if (!counted(a, label[e])) label[e] = -1;
    scale[e] = BACK && label[e] >= 0 ? a.dloss_dev[t] : 0.f;
    lse[e] = BACK && label[e] >= 0 ? a.lse_dev[t] : 0.f;
    m[e] = -INFINITY;
    l[e] = 0.f;
  }
  const int step = (int)gridDim.x * (FEW_THREADS / 32) * FEW_WORDS;
  for (int v0 = ((int)blockIdx.x * (FEW_THREADS / 32) + warp) * FEW_WORDS; v0 < a.vocab; v0 += step) {
    float z[FEW_WORDS * TT];
#pragma unroll
    for (int i = 0; i < FEW_WORDS * TT; ++i) z[i] = 0.f;
    auto fetch = [&](int c, float4* y) {
#pragma unroll
      for (int i = 0; i < FEW_WORDS; ++i)
        y[i] = c < H && v0 + i < a.vocab ? *reinterpret_cast<const float4*>(w + (v0 + i) * a.w_stride + c) : make_float4(0.f, 0.f, 0.f, 0.f);
    };
    float4 y[FEW_WORDS], next[FEW_WORDS];
    fetch(lane * 4, y);
    for (int c = lane * 4; c - lane * 4 < H; c += 128) {
      fetch(c + 128, next);
      if (c < H)
#pragma unroll
        for (int t = 0; t < TT; ++t) {
          const float4 h = *reinterpret_cast<const float4*>(xs + t * H + c);
#pragma unroll
          for (int i = 0; i < FEW_WORDS; ++i)
            z[i * TT + t] = fmaf(y[i].x, h.x, fmaf(y[i].y, h.y, fmaf(y[i].z, h.z, fmaf(y[i].w, h.w, z[i * TT + t]))));
        }
#pragma unroll
      for (int i = 0; i < FEW_WORDS; ++i) y[i] = next[i];
    }
    scatter_sum(z, lane);
    const int v = v0 + k;
    if (!BACK) {
#pragma unroll
      for (int e = 0; e < EACH; ++e)
        if (v < a.vocab) {
          if (v == label[e]) zlab[t0 + e] = z[e];
          const float top = fmaxf(m[e], z[e]), from = top > -INFINITY ? top : 0.f;
          l[e] = l[e] * ex2_fast(__fmul_rn(__fsub_rn(m[e], from), LOG2E)) + ex2_fast(__fmul_rn(__fsub_rn(z[e], from), LOG2E));
          m[e] = top;
        }
    } else {
      float* mine = reinterpret_cast<float*>(dzs[warp]);  // [TT][4]
      __syncwarp();
#pragma unroll
      for (int e = 0; e < EACH; ++e) {
        const float p = ex2_fast(__fmul_rn(__fsub_rn(z[e], lse[e]), LOG2E));
        const float d = label[e] < 0 ? 0.f : __fmul_rn(scale[e], v == label[e] ? __fsub_rn(p, 1.f) : p);
        mine[(t0 + e) * 4 + k] = d;
        if (a.dx_dev && v < a.vocab) dz[(int64_t)v * TT + t0 + e] = d;
      }
      __syncwarp();
      if (a.dw_dev)
        for (int c = lane * 4; c < H; c += 128) {
          float4 s[FEW_WORDS] = {};
#pragma unroll
          for (int t = 0; t < TT; ++t) {
            const float4 h = *reinterpret_cast<const float4*>(xs + t * H + c), d = dzs[warp][t];
            const float ds[4] = {d.x, d.y, d.z, d.w};
#pragma unroll
            for (int i = 0; i < FEW_WORDS; ++i) {
              s[i].x = fmaf(ds[i], h.x, s[i].x);
              s[i].y = fmaf(ds[i], h.y, s[i].y);
              s[i].z = fmaf(ds[i], h.z, s[i].z);
              s[i].w = fmaf(ds[i], h.w, s[i].w);
            }
          }
#pragma unroll
          for (int i = 0; i < FEW_WORDS; ++i)
            if (v0 + i < a.vocab) *reinterpret_cast<float4*>(static_cast<float*>(a.dw_dev) + (v0 + i) * a.dw_stride + c) = s[i];
        }
    }
  }
  if (!BACK) {
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      // lanes of the same token are those of the other words: 32 / FEW_WORDS lanes apart
#pragma unroll
      for (int o = 16; o >= 32 / FEW_WORDS; o >>= 1) {
        const float m2 = __shfl_xor_sync(0xffffffffu, m[e], o), l2 = __shfl_xor_sync(0xffffffffu, l[e], o);
        const float top = fmaxf(m[e], m2), from = top > -INFINITY ? top : 0.f;
        l[e] = l[e] * ex2_fast(__fmul_rn(__fsub_rn(m[e], from), LOG2E)) + l2 * ex2_fast(__fmul_rn(__fsub_rn(m2, from), LOG2E));
        m[e] = top;
      }
      if (k == 0) stats[((int64_t)blockIdx.x * (FEW_THREADS / 32) + warp) * TT + t0 + e] = make_float2(m[e], l[e]);
    }
  }
}

// dx of a part of the vocabulary: sums [parts][TT][pitch] of dz W; a warp 128 columns of every eighth group of words, the next
// group's rows and dz on their way
template <int TT>
__global__ void __launch_bounds__(256, TT <= 16 ? 2 : 1)
    vocab_few_dx_kernel(const __grid_constant__ ra_vocab_loss_args a, const float* dz, float* sums, int per, int pitch) {
  constexpr int AT_ONCE = TT <= 16 ? 8 : 4, PIECES = AT_ONCE * TT / 4, EACH = (PIECES + 31) / 32;  // words of a group; its dz, in fours
  __shared__ float4 sh[4][TT][32];
  __shared__ float4 dzs[8][PIECES];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 128 + lane * 4;
  pdl_wait();
  pdl_trigger();
  const int v1 = min(a.vocab, ((int)blockIdx.y + 1) * per);
  const float* w = static_cast<const float*>(a.w_dev);
  float4 s[TT];
#pragma unroll
  for (int t = 0; t < TT; ++t) s[t] = make_float4(0.f, 0.f, 0.f, 0.f);
  const float4 none = make_float4(0.f, 0.f, 0.f, 0.f);
  auto fetch = [&](int v0, float4 (&y)[AT_ONCE], float4 (&d)[EACH]) {
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) y[i] = c < a.hidden && v0 + i < v1 ? *reinterpret_cast<const float4*>(w + (v0 + i) * a.w_stride + c) : none;
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      const int i = e * 32 + lane;
      d[e] = i < PIECES && v0 + i / (TT / 4) < v1 ? reinterpret_cast<const float4*>(dz + (int64_t)v0 * TT)[i] : none;
    }
  };
  float4 y[AT_ONCE], ny[AT_ONCE], d[EACH];
  int v0 = (int)blockIdx.y * per + warp * AT_ONCE;
  fetch(v0, y, d);
  for (; v0 < v1; v0 += 8 * AT_ONCE) {
    __syncwarp();
#pragma unroll
    for (int e = 0; e < EACH; ++e)
      if (e * 32 + lane < PIECES) dzs[warp][e * 32 + lane] = d[e];
    __syncwarp();
    fetch(v0 + 8 * AT_ONCE, ny, d);
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
#pragma unroll
      for (int q = 0; q < TT / 4; ++q) {
        const float4 g = dzs[warp][i * (TT / 4) + q];
        const float gs[4] = {g.x, g.y, g.z, g.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float4& r = s[4 * q + j];
          r.x = fmaf(gs[j], y[i].x, r.x);
          r.y = fmaf(gs[j], y[i].y, r.y);
          r.z = fmaf(gs[j], y[i].z, r.z);
          r.w = fmaf(gs[j], y[i].w, r.w);
        }
      }
      y[i] = ny[i];
    }
  }
  // the eight warps' sums, halved three times
  for (int half = 4; half >= 1; half >>= 1) {
    if (warp >= half && warp < 2 * half)
#pragma unroll
      for (int t = 0; t < TT; ++t) sh[warp - half][t][lane] = s[t];
    __syncthreads();
    if (warp < half)
#pragma unroll
      for (int t = 0; t < TT; ++t) {
        const float4 o = sh[warp][t][lane];
        s[t].x += o.x;
        s[t].y += o.y;
        s[t].z += o.z;
        s[t].w += o.w;
      }
    __syncthreads();
  }
  if (warp == 0 && c < a.hidden)
#pragma unroll
    for (int t = 0; t < TT; ++t)
      if (t < a.tokens) *reinterpret_cast<float4*>(sums + ((int64_t)blockIdx.y * TT + t) * pitch + c) = s[t];
}
// the parts' sums, added up; nothing for tokens that are not counted
__global__ void __launch_bounds__(128) vocab_few_sum_kernel(const __grid_constant__ ra_vocab_loss_args a, const float* sums, int parts, int64_t part, int pitch) {
  const int t = blockIdx.y, c = (blockIdx.x * 128 + threadIdx.x) * 4;
  pdl_wait();
  pdl_trigger();
  if (c >= a.hidden) return;
  const int label = a.labels_dev[t];
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  if (counted(a, label))
    for (int i0 = 0; i0 < parts; i0 += 8) {
      float4 v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        v[i] = i0 + i < parts ? *reinterpret_cast<const float4*>(sums + (i0 + i) * part + (int64_t)t * pitch + c) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        s.x += v[i].x;
        s.y += v[i].y;
        s.z += v[i].z;
        s.w += v[i].w;
      }
    }
  *reinterpret_cast<float4*>(static_cast<float*>(a.dx_dev) + t * a.dx_stride + c) = s;
}

// ---- the plan -----------------------------------------------------------------------------
struct Plan {
  int planes, dz_planes, rows, chunk;
  int wide, pitch;                // of gathered or split rows: columns to a multiple of 8, 128-byte boundaries
  int pieces, width;              // of the vocabulary, backward (and fp32 forward)
  Pick forward, logits, grads;    // (forward: of its logits)
  int splits_x, splits_w, stats;  // parts of the statistics
  size_t count, index, label, scale, lse, ref, zlab, xc, wc, st, dz, dxs, dws, bytes;
};

constexpr int LOGITS_CHUNK = 16;  // k-blocks of an accumulator of logits, whose error is the loss's: 4e-7 of it

// (the same whether both gradients are wanted or one)
Plan plan(const ra_vocab_loss_args& a) {
  Plan p = {};
  const bool f32 = a.dtype == RA_F32;
  p.planes = f32 ? 3 : 1;
  // bf16: of one row of tiles, where W's bytes and the launches bound and not the products, dz keeps 16 bits: 107 x 359 x 664 trained
  // 29.3 -> 30.5 us, 16 x 32000 x 2048 154 -> 162, and gradients as far from 64 bits as their own rounding (0.0017; with 8 bits 0.0019 at
  // the former).  Of more tokens the second plane's products are paid for: 1024 x 32000 x 256 94 -> 129 us, 4096 x 4096 x 1024 128 -> 167
  p.dz_planes = f32 ? 3 : a.tokens <= prod::BM ? 2 : 1;
  p.chunk = f32 ? 4 : 128;
  p.rows = up(a.tokens > 0 ? a.tokens : 1, ROWS);
  p.wide = up(a.hidden, 8);
  p.pitch = up(a.hidden, 64);
  // pieces of at most 128 MB of dz
  int64_t most = (128ll << 20) / (2ll * p.dz_planes * p.rows) / 256 * 256;
  most = std::max<int64_t>(most, 256);
  p.pieces = parts_of(a.vocab, (int)std::min<int64_t>(most, 1 << 24));
  p.width = up(parts_of(a.vocab, p.pieces), 256);
  p.pieces = parts_of(a.vocab, p.width);

  const int hb = parts_of(a.hidden, prod::BK), terms = prod::terms_of(p.dz_planes, p.planes).n;
  p.logits = prod::pick(a.tokens, p.pieces == 1 || !f32 ? a.vocab : p.width, 1, hb * prod::terms_of(p.planes, p.planes).n, p.planes, p.planes);
  if (p.logits.bn < 128) p.logits.bn = 128;
  p.forward = p.logits;
  if (a.tokens <= prod::BM && !f32) {
    // few tokens: W's bytes bound, so that the tiles had best be as wide as leaves each SM with equal shares of them
    const int waves = parts_of(parts_of(a.vocab, 256), SMS);
    p.forward = {1, std::max(64, std::min(256, up(parts_of(a.vocab, waves * SMS), 32)))};
  }
  p.stats = f32 ? p.pieces * 2 * parts_of(p.width, p.forward.bn) : 2 * parts_of(a.vocab, p.forward.bn);

  const int kx = parts_of(p.width, prod::BK), kw = parts_of(a.tokens > 0 ? a.tokens : 1, prod::BK);
  double best = 1e30;
  for (Pick k : {Pick{1, 64}, Pick{1, 128}, Pick{1, 256}, Pick{2, 256}}) {
    if (k.cg == 2 && (a.tokens <= prod::BM || a.hidden <= 128)) continue;
    if (k.bn > 64 && a.hidden <= k.bn / 2) continue;
    if (!prod::takes(k, p.dz_planes, p.planes)) continue;
    const int64_t nt = parts_of(a.hidden, k.bn);
    const int64_t ux = parts_of(a.tokens, prod::BM * k.cg) * nt, uw = parts_of(p.width, prod::BM * k.cg) * nt;
    const double all = (double)ux * kx + (double)uw * kw, workers = SMS / k.cg;
    // A tile's k-blocks are cut so that none has more than about a share of a worker's part of all of them: dx, whose sums are added
    // up at the end anyway, a sixth, into parts of 16 products at least (4096 tokens, half of them counted, 657 -> 607 us against a
    // third: fewer tokens than were planned for leave its long tiles to the end), dw a third, into parts of 64
    auto cut = [&](int kb, int least, double share) { return std::max(1, std::min(std::min(16, kb * terms / least), (int)(share * kb * workers / std::max(all, 1.)))); };
    const int sx = cut(kx, 16, 6.), cw = cut(kw, 64, 3.), sw = p.pieces == 1 && (int64_t)p.width * a.hidden * 4 * cw <= (128ll << 20) ? cw : 1;
    const double longest = std::max(parts_of(kx, sx), parts_of(kw, sw));
    const double time = (std::max(all / workers, longest) + 0.3 * longest) * terms * prod::block_time(k) + (double)(ux * sx + uw * sw) / workers * 1.;
    if (time < best) {
      best = time;
      p.grads = k;
      p.splits_x = sx;
      p.splits_w = sw;
    }
  }

  size_t at = WS_ZERO;
  auto take = [&](size_t n) {
    const size_t r = at;
    at += (n + 255) / 256 * 256;
    return r;
  };
  p.count = take(4);
  p.index = take((size_t)p.rows * 4);
  p.label = take((size_t)p.rows * 4);
  p.scale = take((size_t)p.rows * 4);
  p.lse = take((size_t)p.rows * 4);
  p.ref = take(4);
  p.zlab = take((size_t)p.rows * 4);
  p.xc = take((size_t)p.planes * p.rows * p.pitch * 2);
  p.wc = take(f32 ? (size_t)3 * p.width * p.pitch * 2 : 0);
  const size_t shared = at;  // what follows is the forward's, or the backward's
  p.st = take((size_t)p.stats * p.rows * sizeof(float2));
  const size_t forward = at;
  at = shared;
  p.dz = take((size_t)p.dz_planes * p.rows * p.width * 2);
  p.dxs = take((size_t)p.splits_x * p.rows * p.pitch * 4);
  p.dws = take(p.splits_w > 1 ? (size_t)p.splits_w * p.width * p.pitch * 4 : 0);
  p.bytes = a.dx_dev || a.dw_dev ? std::max(at, forward) : forward;
  return p;
}

Prep prep_of(const Plan& p, char* ws) {
  Prep r;
  r.count = reinterpret_cast<int*>(ws + p.count);
  r.index = reinterpret_cast<int*>(ws + p.index);
  r.label = reinterpret_cast<int*>(ws + p.label);
  r.scale = reinterpret_cast<float*>(ws + p.scale);
  r.lse = reinterpret_cast<float*>(ws + p.lse);
  r.ref = reinterpret_cast<float*>(ws + p.ref);
  r.x = ws + p.xc;
  r.rows = p.rows;
  r.width = p.wide;
  r.pitch = p.pitch;
  r.planes = p.planes;
  return r;
}
Split split_of(const ra_vocab_loss_args& a, const Plan& p, char* ws, int v0, int width) {
  return {static_cast<const float*>(a.w_dev) + v0 * a.w_stride, a.w_stride, reinterpret_cast<bf16*>(ws + p.wc), width, a.hidden, p.wide, p.pitch};
}
int split_ctas(const Split& s) { return (int)std::min<int64_t>(((int64_t)s.rows * s.width / 4 + 255) / 256, 8 * SMS); }
cudaError_t prepare(const ra_vocab_loss_args& a, const Plan& p, char* ws, const Prep& r, bool backward, cudaStream_t st) {
  const int ctas = std::min(parts_of(a.tokens, 32), 2 * SMS);
  note_launch(1);
  if (a.dtype == RA_BF16) return launch_pdl(vocab_prep_kernel<bf16>, dim3(ctas), dim3(256), 0, st, a, r, (int)backward, ctas, Split{});
  const Split s = split_of(a, p, ws, 0, std::min(p.width, (int)a.vocab));
  return launch_pdl(vocab_prep_kernel<float>, dim3(ctas + split_ctas(s)), dim3(256), 0, st, a, r, (int)backward, ctas, s);
}

VocabArgs args_of(const ra_vocab_loss_args& a, const Plan& p, char* ws) {
  VocabArgs g = {};
  const Prep r = prep_of(p, ws);
  g.err = a.err_dev;
  g.count = r.count;
  g.label = r.label;
  g.scale = r.scale;
  g.lse = r.lse;
  g.ref = r.ref;
  g.stats = reinterpret_cast<float2*>(ws + p.st);
  g.zlab = reinterpret_cast<float*>(ws + p.zlab);
  g.tokens = a.tokens;
  g.hidden = a.hidden;
  g.rows = p.rows;
  g.planes = p.planes;
  g.dtype = a.dtype;
  return g;
}
#define MAP(m, ...)                                                        \
  do {                                                                     \
    if (!tma_map_3d(&(m), __VA_ARGS__)) return cudaErrorInvalidValue;      \
  } while (0)

// the piece's W, K-major boxes of bn rows or MN-major ones of 64; fp32: its planes, made first
// (the first piece's by the launch that numbers the tokens)
cudaError_t piece(const ra_vocab_loss_args& a, const Plan& p, char* ws, VocabArgs& g, int v0, int width, cudaStream_t st) {
  g.v0 = v0;
  g.width = width;
  g.wrow = p.planes == 1 ? v0 : 0;
  if (p.planes == 1 || v0 == 0) return cudaSuccess;
  const Split s = split_of(a, p, ws, v0, width);
  note_launch(1);
  return launch_pdl(vocab_split_kernel, dim3(split_ctas(s)), dim3(256), 0, st, s);
}
cudaError_t w_map(const ra_vocab_loss_args& a, const Plan& p, char* ws, CUtensorMap& m, int width, int box_rows) {
  if (p.planes == 1) MAP(m, a.w_dev, DT_BF16, 1, a.vocab, a.hidden, a.w_stride, 64, box_rows);
  else MAP(m, ws + p.wc, DT_BF16, 3, width, p.wide, p.pitch, 64, box_rows);
  return cudaSuccess;
}
#define DO(x)                                \
  do {                                       \
    const cudaError_t _e = (x);              \
    if (_e != cudaSuccess) return _e;        \
  } while (0)

template <class P>
cudaError_t products(const VocabArgs& g, int64_t units, cudaStream_t st) {
  const int n = (int)std::min<int64_t>(units, 1 << 20);
  return prod::launch<P>(g, g.cg, n, st);
}
// hidden states as given (bf16) and gathered, in boxes of box_rows rows
cudaError_t x_maps(const ra_vocab_loss_args& a, const Plan& p, char* ws, CUtensorMap& given, CUtensorMap& gathered, int box_rows) {
  if (p.planes == 1) MAP(given, a.x_dev, DT_BF16, 1, a.tokens, a.hidden, a.x_stride, 64, box_rows);
  MAP(gathered, ws + p.xc, DT_BF16, p.planes, p.rows, p.wide, p.pitch, 64, box_rows);
  return cudaSuccess;
}

template <int PLANES>
cudaError_t forward(const ra_vocab_loss_args& a, cudaStream_t st) {
  const Plan p = plan(a);
  char* ws = static_cast<char*>(a.workspace_dev);
  const Prep r = prep_of(p, ws);
  VocabArgs g = args_of(a, p, ws);
  g.cg = p.forward.cg;
  g.shape = prod::shape_of(p.forward.bn, p.forward.cg, p.planes, p.planes, std::min(p.chunk, LOGITS_CHUNK));
  // (what may be refused, before anything is enqueued)
  DO(x_maps(a, p, ws, g.x, g.xc, prod::BM));
  if (p.planes == 1) DO(w_map(a, p, ws, g.w, a.vocab, p.forward.bn / p.forward.cg));
  // few tokens in bf16 are one tile's rows, counted or not: their logits need no numbering
  const bool direct = p.planes == 1 && a.tokens <= prod::BM;
  if (direct) {
    g.count = nullptr;
    g.label = a.labels_dev;
  } else {
    DO(prepare(a, p, ws, r, false, st));
  }
  const int step = p.planes == 1 ? a.vocab : p.width;
  for (int v0 = 0; v0 < a.vocab; v0 += step) {
    const int width = std::min(step, a.vocab - v0);
    DO(piece(a, p, ws, g, v0, width, st));
    if (p.planes > 1) DO(w_map(a, p, ws, g.w, width, p.forward.bn / p.forward.cg));
    const int64_t tiles = (int64_t)parts_of(a.tokens, prod::BM * g.cg) * parts_of(width, g.shape.bn);
    DO((products<Logits<false, PLANES, PLANES>>(g, tiles, st)));
    g.stat0 += 2 * parts_of(width, g.shape.bn);
  }
  note_launch(1);
  return launch_pdl(vocab_join_kernel, dim3(parts_of(a.tokens, 8)), dim3(512), 0, st, a, r, (const float2*)g.stats, (const float*)g.zlab, (int)g.stat0, (int)direct);
}

template <typename T, int PLANES, int DZ>
cudaError_t backward(const ra_vocab_loss_args& a, cudaStream_t st) {
  const Plan p = plan(a);
  char* ws = static_cast<char*>(a.workspace_dev);
  const Prep r = prep_of(p, ws);
  VocabArgs g = args_of(a, p, ws), h;
  g.want_x = a.dx_dev != nullptr;
  g.want_w = a.dw_dev != nullptr;
  g.splits_x = p.splits_x;
  g.splits_w = p.splits_w;
  DO(x_maps(a, p, ws, g.x, g.xc, prod::BM));
  DO(x_maps(a, p, ws, g.xm, g.xcm, 64));
  MAP(g.dxs, ws + p.dxs, DT_F32, p.splits_x, p.rows, a.hidden, p.pitch, 16, 32);
  if (a.dw_dev) {
    if (p.splits_w > 1) MAP(g.dw, ws + p.dws, DT_F32, p.splits_w, p.width, a.hidden, p.pitch, 16, 32);
    else MAP(g.dw, a.dw_dev, a.dtype, 1, a.vocab, a.hidden, a.dw_stride, a.dtype == RA_BF16 ? 32 : 16, 32);
  }
  h = g;
  g.cg = p.logits.cg;
  g.shape = prod::shape_of(p.logits.bn, p.logits.cg, p.planes, p.planes, std::min(p.chunk, LOGITS_CHUNK));
  h.cg = p.grads.cg;
  h.shape = prod::shape_of(p.grads.bn, p.grads.cg, DZ, p.planes, p.chunk);
  if (p.planes == 1) {
    DO(w_map(a, p, ws, g.w, a.vocab, p.logits.bn / p.logits.cg));
    DO(w_map(a, p, ws, h.wm, a.vocab, 64));
  }
  DO(prepare(a, p, ws, r, true, st));
  for (int v0 = 0; v0 < a.vocab; v0 += p.width) {
    const int width = std::min(p.width, a.vocab - v0);
    DO(piece(a, p, ws, g, v0, width, st));
    if (p.planes > 1) DO(w_map(a, p, ws, g.w, width, p.logits.bn / p.logits.cg));
    MAP(g.dz, ws + p.dz, DT_BF16, DZ, p.rows, p.width, p.width, 32, 32);
    const int64_t tiles = (int64_t)parts_of(a.tokens, prod::BM * g.cg) * parts_of(width, g.shape.bn);
    DO((products<Logits<true, PLANES, DZ>>(g, tiles, st)));
    h.v0 = v0;
    h.width = width;
    h.wrow = g.wrow;
    if (p.planes > 1) DO(w_map(a, p, ws, h.wm, width, 64));
    MAP(h.dzk, ws + p.dz, DT_BF16, DZ, p.rows, p.width, p.width, 64, prod::BM);
    MAP(h.dzm, ws + p.dz, DT_BF16, DZ, p.rows, p.width, p.width, 64, 64);
    const int64_t nt = parts_of(a.hidden, h.shape.bn);
    DO((products<Grads<PLANES, DZ>>(h, nt * ((h.want_x ? (int64_t)parts_of(a.tokens, prod::BM * h.cg) * h.splits_x : 0) +
                                (h.want_w ? (int64_t)parts_of(width, prod::BM * h.cg) * h.splits_w : 0)), st)));
  }
  if (a.dw_dev && p.splits_w > 1) {
    note_launch(1);
    DO(launch_pdl(vocab_sum_kernel<T>, dim3(std::min(a.vocab, 8 * SMS)), dim3(128), 0, st, (const float*)(ws + p.dws), p.splits_w,
                  (int64_t)p.width * p.pitch, p.pitch, (int)a.hidden, (const int*)nullptr, (int)a.vocab, (const int*)nullptr,
                  static_cast<T*>(a.dw_dev), a.dw_stride));
  }
  if (a.dx_dev) {
    note_launch(1);
    DO(launch_pdl(vocab_sum_kernel<T>, dim3(std::min(a.tokens, 8 * SMS)), dim3(128), 0, st, (const float*)(ws + p.dxs), p.splits_x,
                  (int64_t)p.rows * p.pitch, p.pitch, (int)a.hidden, (const int*)r.count, 0, (const int*)r.index,
                  static_cast<T*>(a.dx_dev), a.dx_stride));
  }
  return cudaSuccess;
}

// ---- few fp32 tokens: the plan and the launches --------------------------------------------
struct FewPlan {
  int tt, ctas, parts, per;  // tokens, CTAs of the logits; parts of the vocabulary for dx, words of one
  size_t stats, zlab, dz, sums, bytes;
};
bool few(const ra_vocab_loss_args& a) {
  const int tt = a.tokens <= 8 ? 8 : a.tokens <= 16 ? 16 : FEW;
  return a.dtype == RA_F32 && a.tokens >= 1 && a.tokens <= FEW && (int64_t)tt * a.hidden * 4 <= FEW_SMEM;
}
FewPlan few_plan(const ra_vocab_loss_args& a) {
  FewPlan p;
  p.tt = a.tokens <= 8 ? 8 : a.tokens <= 16 ? 16 : FEW;
  const int smem = p.tt * a.hidden * 4, each = p.tt <= 16 && smem <= 96 * 1024 ? 2 : 1;
  p.ctas = std::min(parts_of(a.vocab, FEW_WORDS * FEW_THREADS / 32), SMS * each);
  const int blocks = parts_of(a.hidden, 128);
  p.per = up(parts_of(a.vocab, std::max(1, std::min(2 * SMS / blocks, parts_of(a.vocab, 64)))), 8);
  p.parts = parts_of(a.vocab, p.per);
  size_t at = WS_ZERO;
  auto take = [&](size_t n) {
    const size_t r = at;
    at += (n + 255) / 256 * 256;
    return r;
  };
  p.zlab = take((size_t)p.tt * 4);
  p.stats = take((size_t)p.ctas * (FEW_THREADS / 32) * p.tt * sizeof(float2));
  const bool train = a.dx_dev || a.dw_dev;
  p.dz = take(train ? (size_t)a.vocab * p.tt * 4 : 0);
  p.sums = take(train ? (size_t)p.parts * p.tt * up(a.hidden, 4) * 4 : 0);
  p.bytes = at;
  return p;
}
template <int TT>
cudaError_t few_run(const ra_vocab_loss_args& a, bool backward, cudaStream_t st) {
  const FewPlan p = few_plan(a);
  char* ws = static_cast<char*>(a.workspace_dev);
  float2* stats = reinterpret_cast<float2*>(ws + p.stats);
  float *zlab = reinterpret_cast<float*>(ws + p.zlab), *dz = reinterpret_cast<float*>(ws + p.dz), *sums = reinterpret_cast<float*>(ws + p.sums);
  static const cudaError_t attr = [] {
    const cudaError_t e = allow_smem(vocab_few_kernel<TT, false>, FEW_SMEM);
    return e == cudaSuccess ? allow_smem(vocab_few_kernel<TT, true>, FEW_SMEM) : e;
  }();
  if (attr != cudaSuccess) return attr;
  const size_t smem = (size_t)TT * a.hidden * 4;
  if (!backward) {
    note_launch(2);
    DO(launch_pdl(vocab_few_kernel<TT, false>, dim3(p.ctas), dim3(FEW_THREADS), smem, st, a, stats, zlab, (float*)nullptr));
    Prep r = {};
    r.rows = TT;
    return launch_pdl(vocab_join_kernel, dim3(parts_of(a.tokens, 8)), dim3(512), 0, st, a, r, (const float2*)stats, (const float*)zlab,
                      p.ctas * (FEW_THREADS / 32), 1);
  }
  note_launch(1);
  DO(launch_pdl(vocab_few_kernel<TT, true>, dim3(p.ctas), dim3(FEW_THREADS), smem, st, a, stats, zlab, dz));
  if (!a.dx_dev) return cudaSuccess;
  const int blocks = parts_of(a.hidden, 128), pitch = up(a.hidden, 4);
  note_launch(2);
  DO(launch_pdl(vocab_few_dx_kernel<TT>, dim3(blocks, p.parts), dim3(256), 0, st, a, (const float*)dz, sums, p.per, pitch));
  return launch_pdl(vocab_few_sum_kernel, dim3(parts_of(a.hidden, 512), a.tokens), dim3(128), 0, st, a, (const float*)sums, p.parts,
                    (int64_t)TT * pitch, pitch);
}
cudaError_t few_any(const ra_vocab_loss_args& a, bool backward, cudaStream_t st) {
  return a.tokens <= 8 ? few_run<8>(a, backward, st) : a.tokens <= 16 ? few_run<16>(a, backward, st) : few_run<FEW>(a, backward, st);
}

}  // namespace

void vocab_loss_plan(const ra_vocab_loss_args& a, int32_t (&out)[12]) {
  const Plan p = plan(a);
  int32_t* at = out;
  for (int v : {(int)few(a), p.planes, p.pieces, p.width, p.forward.cg, p.forward.bn, p.logits.cg, p.logits.bn, p.grads.cg, p.grads.bn, p.splits_x,
                p.splits_w})
    *at++ = v;
}
size_t vocab_loss_workspace(const ra_vocab_loss_args& a) { return few(a) ? few_plan(a).bytes : plan(a).bytes; }
cudaError_t vocab_loss_fwd(const ra_vocab_loss_args& a, cudaStream_t st) {
  if (few(a)) return few_any(a, false, st);
  return a.dtype == RA_BF16 ? forward<1>(a, st) : forward<3>(a, st);
}
cudaError_t vocab_loss_bwd(const ra_vocab_loss_args& a, cudaStream_t st) {
  if (a.tokens == 0) {
    const size_t es = a.dtype == RA_BF16 ? 2 : 4;
    return cudaMemset2DAsync(a.dw_dev, a.dw_stride * es, 0, a.hidden * es, a.vocab, st);
  }
  if (few(a)) return few_any(a, true, st);
  if (a.dtype == RA_F32) return backward<float, 3, 3>(a, st);
  return plan(a).dz_planes == 2 ? backward<bf16, 1, 2>(a, st) : backward<bf16, 1, 1>(a, st);
}

}  // namespace ra
