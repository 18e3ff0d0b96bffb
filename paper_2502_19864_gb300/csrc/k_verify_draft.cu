// k_verify_draft.cu -- verification of drafted tokens against the target's probabilities.
//
// With p the target's and q the draft's probabilities and u uniform in [0, 1): drafted token x stands when
// u q(x) < p(x), that is with probability min(1, p(x) / q(x)); the first that does not is replaced by a sample of
// max(p - q, 0) / sum, and after all of them comes a sample of p.  For e_v independent and exponentially
// distributed argmax_v r_v / e_v is v with probability r_v / sum r, so a sample needs no sum and no order of
// summation: what comes out is a maximum, the same whichever CTA finds it first.
//
// Of all the probabilities one row of p, one of q and the noise are read, and two values of every drafted place.
// Bound by these reads where the batch is large and by latency where it is small: a sequence's row is cut over
// several CTAs so that the batch fills the SMs once; each finds n for itself, and the last of them to finish (a
// counter) writes the answer and leaves its slot zero.  64 bf16 sequences of 50001 words and 8 drafts: 10.0 us, of it
// three rounds of a thread's 21 tokens, eight at once; one fp32 sequence of 32000 and 4 drafts: 4.2 us.
#include "common.cuh"
#include "operators.h"

namespace ra {
namespace {

constexpr int VT = 128, UN = 8;  // threads; tokens a thread has on their way

// larger score first, then the lower token: a maximum of these is the answer
__device__ __forceinline__ unsigned long long packed(float score, uint32_t v) {
  return ((unsigned long long)__float_as_uint(score) << 32) | (0xffffffffu - v);
}
__device__ __forceinline__ unsigned long long max64(unsigned long long a, unsigned long long b) { return a > b ? a : b; }

// The largest r / e of tokens [v0, v1), from every thread.  Each thread has UN tokens on their way at once; `ready`: the
// noise of the first UN is in e.  The quotient is computed where it can be the largest yet: x / e rounds to more than
// top only if x > top e, and then x is no less than the rounded top e, as rounding keeps the order and x is a float.
template <typename T, bool DIFF>
__device__ unsigned long long race(const T* __restrict__ p, const T* __restrict__ q, const float* __restrict__ noise,
                                   int v0, int v1, float (&e)[UN], bool ready) {
  unsigned long long best = packed(0.f, (uint32_t)v0);
  float top = 0.f;
  for (int base = v0 + (int)threadIdx.x; base < v1; base += VT * UN) {
    float r[UN], d[UN];
#pragma unroll
    for (int i = 0; i < UN; ++i) {
      const int v = base + VT * i;
      r[i] = v < v1 ? to_f(p[v]) : 0.f;
      d[i] = DIFF && v < v1 ? to_f(q[v]) : 0.f;
      if (!ready) e[i] = v < v1 ? noise[v] : 1.f;
    }
    ready = false;
#pragma unroll
    for (int i = 0; i < UN; ++i) {
      float x = fmaxf(r[i], 0.f);  // (a NaN counts as 0)
      if (DIFF) x = fmaxf(x - fmaxf(d[i], 0.f), 0.f);
      if (x > 0.f && x >= top * e[i]) {
        const float s = fmaxf(__fdiv_rn(x, e[i]), 0.f);
        if (s > top) {  // a thread's tokens rise: of equal ones the first stays
          top = s;
          best = packed(s, (uint32_t)(base + VT * i));
        }
      }
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) best = max64(best, __shfl_xor_sync(0xffffffffu, best, o));
  __shared__ unsigned long long warp_best[VT / 32];
  __syncthreads();
  if ((threadIdx.x & 31) == 0) warp_best[threadIdx.x >> 5] = best;
  __syncthreads();
  best = warp_best[0];
#pragma unroll
  for (int i = 1; i < VT / 32; ++i) best = max64(best, warp_best[i]);
  return best;
}

struct VerifySlot {  // of a sequence that is cut, zero between calls
  unsigned long long best;
  unsigned done, pad;
};
static_assert(sizeof(VerifySlot) * WS_SLOTS == WS_ZERO - WS_SLOTS_AT, "the slots' place in a workspace");

template <typename T>
__global__ void __launch_bounds__(VT, 8) verify_draft_kernel(const __grid_constant__ ra_verify_draft_args a, int parts, int per_part) {
  pdl_wait();
  pdl_trigger();
  const int part = blockIdx.x % parts, b = blockIdx.x / parts, tid = threadIdx.x, lane = tid & 31;
  const int K = a.n_draft, V = a.vocab;
  int nd = a.n_drafted_dev ? a.n_drafted_dev[b] : K;
  nd = nd < 0 ? 0 : nd > K ? K : nd;
  // the noise does not wait for n
  const float* noise = a.noise_dev + (int64_t)b * V;
  const int v0 = part * per_part, v1 = v0 + per_part < V ? v0 + per_part : V;
  float e[UN];
#pragma unroll
  for (int i = 0; i < UN; ++i) e[i] = v0 + VT * i + tid < v1 ? noise[v0 + VT * i + tid] : 1.f;
  const T* target = (const T*)a.target_dev + (int64_t)b * (K + 1) * a.target_stride;
  const T* draft = (const T*)a.draft_dev + (int64_t)b * K * a.draft_stride;
  // every warp finds n: the first drafted token that does not stand
  int n = nd;
  for (int base = 0; base < nd; base += 32) {
    const int i = base + lane;
    bool falls = false;
    if (i < nd) {
      const int x = a.tokens_dev[(int64_t)b * K + i];
      falls = true;
      if ((uint32_t)x < (uint32_t)V) {
        const float p = fmaxf(to_f(target[(int64_t)i * a.target_stride + x]), 0.f);
        const float q = fmaxf(to_f(draft[(int64_t)i * a.draft_stride + x]), 0.f);
        // The sign of the exact u q - p.  Where that is not 0, u q is a multiple of 2^-197 if it is near a p (of 2^-149 at
        // least): times 2^64 the difference is not lost below the least float
        const float s = 0x1p64f;
        falls = !(fmaf(a.uniform_dev[(int64_t)b * K + i] * s, q, -p * s) < 0.f);
      }
    }
    const uint32_t f = __ballot_sync(0xffffffffu, falls);
    if (f) {
      n = base + __ffs(f) - 1;
      break;
    }
  }
  const T* p = target + (int64_t)n * a.target_stride;
  const T* q = draft + (int64_t)n * a.draft_stride;
  unsigned long long best = n < nd ? race<T, true>(p, q, noise, v0, v1, e, true) : race<T, false>(p, q, noise, v0, v1, e, true);
  if (parts > 1) {
    VerifySlot* slot = (VerifySlot*)((char*)a.workspace_dev + WS_SLOTS_AT) + b;
    __shared__ bool last;
    __shared__ unsigned long long all;
    if (tid == 0) {
      atomicMax(&slot->best, best);
      __threadfence();
      last = atomicAdd(&slot->done, 1u) == (unsigned)parts - 1;
      if (last) {
        __threadfence();
        all = atomicExch(&slot->best, 0ull);
        slot->done = 0;
      }
    }
    __syncthreads();
    if (!last) return;
    best = all;
  }
  if (n < nd && (best >> 32) == 0) best = race<T, false>(p, q, noise, 0, V, e, false);  // p is nowhere above q
  const int32_t next = (int32_t)(0xffffffffu - (uint32_t)best);
  if (tid == 0) a.accepted_dev[b] = n;
  for (int i = tid; i <= K; i += VT)
    a.out_tokens_dev[(int64_t)b * (K + 1) + i] = i < n ? a.tokens_dev[(int64_t)b * K + i] : i == n ? next : -1;
}

}  // namespace

size_t verify_draft_workspace(const ra_verify_draft_args&) { return WS_ZERO; }

cudaError_t verify_draft(const ra_verify_draft_args& a, cudaStream_t st) {
  // the SMs filled once, with eight small CTAs each (64 rows of 50001: three of 512 threads 10.7 us, four of 256 10.0, these 9.9; a
  // second round of a few CTAs 13.6), none with fewer than four tokens a thread.  From 609 sequences on, with 152 SMs, none is
  // cut; none may be beyond the slots
  const int want = 8 * device_sm_count() / a.batch, most = (a.vocab + 4 * VT - 1) / (4 * VT);
  int parts = want < 1 || a.batch > WS_SLOTS ? 1 : want < most ? want : most;
  const int per = (a.vocab + parts - 1) / parts;
  parts = (a.vocab + per - 1) / per;
  const dim3 grid((unsigned)parts * (unsigned)a.batch);
  if ((int64_t)parts * a.batch > INT32_MAX) return cudaErrorNotSupported;
  cudaError_t e = a.dtype == RA_BF16 ? launch_pdl(verify_draft_kernel<bf16>, grid, dim3(VT), 0, st, a, parts, per)
                                     : launch_pdl(verify_draft_kernel<float>, grid, dim3(VT), 0, st, a, parts, per);
  note_launch(1);
  return e;
}

}  // namespace ra
