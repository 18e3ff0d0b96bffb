// window_tc.cuh -- what the windowed attention kernels share: TMA of 64-column boxes of one sequence, products with an A
// operand in TMEM, and barriers of a part of the CTA.
#pragma once

#include <cuda.h>

#include "tcgen05.cuh"

namespace ra {
namespace tc {

__device__ __forceinline__ void tma_load3(const CUtensorMap* tm, uint32_t dst, uint64_t* bar, int c0, int c1, int c2) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst), "l"(reinterpret_cast<uint64_t>(tm)), "r"(c0), "r"(c1), "r"(c2),
      "r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void tma_load4(const CUtensorMap* tm, uint32_t dst, uint64_t* bar, int c0, int c1, int c2, int c3) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst), "l"(reinterpret_cast<uint64_t>(tm)), "r"(c0), "r"(c1), "r"(c2), "r"(c3),
      "r"(smem_u32(bar)) : "memory");
}
// The low words of the operands' descriptors (address and leading byte offset), in a uniform register, and the whole: what
// a product's issue costs is the moves of its operands into uniform registers, so that a base goes there once and steps
// are added to it (the address is the lowest field; 16 bytes count one)
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return __shfl_sync(0xffffffffu, x, 0); }
__device__ __forceinline__ uint32_t desc_lo_k(uint32_t saddr) { return uniform(((saddr & 0x3FFFFu) >> 4) | (1u << 16)); }
__device__ __forceinline__ uint32_t desc_lo_mn(uint32_t saddr, uint32_t lbo) { return uniform(((saddr & 0x3FFFFu) >> 4) | (((lbo >> 4) & 0x3FFFu) << 16)); }
__device__ __forceinline__ uint64_t desc_of(uint32_t lo) { return ((uint64_t)((1024u >> 4) | (1u << 14) | (2u << 29)) << 32) | lo; }
// D[tmem] (+)= A[tmem, 128 x 16 bf16] B
__device__ __forceinline__ void umma_bf16_ts(uint32_t d, uint32_t a, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\n"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(d), "r"(a), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(addr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
      "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
__device__ __forceinline__ void tmem_st8(uint32_t addr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]),
               "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ uint32_t pk2(float a, float b) {
  __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<uint32_t*>(&h);
}
// Four 16-byte pieces a lane, of four lanes' rows in turn: afterwards piece i is row (lane & ~3) + i's, its (lane & 3)-th.  A
// store of a piece a lane then writes 64 bytes of each of eight rows, where a row a lane it would touch 32 lines
__device__ __forceinline__ void transpose4(uint32_t* w, int lane) {
#pragma unroll
  for (int b = 1; b < 4; b <<= 1)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (!(i & b))
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          uint32_t &lo = w[4 * i + e], &hi = w[4 * (i | b) + e];
          const uint32_t got = __shfl_xor_sync(0xffffffffu, lane & b ? lo : hi, b);
          if (lane & b) lo = got;
          else hi = got;
        }
}
__device__ __forceinline__ void named_sync(int id, int threads) {
  asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}
// bits 0 .. n - 1
__device__ __forceinline__ uint32_t below(int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1u; }
// The rows from `dead` on of a [128][DH] operand block (64-wide swizzle atoms of [128][128 bytes]) become zero, by one warp:
// memory past a sequence's end may hold anything, and 0 times NaN is not 0
template <int DH>
__device__ __forceinline__ void zero_rows(uint8_t* block, int dead, int lane) {
  for (int e = lane; e < (128 - dead) * (DH / 8); e += 32) {
    const int r = dead + e / (DH / 8), c = e % (DH / 8);
    *reinterpret_cast<uint4*>(block + (c >> 3) * (128 * 128) + r * 128 + ((c & 7) << 4)) = make_uint4(0, 0, 0, 0);
  }
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  __syncwarp();
}

}  // namespace tc
}  // namespace ra
