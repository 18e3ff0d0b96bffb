// simt_tile.cuh -- a 64 x 64 tile of a product in fp32 on the CUDA cores, with operands and results through functions.
#pragma once

#include "common.cuh"

namespace ra {

constexpr int ST_THREADS = 256;
struct SimtTile {
  float a[16][68], b[16][68];
};
// acc[i][j] += sum_k A(m0 + 4 ty + i, k) B(n0 + 4 tx + j, k) over [k0, k1), with tx = thread % 16 and ty = thread / 16; A and B
// give 0 outside their operands.  ka, kb: whether k is the operand's contiguous index.
template <bool KA, bool KB, typename FA, typename FB>
__device__ __forceinline__ void simt_tile(SimtTile& sh, float (&acc)[4][4], int m0, int n0, int k0, int k1, FA A, FB B) {
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
  for (int kk = k0; kk < k1; kk += 16) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int e = tid + 256 * i;
      const int ak = KA ? e & 15 : e >> 6, am = KA ? e >> 4 : e & 63;
      sh.a[ak][am] = kk + ak < k1 ? A(m0 + am, kk + ak) : 0.f;
      const int bk = KB ? e & 15 : e >> 6, bn = KB ? e >> 4 : e & 63;
      sh.b[bk][bn] = kk + bk < k1 ? B(n0 + bn, kk + bk) : 0.f;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      const float4 x = *reinterpret_cast<const float4*>(&sh.a[k][4 * ty]);
      const float4 y = *reinterpret_cast<const float4*>(&sh.b[k][4 * tx]);
      const float xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(xs[i], ys[j], acc[i][j]);
    }
  }
}

}  // namespace ra
