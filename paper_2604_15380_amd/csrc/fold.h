// The norms' reverse passes: the blocks' partial column sums added, in the
// order of the blocks.
#pragma once

#include "ops.h"

namespace ops {

// part [n][2][cols]: the sums of its rows 0 to dgamma (blockIdx.y = 0), 1 to
// dbeta (1): 32 columns per block at a time, the partial rows in 32 slices, in S.
template <class T, class S>
__global__ void __launch_bounds__(1024) k_fold(int n, int cols, const float* __restrict__ part, T* __restrict__ dgamma,
                                               T* __restrict__ dbeta) {
  __shared__ S s[32][33];
  const int q = threadIdx.x >> 5, l = threadIdx.x & 31;
  for (int c0 = blockIdx.x * 32; c0 < cols; c0 += gridDim.x * 32) {
    const int c = c0 + l;
    S a = 0;
    if (c < cols) {
#pragma unroll 8
      for (int k = q; k < n; k += 32) a += part[((size_t)k * 2 + blockIdx.y) * cols + c];
    }
    s[q][l] = a;
    __syncthreads();
    if (q == 0 && c < cols) {
      a = 0;
#pragma unroll
      for (int k = 0; k < 32; ++k) a += s[k][l];
      const float sum = (float)a;
      store<1>((blockIdx.y ? dbeta : dgamma) + c, &sum);
    }
    __syncthreads();
  }
}

template <class T, class S>
void fold_columns(hipStream_t stream, int n, int cols, const float* part, T* dgamma, T* dbeta) {
  constexpr int most = 65536;       // blocks along the columns
  const long long blocks = ((long long)cols + 31) / 32;
  k_fold<T, S><<<dim3((unsigned)(blocks < most ? blocks : most), 2), 1024, 0, stream>>>(n, cols, part, dgamma, dbeta);
}

}  // namespace ops
