// Logits of consecutive samples under one replica's parameters, for the log probabilities of the softmax and MLP models.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "../../include/straggler_sim.h"

namespace ssim {

// z[i][c] = bias[c] + sum_j x[i][j] w[c sc + j sj] in fp32.  A warp takes four rows, a lane every 32nd feature: the rows are read once, the parameters of
// up to sixteen classes once for four rows, from L1 and L2.
__global__ void __launch_bounds__(256) row_logits_kernel(const float* x, long long rows, int d, const float* w, int sc, int sj, const float* bias, int C, float* z) {
  const int lane = threadIdx.x & 31;
  const long long row0 = 4 * ((long long)blockIdx.x * 8 + (threadIdx.x >> 5));
  if (row0 >= rows) return;
  float acc[4][SIM_MAX_CLASSES];
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int c = 0; c < SIM_MAX_CLASSES; ++c) acc[r][c] = 0.f;
  for (int j = lane; j < d; j += 32) {
    float v[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = row0 + r < rows ? x[(row0 + r) * d + j] : 0.f;
#pragma unroll
    for (int c = 0; c < SIM_MAX_CLASSES; ++c) {
      if (c >= C) break;
      const float p = w[(long long)c * sc + (long long)j * sj];
#pragma unroll
      for (int r = 0; r < 4; ++r) acc[r][c] = fmaf(v[r], p, acc[r][c]);
    }
  }
#pragma unroll
  for (int c = 0; c < SIM_MAX_CLASSES; ++c) {
    if (c >= C) break;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      float s = acc[r][c];
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
      if (lane == 0 && row0 + r < rows) z[(row0 + r) * C + c] = s + (bias ? bias[c] : 0.f);
    }
  }
}

__global__ void __launch_bounds__(256) round_bf16_kernel(const float* x, long long n, __nv_bfloat16* out) {
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256) out[i] = __float2bfloat16_rn(x[i]);
}

}  // namespace ssim
