// Full-data risk from logits that a 4-bit product left as z [R C][rows] (row r C + c: class c of replica r): per replica and segment of
// rows an fp64 partial sum of the losses, then the segments in order.  Bound by reading z once.
#pragma once
#include "linear_kernel.cuh"

namespace ssim {

constexpr int MXE_SEG = 4096;       // rows of a partial sum

__global__ void __launch_bounds__(256) mx_loss_kernel(const float* z, long long ldz, const void* y, int model, int C, long long row0, int rows, double* partial,
                                                      int segments, int first_segment) {
  __shared__ double sum_s[256];
  const int r = blockIdx.y, seg = blockIdx.x, begin = seg * MXE_SEG, end = min(rows, begin + MXE_SEG);
  const float* zr = z + (long long)r * C * ldz;
  double s = 0.0;
  for (int i = begin + threadIdx.x; i < end; i += 256) {
    if (model == M_LSQ) {
      const float e = zr[i] - static_cast<const float*>(y)[row0 + i];
      s += (double)(0.5f * e * e);
    } else if (model == M_LOGISTIC) {
      const float v = zr[i], b = (float)static_cast<const int*>(y)[row0 + i];
      s += (double)(fmaxf(v, 0.f) + log1pf(expf(-fabsf(v))) - b * v);
    } else {
      float top = zr[i];
      for (int c = 1; c < C; ++c) top = fmaxf(top, zr[(long long)c * ldz + i]);
      float e = 0.f;
      for (int c = 0; c < C; ++c) e += expf(zr[(long long)c * ldz + i] - top);
      s += (double)(top + logf(e) - zr[(long long)static_cast<const int*>(y)[row0 + i] * ldz + i]);
    }
  }
  sum_s[threadIdx.x] = s;
  __syncthreads();
  for (int off = 128; off > 0; off >>= 1) {
    if ((int)threadIdx.x < off) sum_s[threadIdx.x] += sum_s[threadIdx.x + off];
    __syncthreads();
  }
  if (threadIdx.x == 0) partial[(long long)r * segments + first_segment + seg] = sum_s[0];
}

__global__ void mx_loss_finish_kernel(const double* partial, int segments, long long n, int R, float* loss) {
  const int r = blockIdx.x * blockDim.x + threadIdx.x;
  if (r >= R) return;
  double s = 0.0;
  for (int k = 0; k < segments; ++k) s += partial[(long long)r * segments + k];
  loss[r] = (float)(s / (double)n);
}

}  // namespace ssim
