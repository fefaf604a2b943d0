// The arithmetic of one AdamW step (formulas: adamw_kernel.cuh), shared by the step over a list of tensors and by the simulated
// server's update.
#pragma once
#include <cuda_runtime.h>

namespace ssim {

// What a step multiplies with.  The mean over pushes is folded in: c1 = (1 - b1) grad_scale / K and s2 = sqrt(1 - b2) grad_scale / K,
// so that m' = b1 m + c1 G and v' = b2 v + (s2 G)^2 with G the plain sum; sb2 = sqrt(b2) does the same for r: v' = (sb2 r)^2 + (s2 G)^2.
struct AdamwCoef { float b1, c1, b2, sb2, s2, lr, lr_bc1, rbc2, eps; };

__host__ __device__ inline AdamwCoef adamw_coef(double beta1, double beta2, float eps, double mean, float lr, long long step) {
  AdamwCoef c;
  c.b1 = (float)beta1; c.c1 = (float)((1.0 - beta1) * mean); c.b2 = (float)beta2; c.sb2 = (float)sqrt(beta2); c.s2 = (float)(sqrt(1.0 - beta2) * mean);
  c.lr = lr; c.eps = eps;
  // 1 - beta^t without cancellation for small t and beta near 1 (beta = 0: 1)
  const double bc1 = beta1 > 0.0 ? -expm1((double)step * log(beta1)) : 1.0, bc2 = beta2 > 0.0 ? -expm1((double)step * log(beta2)) : 1.0;
  c.lr_bc1 = (float)((double)lr / bc1);
  c.rbc2 = (float)(1.0 / sqrt(bc2));
  return c;
}

// relative error of each at most 2^-22; magnitudes under 2^-126 count as zero (v that small is far below eps^2 of any use, and
// the divisor is at least eps, which the host requires to be a normal number)
__device__ __forceinline__ float sqrt_fast(float x) {
  float r;
  asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float reciprocal_fast(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// p' from p, m' and r = sqrt(v')
__device__ __forceinline__ float adamw_param(const AdamwCoef& c, float keep, float p, float m, float r) {
  return fmaf(p, keep, -(c.lr_bc1 * m) * reciprocal_fast(fmaf(r, c.rbc2, c.eps)));
}

}  // namespace ssim
