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

// Root of x >= 0, relative error at most 2^-22.  The instruction takes what lies under 2^-126 for zero, which with a small eps would leave
// eps alone in the divisor: such x go through it 2^48 larger (exact, as is the way back).  Correctly rounded roots and divisions cost 205 M
// elements with 8-bit states 0.49 -> 0.55 ms and a list of 400 small tensors 8.3 -> 10.2 us; the step is lr times this quotient, so that
// what they would add lies far under p's own rounding.
constexpr float ROOT_NORMAL = 1.17549435e-38f;                // 2^-126
__device__ __forceinline__ float root_normal(float x) {        // x is zero or at least ROOT_NORMAL
  float r;
  asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float root(float x) {
  const bool low = x < ROOT_NORMAL;
  return root_normal(low ? x * 281474976710656.f : x) * (low ? 5.9604644775390625e-8f : 1.f);
}
// The instruction takes divisors under 2^-126 for zero and gives zero for those over 2^126.  eps is in the divisor, and sqrt(v / (1 - b2^t)) is
// under 2^92 (v an fp32 number, 1 - b2 at least 2^-53), so with eps in this range neither happens.
inline bool adamw_eps_ok(float eps) { return eps >= 1.17549435e-38f && eps <= 4.25352959e37f; }       // 2^-126, 2^125
// relative error at most 2^-22
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
