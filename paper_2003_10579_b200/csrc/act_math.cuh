// Activations of a layer and their derivatives, in fp32:
//   relu(z) = max(z, 0)
//   gelu(z) = z / 2 (1 + tanh(sqrt(2 / pi) (z + 0.044715 z^3))) = z s(u),  u = 2 sqrt(2 / pi) (z + 0.044715 z^3)
//   silu(z) = z s(z),  s the logistic function 1 / (1 + e^-z)
// Through s one exponential and one reciprocal do, and nothing cancels for z far below zero, where 1 + tanh would.
#pragma once
#include <cuda_runtime.h>
#include <cstdint>

namespace ssim {

enum : int { ACT_NONE = 0, ACT_RELU = 1, ACT_GELU = 2, ACT_SILU = 3 };

constexpr float GELU_C = 1.5957691216057308f, GELU_A = 0.044715f;      // 2 sqrt(2 / pi)
constexpr float LOG2E = 1.4426950408889634f;

__device__ __forceinline__ float exp2_fast(float d) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(d)); return r; }
__device__ __forceinline__ float rcp_fast(float d) { float r; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(d)); return r; }

// 1 / (1 + 2^-d).  The approximate power and reciprocal are off by about 2^-21 of the value at most, far below a 16-bit type's half step and eight of fp32's.  Values under
// 2^-126 are taken as zero: silu below -87.3 is, where it is 1e-36 and less.
__device__ __forceinline__ float logistic2(float d) { return rcp_fast(1.f + exp2_fast(-d)); }

template <int ACT>
__device__ __forceinline__ float act_value(float z) {
  if (ACT == ACT_RELU) return z > 0.f ? z : z != z ? z : 0.f;
  if (ACT == ACT_GELU) return z * logistic2(z * fmaf(LOG2E * GELU_C * GELU_A * z, z, LOG2E * GELU_C));
  if (ACT == ACT_SILU) return z * logistic2(LOG2E * z);
  return z;
}
// The derivative at a finite z; relu's at zero is zero.  With q = s(u): (z s(u))' = q (1 + z u'(z) (1 - q)).  Beyond the limits it is 0 or 1, and the powers
// of z would only raise the error of 1 - q.
template <int ACT>
__device__ __forceinline__ float act_slope(float z) {
  if (ACT == ACT_RELU) return z > 0.f ? 1.f : 0.f;
  if (ACT == ACT_GELU) {
    const float t = fminf(fmaxf(z, -10.f), 10.f), t2 = t * t;
    const float q = logistic2(t * fmaf(LOG2E * GELU_C * GELU_A, t2, LOG2E * GELU_C));
    return q * fmaf(t * fmaf(3.f * GELU_C * GELU_A, t2, GELU_C), 1.f - q, 1.f);
  }
  if (ACT == ACT_SILU) {
    const float t = fminf(fmaxf(z, -80.f), 80.f), q = logistic2(LOG2E * t);
    return q * fmaf(t, 1.f - q, 1.f);
  }
  return 1.f;
}

}  // namespace ssim
