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

// The approximate exponential and reciprocal are off by about 2^-21 of the value at most, far below a 16-bit type's half step.
__device__ __forceinline__ float logistic(float z) { return __fdividef(1.f, 1.f + __expf(-z)); }

template <int ACT>
__device__ __forceinline__ float act_value(float z) {
  if (ACT == ACT_RELU) return z > 0.f ? z : z != z ? z : 0.f;
  if (ACT == ACT_GELU) return z * logistic(GELU_C * z * fmaf(GELU_A * z, z, 1.f));
  if (ACT == ACT_SILU) return z * logistic(z);
  return z;
}
// The derivative; relu's at zero is zero.
template <int ACT>
__device__ __forceinline__ float act_slope(float z) {
  if (ACT == ACT_RELU) return z > 0.f ? 1.f : z != z ? z : 0.f;
  if (ACT == ACT_GELU) {
    const float t = fminf(fmaxf(z, -10.f), 10.f);                      // beyond, it is 0 or 1, and the cube would only raise the error of 1 - q
    const float q = logistic(GELU_C * t * fmaf(GELU_A * t, t, 1.f));
    const float d = fmaf(t * q * (1.f - q), GELU_C * fmaf(3.f * GELU_A * t, t, 1.f), q);
    return z != z ? z : d;
  }
  if (ACT == ACT_SILU) {
    const float t = fminf(fmaxf(z, -80.f), 80.f);
    const float q = logistic(t), d = fmaf(t * q, 1.f - q, q);
    return z != z ? z : d;
  }
  return 1.f;
}

}  // namespace ssim
