// AdamW over a list of tensors, one launch: the step of a parameter server that averages K pushed gradients.
//
//   g  = (grad_scale / K) sum_{l<K} g_l            (in arrival order, fp32)
//   m' = b1 m + (1 - b1) g,   v' = b2 v + (1 - b2) g^2
//   p' = p (1 - lr wd) - lr (m' / (1 - b1^t)) / (sqrt(v') / sqrt(1 - b2^t) + eps)
//
// States in 32 bits: m and v in fp32.  States in 8 bits: m and r = sqrt(v) as E4M3 codes in blocks of 32 with a power-of-two
// scale (lowbits.cuh).  The root is stored because E4M3 spans 2^17.8 inside a block: as many binades of v as 2^35.6 has, and
// the step needs the root anyway.  The step itself uses the fp32 m' and v'; only what is kept for the next step is rounded, and
// stochastically: v' moves by 1 - b2 = 0.001 of itself a step, far less than half an 8-bit step, so that rounding to nearest would
// never let it decay.  The 16-bit random number of an element comes from Philox (key = seed; counter = group of eight in the tensor,
// step, tensor), so results depend neither on the launch shape nor on the order of blocks; r takes the number with its bytes
// swapped, so that both roundings are unbiased without a second draw.  A positive r is never stored as zero: the next step would
// divide m by eps.
//
// Bound by HBM (at fp32 p, bf16 g: 26 bytes an element with 32-bit states, 14 with 8-bit ones).  A thread owns eight
// consecutive elements, so all streams are 16-byte accesses; four neighbouring lanes own a block of 32 and find its largest
// magnitude with two shuffles.  Chunks of 2048 elements of any tensor are dealt to a grid that fills the machine once, from a
// table made when the list was bound.
#pragma once
#include "lowbits.cuh"

namespace ssim {

constexpr int ADAMW_THREADS = 256;
constexpr int ADAMW_CHUNK = 8 * ADAMW_THREADS;

struct AdamwTensor {
  void* p; void* m; void* v;
  uint8_t* m_scale; uint8_t* v_scale;
  uint16_t* shadow;        // bf16 copy of p, or null
  long long n;
  float decay;
  int vec;                 // every stream allows 16-byte (8-bit states: 8-byte, MXFP4 pushes: 4-byte) accesses
};
struct AdamwChunk { uint32_t tensor, chunk; };      // elements [2048 chunk, 2048 (chunk + 1)) of that tensor

struct AdamwArgs {
  const AdamwTensor* tensors;
  const AdamwChunk* chunks;
  const void* const* g;            // [K_max][n_tensors]
  const uint8_t* const* g_scale;   // [K_max][n_tensors], MXFP4 pushes
  int n_tensors, K;
  uint32_t n_chunks;
  double beta1, beta2;
  float eps, grad_scale;           // grad_scale / K
  float lr;
  long long step;
  const float* lr_dev;             // read instead of lr / step when not null (captured steps)
  const long long* step_dev;
  uint64_t seed;
};

struct AdamwCoef { float b1, c1, b2, c2, lr, lr_bc1, rbc2, eps; };

__host__ __device__ inline AdamwCoef adamw_coef(double beta1, double beta2, float eps, float lr, long long step) {
  AdamwCoef c;
  c.b1 = (float)beta1; c.c1 = (float)(1.0 - beta1); c.b2 = (float)beta2; c.c2 = (float)(1.0 - beta2);
  c.lr = lr; c.eps = eps;
  // 1 - beta^t without cancellation for small t and beta near 1 (beta = 0: 1)
  const double bc1 = beta1 > 0.0 ? -expm1((double)step * log(beta1)) : 1.0, bc2 = beta2 > 0.0 ? -expm1((double)step * log(beta2)) : 1.0;
  c.lr_bc1 = (float)((double)lr / bc1);
  c.rbc2 = (float)(1.0 / sqrt(bc2));
  return c;
}

__device__ __forceinline__ float sqrt_approx(float x) {   // relative error at most 2^-23
  float r;
  asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// One element: updates p, m, v and returns sqrt(v').
__device__ __forceinline__ float adamw_element(const AdamwCoef& c, float keep, float g, float& p, float& m, float& v) {
  m = fmaf(c.b1, m, c.c1 * g);
  v = fmaf(c.b2, v, c.c2 * g * g);
  const float r = sqrt_approx(v);
  p = fmaf(p, keep, -__fdividef(c.lr_bc1 * m, fmaf(r, c.rbc2, c.eps)));   // the divisor stays below 2^66: no special range
  return r;
}

// E4M3 form of a block of 32 that four neighbouring lanes hold, eight each -> two words of codes, the scale byte
template <bool KEEP, bool SWAP>
__device__ __forceinline__ uint32_t encode_e4m3(const float (&x)[8], const U4& u, uint32_t (&codes)[2]) {
  uint32_t amax = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) amax = max(amax, __float_as_uint(x[e]) & ABS_MASK);
  amax = max(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, 1));
  amax = max(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, 2));
  const uint32_t code = scale_code_e4m3(amax);
  const float inv = scale_inverse(code);
  float q[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    uint32_t k16 = half_word(u, e);
    if (SWAP) k16 = __byte_perm(k16, 0u, 0x4401);
    const float a = fabsf(x[e]) * inv;
    float r = round_stochastic<3, -6>(a, k16);
    if (KEEP) r = a > 0.f ? fmaxf(r, 0.001953125f) : r;         // 2^-9, the smallest E4M3 value
    q[e] = copysignf(r, x[e]);
  }
#pragma unroll
  for (int w = 0; w < 2; ++w) codes[w] = to_e4m3x2(q[4 * w], q[4 * w + 1]) | to_e4m3x2(q[4 * w + 2], q[4 * w + 3]) << 16;
  return code;
}

__device__ __forceinline__ void decode_e4m3(const uint32_t (&codes)[2], float scale, float (&x)[8]) {
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float2 t = from_e4m3x2((codes[w >> 1] >> (16 * (w & 1))) & 0xFFFFu);
    x[2 * w] = t.x * scale;
    x[2 * w + 1] = t.y * scale;
  }
}

// Sum of the K pushes at elements [i, i + 8); n8 of them exist.
template <int GT>
__device__ __forceinline__ void sum_pushes(const AdamwArgs& a, uint32_t t, long long i, int n8, bool vec, float (&g)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) g[e] = 0.f;
  for (int l = 0; l < a.K; ++l) {
    const void* src = a.g[(size_t)l * a.n_tensors + t];
    float x[8];
    if constexpr (GT == T_MXFP4) {
      const uint8_t* c = static_cast<const uint8_t*>(src) + (i >> 1);
      uint32_t w = 0;
      if (vec && n8 == 8) {
        w = *reinterpret_cast<const uint32_t*>(c);
      } else {
        for (int b = 0; 2 * b < n8; ++b) w |= (uint32_t)c[b] << (8 * b);
        if (n8 & 1) w &= (1u << (4 * n8)) - 1u;                  // the last byte's high half belongs to no element
      }
      const float s = n8 > 0 ? scale_value(a.g_scale[(size_t)l * a.n_tensors + t][i >> 5]) : 0.f;
      e2m1x8(w, x);
#pragma unroll
      for (int e = 0; e < 8; ++e) g[e] = fmaf(x[e], s, g[e]);    // the product is exact: one rounding, that of the sum
    } else {
      if (vec && n8 == 8) {
        Elem<GT>::get8(src, i, x);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = e < n8 ? Elem<GT>::get(src, i + e) : 0.f;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) g[e] += x[e];
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) g[e] *= a.grad_scale;
}

template <int PT, int GT, int BITS>
__global__ void __launch_bounds__(ADAMW_THREADS) adamw_kernel(AdamwArgs a) {
  __shared__ AdamwCoef coef_s;
  if (threadIdx.x == 0)
    coef_s = adamw_coef(a.beta1, a.beta2, a.eps, a.lr_dev ? *a.lr_dev : a.lr, a.step_dev ? *a.step_dev : a.step);
  const uint32_t step32 = (uint32_t)(a.step_dev ? *a.step_dev : a.step);
  __syncthreads();
  const AdamwCoef c = coef_s;
  for (uint32_t k = blockIdx.x; k < a.n_chunks; k += gridDim.x) {
    const AdamwChunk ch = a.chunks[k];
    const AdamwTensor t = a.tensors[ch.tensor];
    const float keep = fmaf(-c.lr, t.decay, 1.f);
    const bool vec = t.vec != 0;
    const long long i = (long long)ch.chunk * ADAMW_CHUNK + 8 * (int)threadIdx.x;
    const int n8 = (int)max(0ll, min(8ll, t.n - i));
    float g[8], p[8], m[8], v[8];
    sum_pushes<GT>(a, ch.tensor, i, n8, vec, g);
    if (vec && n8 == 8) {
      Elem<PT>::get8(t.p, i, p);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] = e < n8 ? Elem<PT>::get(t.p, i + e) : 0.f;
    }
    if constexpr (BITS == 32) {
      if (vec && n8 == 8) {
        Elem<T_F32>::get8(t.m, i, m);
        Elem<T_F32>::get8(t.v, i, v);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) { m[e] = e < n8 ? Elem<T_F32>::get(t.m, i + e) : 0.f; v[e] = e < n8 ? Elem<T_F32>::get(t.v, i + e) : 0.f; }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) adamw_element(c, keep, g[e], p[e], m[e], v[e]);
      if (vec && n8 == 8) {
        Elem<T_F32>::put8(t.m, i, m);
        Elem<T_F32>::put8(t.v, i, v);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e < n8) { Elem<T_F32>::put(t.m, i + e, m[e]); Elem<T_F32>::put(t.v, i + e, v[e]); }
      }
    } else {
      uint8_t* mc = static_cast<uint8_t*>(t.m) + i;
      uint8_t* vc = static_cast<uint8_t*>(t.v) + i;
      uint32_t cm[2] = {0u, 0u}, cv[2] = {0u, 0u};
      float sm = 0.f, sv = 0.f;
      if (n8 > 0) { sm = scale_value(t.m_scale[i >> 5]); sv = scale_value(t.v_scale[i >> 5]); }
      if (vec && n8 == 8) {
        const uint2 x = *reinterpret_cast<const uint2*>(mc), y = *reinterpret_cast<const uint2*>(vc);
        cm[0] = x.x; cm[1] = x.y; cv[0] = y.x; cv[1] = y.y;
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e < n8) { cm[e >> 2] |= (uint32_t)mc[e] << (8 * (e & 3)); cv[e >> 2] |= (uint32_t)vc[e] << (8 * (e & 3)); }
      }
      decode_e4m3(cm, sm, m);
      decode_e4m3(cv, sv, v);
      float r[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        v[e] *= v[e];
        r[e] = adamw_element(c, keep, g[e], p[e], m[e], v[e]);
        if (e >= n8) { m[e] = 0.f; r[e] = 0.f; }                 // elements past the end stay out of their block's scale
      }
      const unsigned long long grp = (unsigned long long)(i >> 3);
      const U4 u = philox4x32_10((uint32_t)a.seed, (uint32_t)(a.seed >> 32), (uint32_t)grp, (2u << 24) | (uint32_t)(grp >> 32), step32, ch.tensor);
      const uint32_t km = encode_e4m3<false, false>(m, u, cm), kv = encode_e4m3<true, true>(r, u, cv);
      if (vec && n8 == 8) {
        *reinterpret_cast<uint2*>(mc) = make_uint2(cm[0], cm[1]);
        *reinterpret_cast<uint2*>(vc) = make_uint2(cv[0], cv[1]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e < n8) { mc[e] = (uint8_t)(cm[e >> 2] >> (8 * (e & 3))); vc[e] = (uint8_t)(cv[e >> 2] >> (8 * (e & 3))); }
      }
      if ((threadIdx.x & 3) == 0 && n8 > 0) { t.m_scale[i >> 5] = (uint8_t)km; t.v_scale[i >> 5] = (uint8_t)kv; }
    }
    if (vec && n8 == 8) {
      Elem<PT>::put8(t.p, i, p);
      if (PT == T_F32 && t.shadow) Elem<T_BF16>::put8(t.shadow, i, p);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < n8) {
          Elem<PT>::put(t.p, i + e, p[e]);
          if (PT == T_F32 && t.shadow) Elem<T_BF16>::put(t.shadow, i + e, p[e]);
        }
    }
  }
}

}  // namespace ssim
