// Conversions between fp32 and block-scaled 8- and 4-bit floats, device side.
//
// A block is 32 consecutive elements with one scale 2^k, stored as the byte k + 127 (E8M0; 0xFF: the block held an
// infinity or a NaN and reads as NaN).  k is the smallest exponent >= -127 for which no magnitude of the block exceeds
// L 2^k, L the format's largest value: 448 = 1.75 * 2^8 for E4M3, 6 = 1.5 * 2^2 for E2M1.  So nothing saturates and
// every element is off by at most half a step (nearest) or less than one step (stochastic).
//
// Stochastic rounding takes |x| to step * floor(|x| / step + u), u = k16 / 2^16.  Below the leading bits that a format keeps,
// an fp32 magnitude holds |x| / step's fraction; adding u at that place and clearing what lies below is that formula in
// integer arithmetic, exactly.  Magnitudes under the format's smallest normal have a fixed step: they are moved up to it first,
// rounding towards zero, which cannot cross the points k16 / 2^16 that the addition compares with.
#pragma once
#include "device_rng.cuh"

namespace ssim {

constexpr uint32_t ABS_MASK = 0x7FFFFFFFu, INF_BITS = 0x7F800000u;

// Scale byte of a block whose largest magnitude has the bits `amax`; TOP is the mantissa of L, EMAX its exponent.
template <uint32_t TOP, int EMAX>
__device__ __forceinline__ uint32_t block_scale_code(uint32_t amax) {
  if (amax >= INF_BITS) return 255u;
  const int code = (int)(amax >> 23) - EMAX + ((amax & 0x7FFFFFu) > TOP ? 1 : 0);
  return (uint32_t)max(code, 0);
}
__device__ __forceinline__ uint32_t scale_code_e4m3(uint32_t amax) { return block_scale_code<0x600000u, 8>(amax); }
__device__ __forceinline__ uint32_t scale_code_e2m1(uint32_t amax) { return block_scale_code<0x400000u, 2>(amax); }

// 2^k of a scale byte (2^-127 is subnormal in fp32; 0xFF is NaN), and 2^-k (a NaN block: 2^-127, its codes do not matter)
__device__ __forceinline__ float scale_value(uint32_t code) {
  return __uint_as_float(code == 0u ? 0x00400000u : code == 255u ? 0x7FC00000u : code << 23);
}
__device__ __forceinline__ float scale_inverse(uint32_t code) { return __uint_as_float(code == 255u ? 0x00400000u : (254u - code) << 23); }

// x / scale (any sign) on a format of MBITS mantissa bits whose smallest normal is 2^EMIN, rounded stochastically with k16 in
// [0, 2^16).  round_normal: |x| / scale is at least the smallest normal (or x is zero and k16 does not matter: see the mask).
template <int MBITS>
__device__ __forceinline__ float round_normal(float a, uint32_t k16) {
  constexpr int LOW = 23 - MBITS;                               // bits that go
  return __uint_as_float((k16 * (1u << (LOW - 16)) + __float_as_uint(a)) & ~((1u << LOW) - 1u));
}
template <int MBITS, int EMIN>
__device__ __forceinline__ float round_stochastic(float a, uint32_t k16) {
  constexpr float NORMAL = EMIN == 0 ? 1.f : 1.f / (float)(1 << -EMIN);
  const float mag = fabsf(a);
  float base;                                                     // NORMAL or zero
  if (EMIN == 0) asm("set.lt.f32.f32 %0, %1, %2;" : "=f"(base) : "f"(mag), "f"(1.f));
  else base = mag < NORMAL ? NORMAL : 0.f;
  return copysignf(round_normal<MBITS>(__fadd_rz(mag, base), k16) - base, a);
}

// largest magnitude of three, NaN if one is NaN
__device__ __forceinline__ float max3_abs(float a, float b, float c) {
  float r;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ float min3_abs(float a, float b, float c) {
  float r;
  asm("min.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ uint32_t amax8(const float (&x)[8]) {   // bits of the largest magnitude; at least INF_BITS if one is not finite
  return __float_as_uint(max3_abs(max3_abs(x[0], x[1], x[2]), max3_abs(x[3], x[4], x[5]), max3_abs(x[6], x[7], 0.f))) & ABS_MASK;
}
__device__ __forceinline__ float amin8(const float (&x)[8]) {
  return min3_abs(min3_abs(x[0], x[1], x[2]), min3_abs(x[3], x[4], x[5]), fminf(fabsf(x[6]), fabsf(x[7])));
}

// Philox4x32-10 (device_rng.cuh) with the ten round keys worked out once, where the key is the same for a whole launch
struct PhiloxKeys { uint32_t k[20]; };
__host__ inline PhiloxKeys philox_keys(uint64_t seed) {
  PhiloxKeys q;
  uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
  for (int r = 0; r < 10; ++r) {
    q.k[2 * r] = k0; q.k[2 * r + 1] = k1;
    k0 += 0x9E3779B9u; k1 += 0xBB67AE85u;
  }
  return q;
}
__device__ __forceinline__ U4 philox_keyed(const PhiloxKeys& q, uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3) {
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t p0 = (uint64_t)0xD2511F53u * c0, p1 = (uint64_t)0xCD9E8D57u * c2;
    const uint32_t n0 = (uint32_t)(p1 >> 32) ^ c1 ^ q.k[2 * r], n2 = (uint32_t)(p0 >> 32) ^ c3 ^ q.k[2 * r + 1];
    c0 = n0; c1 = (uint32_t)p1; c2 = n2; c3 = (uint32_t)p0;
  }
  return U4{c0, c1, c2, c3};
}

// the 16-bit number of element e of a group of eight
__device__ __forceinline__ uint32_t half_word(const U4& u, int e) {
  const uint32_t w = e < 2 ? u.x : e < 4 ? u.y : e < 6 ? u.z : u.w;
  return __byte_perm(w, 0u, (e & 1) ? 0x4432 : 0x4410);
}
__device__ __forceinline__ uint32_t half_word_swapped(const U4& u, int e) {   // the same with its two bytes swapped
  const uint32_t w = e < 2 ? u.x : e < 4 ? u.y : e < 6 ? u.z : u.w;
  return __byte_perm(w, 0u, (e & 1) ? 0x4423 : 0x4401);
}

// two values that E4M3 / E2M1 holds exactly, or rounded to nearest even -> codes, `lo` in the low byte / nibble
__device__ __forceinline__ uint32_t to_e4m3x2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ float2 from_e4m3x2(uint32_t codes) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)codes));
  float2 v;
  asm("{\n\t.reg .b16 l, u;\n\tmov.b32 {l, u}, %2;\n\tcvt.f32.f16 %0, l;\n\tcvt.f32.f16 %1, u;\n\t}" : "=f"(v.x), "=f"(v.y) : "r"(h));
  return v;
}
// eight values -> eight E2M1 codes, the first in the lowest nibble (one block of assembly: the conversions then write into place)
__device__ __forceinline__ uint32_t to_e2m1x8(const float (&x)[8]) {
  uint32_t r;
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\tmov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(r) : "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]));
  return r;
}
__device__ __forceinline__ uint32_t to_e4m3x4(float a, float b, float c, float d) {
  uint32_t r;
  asm("{\n\t.reg .b16 l, h;\n\tcvt.rn.satfinite.e4m3x2.f32 l, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 h, %4, %3;\n\tmov.b32 %0, {l, h};\n\t}"
      : "=r"(r) : "f"(a), "f"(b), "f"(c), "f"(d));
  return r;
}
__device__ __forceinline__ float2 from_e2m1x2(uint32_t codes) {
  uint32_t h;
  asm("{\n\t.reg .b8 c, d1, d2, d3;\n\tmov.b32 {c, d1, d2, d3}, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, c;\n\t}" : "=r"(h) : "r"(codes));
  float2 v;
  asm("{\n\t.reg .b16 l, u;\n\tmov.b32 {l, u}, %2;\n\tcvt.f32.f16 %0, l;\n\tcvt.f32.f16 %1, u;\n\t}" : "=f"(v.x), "=f"(v.y) : "r"(h));
  return v;
}

// ---- eight consecutive elements of a tensor, as fp32 --------------------------------------------------------------------
enum : int { T_F32 = 0, T_BF16 = 1, T_F16 = 2, T_MXFP4 = 3 };

__device__ __forceinline__ float bf16_to_float(uint32_t h) { return __uint_as_float(h << 16); }
__device__ __forceinline__ uint32_t float_to_bf16x2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t float_to_f16x2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ float f16_to_float(uint32_t h) {
  float v;
  asm("cvt.f32.f16 %0, %1;" : "=f"(v) : "h"((uint16_t)h));
  return v;
}

__device__ __forceinline__ void store32(void* p, const uint32_t (&w)[8]) {      // one aligned 32-byte sector
  asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
}
__device__ __forceinline__ void load32(const void* p, uint32_t (&w)[8]) {
  asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p));
}
template <int T> struct Elem;
template <> struct Elem<T_F32> {
  static constexpr int bytes = 4;
  static __device__ __forceinline__ float get(const void* p, long long i) { return static_cast<const float*>(p)[i]; }
  static __device__ __forceinline__ void put(void* p, long long i, float v) { static_cast<float*>(p)[i] = v; }
  static __device__ __forceinline__ void get8(const void* p, long long i, float (&v)[8]) {   // 16-byte aligned
    const float4* q = reinterpret_cast<const float4*>(static_cast<const float*>(p) + i);
    const float4 a = q[0], b = q[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
  static __device__ __forceinline__ void put8(void* p, long long i, const float (&v)[8]) {
    float4* q = reinterpret_cast<float4*>(static_cast<float*>(p) + i);
    q[0] = make_float4(v[0], v[1], v[2], v[3]);
    q[1] = make_float4(v[4], v[5], v[6], v[7]);
  }
};
template <> struct Elem<T_BF16> {
  static constexpr int bytes = 2;
  static __device__ __forceinline__ float get(const void* p, long long i) { return bf16_to_float(static_cast<const uint16_t*>(p)[i]); }
  static __device__ __forceinline__ void put(void* p, long long i, float v) { static_cast<uint16_t*>(p)[i] = (uint16_t)float_to_bf16x2(v, 0.f); }
  static __device__ __forceinline__ void get8(const void* p, long long i, float (&v)[8]) {
    const uint4 a = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + i);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) { v[2 * k] = __uint_as_float(w[k] << 16); v[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u); }
  }
  static __device__ __forceinline__ void put8(void* p, long long i, const float (&v)[8]) {
    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p) + i) =
        make_uint4(float_to_bf16x2(v[0], v[1]), float_to_bf16x2(v[2], v[3]), float_to_bf16x2(v[4], v[5]), float_to_bf16x2(v[6], v[7]));
  }
};
template <> struct Elem<T_F16> {
  static constexpr int bytes = 2;
  static __device__ __forceinline__ float get(const void* p, long long i) { return f16_to_float(static_cast<const uint16_t*>(p)[i]); }
  static __device__ __forceinline__ void put(void* p, long long i, float v) { static_cast<uint16_t*>(p)[i] = (uint16_t)float_to_f16x2(v, 0.f); }
  static __device__ __forceinline__ void get8(const void* p, long long i, float (&v)[8]) {
    const uint4 a = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + i);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) { v[2 * k] = f16_to_float(w[k] & 0xFFFFu); v[2 * k + 1] = f16_to_float(w[k] >> 16); }
  }
};

// ---- eight consecutive elements as they are stored: their largest magnitude without unpacking 16-bit types ----------------
template <int T> struct Raw8;
template <> struct Raw8<T_F32> {
  uint32_t w[8];
  __device__ __forceinline__ void load(const void* p, long long i) {
    const uint4* q = reinterpret_cast<const uint4*>(static_cast<const float*>(p) + i);
    const uint4 a = q[0], b = q[1];
    w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w; w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
  }
  __device__ __forceinline__ void load_some(const void* p, long long i, int n) {
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = e < n ? static_cast<const uint32_t*>(p)[i + e] : 0u;
  }
  __device__ __forceinline__ float value(int e) const { return __uint_as_float(w[e]); }
  __device__ __forceinline__ uint32_t amax() const {
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(w[e]);
    return amax8(v);
  }
};
__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
template <int T> struct Raw16 {      // bf16 and fp16: two elements a word
  uint32_t w[4];
  __device__ __forceinline__ void load(const void* p, long long i) {
    const uint4 a = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + i);
    w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
  }
  __device__ __forceinline__ void load_some(const void* p, long long i, int n) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t lo = 2 * k < n ? static_cast<const uint16_t*>(p)[i + 2 * k] : 0u, hi = 2 * k + 1 < n ? static_cast<const uint16_t*>(p)[i + 2 * k + 1] : 0u;
      w[k] = lo | hi << 16;
    }
  }
  __device__ __forceinline__ float value(int e) const {
    const uint32_t x = w[e >> 1];
    if (T == T_BF16) return __uint_as_float((e & 1) ? x & 0xFFFF0000u : x << 16);
    return f16_to_float((e & 1) ? x >> 16 : x & 0xFFFFu);
  }
  // magnitudes compare as the integers that their bits are (an infinity or a NaN above every number)
  __device__ __forceinline__ uint32_t amax() const {
    const uint32_t m = max_u16x2(max_u16x2(w[0] & 0x7FFF7FFFu, w[1] & 0x7FFF7FFFu), max_u16x2(w[2] & 0x7FFF7FFFu, w[3] & 0x7FFF7FFFu));
    return widen(max(m >> 16, m & 0xFFFFu));
  }
  static __device__ __forceinline__ uint32_t widen(uint32_t h) { return T == T_BF16 ? h << 16 : __float_as_uint(f16_to_float(h)); }
};
template <> struct Raw8<T_BF16> : Raw16<T_BF16> {};
template <> struct Raw8<T_F16> : Raw16<T_F16> {};

// eight MXFP4 codes of one word -> values in units of the scale
__device__ __forceinline__ void e2m1x8(uint32_t w, float (&v)[8]) {
  asm("{\n\t.reg .b8 a, b, c, d;\n\t.reg .b32 p, q, r, s;\n\t.reg .b16 l, h;\n\tmov.b32 {a, b, c, d}, %8;\n\t"
      "cvt.rn.f16x2.e2m1x2 p, a;\n\tcvt.rn.f16x2.e2m1x2 q, b;\n\tcvt.rn.f16x2.e2m1x2 r, c;\n\tcvt.rn.f16x2.e2m1x2 s, d;\n\t"
      "mov.b32 {l, h}, p;\n\tcvt.f32.f16 %0, l;\n\tcvt.f32.f16 %1, h;\n\tmov.b32 {l, h}, q;\n\tcvt.f32.f16 %2, l;\n\tcvt.f32.f16 %3, h;\n\t"
      "mov.b32 {l, h}, r;\n\tcvt.f32.f16 %4, l;\n\tcvt.f32.f16 %5, h;\n\tmov.b32 {l, h}, s;\n\tcvt.f32.f16 %6, l;\n\tcvt.f32.f16 %7, h;\n\t}"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]) : "r"(w));
}

}  // namespace ssim
