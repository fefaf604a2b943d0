// AdamW over a list of tensors, a launch per combination of types: the step of a parameter server that averages K pushed gradients.
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
// Bound by HBM (at fp32 p, bf16 g: 26 bytes an element with 32-bit states, 14 with 8-bit ones): 257 M elements with a bf16 copy 1.05 ms, 6.8
// TB/s.  With 8-bit states the arithmetic is close behind (about 57 instructions an element, most of them the two roundings and
// Philox): 205 M elements 0.49 to 0.54 ms by the clock, 5.4 to 5.9 TB/s.  With four MXFP4 pushes to decode, 56.6 M elements 0.23 ms, neither HBM (60 %)
// nor the issue slots (58 %, 80 instructions an element) are full: a chunk's loads start when the last chunk is stored.  A thread owns eight
// consecutive elements, so all streams are 16-byte accesses; four neighbouring lanes own a block of 32 and find its largest
// magnitude with two shuffles.  Chunks of 2048 elements of any tensor come from a table made when the list
// was bound.
#pragma once
#include "adamw_math.cuh"
#include "lowbits.cuh"

namespace ssim {

constexpr int ADAMW_THREADS = 256;
constexpr int ADAMW_CHUNK = 8 * ADAMW_THREADS;

struct AdamwTensor {
  void* p; void* m; void* v;
  uint8_t* m_scale; uint8_t* v_scale;
  uint16_t* shadow;        // bf16 copy of p, or null
  const void* g0;          // the first push (the others: AdamwArgs::g)
  const uint8_t* g0_scale;
  long long n;
  float decay;
  int vec;                 // every stream allows 16-byte (8-bit states: 8-byte, MXFP4 pushes: 4-byte) accesses
};
struct AdamwChunk { uint32_t tensor, chunk; };      // elements [ADAMW_CHUNK chunk, ADAMW_CHUNK (chunk + 1)) of that tensor

struct AdamwArgs {
  const AdamwTensor* tensors;
  const AdamwChunk* chunks;
  const void* const* g;            // [K_max][n_tensors]
  const uint8_t* const* g_scale;   // [K_max][n_tensors], MXFP4 pushes
  int n_tensors, K;
  uint32_t n_chunks, step32;
  AdamwCoef coef;
  const float* lr_dev;             // when not null, lr and step are read here and the coefficients worked out on the device
  const long long* step_dev;
  double beta1, beta2, mean;       // mean: grad_scale / K
  PhiloxKeys keys;
};

// E4M3 form of a block of 32 that four neighbouring lanes hold, eight each -> two words of codes, the scale byte.
// KEEP (r): magnitudes are positive, and a positive one never becomes zero; the random number has its bytes swapped.
template <bool KEEP>
__device__ __forceinline__ uint32_t encode_e4m3(const float (&x)[8], const U4& u, uint32_t (&codes)[2]) {
  uint32_t amax = amax8(x);
  amax = max(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, 1));
  amax = max(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, 2));
  const uint32_t code = scale_code_e4m3(amax);
  const float inv = scale_inverse(code);
  float q[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) q[e] = x[e] * inv;
  if (amin8(q) >= 0.015625f) {                                   // all normal in E4M3: almost always
#pragma unroll
    for (int e = 0; e < 8; ++e) q[e] = round_normal<3>(q[e], KEEP ? half_word_swapped(u, e) : half_word(u, e));
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float r = round_stochastic<3, -6>(q[e], KEEP ? half_word_swapped(u, e) : half_word(u, e));
      q[e] = KEEP && q[e] > 0.f ? fmaxf(r, 0.001953125f) : r;    // 2^-9, the smallest E4M3 value
    }
  }
#pragma unroll
  for (int w = 0; w < 2; ++w) codes[w] = to_e4m3x4(q[4 * w], q[4 * w + 1], q[4 * w + 2], q[4 * w + 3]);
  return code;
}

// codes -> values times s
__device__ __forceinline__ void decode_e4m3(const uint32_t (&codes)[2], float s, float (&x)[8]) {
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float2 t = from_e4m3x2((w & 1) ? codes[w >> 1] >> 16 : codes[w >> 1]);
    x[2 * w] = t.x * s;
    x[2 * w + 1] = t.y * s;
  }
}

// Elements [i, i + 8) of one push, added to the sum or (FIRST) as its start; n8 of them exist.
template <int GT, bool FIRST>
__device__ __forceinline__ void add_push(const void* src, const uint8_t* scale, long long i, int n8, float (&g)[8]) {
  float x[8];
  if constexpr (GT == T_MXFP4) {
    const uint8_t* c = static_cast<const uint8_t*>(src) + (i >> 1);
    uint32_t w = 0;
    if (n8 == 8) {
      w = *reinterpret_cast<const uint32_t*>(c);
    } else {
      for (int b = 0; 2 * b < n8; ++b) w |= (uint32_t)c[b] << (8 * b);
      if (n8 & 1) w &= (1u << (4 * n8)) - 1u;                    // the last byte's high half belongs to no element
    }
    const float s = n8 > 0 ? scale_value(scale[i >> 5]) : 0.f;
    e2m1x8(w, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) g[e] = FIRST ? x[e] * s : fmaf(x[e], s, g[e]);   // the product is exact: one rounding, that of the sum
  } else {
    if (n8 == 8) {
      Elem<GT>::get8(src, i, x);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = e < n8 ? Elem<GT>::get(src, i + e) : 0.f;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) g[e] = FIRST ? x[e] : g[e] + x[e];
  }
}
template <int GT>
__device__ __forceinline__ float push_element(const void* src, const uint8_t* scale, long long i) {
  if constexpr (GT == T_MXFP4) {
    const uint32_t byte = static_cast<const uint8_t*>(src)[i >> 1];
    return from_e2m1x2((i & 1) ? byte >> 4 : byte & 15u).x * scale_value(scale[i >> 5]);
  } else {
    return Elem<GT>::get(src, i);
  }
}

// Tensors whose streams allow wide accesses: a thread owns eight consecutive elements (FULL: the chunk ends inside the tensor, all exist).
template <int PT, int GT, int BITS, bool MULTI, bool FULL>
__device__ __forceinline__ void adamw_chunk_wide(const AdamwArgs& a, const AdamwCoef& c, uint32_t step32, const AdamwTensor& t, const AdamwChunk ch) {
  const float keep = fmaf(-c.lr, t.decay, 1.f);
  const long long i = (long long)ch.chunk * ADAMW_CHUNK + 8 * (int)threadIdx.x;
  float p[8], g[8], m[8], v[8];      // m, v: 32-bit states
  uint32_t cm[2], cv[2];             // 8-bit states
  float sm, sv;
  const int n8 = FULL ? 8 : (int)max(0ll, min(8ll, t.n - i));
  add_push<GT, true>(t.g0, t.g0_scale, i, n8, g);
  if (n8 == 8) {
    Elem<PT>::get8(t.p, i, p);
    if constexpr (BITS == 32) {
      Elem<T_F32>::get8(t.m, i, m);
      Elem<T_F32>::get8(t.v, i, v);
    } else {
      const uint2 x = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(t.m) + i), y = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(t.v) + i);
      cm[0] = x.x; cm[1] = x.y; cv[0] = y.x; cv[1] = y.y;
    }
  } else {
    if constexpr (BITS == 8) cm[0] = cm[1] = cv[0] = cv[1] = 0u;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const bool in = e < n8;
      p[e] = in ? Elem<PT>::get(t.p, i + e) : 0.f;
      if constexpr (BITS == 32) {
        m[e] = in ? static_cast<const float*>(t.m)[i + e] : 0.f;
        v[e] = in ? static_cast<const float*>(t.v)[i + e] : 0.f;
      } else if (in) {
        cm[e >> 2] |= (uint32_t)static_cast<const uint8_t*>(t.m)[i + e] << (8 * (e & 3));
        cv[e >> 2] |= (uint32_t)static_cast<const uint8_t*>(t.v)[i + e] << (8 * (e & 3));
      }
    }
  }
  if constexpr (BITS == 8) {
    sm = sv = 0.f;
    if (n8 > 0) { sm = scale_value(t.m_scale[i >> 5]); sv = scale_value(t.v_scale[i >> 5]); }
  }
#pragma unroll 4
  for (int l = 1; MULTI && l < a.K; ++l) {
    const void* src = a.g[(size_t)l * a.n_tensors + ch.tensor];
    const uint8_t* scale = GT == T_MXFP4 ? a.g_scale[(size_t)l * a.n_tensors + ch.tensor] : nullptr;
    add_push<GT, false>(src, scale, i, n8, g);
  }
  if constexpr (BITS == 32) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float s = c.s2 * g[e];
      m[e] = fmaf(c.b1, m[e], c.c1 * g[e]);
      v[e] = fmaf(c.b2, v[e], s * s);
      p[e] = adamw_param(c, keep, p[e], m[e], root(v[e]));
    }
  } else {
    float mq[8], r[8];
    decode_e4m3(cm, c.b1 * sm, mq);
    decode_e4m3(cv, c.sb2 * sv, r);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float s = c.s2 * g[e];
      mq[e] = fmaf(c.c1, g[e], mq[e]);
      r[e] = fmaf(r[e], r[e], s * s);
    }
    if (amin8(r) >= ROOT_NORMAL) {                          // one look for all eight: 205 M elements 0.49 ms, each looked at 0.50 ms
#pragma unroll
      for (int e = 0; e < 8; ++e) r[e] = root_normal(r[e]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) r[e] = root(r[e]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) p[e] = adamw_param(c, keep, p[e], mq[e], r[e]);
    if (n8 < 8) {                                           // elements past the end stay out of their block's scale
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e >= n8) { mq[e] = 0.f; r[e] = 0.f; }
    }
    const unsigned long long grp = (unsigned long long)(i >> 3);
    const U4 u = philox_keyed(a.keys, (uint32_t)grp, (2u << 24) | (uint32_t)(grp >> 32), step32, ch.tensor);
    const uint32_t km = encode_e4m3<false>(mq, u, cm), kv = encode_e4m3<true>(r, u, cv);
    if ((threadIdx.x & 3) == 0 && n8 > 0) { t.m_scale[i >> 5] = (uint8_t)km; t.v_scale[i >> 5] = (uint8_t)kv; }
  }
  if (n8 == 8) {
    Elem<PT>::put8(t.p, i, p);
    if (PT == T_F32 && t.shadow) Elem<T_BF16>::put8(t.shadow, i, p);
    if constexpr (BITS == 32) {
      Elem<T_F32>::put8(t.m, i, m);
      Elem<T_F32>::put8(t.v, i, v);
    } else {
      *reinterpret_cast<uint2*>(static_cast<uint8_t*>(t.m) + i) = make_uint2(cm[0], cm[1]);
      *reinterpret_cast<uint2*>(static_cast<uint8_t*>(t.v) + i) = make_uint2(cv[0], cv[1]);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n8) {
        Elem<PT>::put(t.p, i + e, p[e]);
        if (PT == T_F32 && t.shadow) Elem<T_BF16>::put(t.shadow, i + e, p[e]);
        if constexpr (BITS == 32) {
          static_cast<float*>(t.m)[i + e] = m[e];
          static_cast<float*>(t.v)[i + e] = v[e];
        } else {
          static_cast<uint8_t*>(t.m)[i + e] = (uint8_t)(cm[e >> 2] >> (8 * (e & 3)));
          static_cast<uint8_t*>(t.v)[i + e] = (uint8_t)(cv[e >> 2] >> (8 * (e & 3)));
        }
      }
  }
}

// Any other alignment: neighbouring lanes take neighbouring elements, a warp a block of 32.
template <int PT, int GT, int BITS, bool MULTI>
__device__ __forceinline__ void adamw_chunk_narrow(const AdamwArgs& a, const AdamwCoef& c, uint32_t step32, const AdamwTensor& t, const AdamwChunk ch) {
  const float keep = fmaf(-c.lr, t.decay, 1.f);
  const long long first = (long long)ch.chunk * ADAMW_CHUNK + (int)threadIdx.x;
  constexpr int ROUNDS = ADAMW_CHUNK / ADAMW_THREADS, BATCH = 4;
#pragma unroll 1
  for (int at = 0; at < ROUNDS; at += BATCH) {
    if (first - (int)threadIdx.x + at * ADAMW_THREADS >= t.n) break;      // the whole block agrees
    float p[BATCH], g[BATCH], m[BATCH], v[BATCH];
#pragma unroll
    for (int k = 0; k < BATCH; ++k) {
      const long long i = first + (at + k) * ADAMW_THREADS;
      const bool in = i < t.n;
      g[k] = in ? push_element<GT>(t.g0, t.g0_scale, i) : 0.f;
      p[k] = in ? Elem<PT>::get(t.p, i) : 0.f;
      if constexpr (BITS == 32) {
        m[k] = in ? static_cast<const float*>(t.m)[i] : 0.f;
        v[k] = in ? static_cast<const float*>(t.v)[i] : 0.f;
      } else {
        m[k] = in ? from_e4m3x2(static_cast<const uint8_t*>(t.m)[i]).x * scale_value(t.m_scale[i >> 5]) : 0.f;
        v[k] = in ? from_e4m3x2(static_cast<const uint8_t*>(t.v)[i]).x * scale_value(t.v_scale[i >> 5]) : 0.f;
      }
    }
    for (int l = 1; MULTI && l < a.K; ++l) {
      const void* src = a.g[(size_t)l * a.n_tensors + ch.tensor];
      const uint8_t* scale = GT == T_MXFP4 ? a.g_scale[(size_t)l * a.n_tensors + ch.tensor] : nullptr;
#pragma unroll
      for (int k = 0; k < BATCH; ++k) {
        const long long i = first + (at + k) * ADAMW_THREADS;
        if (i < t.n) g[k] += push_element<GT>(src, scale, i);
      }
    }
#pragma unroll
    for (int k = 0; k < BATCH; ++k) {
      const long long i = first + (at + k) * ADAMW_THREADS;
      const bool in = i < t.n;
      const float s = c.s2 * g[k];
      float r;
      if constexpr (BITS == 32) {
        m[k] = fmaf(c.b1, m[k], c.c1 * g[k]);
        v[k] = fmaf(c.b2, v[k], s * s);
        r = root(v[k]);
      } else {
        m[k] = fmaf(c.c1, g[k], c.b1 * m[k]);
        const float old = c.sb2 * v[k];
        r = root(fmaf(old, old, s * s));
      }
      p[k] = adamw_param(c, keep, p[k], m[k], r);
      if (in) {
        Elem<PT>::put(t.p, i, p[k]);
        if (PT == T_F32 && t.shadow) Elem<T_BF16>::put(t.shadow, i, p[k]);
        if constexpr (BITS == 32) {
          static_cast<float*>(t.m)[i] = m[k];
          static_cast<float*>(t.v)[i] = v[k];
        }
      }
      if constexpr (BITS == 8) {
        const unsigned long long grp = (unsigned long long)(i >> 3);
        const U4 u = philox_keyed(a.keys, (uint32_t)grp, (2u << 24) | (uint32_t)(grp >> 32), step32, ch.tensor);
        const int e = (int)(i & 7);
        const uint32_t w = e < 4 ? (e < 2 ? u.x : u.y) : (e < 6 ? u.z : u.w), k16 = (e & 1) ? w >> 16 : w & 0xFFFFu;
        const float mv = in ? m[k] : 0.f, rv = in ? r : 0.f;
        const uint32_t km = scale_code_e4m3(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(mv) & ABS_MASK));
        const uint32_t kv = scale_code_e4m3(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(rv) & ABS_MASK));
        const float qm = round_stochastic<3, -6>(mv * scale_inverse(km), k16);
        const float ar = rv * scale_inverse(kv);
        float qr = round_stochastic<3, -6>(ar, (k16 & 0xFFu) << 8 | k16 >> 8);
        if (ar > 0.f) qr = fmaxf(qr, 0.001953125f);
        if (in) {
          static_cast<uint8_t*>(t.m)[i] = (uint8_t)to_e4m3x2(qm, 0.f);
          static_cast<uint8_t*>(t.v)[i] = (uint8_t)to_e4m3x2(qr, 0.f);
          if ((threadIdx.x & 31) == 0) { t.m_scale[i >> 5] = (uint8_t)km; t.v_scale[i >> 5] = (uint8_t)kv; }
        }
      }
    }
  }
}

// MULTI: more than one push.  With 32-bit states a block per chunk (the hardware deals them: 257 M elements with a bf16 copy 1.04 ms, a grid
// that stays 1.28 ms); with 8-bit states, where the arithmetic counts, a grid that fills the machine once and stays (205 M elements 0.49 ms, a
// block per chunk 0.56 ms).  Four blocks of 64 registers a multiprocessor: fp32 pushes with K > 1 spill 12 to 16 bytes a thread, which does not
// show (50 M elements, four pushes: 290 us with 32-bit states, 214 us with 8-bit ones; their bytes take 306 and 215).  Step and rate read on the device: every block works the coefficients out (257 M elements 1.05 ms, 12.9 M
// 50 against 47 us).
template <int PT, int GT, int BITS, bool MULTI>
__global__ void __launch_bounds__(ADAMW_THREADS, 4) adamw_kernel(const __grid_constant__ AdamwArgs a) {
  __shared__ AdamwCoef coef_s;
  AdamwCoef c = a.coef;
  uint32_t step32 = a.step32;
  if (a.step_dev) {
    const long long step = *a.step_dev;
    if (threadIdx.x == 0) coef_s = adamw_coef(a.beta1, a.beta2, a.coef.eps, a.mean, *a.lr_dev, step);
    __syncthreads();
    c = coef_s;
    step32 = (uint32_t)step;
  }
  AdamwChunk next = a.chunks[blockIdx.x];
  for (uint32_t k = blockIdx.x; k < a.n_chunks; k += gridDim.x) {
    const AdamwChunk ch = next;
    if (k + gridDim.x < a.n_chunks) next = a.chunks[k + gridDim.x];
    const AdamwTensor t = a.tensors[ch.tensor];
    if (t.vec && (long long)(ch.chunk + 1ull) * ADAMW_CHUNK <= t.n) adamw_chunk_wide<PT, GT, BITS, MULTI, true>(a, c, step32, t, ch);
    else if (t.vec) adamw_chunk_wide<PT, GT, BITS, MULTI, false>(a, c, step32, t, ch);
    else adamw_chunk_narrow<PT, GT, BITS, MULTI>(a, c, step32, t, ch);
  }
}

}  // namespace ssim
