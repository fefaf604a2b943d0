// Log probabilities of given tokens, entropies, the likeliest alternatives, and the gradient by the logits, at vocabulary size.
//
// With l = x / T and c = log2(e) / T everything is taken in powers of two: d = c x - m for a whole number m near the largest c x,
//   s = sum 2^d,  q = sum 2^d d,   lse = (m + log2 s) ln 2,  log p = (d - log2 s) ln 2,  H = (log2 s - q / s) ln 2,
// one pass over the row with running m, s, q a thread.  m being whole, moving it scales s and q exactly, and a thread moves it only
// when a logit is over 2^8 times (in 2^d) beyond it, so the rescaling's exponential is rare.  s and q are fp32: a thread adds at most
// vocab / threads terms, then the threads meet in a tree.  m is kept in quarters, m4 = m / 4: a row of nothing but the lowest fp32
// number would overflow as c x.  Where m is beyond 2^28 c x is rounded to steps of 16 and more: fp32 logits one step apart would come out up to 32 off, or equal, so
// that there the reference is the largest logit x0 itself, d = c (x - x0).  16-bit logits of that size are 2^17 and more apart where they differ.
//
// The gradient by x_v is (g (1[v = token] - p_v) - h p_v (log p_v + H)) / T: a second look at the row, which L2 still holds.
//
// The `top` largest logits: the first pass leaves each thread's largest one; the top-th of those is a bound that at least `top`
// logits reach, and every logit that reaches it lies in a thread's share that does.  Those few shares are looked through
// again, a warp a share, and what reaches the bound is ranked by counting, the lower index first among equals.  Where more reach it than the
// list takes (rows of equal logits), the largest is taken `top` times, each time only the share that gave it searched again.
//
// Floor: HBM, the row read once (and the gradient written once).  Measured: 4096 x 131072 bf16 184 us, with eight alternatives 220 (floor 164: 5.8 and 4.9
// TB/s; issue slots 64 %, the special-function unit 56 %: an exponential, and some nine other instructions, an element); 8192 x 50021 bf16 with the
// gradient 361 us (floor 251; more rows are under way than L2 holds, so half of the second look comes from memory); 65536 x 10 fp32 9 us.
#pragma once
#include "act_math.cuh"
#include "lowbits.cuh"
#include "ptx_util.cuh"

namespace ssim {

constexpr int LP_MAX_TOP = 32;
constexpr int LP_THREADS = 1536;            // a multiprocessor's, of the kernel for long rows
constexpr int LP_LIST = 1024;               // logits that may reach the bound
constexpr float LP_LN2 = 0.6931471805599453f;
constexpr float LP_NONE = -200.f;           // 2^-200 is zero

struct LogpArgs {
  const void* x;
  long long rows, vocab, ld;
  const void* tokens;                       // or null
  int token64;
  float c, c4, inv_t;                       // log2(e) / T, a quarter of it, 1 / T
  int top;
  float *logp, *entropy, *lse, *top_logp;   // any may be null
  int* top_ids;
  const float *d_logp, *d_entropy;          // may be null: zero
  void* out;                                // gradient, or null
  long long ldo;
};

__device__ __forceinline__ float max_nan(float a, float b) { float r; asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ uint32_t max_nan_bf16x2(uint32_t a, uint32_t b) { uint32_t r; asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b)); return r; }
constexpr uint32_t LP_LOW_BF16X2 = 0xF149F149u;      // -1e30 twice
__device__ __forceinline__ float neg_inf() { return __uint_as_float(0xFF800000u); }
__device__ __forceinline__ float quiet_nan() { return __uint_as_float(0x7FC00000u); }

// Whole numbers in the order of the logits, NaN above all, both zeros alike; 0 is none and so is 2^32 - 1.  Back: the logit.
__device__ __forceinline__ uint32_t logit_key(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return x != x ? 0xFFFFFFFEu : b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float logit_of_key(uint32_t k) {
  return k > 0xFF800000u ? quiet_nan() : __uint_as_float((k & 0x80000000u) ? k ^ 0x80000000u : ~k);
}
// bits of a key that are the same for all values of one sign of a type
template <int T> struct KeyShift { static constexpr int value = T == T_BF16 ? 16 : T == T_F16 ? 13 : 0; };

// Running reference and sums of some logits of type T.  What the loops need of the reference is kept ready: where the next move is due, the addend of c x.
template <int T>
struct LogSum {
  static constexpr bool FINE = T == T_F32;                   // a far reference is a logit (16-bit logits take their products' differences: 2 % faster)
  float m4 = neg_inf(), s = 0.f, q = 0.f;
  float due = neg_inf(), off = 0.f;                          // m4 + 2; -4 m4 (0 for none)
  bool far = false;                                          // c x may overflow; FINE: off is the reference, m4 its product with c4, due just below that
  static __device__ __forceinline__ bool is_far(float to4) { return fabsf(to4) > 67108864.f && to4 != neg_inf(); }       // up to there the rounding of m4 moves d by 16 at most, for all logits alike
  __device__ __forceinline__ void set(float to4, float x) {  // FINE: x is the logit that gave to4, or a far reference's off
    m4 = to4;
    far = is_far(to4);
    due = FINE && far ? fmaf(fabsf(to4), -2.384185791015625e-7f, to4) : to4 + 2.f;
    off = FINE && far ? (to4 - to4 == 0.f ? x : quiet_nan()) : to4 == neg_inf() ? 0.f : -4.f * to4;   // a product beyond the range counts as infinite: every distance is NaN
  }
  __device__ __forceinline__ void move(float to4, float x, float c4) {          // to a reference to4 >= m4
    float by = 4.f * (to4 - m4);
    if (FINE && (far || is_far(to4))) {
      const float c = 4.f * c4;
      if (far && is_far(to4) && !(x > off)) return;          // its product rounded alike
      by = !is_far(to4) ? -fmaf(off, c, -4.f * to4) : far ? (x - off) * c : m4 == neg_inf() ? 250.f : fmaf(x, c, off);
    }
    if (by < 250.f) {
      const float f = exp2_fast(-by);
      q = (q - by * s) * f;
      s *= f;
    } else {
      s = s == s ? 0.f : s;                                  // a NaN stays
      q = s;
    }
    set(to4, x);
  }
  __device__ __forceinline__ void reach(float most, float c4) {
    const float top4 = __fmul_rn(most, c4);
    if (top4 > due) move(fabsf(top4) < 1048576.f ? rintf(4.f * top4) * 0.25f : top4, most, c4);
  }
  __device__ __forceinline__ float dist4(float x, float c4) const { return FINE ? (x - off) * c4 : __fmul_rn(x, c4) - m4; }      // a quarter of it, of a far reference
  __device__ __forceinline__ float dist(float x, float c, float c4) const { return far ? 4.f * dist4(x, c4) : fmaf(x, c, off); }
  __device__ __forceinline__ void add(float d) {             // d >= LP_NONE or NaN
    const float e = exp2_fast(d);
    s += e;
    q = fmaf(e, d, q);
  }
  template <int N>
  __device__ __forceinline__ void add_far(const float (&x)[N], float c4) {
#pragma unroll
    for (int e = 0; e < N; ++e) add(max_nan(4.f * dist4(x[e], c4), LP_NONE));
  }
  template <int N>
  __device__ __forceinline__ float take(const float (&x)[N], float c, float c4) {
    float most = x[0];
#pragma unroll
    for (int e = 1; e < N; ++e) most = max_nan(most, x[e]);
    reach(most, c4);
    if (far) add_far(x, c4);
    else
#pragma unroll
      for (int e = 0; e < N; ++e) add(max_nan(fmaf(x[e], c, off), LP_NONE));
    return most;
  }
  // Eight logits as they are stored.  bf16: the largest and the way out of -inf two at a time - a logit under -1e30 stands for any such, and its
  // probability is zero without the product 0 (-inf) - unless they all are that small.
  __device__ __forceinline__ float take8(const Raw8<T>& r, float c, float c4) {
    if constexpr (T == T_BF16) {
      const uint32_t m = max_nan_bf16x2(max_nan_bf16x2(r.w[0], r.w[1]), max_nan_bf16x2(r.w[2], r.w[3]));
      const float most = max_nan(__uint_as_float(m << 16), __uint_as_float(m & 0xFFFF0000u));
      reach(most, c4);
      float x[8];
      if (far) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = r.value(e);
        add_far(x, c4);
        return most;
      }
      Raw8<T> f;
#pragma unroll
      for (int k = 0; k < 4; ++k) f.w[k] = max_nan_bf16x2(r.w[k], LP_LOW_BF16X2);
#pragma unroll
      for (int e = 0; e < 8; ++e) add(fmaf(f.value(e), c, off));
      return most;
    } else {
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = r.value(e);
      return take(x, c, c4);
    }
  }
  // The sums of groups of G lanes, in each of them: first the largest reference, then one move, then two trees
  template <int G>
  __device__ __forceinline__ void join_lanes(float c4) {
    float to = m4, x = off;
#pragma unroll
    for (int k = G / 2; k > 0; k >>= 1) to = fmaxf(to, __shfl_xor_sync(0xFFFFFFFFu, to, k));
    if (FINE && __any_sync(0xFFFFFFFFu, is_far(to))) {       // several logits may have this product: the largest
      x = m4 == to ? off : neg_inf();
#pragma unroll
      for (int k = G / 2; k > 0; k >>= 1) x = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, k));
    }
    if (m4 != to || (FINE && far)) move(to, x, c4);
#pragma unroll
    for (int k = G / 2; k > 0; k >>= 1) {
      s += __shfl_xor_sync(0xFFFFFFFFu, s, k);
      q += __shfl_xor_sync(0xFFFFFFFFu, q, k);
    }
  }
};

// What a row's sums say
template <int T>
struct LogRow {
  LogSum<T> t;
  float l2;                                 // log2 s
  bool none;                                // nothing but -inf
  __device__ __forceinline__ explicit LogRow(const LogSum<T>& sum) : t(sum), l2(log2f(sum.s)), none(sum.s == 0.f) {}
  __device__ __forceinline__ float lse() const { return none ? neg_inf() : t.far ? (l2 == l2 ? t.m4 * (4.f * LP_LN2) : l2) : fmaf(4.f, t.m4, l2) * LP_LN2; }
  __device__ __forceinline__ float logp(float x, float c, float c4) const {
    if (none) return neg_inf();
    const float lp = t.far ? (t.dist4(x, c4) - 0.25f * l2) * (4.f * LP_LN2) :
                     fabsf(x) < 1e30f ? (fmaf(x, c, t.off) - l2) * LP_LN2 : (__fmul_rn(x, c4) - t.m4 - 0.25f * l2) * (4.f * LP_LN2);      // c x may overflow
    return lp > 0.f ? 0.f : lp;                              // by rounding only
  }
  __device__ __forceinline__ float entropy() const {
    const float h = (l2 - t.q / t.s) * LP_LN2;
    return none || h < 0.f ? 0.f : h;
  }
};

// The gradient by a logit, p (a lp + b) with lp = log2 p = d - log2 s, as 2^d (a' d + b'), a' = a / s, b' = (b - a log2 s) / s; at the token plus g / T.  d is what the sums
// took: log2 s joined to the addend of c x loses its digits beside a far reference (logits around 1e6: p off by 1.6 %, and a row's gradients then
// do not sum to zero).
template <int T>
struct LogGrad {
  LogSum<T> t;
  float c, c4, a, b, g;                     // a and b: the ones above with a dash
  uint32_t low;                             // twice, in bf16: a logit whose d is LP_NONE or below, by the rounding's step at most
  bool none;
  __device__ __forceinline__ LogGrad(const LogpArgs& k, const LogRow<T>& r, float g_, float h) {
    t = r.t; c = k.c; c4 = k.c4; none = r.none;
    const float by_lp = -h * LP_LN2 * k.inv_t, inv_s = 1.f / r.t.s;
    a = by_lp * inv_s;
    b = (-(g_ + h * r.entropy()) * k.inv_t - by_lp * r.l2) * inv_s;
    g = none ? 0.f : g_ * k.inv_t;
    const uint32_t w = __float_as_uint((LP_NONE - t.off) / c);
    low = ((int32_t)w < 0 ? (w + 0xFFFFu) >> 16 : w >> 16) * 0x10001u;          // rounded down
  }
  __device__ __forceinline__ float at(float x) const {
    if (none) return 0.f;
    const float d = max_nan(t.dist(x, c, c4), LP_NONE);
    return exp2_fast(d) * fmaf(a, d, b);
  }
  // bf16: logits are kept at `low` or above two at a time, so that no d is far below LP_NONE: with -inf, or a mask's lowest number, a d + b could be
  // infinite beside the probability zero (-1e30 as the least: NaN from d_entropy = 342 on at T = 0.001)
  __device__ __forceinline__ void at8(const Raw8<T>& r, float (&x)[8]) const {
    if constexpr (T == T_BF16) {
      if (!t.far && !none) {
        Raw8<T> f;
#pragma unroll
        for (int k = 0; k < 4; ++k) f.w[k] = max_nan_bf16x2(r.w[k], low);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float d = fmaf(f.value(e), c, t.off);
          x[e] = exp2_fast(d) * fmaf(a, d, b);
        }
        return;
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = at(r.value(e));
  }
};

__device__ __forceinline__ long long token_of(const LogpArgs& a, long long row) {
  if (!a.tokens) return -1;
  return a.token64 ? static_cast<const long long*>(a.tokens)[row] : (long long)static_cast<const int*>(a.tokens)[row];
}
__device__ __forceinline__ float token_weight(const LogpArgs& a, long long row, long long token) {   // derivative of the loss by logp
  if (token < 0 || !a.d_logp) return 0.f;
  return token < a.vocab ? a.d_logp[row] : quiet_nan();
}
template <int T>
__device__ __forceinline__ void write_row(const LogpArgs& a, const LogRow<T>& r, long long row, long long token) {
  if (a.lse) a.lse[row] = r.lse();
  if (a.entropy) a.entropy[row] = r.entropy();
  if (a.logp) a.logp[row] = token < 0 ? 0.f : token >= a.vocab ? quiet_nan() : r.logp(Elem<T>::get(a.x, row * a.ld + token), a.c, a.c4);
}

// ---- short rows: G lanes a row, E logits a lane, in registers ---------------------------------------------------------------
template <int T, int G, int E>
__global__ void __launch_bounds__(128) logp_short_kernel(const __grid_constant__ LogpArgs a) {
  const long long row = (long long)blockIdx.x * (128 / G) + threadIdx.x / G;
  const int lane = threadIdx.x % G, vocab = (int)a.vocab;
  const bool live = row < a.rows;
  const long long base = live ? row * a.ld : 0;
  float x[E];
  LogSum<T> t;
#pragma unroll
  for (int i = 0; i < E; ++i) x[i] = live && i * G + lane < vocab ? Elem<T>::get(a.x, base + i * G + lane) : neg_inf();
  t.take(x, a.c, a.c4);
  if (G > 1) t.template join_lanes<G>(a.c4);
  const LogRow<T> r(t);
  const long long token = live ? token_of(a, row) : -1;
  if (live && lane == 0) write_row<T>(a, r, row, token);
  if (a.top) {
    uint32_t key[E];
#pragma unroll
    for (int i = 0; i < E; ++i) key[i] = i * G + lane < vocab ? logit_key(x[i]) : 0u;
    for (int k = 0; k < a.top; ++k) {
      uint32_t best = 0;
#pragma unroll
      for (int i = 0; i < E; ++i) best = max(best, key[i]);
      uint32_t all = best;
#pragma unroll
      for (int o = G / 2; o > 0; o >>= 1) all = max(all, __shfl_xor_sync(0xFFFFFFFFu, all, o));
      int id = 0x7FFFFFFF;
#pragma unroll
      for (int i = E - 1; i >= 0; --i)
        if (key[i] == all && all != 0u) id = i * G + lane;
#pragma unroll
      for (int o = G / 2; o > 0; o >>= 1) id = min(id, __shfl_xor_sync(0xFFFFFFFFu, id, o));
#pragma unroll
      for (int i = 0; i < E; ++i)
        if (i * G + lane == id) key[i] = 0u;
      if (live && lane == 0) {
        if (a.top_ids) a.top_ids[row * a.top + k] = id;
        if (a.top_logp) a.top_logp[row * a.top + k] = r.logp(logit_of_key(all), a.c, a.c4);
      }
    }
  }
  __syncwarp();              // the token's logit has been read: the gradient may go over the logits
  if (a.out && live) {
    const LogGrad<T> d(a, r, token_weight(a, row, token), a.d_entropy ? a.d_entropy[row] : 0.f);
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int v = i * G + lane;
      if (v < vocab) Elem<T>::put(a.out, row * a.ldo + v, d.at(x[i]) + (v == token ? d.g : 0.f));
    }
  }
}

// ---- long rows: a block a row, or a cluster of blocks with a slice each -----------------------------------------------------------
// A slice: elements before the first 16-byte boundary, groups of eight from there, elements behind the last group
template <int T>
struct Slice {
  static constexpr int EB = Elem<T>::bytes;
  const char* at;
  int n, head, groups, tail;                // a slice has less than 2^31 elements
  __device__ __forceinline__ Slice(const void* x, long long first, int n_) : at(static_cast<const char*>(x) + first * EB), n(n_) {
    head = min(n, (int)((-(intptr_t)at) & 15) / EB);
    groups = (n - head) >> 3;
    tail = n - head - 8 * groups;
  }
  __device__ __forceinline__ int index(int group) const { return head + 8 * group; }
  __device__ __forceinline__ int tail_index() const { return head + 8 * groups; }
  __device__ __forceinline__ float one(int i) const { return Elem<T>::get(at, i); }
  __device__ __forceinline__ void load(int group, Raw8<T>& r) const { r.load(at, index(group)); }
};
// Calls f(index in the slice, logit) for the elements of thread t's share
template <int T, int NT, typename F>
__device__ __forceinline__ void each_of_share(const Slice<T>& sl, int t, F f) {
  if (t < sl.head) f(t, sl.one(t));
  for (int g = t; g < sl.groups; g += NT) {
    Raw8<T> r;
    sl.load(g, r);
#pragma unroll
    for (int e = 0; e < 8; ++e) f(sl.index(g) + e, r.value(e));
  }
  if (t < sl.tail) f(sl.tail_index() + t, sl.one(sl.tail_index() + t));
}

// Eight results that nobody reads soon
template <int T>
__device__ __forceinline__ void put8_past(void* p, long long i, const float (&v)[8]) {
  if (T == T_F32) {
    float4* q = reinterpret_cast<float4*>(static_cast<float*>(p) + i);
    __stcs(q, make_float4(v[0], v[1], v[2], v[3]));
    __stcs(q + 1, make_float4(v[4], v[5], v[6], v[7]));
  } else {
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = T == T_BF16 ? float_to_bf16x2(v[2 * k], v[2 * k + 1]) : float_to_f16x2(v[2 * k], v[2 * k + 1]);
    __stcs(reinterpret_cast<uint4*>(static_cast<uint16_t*>(p) + i), make_uint4(w[0], w[1], w[2], w[3]));
  }
}

template <int NT>
struct LogpShared {
  float m4[NT / 32], s[NT / 32], q[NT / 32], off[NT / 32];
  float row[4];                                      // the block's own sums, for the others of the cluster
  unsigned long long list[LP_LIST], best[LP_MAX_TOP], pick[NT / 32];
  int share[NT], shares, listed;
  uint32_t bound;
};

__device__ __forceinline__ unsigned long long rank_word(uint32_t key, uint32_t index) { return (unsigned long long)key << 32 | (0xFFFFFFFFu - index); }

// words [n] in shared memory, all different where not zero -> the first `top` in falling order (zeros where there are fewer)
template <int NT>
__device__ __forceinline__ void rank_words(const unsigned long long* words, int n, int top, unsigned long long* best) {
  if ((int)threadIdx.x < top) best[threadIdx.x] = 0ull;
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += NT) {
    const unsigned long long w = words[i];
    int above = 0;
#pragma unroll 8
    for (int j = 0; j < n; ++j) above += words[j] > w ? 1 : 0;
    if (w && above < top) best[above] = w;
  }
  __syncthreads();
}

template <int T, int NT>
__device__ __noinline__ void top_of_slice(LogpShared<NT>& sh, const Slice<T>& sl, uint32_t first, int top, uint32_t kmax) {
  constexpr int SHIFT = KeyShift<T>::value, PER = NT / 32;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  sh.share[tid] = (int)(kmax >> SHIFT);                                 // not zero where there is a logit
  if (tid == 0) sh.listed = 0;
  __syncthreads();
  if (warp == 0) {                       // one warp finds the bound, bit by bit, and the shares that reach it
    uint32_t key[PER], bound = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) key[i] = (uint32_t)sh.share[32 * i + lane];
    for (int bit = 31 - SHIFT; bit >= 0; --bit) {
      const uint32_t trial = bound | 1u << bit;
      int n = 0;
#pragma unroll
      for (int i = 0; i < PER; ++i) n += key[i] >= trial ? 1 : 0;
      if ((int)__reduce_add_sync(0xFFFFFFFFu, (unsigned)n) >= top) bound = trial;
    }
    int n = 0;
    __syncwarp();
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const bool in = key[i] != 0u && key[i] >= bound;
      const uint32_t who = __ballot_sync(0xFFFFFFFFu, in);
      if (in) sh.share[n + __popc(who & ((1u << lane) - 1u))] = 32 * i + lane;
      n += __popc(who);
    }
    if (lane == 0) { sh.shares = n; sh.bound = bound; }
  }
  __syncthreads();
  const uint32_t bound = sh.bound;
  auto list = [&](int i, float x) {
    const uint32_t key = logit_key(x);
    if ((key >> SHIFT) >= bound) {
      const int at = atomicAdd(&sh.listed, 1);
      if (at < LP_LIST) sh.list[at] = rank_word(key, first + (uint32_t)i);
    }
  };
  for (int k = warp; k < sh.shares; k += NT / 32) {
    const int t = sh.share[k];
    if (lane == 0 && t < sl.head) list(t, sl.one(t));
    if (lane == 1 && t < sl.tail) list(sl.tail_index() + t, sl.one(sl.tail_index() + t));
    for (int g = t + lane * NT; g < sl.groups; g += 32 * NT) {
      Raw8<T> r;
      sl.load(g, r);
#pragma unroll
      for (int e = 0; e < 8; ++e) list(sl.index(g) + e, r.value(e));
    }
  }
  __syncthreads();
  if (sh.listed <= LP_LIST) {
    rank_words<NT>(sh.list, sh.listed, top, sh.best);
    return;
  }
  // the largest, `top` times
  unsigned long long mine = 0, under = ~0ull;
  auto look = [&](int i, float x) {
    const unsigned long long w = rank_word(logit_key(x), first + (uint32_t)i);
    if (w < under && w > mine) mine = w;
  };
  each_of_share<T, NT>(sl, tid, look);
  for (int k = 0; k < top; ++k) {
    unsigned long long w = mine;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const unsigned long long other = __shfl_xor_sync(0xFFFFFFFFu, w, o);
      w = other > w ? other : w;
    }
    if (lane == 0) sh.pick[warp] = w;
    __syncthreads();
    w = sh.pick[0];
    for (int j = 1; j < NT / 32; ++j) w = sh.pick[j] > w ? sh.pick[j] : w;
    if (tid == 0) sh.best[k] = w;
    if (w && mine == w) {
      under = w;
      mine = 0;
      each_of_share<T, NT>(sl, tid, look);
    }
    __syncthreads();
  }
}

template <int T, int NT>
__global__ void __launch_bounds__(NT, LP_THREADS / NT) logp_row_kernel(const __grid_constant__ LogpArgs a, int slices, int slice_len) {
  __shared__ LogpShared<NT> sh;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const long long row = blockIdx.x / (unsigned)slices;
  const int part = (int)(blockIdx.x % (unsigned)slices);               // = the rank in the cluster
  const long long first = (long long)part * slice_len;
  const Slice<T> sl(a.x, row * a.ld + first, (int)max(0ll, min((long long)slice_len, a.vocab - first)));

  LogSum<T> t;
  float most = neg_inf();                                              // of the thread's share
  auto some = [&](const Raw8<T>& r) { most = max_nan(most, t.take8(r, a.c, a.c4)); };
  auto single = [&](float v) {
    const float x[1] = {v};
    most = max_nan(most, t.take(x, a.c, a.c4));
  };
  if (tid < sl.head) single(sl.one(tid));
  if (tid < sl.tail) single(sl.one(sl.tail_index() + tid));
  constexpr int AHEAD = Elem<T>::bytes == 4 ? 2 : 4;                    // groups whose loads are in flight together
  int g = tid;
  for (; g + (AHEAD - 1) * NT < sl.groups; g += AHEAD * NT) {
    Raw8<T> r[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) sl.load(g + k * NT, r[k]);
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) some(r[k]);
  }
  if (g < sl.groups) {                                                  // the last few, also together
    Raw8<T> r[AHEAD - 1];
#pragma unroll
    for (int k = 0; k < AHEAD - 1; ++k)
      if (g + k * NT < sl.groups) sl.load(g + k * NT, r[k]);
#pragma unroll
    for (int k = 0; k < AHEAD - 1; ++k)
      if (g + k * NT < sl.groups) some(r[k]);
  }
  t.template join_lanes<32>(a.c4);
  if (lane == 0) { sh.m4[warp] = t.m4; sh.s[warp] = t.s; sh.q[warp] = t.q; sh.off[warp] = t.off; }
  __syncthreads();
  constexpr int WARPS = NT / 32;
  t = LogSum<T>();                                                          // every warp joins the warps' sums: the same in all
  if (lane < WARPS) { t.set(sh.m4[lane], sh.off[lane]); t.s = sh.s[lane]; t.q = sh.q[lane]; }
  t.template join_lanes<32>(a.c4);
  if (a.top) {
    const bool any = tid < sl.groups || tid < sl.head || tid < sl.tail;
    top_of_slice<T, NT>(sh, sl, (uint32_t)first, a.top, any ? logit_key(most) : 0u);
  }
  if (slices > 1) {
    if (tid == 0) { sh.row[0] = t.m4; sh.row[1] = t.s; sh.row[2] = t.q; sh.row[3] = t.off; }
    __syncthreads();
    cluster_sync_all();
    t = LogSum<T>();
    if (lane < slices) {
      const uint32_t from = cluster_addr(smem_addr(sh.row), (uint32_t)lane);
      t.set(ld_cluster1(from), ld_cluster1(from + 12)); t.s = ld_cluster1(from + 4); t.q = ld_cluster1(from + 8);
    }
    t.template join_lanes<32>(a.c4);
    if (a.top && part == 0) {
      for (int i = tid; i < slices * a.top; i += NT)
        sh.list[i] = ld_cluster64(cluster_addr(smem_addr(sh.best + i % a.top), (uint32_t)(i / a.top)));
      __syncthreads();
    }
    cluster_sync_all();                                                  // the others' sums and lists have been read
    if (a.top && part == 0) rank_words<NT>(sh.list, slices * a.top, a.top, sh.best);
  }
  const LogRow<T> r(t);
  const long long token = token_of(a, row);
  if (part == 0) {
    if (tid == 0) write_row<T>(a, r, row, token);
    if (tid < a.top) {
      const unsigned long long w = sh.best[tid];
      if (a.top_ids) a.top_ids[row * a.top + tid] = (int)(0xFFFFFFFFu - (uint32_t)w);
      if (a.top_logp) a.top_logp[row * a.top + tid] = r.logp(logit_of_key((uint32_t)(w >> 32)), a.c, a.c4);
    }
  }
  if (a.out) {
    // The token's logit was read by thread 0 of the first slice, possibly of another block: where the gradient goes over the
    // logits, nobody writes before that.
    if (slices > 1) cluster_sync_all();
    else __syncthreads();
    const LogGrad<T> d(a, r, token_weight(a, row, token), a.d_entropy ? a.d_entropy[row] : 0.f);
    const int tok = token >= first && token < first + sl.n ? (int)(token - first) : -1;
    char* out = static_cast<char*>(a.out) + (row * a.ldo + first) * Elem<T>::bytes;
    const bool wide = ((reinterpret_cast<uintptr_t>(out) + sl.head * Elem<T>::bytes) & 15) == 0;
    auto put = [&](int i, float x) { Elem<T>::put(out, i, d.at(x) + (i == tok ? d.g : 0.f)); };
    if (tid < sl.head) put(tid, sl.one(tid));
    if (tid < sl.tail) put(sl.tail_index() + tid, sl.one(sl.tail_index() + tid));
    // from the end of the row: what was read last is what L2 still holds when the rows of all blocks are more than it takes; the gradient goes out past it
    for (g = sl.groups - 1 - tid; g >= 0; g -= AHEAD * NT) {
      Raw8<T> raw[AHEAD];
#pragma unroll
      for (int k = 0; k < AHEAD; ++k)
        if (g - k * NT >= 0) sl.load(g - k * NT, raw[k]);
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) {
        if (g - k * NT < 0) break;
        const int at = sl.index(g - k * NT);
        float x[8];
        d.at8(raw[k], x);
        if ((unsigned)(tok - at) < 8u) {
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] += at + e == tok ? d.g : 0.f;
        }
        if (wide) put8_past<T>(out, at, x);
        else
#pragma unroll
          for (int e = 0; e < 8; ++e) Elem<T>::put(out, at + e, x[e]);
      }
    }
  }
}

}  // namespace ssim
