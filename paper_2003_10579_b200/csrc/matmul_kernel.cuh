// c = tail(sum_k a[m, k] b[n, k]) for 16-bit operands on the tensor cores, fp32 accumulators, the tail in fp32, one rounding at the end:
//   tail(s) = act(s + bias) + residual,  s + bias optionally kept in 8 bits as well (ckpt_kernel.cuh), or
//   tail(s) = s act'(z) + residual with z kept in 8 bits.
// Either operand may lie in memory with its rows along k ([m][k]) or along its other axis ([k][m]): TMA brings both into 128-byte swizzled
// tiles as they are, and the instruction takes K-major or MN-major tiles, so a layer's forward product and the two of its backward pass read the
// same tensors without a transposition.
//
// Two kernels.  mm_pair_kernel: pairs of multiprocessors on 256 x 256 tiles (cta_group::2), persistent, two sets of accumulators, for
// large products.  mm_tile_kernel: a 128 x BN tile a block, the blocks of a cluster sharing one along k where there are few; with
// SWAP the operand with few rows is the instruction's N side (16, 32 or 64), so that nothing is multiplied for rows that do not exist.
// Bounds: large products the tensor cores and, over longer runs, the power limit (4096 x 8192 x 8192 436 to 450 us in a user's calls one after
// the other, where a library's product alone takes 420; in runs too short for the limit 348 us = 1.58 PFLOP/s and 356); middling ones a block's chain of stages (300 cycles each: 256 of MMA) beside
// about 4 us of launch, set-up and tail (2048 x 1024 x 512 7.7 us, 600^3 6.7); few rows the weights' way from memory (1 x 4096 x 12288 20.3 us, floor 15.4).
// The tensor cores add fp32 and round towards zero, in their own order: at k = 8192 a sum is 9e-6 of itself off on average (k = 512: 5e-7), a library's 16-bit
// product exactly as much, sums in fp32 instructions 1e-6.  One bf16 result in 217 then comes out a place beside the rounded 64-bit value (fp32 sums: one in 1800).
// Waits are bounded; where one runs out the tile is written as NaN.
#pragma once
#include <type_traits>

#include "act_math.cuh"
#include "ckpt_kernel.cuh"
#include "lowbits.cuh"
#include "ptx_util.cuh"

namespace ssim {

struct MmArgs {
  long long M, N;             // of c
  int kb, kb_split;           // 64-element blocks of k; of them for each block of a cluster
  int tiles_a, tiles_b;       // the instruction's operands: A (128 or 256 rows a tile) and B
  int a_t, b_t;               // operand with its rows along its other axis
  int stage_bytes, stages;    // mm_tile_kernel's ring
  uint32_t idesc;
  // the tail
  int act, grad, bias_type;   // grad: s act'(z)
  const void* bias;
  uint8_t* z_codes;
  uint8_t* z_scales;
  const void* res;
  void* c;
  long long ldr, ldc;
  int vec_c, vec_r;           // rows on 16-byte boundaries (vec_c 2: on 32-byte ones)
};

// ---- the tail -----------------------------------------------------------------------------------------------------------------------
// A lane holds 32 columns of its row, as tensor memory gives them: a block of the 8-bit form needs no exchange between lanes, and a lane
// reads and writes whole 32-byte sectors.  (Four columns a lane through shared memory, so that a warp accesses one row at a time, took three
// times the instructions: 1531 x 2731 outputs 2.1 us plain, 6.2 us with silu and the 8-bit form, against 1.1 and 3.4.)
// Rows off 16-byte boundaries go through a patch of shared memory of the warp's own, sixteen words a row, so that lanes access neighbours.
constexpr int MM_PATCH = 32 * 17 * 4;            // a multiple of 16: bias is read from it four at a time

// 16 words a lane, 32 columns of a 16-bit type or 16 of fp32, to or from rows at any alignment of their elements
template <int T, bool WRITE>
__device__ __forceinline__ void mm_patch_rows(uint32_t* patch, int lane, uint32_t (&w)[16], void* rows, long long ld, long long row0, long long n_rows, long long col0, long long n_cols) {
  if (WRITE) {
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 16; ++j) patch[lane * 17 + j] = w[j];
  }
  __syncwarp();
  // a warp a row of 32 elements of 16 bits, or two rows of 16 of fp32
  constexpr int STEP = T == T_F32 ? 2 : 1;
  const int r0 = T == T_F32 ? lane >> 4 : 0, c = T == T_F32 ? lane & 15 : lane;
  const int left = col0 + c < n_cols ? (int)min(32ll, n_rows - row0) : 0;
  const long long step = STEP * ld;
  using E = typename std::conditional<T == T_F32, uint32_t, uint16_t>::type;
  constexpr int PITCH = 68 / sizeof(E);      // of the patch's rows
  E* at = static_cast<E*>(rows) + ((row0 + r0) * ld + col0 + c);
  E* in = reinterpret_cast<E*>(patch) + r0 * PITCH + c;
  if (WRITE) {
#pragma unroll 8
    for (int r = r0; r < left; r += STEP, at += step, in += STEP * PITCH) *at = *in;
  } else {
    // sixteen loads under way (one behind the other, each waiting for its place in the patch: 1531 x 2731 x 1001 with a residual 32.4 us, 23.0 so)
#pragma unroll 1
    for (int r = r0; r < 32; r += 16 * STEP) {
      E t[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) t[i] = r + i * STEP < left ? at[i * step] : (E)0;
#pragma unroll
      for (int i = 0; i < 16; ++i) in[i * STEP * PITCH] = t[i];
      at += 16 * step;
      in += 16 * STEP * PITCH;
    }
  }
  __syncwarp();
  if (!WRITE) {
#pragma unroll
    for (int j = 0; j < 16; ++j) w[j] = patch[lane * 17 + j];
    __syncwarp();
  }
}
__device__ __forceinline__ void load16(const void* p, uint32_t (&w)[16]) {
  const uint4* q = static_cast<const uint4*>(p);
#pragma unroll
  for (int k = 0; k < 4; ++k) { const uint4 a = q[k]; w[4 * k] = a.x; w[4 * k + 1] = a.y; w[4 * k + 2] = a.z; w[4 * k + 3] = a.w; }
}
// 64 bytes on a boundary of 16 (sectors: of 32)
__device__ __forceinline__ void store16(void* p, const uint32_t (&w)[16], bool sectors) {
  if (sectors) {
    const uint32_t a[8] = {w[0], w[1], w[2], w[3], w[4], w[5], w[6], w[7]}, b[8] = {w[8], w[9], w[10], w[11], w[12], w[13], w[14], w[15]};
    store32(p, a);
    store32(static_cast<char*>(p) + 32, b);
  } else {
    uint4* q = static_cast<uint4*>(p);
#pragma unroll
    for (int k = 0; k < 4; ++k) q[k] = make_uint4(w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]);
  }
}
template <int T>
__device__ __forceinline__ float half_value(uint32_t w, int odd) {       // of two 16-bit elements in a word
  if (T == T_BF16) return __uint_as_float(odd ? w & 0xFFFF0000u : w << 16);
  return f16_to_float(odd ? w >> 16 : w & 0xFFFFu);
}
template <int ACT>
__device__ __forceinline__ void act_row(float (&v)[32]) {
#pragma unroll
  for (int j = 0; j < 32; ++j) v[j] = act_value<ACT>(v[j]);
}
template <int ACT>
__device__ __forceinline__ void slope_row(float (&v)[32], const uint4& a, const uint4& b, float scale) {
  const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    float z[4];
    ckpt_values4(w[k], scale, z);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[4 * k + e] *= act_slope<ACT>(z[e]);
  }
}

// One element of bias as it is stored, and its value
__device__ __forceinline__ uint32_t mm_bias_raw(const MmArgs& g, long long col) {
  if (!g.bias || col >= g.N) return 0u;
  return g.bias_type == T_F32 ? static_cast<const uint32_t*>(g.bias)[col] : static_cast<const uint16_t*>(g.bias)[col];
}
__device__ __forceinline__ float mm_bias_value(const MmArgs& g, uint32_t raw) {
  return g.bias_type == T_F32 ? __uint_as_float(raw) : g.bias_type == T_BF16 ? __uint_as_float(raw << 16) : f16_to_float(raw);
}
template <int T>
__device__ __forceinline__ uint32_t raw_of(const void* p, long long i) { return T == T_F32 ? static_cast<const uint32_t*>(p)[i] : static_cast<const uint16_t*>(p)[i]; }
template <int T>
__device__ __forceinline__ float value_of(uint32_t raw) { return T == T_F32 ? __uint_as_float(raw) : half_value<T>(raw, 0); }

__device__ __forceinline__ void prefetch_l2(const void* p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }
// Asks L2 for what the tail will read of 32 x 32 elements
template <int T>
__device__ __forceinline__ void mm_ahead(const MmArgs& g, long long row, long long col0) {
  if (row >= g.M || col0 >= g.N) return;
  if (g.res) prefetch_l2(static_cast<const char*>(g.res) + (row * g.ldr + col0) * Elem<T>::bytes);
  if (g.grad) prefetch_l2(g.z_codes + (row * ((g.N + 31) >> 5) << 5) + col0);
}

// Of a warp's 32 rows from row0 on, the 32 columns from col0 on (a multiple of 32).  Every lane takes part, whatever exists.  Made before the sums are read:
// what else the tail reads is then under way, and stays as it is stored (a conversion would wait for it).  Asking for it a chunk ahead, in registers,
// cost more in moves than it hid; instead L2 is asked for a tile's lines while the products run (mm_ahead).
template <int T>
struct MmRows {
  long long row, row0, col0;
  int cols;                                  // of the 32 that exist; none in a row behind the last
  bool wide_res;
  uint4 za, zb;
  uint32_t zs, bias;                         // bias: of column col0 + lane
  uint32_t r[T == T_F32 ? 32 : 16];
  __device__ __forceinline__ MmRows() {}
  __device__ __forceinline__ MmRows(const MmArgs& g, long long row0_, long long col0_, int lane, uint32_t bias_) : row(row0_ + lane), row0(row0_), col0(col0_), bias(bias_) {
    cols = row < g.M ? (int)max(0ll, min(32ll, g.N - col0)) : 0;
    if (g.grad && cols > 0) {
      const long long at = row * ((g.N + 31) >> 5) + (col0 >> 5);
      const uint4* codes = reinterpret_cast<const uint4*>(g.z_codes + 32 * at);
      za = codes[0]; zb = codes[1];
      zs = g.z_scales[at];
    }
    wide_res = g.vec_r && col0 + 32 <= g.N;
    if (g.res && wide_res && cols > 0) {
#pragma unroll
      for (int h = 0; h < (T == T_F32 ? 2 : 1); ++h) {
        uint32_t w[16];
        load16(static_cast<const char*>(g.res) + (row * g.ldr + col0 + 16 * h) * Elem<T>::bytes, w);
#pragma unroll
        for (int j = 0; j < 16; ++j) r[16 * h + j] = w[j];
      }
    }
  }
  __device__ __forceinline__ void finish(const MmArgs& g, float (&v)[32], int lane, uint32_t* patch) {
    if (g.grad) {
      if (cols > 0) {
        const float scale = scale_value(zs);
        if (g.act == ACT_RELU) slope_row<ACT_RELU>(v, za, zb, scale);
        else if (g.act == ACT_GELU) slope_row<ACT_GELU>(v, za, zb, scale);
        else if (g.act == ACT_SILU) slope_row<ACT_SILU>(v, za, zb, scale);
        if (zs == 255u) {                    // a NaN block
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] = scale;
        }
      }
    } else {
      if (g.bias) {                          // each lane's column to all lanes
        __syncwarp();
        patch[lane] = __float_as_uint(mm_bias_value(g, bias));
        __syncwarp();
        const float4* q = reinterpret_cast<const float4*>(patch);
#pragma unroll
        for (int k = 0; k < 8; ++k) { const float4 c = q[k]; v[4 * k] += c.x; v[4 * k + 1] += c.y; v[4 * k + 2] += c.z; v[4 * k + 3] += c.w; }
        __syncwarp();
      }
      if (g.z_codes) {
        if (cols < 32) {
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] = j < cols ? v[j] : 0.f;      // the tail of a row of codes is zero
        }
        float most = 0.f;
#pragma unroll
        for (int j = 0; j < 32; j += 2) most = max3_abs(most, v[j], v[j + 1]);
        const uint32_t code = scale_code_e4m3(__float_as_uint(most) & ABS_MASK);
        const float inv = scale_inverse(code);
        uint32_t w[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) w[k] = to_e4m3x4(v[4 * k] * inv, v[4 * k + 1] * inv, v[4 * k + 2] * inv, v[4 * k + 3] * inv);
        if (cols > 0) {
          const long long at = row * ((g.N + 31) >> 5) + (col0 >> 5);
          uint4* to = reinterpret_cast<uint4*>(g.z_codes + 32 * at);
          to[0] = make_uint4(w[0], w[1], w[2], w[3]);
          to[1] = make_uint4(w[4], w[5], w[6], w[7]);
          g.z_scales[at] = (uint8_t)code;
        }
      }
      if (g.act == ACT_RELU) act_row<ACT_RELU>(v);
      else if (g.act == ACT_GELU) act_row<ACT_GELU>(v);
      else if (g.act == ACT_SILU) act_row<ACT_SILU>(v);
    }
    if (g.res) {
      if (!wide_res) {
#pragma unroll
        for (int h = 0; h < (T == T_F32 ? 2 : 1); ++h) {
          uint32_t w[16];
          mm_patch_rows<T, false>(patch, lane, w, const_cast<void*>(g.res), g.ldr, row0, g.M, col0 + 16 * h, g.N);
#pragma unroll
          for (int j = 0; j < 16; ++j) r[16 * h + j] = w[j];
        }
      }
#pragma unroll
      for (int j = 0; j < 32; ++j) v[j] += T == T_F32 ? __uint_as_float(r[j]) : half_value<T>(r[T == T_F32 ? 0 : j >> 1], j & 1);
    }
    const bool wide = g.vec_c && col0 + 32 <= g.N;
#pragma unroll
    for (int h = 0; h < (T == T_F32 ? 2 : 1); ++h) {
      uint32_t w[16];
#pragma unroll
      for (int j = 0; j < 16; ++j)
        w[j] = T == T_F32 ? __float_as_uint(v[(16 * h + j) & 31]) : T == T_BF16 ? float_to_bf16x2(v[2 * j], v[2 * j + 1]) : float_to_f16x2(v[2 * j], v[2 * j + 1]);
      if (!wide) mm_patch_rows<T, true>(patch, lane, w, g.c, g.ldc, row0, g.M, col0 + 16 * h, g.N);
      else if (cols > 0) store16(static_cast<char*>(g.c) + (row * g.ldc + col0 + 16 * h) * Elem<T>::bytes, w, g.vec_c == 2);
    }
  }
};

// With the operands swapped a lane holds one column of eight of the few rows; 32 lanes are a block of the 8-bit form, and neighbours.
template <int T>
struct MmFew {
  long long row0, col;
  uint32_t r[8], z[8], zs[8], bias;
  __device__ __forceinline__ MmFew() {}
  __device__ __forceinline__ MmFew(const MmArgs& g, long long row0_, long long col_, uint32_t bias_) : row0(row0_), col(col_), bias(bias_) {
    const long long blocks = (g.N + 31) >> 5;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const bool here = col < g.N && row0 + j < g.M;
      if (g.res && here) r[j] = raw_of<T>(g.res, (row0 + j) * g.ldr + col);
      if (g.grad && here) { z[j] = g.z_codes[(row0 + j) * blocks * 32 + col]; zs[j] = g.z_scales[(row0 + j) * blocks + (col >> 5)]; }
    }
  }
  __device__ __forceinline__ void finish(const MmArgs& g, float (&v)[8]) {
    const bool in = col < g.N;
    if (!g.grad) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] += mm_bias_value(g, bias);
      if (g.z_codes) {
        const long long blocks = (g.N + 31) >> 5;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float x = in ? v[j] : 0.f;
          const uint32_t code = scale_code_e4m3(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(x) & ABS_MASK));
          if (row0 + j < g.M && col < 32 * blocks) {
            g.z_codes[(row0 + j) * blocks * 32 + col] = (uint8_t)to_e4m3x2(x * scale_inverse(code), 0.f);
            if ((col & 31) == 0) g.z_scales[(row0 + j) * blocks + (col >> 5)] = (uint8_t)code;
          }
        }
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (!in || row0 + j >= g.M) continue;
      const float at = g.grad ? from_e4m3x2(z[j]).x * scale_value(zs[j]) : v[j];
      if (g.act == ACT_RELU) v[j] = g.grad ? v[j] * act_slope<ACT_RELU>(at) : act_value<ACT_RELU>(at);
      else if (g.act == ACT_GELU) v[j] = g.grad ? v[j] * act_slope<ACT_GELU>(at) : act_value<ACT_GELU>(at);
      else if (g.act == ACT_SILU) v[j] = g.grad ? v[j] * act_slope<ACT_SILU>(at) : act_value<ACT_SILU>(at);
      if (g.grad && zs[j] == 255u) v[j] = at;                // a NaN block
      if (g.res) v[j] += value_of<T>(r[j]);
      Elem<T>::put(g.c, (row0 + j) * g.ldc + col, v[j]);
    }
  }
};

// ---- loads and instructions ---------------------------------------------------------------------------------------------------------
// fp32 accumulators; bf: bf16 operands (else fp16); m, n: the instruction's shape
__host__ __device__ inline uint32_t mm_idesc(int m, int n, int bf, int a_t, int b_t) {
  return (1u << 4) | ((uint32_t)bf << 7) | ((uint32_t)bf << 10) | ((uint32_t)a_t << 15) | ((uint32_t)b_t << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
__device__ __forceinline__ uint64_t mm_desc(uint32_t saddr, int t) { return t ? tc_desc_mnmajor(saddr, 8192, 1024) : tc_desc_kmajor(saddr); }
// sixteen elements of k further: 32 bytes along a row, or sixteen rows of 128 bytes (descriptors count in 16 bytes)
__device__ __forceinline__ uint32_t mm_desc_step(int t) { return t ? 128u : 2u; }

// The first lane's value, which the compiler then knows to be the same in all: the role of a warp and what its MMAs take stay in uniform registers (a
// stage of four MMAs was issued in 550 cycles without it)
template <typename V>
__device__ __forceinline__ V uniform(V v) { return __shfl_sync(0xFFFFFFFFu, v, 0); }

// Where operands are copied first, the product is launched while the copy runs and sets itself up; the warp that loads the operands, the only one that touches
// what the copy writes, waits here until all of that is done, and the others for it at a barrier: no wait with a limit begins before.  The copy itself
// is launched behind everything before it, so what else the product reads and writes is in order.  Without a copy this returns at once.  (37 x 2051 x 5003
// 24.1 -> 22.5 us, a block of 1531 x 1001 x 2731 forward and backward 227 -> 215; both since faster by their copies' rows on lines.)
__device__ __forceinline__ void await_copies() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// Issued by one elected lane of a converged warp
__device__ __forceinline__ void mm_mma(uint32_t d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\telect.sync _|q, 0xFFFFFFFF;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void mm_mma_pair(uint32_t d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\telect.sync _|q, 0xFFFFFFFF;\n\t"
      "@q tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}

// ---- a 128 x BN tile a block --------------------------------------------------------------------------------------------------------
//   warp 0     producer: TMA loads into the ring
//   warp 1     allocates tensor memory; one lane issues the MMAs
//   all eight  the tail, each 32 lanes of tensor memory and half of the columns.  In a cluster the sums go to shared memory (over the ring, which
//              every MMA has read by then), and each block takes its share of the tile over the blocks, in their order: the same bits every time
constexpr int MM_THREADS = 256, MM_MAX_STAGES = 12, MM_A_BYTES = 16384;
constexpr int MM_RING = 98304, MM_RING_WIDE = 2 * MM_RING, MM_RING_NARROW = 73728;    // bytes, with what else there is: for two blocks to a multiprocessor, for one, for three
constexpr int MM_OFF_PATCH = MM_RING - 8 * MM_PATCH;            // the warps' patches, behind the sums
__host__ __device__ constexpr int mm_pitch(int bn, bool swap) { return swap ? 132 : bn + 4; }     // floats between lines of sums: rows, or (swap) columns of tensor memory
__host__ __device__ constexpr int mm_part_bytes(int bn, bool swap) { return (swap ? bn : 128) * mm_pitch(bn, swap) * 4; }

// Columns [col, col + 32) of rows [row, row + 32) of the sums that the n blocks of a cluster hold in shared memory at `part`, added in the blocks'
// order; a lane gets its row.  Read four rows of 128 bytes at a time (a row a lane took twice as long) and left in this block's place of the
// chunk, which nobody else reads.
template <int PITCH>
__device__ __forceinline__ void mm_sum_chunk(float* part, uint32_t part_addr, int row, int col, int n, int lane, float (&v)[32]) {
  const uint32_t at = (uint32_t)((row + (lane >> 3)) * PITCH + col + (lane & 7) * 4);
#pragma unroll 1
  for (int k0 = 0; k0 < 8; k0 += 4) {
    float4 t[4];
#pragma unroll 1
    for (int r = 0; r < n; ++r) {
      const uint32_t from = cluster_addr(part_addr + 4u * at, (uint32_t)r) + 16u * (uint32_t)(PITCH * k0);
      float4 p[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) p[k] = ld_cluster4(from + 16u * (uint32_t)(PITCH * k));
#pragma unroll
      for (int k = 0; k < 4; ++k) t[k] = r == 0 ? p[k] : make_float4(t[k].x + p[k].x, t[k].y + p[k].y, t[k].z + p[k].z, t[k].w + p[k].w);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) *reinterpret_cast<float4*>(part + at + 4 * PITCH * (k0 + k)) = t[k];
  }
  __syncwarp();
  const float* mine = part + (row + lane) * PITCH + col;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const float4 q = *reinterpret_cast<const float4*>(mine + 4 * k);
    v[4 * k] = q.x; v[4 * k + 1] = q.y; v[4 * k + 2] = q.z; v[4 * k + 3] = q.w;
  }
}

template <int BN, int T, bool SWAP, bool SPLIT>
__global__ void __launch_bounds__(MM_THREADS, 2) mm_tile_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ MmArgs g) {
  extern __shared__ unsigned char smem_raw[];
  __shared__ __align__(8) unsigned long long bars_s[2 * MM_MAX_STAGES + 1];
  __shared__ uint32_t tmem_slot;
  const uint32_t raw = smem_addr(smem_raw), base = (raw + 1023u) & ~1023u;
  unsigned char* base_p = smem_raw + (base - raw);
  const int tid = threadIdx.x, lane = tid & 31, warp = uniform(tid >> 5);
  const uint32_t bars = smem_addr(bars_s);
  auto full = [&](int s) { return bars + 8u * s; };
  auto empty = [&](int s) { return bars + 8u * (MM_MAX_STAGES + s); };
  const uint32_t acc_bar = bars + 16u * MM_MAX_STAGES;
  constexpr int TMEM_COLS = BN < 32 ? 32 : BN;

  // tiles in bands of eight of A: neighbouring blocks share rows of both operands in L2
  const int tile = blockIdx.x, band = tile / (8 * g.tiles_b), in_band = tile % (8 * g.tiles_b);
  const int band_rows = min(8, g.tiles_a - band * 8);
  const int a0 = (band * 8 + in_band % band_rows) * 128, b0 = in_band / band_rows * BN;
  const int k_begin = SPLIT ? (int)blockIdx.y * g.kb_split : 0, n_it = (SPLIT ? min(g.kb, k_begin + g.kb_split) : g.kb) - k_begin;

  // the loads of one stage, which the producer has found empty, by the lane that is `on` of a converged warp
  auto load = [&](uint32_t on, int it, int s) {
    const uint32_t at = base + (uint32_t)(s * g.stage_bytes), to_b = at + MM_A_BYTES;
    const int k0 = (k_begin + it) * 64;
    mbar_arrive_expect_tx_if(on, full(s), (uint32_t)g.stage_bytes);
    if (g.a_t) {
      tma_load_2d_if(on, at, &map_a, a0, k0, full(s));
      tma_load_2d_if(on, at + 8192, &map_a, a0 + 64, k0, full(s));
    } else {
      tma_load_2d_if(on, at, &map_a, k0, a0, full(s));
    }
    if (g.b_t) {
      tma_load_2d_if(on, to_b, &map_b, b0, k0, full(s));
      if (BN > 64) tma_load_2d_if(on, to_b + 8192, &map_b, b0 + 64, k0, full(s));
    } else {
      tma_load_2d_if(on, to_b, &map_b, k0, b0, full(s));
    }
  };
  const uint32_t on = lane == 0;
  if (warp == 0) {
    if (lane == 0) {
      for (int s = 0; s < g.stages; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
      mbar_init(acc_bar, 1);
      mbar_fence_init();
    }
    __syncwarp();
    await_copies();
    for (int it = 0; it < min(n_it, g.stages); ++it) load(on, it, it);       // the first round of the ring needs nobody else
  }
  if (warp == 1) tc_alloc(smem_addr(&tmem_slot), TMEM_COLS);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = uniform(tmem_slot);
  bool failed = false;
  if (warp == 0) {
    int s = 0, issued = min(n_it, g.stages);
    uint32_t phase = 0;
    for (int it = g.stages; it < n_it; ++it) {
      if (!mbar_wait_all(empty(s), phase)) { failed = true; break; }
      load(on, it, s);
      issued = it + 1;
      if (++s == g.stages) { s = 0; phase ^= 1u; }
    }
    if (failed)     // let what is in flight land (a bounded time) before the block gives up its shared memory
      for (int it = max(0, issued - g.stages); it < issued; ++it) mbar_wait_all(full(it % g.stages), (uint32_t)((it / g.stages) & 1), 1u << 14);
  } else if (warp == 1) {
    const uint64_t adesc = mm_desc(base, g.a_t), bdesc = mm_desc(base + MM_A_BYTES, g.b_t);
    const uint32_t astep = mm_desc_step(g.a_t), bstep = mm_desc_step(g.b_t);
    int s = 0;
    uint32_t phase = 0;
    bool there = false;                      // the stage's operands are known to have landed
    for (int it = 0; it < n_it; ++it) {
      if (!there && !mbar_wait_all(full(s), phase)) { failed = true; break; }
      tc_fence_after();
      const uint32_t at = (uint32_t)(s * g.stage_bytes) >> 4;
      mm_mma(tmem, adesc + at, bdesc + at, g.idesc, it > 0 ? 1u : 0u);
      mm_mma(tmem, adesc + at + astep, bdesc + at + bstep, g.idesc, 1u);
      const int s_now = s;
      if (++s == g.stages) { s = 0; phase ^= 1u; }
      there = __all_sync(0xFFFFFFFFu, mbar_test(full(s), phase));                   // looked at while this stage's MMAs are queued
      mm_mma(tmem, adesc + at + 2 * astep, bdesc + at + 2 * bstep, g.idesc, 1u);
      mm_mma(tmem, adesc + at + 3 * astep, bdesc + at + 3 * bstep, g.idesc, 1u);
      tc_commit_elected(empty(s_now));
      if (it == n_it - 1) tc_commit_elected(acc_bar);
    }
  }
  __syncwarp();
  const int q = warp & 3, half = warp >> 2;
  const uint32_t trow = tmem + ((uint32_t)(32 * q) << 16);
  uint32_t* patch = reinterpret_cast<uint32_t*>(base_p + MM_OFF_PATCH + warp * MM_PATCH);
  float* part = reinterpret_cast<float*>(base_p);
  constexpr int PITCH = mm_pitch(BN, SWAP), CHUNKS = SWAP ? BN / 8 : BN / 32, WIDTH = BN / CHUNKS;     // columns of tensor memory, 8 or 32 at a time
  // what the tail reads besides the sums: of the lane's column (SWAP) or of the 32 columns of each of the warp's chunks, before the wait
  uint32_t bias[2] = {0u, 0u};
  if (SWAP) bias[0] = mm_bias_raw(g, a0 + 32 * q + lane);
  else
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (half + 2 * i < CHUNKS) {
        bias[i] = mm_bias_raw(g, b0 + 32 * (half + 2 * i) + lane);
        if (!SPLIT) mm_ahead<T>(g, a0 + 32 * q + lane, b0 + 32 * (half + 2 * i));
      }
  if (n_it > 0 && !mbar_wait_warp_long(acc_bar, 0)) failed = true;
  tc_fence_after();
#pragma unroll 1
  for (int ch = half; ch < CHUNKS; ch += 2) {
    if (SWAP && b0 + 8 * ch >= g.M) break;
    MmFew<T> few;
    MmRows<T> rows;
    if constexpr (!SPLIT && SWAP) few = MmFew<T>(g, b0 + 8 * ch, a0 + 32 * q + lane, bias[0]);
    if constexpr (!SPLIT && !SWAP) rows = MmRows<T>(g, a0 + 32 * q, b0 + 32 * ch, lane, ch == half ? bias[0] : bias[1]);
    float v[WIDTH];
    uint32_t w[WIDTH];
    if constexpr (SWAP) tc_ld8_async(trow + 8 * ch, w);
    else tc_ld32_async(trow + 32 * ch, w);
    tc_ld_wait();
#pragma unroll
    for (int j = 0; j < WIDTH; ++j) v[j] = __uint_as_float(failed ? 0x7FC00000u : n_it == 0 ? 0u : w[j]);       // no k at all: sums of nothing
    if constexpr (SPLIT && SWAP) {
#pragma unroll
      for (int j = 0; j < 8; ++j) part[(8 * ch + j) * PITCH + 32 * q + lane] = v[j];
    } else if constexpr (SPLIT) {
#pragma unroll
      for (int j = 0; j < 32; j += 4) *reinterpret_cast<float4*>(part + (32 * q + lane) * PITCH + 32 * ch + j) = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
    } else if constexpr (SWAP) {
      few.finish(g, v);
    } else {
      rows.finish(g, v, lane, patch);
    }
  }
  if constexpr (SPLIT) {
    // chunks of 32 lanes, dealt to the blocks and then to their warps
    const int rank = (int)cluster_rank(), n = (int)gridDim.y, tasks = 4 * (SWAP ? (int)min((long long)CHUNKS, (g.M - b0 + 7) / 8) : CHUNKS);     // of rows that exist
    int task = rank + n * warp;
    auto ahead = [&]() {                                                             // under way while the blocks meet
      if (task >= tasks) return 0u;
      if (!SWAP) mm_ahead<T>(g, a0 + 32 * (task & 3) + lane, b0 + 32 * (task >> 2));
      return mm_bias_raw(g, SWAP ? a0 + 32 * (task & 3) + lane : b0 + 32 * (task >> 2) + lane);
    };
    uint32_t raw = ahead();
    __syncthreads();
    cluster_sync_all();
#pragma unroll 1
    while (task < tasks) {
      const int tq = task & 3, ch = task >> 2;
      if constexpr (SWAP) {
        MmFew<T> few(g, b0 + 8 * ch, a0 + 32 * tq + lane, raw);
        const uint32_t from = base + 4u * (uint32_t)(8 * ch * PITCH + 32 * tq + lane);
        float v[8], p[4][8];                                                         // four blocks at a time
#pragma unroll 1
        for (int r = 0; r < n; r += 4) {
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (r + k < n) {
              const uint32_t at = cluster_addr(from, (uint32_t)(r + k));
#pragma unroll
              for (int j = 0; j < 8; ++j) p[k][j] = ld_cluster1(at + 4u * (uint32_t)(j * PITCH));
            }
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (r + k < n) {
#pragma unroll
              for (int j = 0; j < 8; ++j) v[j] = r + k == 0 ? p[k][j] : v[j] + p[k][j];
            }
        }
        few.finish(g, v);
      } else {
        MmRows<T> rows(g, a0 + 32 * tq, b0 + 32 * ch, lane, raw);
        float v[32];
        mm_sum_chunk<PITCH>(part, base, 32 * tq, 32 * ch, n, lane, v);
        rows.finish(g, v, lane, patch);
      }
      task += n * (MM_THREADS / 32);
      raw = ahead();
    }
    cluster_sync_all();                  // nobody leaves while its sums may still be read
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) tc_dealloc(tmem, TMEM_COLS);
}

// ---- two multiprocessors on a 256 x 256 tile -----------------------------------------------------------------------------------------
//   warp 0      TMA loads (leader's barrier): each block its 128 rows of A and its half of B's
//   warp 1      tensor memory; in the leader one lane issues the MMAs for both
//   warps 2-9   the tail: a warp takes 32 rows x 128 columns, 32 columns at a time
// Two sets of accumulators (2 x 256 columns of tensor memory): a tile's tail runs beside the next one's MMAs.
// (Two pairs of a cluster sharing a tile along k were built and dropped: 256 x 8192 x 8192 38.9 -> 35.0 us, 300 x 4096 x 4096 21.8 -> 21.1, others slower;
// clusters of four blocks of this size fit the device 32 times at most.)
constexpr int MMP_THREADS = 320, MMP_STAGES = 6, MMP_HALF = 128 * 128, MMP_STAGE = 2 * MMP_HALF;
constexpr int MMP_OFF_STORE = MMP_STAGES * MMP_STAGE;
constexpr int MMP_OFF_BARS = MMP_OFF_STORE + 8 * MM_PATCH;
constexpr int MMP_SMEM = MMP_OFF_BARS + 8 * (2 * MMP_STAGES + 4) + 16 + 1024;
static_assert(MMP_SMEM <= 227 * 1024, "the ring and the tail's patches must fit");


template <int T>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(MMP_THREADS, 1)
mm_pair_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ MmArgs g) {
  extern __shared__ unsigned char smem_raw[];
  const uint32_t raw = smem_addr(smem_raw), base = (raw + 1023u) & ~1023u;      // the same offset in both blocks
  unsigned char* base_p = smem_raw + (base - raw);
  const int tid = threadIdx.x, lane = tid & 31, warp = uniform(tid >> 5);
  const uint32_t rank = cluster_rank();
  const uint32_t bars = base + MMP_OFF_BARS;
  auto full = [&](int s) { return bars + 8u * s; };                             // both blocks' operands have landed: the leader's count
  auto empty = [&](int s) { return bars + 8u * (MMP_STAGES + s); };
  auto acc_full = [&](int b) { return bars + 8u * (2 * MMP_STAGES + b); };
  auto acc_empty = [&](int b) { return bars + 8u * (2 * MMP_STAGES + 2 + b); };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(base_p + MMP_OFF_BARS + 8 * (2 * MMP_STAGES + 4));

  if (tid == 0) {
    for (int s = 0; s < MMP_STAGES; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
    for (int b = 0; b < 2; ++b) { mbar_init(acc_full(b), 1); mbar_init(acc_empty(b), 16); }      // eight warps of each block
    mbar_fence_init();
    prefetch_map(&map_a); prefetch_map(&map_b);
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(tmem_slot)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  if (warp == 0) await_copies();
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();                                                           // barriers of both blocks are set up
  tc_fence_after();
  const uint32_t tmem = uniform(*tmem_slot);
  const int n_tiles = g.tiles_a * g.tiles_b, pairs = (int)gridDim.x >> 1;
  bool failed = false;

  // tiles in bands of eight of A: pairs that run together share rows of both operands in L2
  auto tile_at = [&](int tile, int& a0, int& b0) {
    const int band = tile / (8 * g.tiles_b), in_band = tile % (8 * g.tiles_b), band_rows = min(8, g.tiles_a - band * 8);
    a0 = (band * 8 + in_band % band_rows) * 256 + (int)rank * 128;
    b0 = in_band / band_rows * 256;
  };

  if (warp == 0) {
    const uint32_t on = lane == 0, on_leader = on && rank == 0;
    Ring r(1);
    for (int tile = (int)blockIdx.x >> 1; tile < n_tiles && !failed; tile += pairs) {
      int a0, b0;
      tile_at(tile, a0, b0);
      b0 += (int)rank * 128;
      for (int it = 0; it < g.kb; ++it, r.step<MMP_STAGES>()) {
        if (!mbar_wait_all(empty(r.s), r.phase)) { failed = true; break; }
        const uint32_t at = base + (uint32_t)r.s * MMP_STAGE, to_b = at + MMP_HALF, bar = cluster_addr(full(r.s), 0);
        const int k0 = it * 64;
        mbar_arrive_expect_tx_if(on_leader, full(r.s), 2u * MMP_STAGE);
        if (g.a_t) {
          tma_load_2d_pair_if(on, at, &map_a, a0, k0, bar);
          tma_load_2d_pair_if(on, at + 8192, &map_a, a0 + 64, k0, bar);
        } else {
          tma_load_2d_pair_if(on, at, &map_a, k0, a0, bar);
        }
        if (g.b_t) {
          tma_load_2d_pair_if(on, to_b, &map_b, b0, k0, bar);
          tma_load_2d_pair_if(on, to_b + 8192, &map_b, b0 + 64, k0, bar);
        } else {
          tma_load_2d_pair_if(on, to_b, &map_b, k0, b0, bar);
        }
      }
    }
    if (failed)
      for (int i = 0; i < 1000; ++i) __nanosleep(1000);                         // let what is in flight land
    __syncwarp();
  } else if (warp == 1) {
    if (rank == 0) {
      const uint64_t adesc = mm_desc(base, g.a_t), bdesc = mm_desc(base + MMP_HALF, g.b_t);
      const uint32_t astep = mm_desc_step(g.a_t), bstep = mm_desc_step(g.b_t);
      Ring r(0);
      int buf = 0;
      uint32_t acc_phase = 1;
      bool there = false;                                                       // the stage's operands are known to have landed
      for (int tile = (int)blockIdx.x >> 1; tile < n_tiles && !failed; tile += pairs) {
        if (!mbar_wait_all(acc_empty(buf), acc_phase)) { failed = true; break; }
        tc_fence_after();
        const uint32_t d = tmem + 256u * buf;
        for (int it = 0; it < g.kb; ++it) {
          if (!there && !mbar_wait_all(full(r.s), r.phase)) { failed = true; break; }
          tc_fence_after();
          const uint32_t at = (uint32_t)(r.s * (MMP_STAGE / 16));
          mm_mma_pair(d, adesc + at, bdesc + at, g.idesc, it > 0 ? 1u : 0u);
          mm_mma_pair(d, adesc + at + astep, bdesc + at + bstep, g.idesc, 1u);
          const int s_now = r.s;
          r.step<MMP_STAGES>();
          there = __all_sync(0xFFFFFFFFu, mbar_test(full(r.s), r.phase));       // looked at while this stage's MMAs are queued
          mm_mma_pair(d, adesc + at + 2 * astep, bdesc + at + 2 * bstep, g.idesc, 1u);
          mm_mma_pair(d, adesc + at + 3 * astep, bdesc + at + 3 * bstep, g.idesc, 1u);
          tc_commit_pair(empty(s_now));
          if (it == g.kb - 1) tc_commit_pair(acc_full(buf));
        }
        buf ^= 1;
        if (buf == 0) acc_phase ^= 1u;
      }
    }
    __syncwarp();
  } else {
    const int q = warp & 3, half = (warp - 2) >> 2;
    uint32_t* patch = reinterpret_cast<uint32_t*>(base_p + MMP_OFF_STORE + (warp - 2) * MM_PATCH);
    int buf = 0;
    uint32_t phase = 0;
    for (int tile = (int)blockIdx.x >> 1; tile < n_tiles; tile += pairs) {
      int a0, b0;
      tile_at(tile, a0, b0);
      const uint32_t trow = tmem + ((uint32_t)(32 * q) << 16) + 256u * buf + 128 * half, done = cluster_addr(acc_empty(buf), 0);
      a0 += 32 * q;
      b0 += 128 * half;
      uint32_t bias[4];
#pragma unroll
      for (int ch = 0; ch < 4; ++ch) {
        bias[ch] = mm_bias_raw(g, b0 + 32 * ch + lane);
        mm_ahead<T>(g, a0 + lane, b0 + 32 * ch);
      }
      if (!failed && !mbar_wait_warp_long(acc_full(buf), phase)) failed = true;           // from then on every tile of this block is NaN
      tc_fence_after();
#pragma unroll 1
      for (int ch = 0; ch < 4; ++ch) {
        uint32_t w[32];
        tc_ld32_async(trow + 32 * ch, w);
        MmRows<T> rows(g, a0, b0 + 32 * ch, lane, ch < 2 ? (ch == 0 ? bias[0] : bias[1]) : ch == 2 ? bias[2] : bias[3]);
        tc_ld_wait();
        if (ch == 3) {                                                          // the accumulators are read: the tile after the next may start
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive_cluster(done);
        }
        float v[32];
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(failed ? 0x7FC00000u : w[j]);
        rows.finish(g, v, lane, patch);
      }
      buf ^= 1;
      if (buf == 0) phase ^= 1u;
    }
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();                        // nobody leaves while the other may still load, commit or arrive here
  if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
}

// ---- operands that TMA cannot read -----------------------------------------------------------------------------------------------------
// Rows that do not start on 16-byte boundaries are copied to rows that do before the product: one read
// and one write more of an operand that the tiles read many times.
struct MmRepack {
  struct One { const uint16_t* x; uint16_t* out; long long rows, cols, ld, pitch; } of[2];
  int n;
};
// 16 bytes from any even address, from the two aligned pieces that hold them (5003 x 2051 from memory: 8.7 us, element by element 8.9)
__device__ __forceinline__ uint4 unaligned16(const uint16_t* p) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p);
  const uint4* q = reinterpret_cast<const uint4*>(a & ~(uintptr_t)15);
  const uint4 lo = q[0], hi = q[1];
  uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
  const int by = (int)(a & 15) >> 1;                       // elements
  if (by & 4)
#pragma unroll
    for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
  if (by & 2)
#pragma unroll
    for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
  if (by & 1)
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 16);
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__global__ void __launch_bounds__(256) mm_repack_kernel(const __grid_constant__ MmRepack r) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");        // once every block has started, the product's may
  for (int i = 0; i < r.n; ++i) {
    const MmRepack::One o = r.of[i];
    const uint32_t pieces = (uint32_t)((o.cols + 7) / 8);
    const uintptr_t first = reinterpret_cast<uintptr_t>(o.x), last = reinterpret_cast<uintptr_t>(o.x + (o.rows - 1) * o.ld + o.cols);
    for (PieceWalk at((long long)blockIdx.x * 256 + threadIdx.x, (long long)gridDim.x * 256, pieces); at.row < o.rows; at.next()) {
      const long long c = 8ll * at.at;
      const uint16_t* src = o.x + at.row * o.ld + c;
      const uintptr_t from = reinterpret_cast<uintptr_t>(src) & ~(uintptr_t)15;
      uint4 v;
      if (from >= first && from + 32 <= last) {              // both pieces lie inside the matrix
        v = unaligned16(src);
        if (c + 8 > o.cols) {                                // what follows a row is not its own
          uint32_t* w = &v.x;
#pragma unroll
          for (int k = 0; k < 4; ++k) w[k] &= c + 2 * k + 1 < o.cols ? 0xFFFFFFFFu : c + 2 * k < o.cols ? 0xFFFFu : 0u;
        }
      } else {
        uint32_t e[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) e[k] = c + k < o.cols ? src[k] : 0u;
        v = make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
      }
      *reinterpret_cast<uint4*>(o.out + at.row * o.pitch + c) = v;
    }
  }
}

}  // namespace ssim
