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
// Waits are bounded; where one runs out the tile is written as NaN.
#pragma once
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
  int vec_c, vec_r, vec_b;    // four neighbours at once
};

// ---- the tail, on four neighbours of a row --------------------------------------------------------------------------------------
template <int T>
__device__ __forceinline__ void load4(const void* p, long long i, float (&v)[4]) {     // aligned to four elements
  if (T == T_F32) {
    const float4 a = *reinterpret_cast<const float4*>(static_cast<const float*>(p) + i);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
  } else {
    const uint2 a = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(p) + i);
    if (T == T_BF16) {
      v[0] = __uint_as_float(a.x << 16); v[1] = __uint_as_float(a.x & 0xFFFF0000u); v[2] = __uint_as_float(a.y << 16); v[3] = __uint_as_float(a.y & 0xFFFF0000u);
    } else {
      v[0] = f16_to_float(a.x & 0xFFFFu); v[1] = f16_to_float(a.x >> 16); v[2] = f16_to_float(a.y & 0xFFFFu); v[3] = f16_to_float(a.y >> 16);
    }
  }
}
template <int T>
__device__ __forceinline__ void store4(void* p, long long i, const float (&v)[4]) {
  if (T == T_F32) *reinterpret_cast<float4*>(static_cast<float*>(p) + i) = make_float4(v[0], v[1], v[2], v[3]);
  else if (T == T_BF16) *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p) + i) = make_uint2(float_to_bf16x2(v[0], v[1]), float_to_bf16x2(v[2], v[3]));
  else *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p) + i) = make_uint2(float_to_f16x2(v[0], v[1]), float_to_f16x2(v[2], v[3]));
}
template <int T>
__device__ __forceinline__ void load4_of(const void* p, long long i, int n, bool vec, float (&v)[4]) {   // n of them exist
  if (vec && n >= 4) load4<T>(p, i, v);
  else
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = e < n ? Elem<T>::get(p, i + e) : 0.f;
}

// What the tail of four elements at (row, col) reads besides the sum
struct MmTail {
  float r[4];
  uint32_t z;
  uint8_t zs;
};
template <int T>
__device__ __forceinline__ void mm_tail_load(const MmArgs& g, long long row, long long col, MmTail& t) {
  const int n = row < g.M ? (int)max(0ll, min(4ll, g.N - col)) : 0;
  if (g.res) load4_of<T>(g.res, row * g.ldr + col, n, g.vec_r, t.r);
  if (g.grad && n > 0) {
    const long long blocks = (g.N + 31) >> 5;
    t.z = *reinterpret_cast<const uint32_t*>(g.z_codes + row * blocks * 32 + col);
    t.zs = g.z_scales[row * blocks + (col >> 5)];
  }
}
template <int ACT>
__device__ __forceinline__ void act4(float (&v)[4]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = act_value<ACT>(v[e]);
}
template <int ACT>
__device__ __forceinline__ void slope4(float (&v)[4], const float (&z)[4]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] *= act_slope<ACT>(z[e]);
}
// Every lane of the warp takes part; eight neighbouring lanes hold a block of 32 columns.  col is a multiple of four.
template <int T>
__device__ __forceinline__ void mm_tail(const MmArgs& g, long long row, long long col, float (&v)[4], const MmTail& t) {
  const int n = row < g.M ? (int)max(0ll, min(4ll, g.N - col)) : 0;
  if (g.grad) {
    if (n > 0) {
      float z[4];
      ckpt_values4(t.z, scale_value(t.zs), z);
      if (g.act == ACT_RELU) slope4<ACT_RELU>(v, z);
      else if (g.act == ACT_GELU) slope4<ACT_GELU>(v, z);
      else if (g.act == ACT_SILU) slope4<ACT_SILU>(v, z);
    }
  } else {
    if (g.bias && n > 0) {
      float b[4];
      if (g.bias_type == T_F32) load4_of<T_F32>(g.bias, col, n, g.vec_b, b);
      else if (g.bias_type == T_BF16) load4_of<T_BF16>(g.bias, col, n, g.vec_b, b);
      else load4_of<T_F16>(g.bias, col, n, g.vec_b, b);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += b[e];
    }
    if (g.z_codes) {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = e < n ? v[e] : 0.f;
      uint32_t most = __float_as_uint(max3_abs(max3_abs(v[0], v[1], v[2]), v[3], 0.f)) & ABS_MASK;
#pragma unroll
      for (int k = 1; k < 8; k <<= 1) most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, k));
      const uint32_t code = scale_code_e4m3(most);
      const float inv = scale_inverse(code);
      const long long blocks = (g.N + 31) >> 5;
      if (row < g.M && col < 32 * blocks) {
        *reinterpret_cast<uint32_t*>(g.z_codes + row * blocks * 32 + col) = to_e4m3x4(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
        if ((col & 31) == 0) g.z_scales[row * blocks + (col >> 5)] = (uint8_t)code;
      }
    }
    if (g.act == ACT_RELU) act4<ACT_RELU>(v);
    else if (g.act == ACT_GELU) act4<ACT_GELU>(v);
    else if (g.act == ACT_SILU) act4<ACT_SILU>(v);
  }
  if (n <= 0) return;
  if (g.res) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] += t.r[e];
  }
  if (g.vec_c && n == 4) store4<T>(g.c, row * g.ldc + col, v);
  else
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < n) Elem<T>::put(g.c, row * g.ldc + col + e, v[e]);
}

// ---- loads and instructions ---------------------------------------------------------------------------------------------------------
// fp32 accumulators; bf: bf16 operands (else fp16); m, n: the instruction's shape
__host__ __device__ inline uint32_t mm_idesc(int m, int n, int bf, int a_t, int b_t) {
  return (1u << 4) | ((uint32_t)bf << 7) | ((uint32_t)bf << 10) | ((uint32_t)a_t << 15) | ((uint32_t)b_t << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
__device__ __forceinline__ uint64_t mm_desc(uint32_t saddr, int t) { return t ? tc_desc_mnmajor(saddr, 8192, 1024) : tc_desc_kmajor(saddr); }
// sixteen elements of k further: 32 bytes along a row, or sixteen rows of 128 bytes (descriptors count in 16 bytes)
__device__ __forceinline__ uint32_t mm_desc_step(int t) { return t ? 128u : 2u; }

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
//   warps 2-5  accumulators from tensor memory to shared memory (over the ring, which every MMA has read by then)
//   all        the tail; in a cluster each block adds its share of the tile over the blocks, in their order: the same bits each time
constexpr int MM_THREADS = 192, MM_MAX_STAGES = 8, MM_A_BYTES = 16384;
__host__ __device__ constexpr int mm_pitch(int bn, bool swap) { return swap ? 132 : bn + 4; }     // floats between lines of partial sums
__host__ __device__ constexpr int mm_part_bytes(int bn, bool swap) { return (swap ? bn : 128) * mm_pitch(bn, swap) * 4; }

template <int BN, int T, bool SWAP, bool SPLIT>
__global__ void __launch_bounds__(MM_THREADS) mm_tile_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ MmArgs g) {
  extern __shared__ unsigned char smem_raw[];
  __shared__ __align__(8) unsigned long long bars_s[2 * MM_MAX_STAGES + 1];
  __shared__ uint32_t tmem_slot;
  const uint32_t raw = smem_addr(smem_raw), base = (raw + 1023u) & ~1023u;
  unsigned char* base_p = smem_raw + (base - raw);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
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

  if (tid == 0) {
    for (int s = 0; s < g.stages; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
    mbar_init(acc_bar, 1);
    mbar_fence_init();
    if (n_it > 0) { prefetch_map(&map_a); prefetch_map(&map_b); }
  }
  if (warp == 1) tc_alloc(smem_addr(&tmem_slot), TMEM_COLS);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  bool failed = false;

  if (warp == 0) {
    if (lane == 0) {
      int s = 0, issued = 0;
      uint32_t phase = 1;
      for (int it = 0; it < n_it; ++it) {
        if (!mbar_wait(empty(s), phase)) { failed = true; break; }
        const uint32_t at = base + (uint32_t)(s * g.stage_bytes), to_b = at + MM_A_BYTES;
        const int k0 = (k_begin + it) * 64;
        mbar_arrive_expect_tx(full(s), (uint32_t)g.stage_bytes);
        if (g.a_t) {
          tma_load_2d(at, &map_a, a0, k0, full(s));
          tma_load_2d(at + 8192, &map_a, a0 + 64, k0, full(s));
        } else {
          tma_load_2d(at, &map_a, k0, a0, full(s));
        }
        if (g.b_t) {
          tma_load_2d(to_b, &map_b, b0, k0, full(s));
          if (BN > 64) tma_load_2d(to_b + 8192, &map_b, b0 + 64, k0, full(s));
        } else {
          tma_load_2d(to_b, &map_b, k0, b0, full(s));
        }
        issued = it + 1;
        if (++s == g.stages) { s = 0; phase ^= 1u; }
      }
      if (failed)     // let what is in flight land (a bounded time) before the block gives up its shared memory
        for (int it = max(0, issued - g.stages); it < issued; ++it) mbar_wait(full(it % g.stages), (uint32_t)((it / g.stages) & 1), 1u << 14);
    }
    __syncwarp();
  } else if (warp == 1) {
    const uint64_t adesc = mm_desc(base, g.a_t), bdesc = mm_desc(base + MM_A_BYTES, g.b_t);
    const uint32_t astep = mm_desc_step(g.a_t), bstep = mm_desc_step(g.b_t);
    int s = 0;
    uint32_t phase = 0;
    for (int it = 0; it < n_it; ++it) {
      if (!mbar_wait_warp(full(s), phase)) { failed = true; break; }
      tc_fence_after();
      const uint32_t at = (uint32_t)(s * g.stage_bytes) >> 4;
#pragma unroll
      for (int k = 0; k < 4; ++k) mm_mma(tmem, adesc + at + k * astep, bdesc + at + k * bstep, g.idesc, it > 0 || k > 0 ? 1u : 0u);
      tc_commit_elected(empty(s));
      if (it == n_it - 1) tc_commit_elected(acc_bar);
      if (++s == g.stages) { s = 0; phase ^= 1u; }
    }
  } else {
    if (n_it > 0 && !mbar_wait_warp(acc_bar, 0)) failed = true;
    tc_fence_after();
    const int q = warp & 3, row = 32 * q + lane;
    const uint32_t trow = tmem + ((uint32_t)(32 * q) << 16);
    float* part = reinterpret_cast<float*>(base_p);
    constexpr int CH = BN < 32 ? 16 : 32;
#pragma unroll 1
    for (int ch = 0; ch < BN / CH; ++ch) {
      uint32_t v[32];
      if (CH == 32) {
        tc_ld32_async(trow + ch * 32, v);
      } else {
        asm volatile(
            "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
            : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
              "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]) : "r"(trow));
      }
      tc_ld_wait();
      if (failed || n_it == 0) {                                  // no k at all: sums of nothing
#pragma unroll
        for (int j = 0; j < CH; ++j) v[j] = failed ? 0x7FC00000u : 0u;
      }
      if (SWAP) {
#pragma unroll
        for (int j = 0; j < CH; ++j) part[(ch * CH + j) * mm_pitch(BN, SWAP) + row] = __uint_as_float(v[j]);
      } else {
#pragma unroll
        for (int j = 0; j < CH; j += 4) *reinterpret_cast<uint4*>(part + row * mm_pitch(BN, SWAP) + ch * CH + j) = make_uint4(v[j], v[j + 1], v[j + 2], v[j + 3]);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (SPLIT) cluster_sync_all();

  // A warp takes a unit of 32 groups of four: a line of 128 columns (SWAP: of one of the few rows), or a few shorter lines
  const int rank = SPLIT ? (int)cluster_rank() : 0, n = SPLIT ? (int)gridDim.y : 1;
  constexpr int GROUPS = SWAP ? 32 : BN / 4, LINES = 32 / GROUPS;          // groups of four a line, lines a unit
  for (int u = BN * rank / n + warp; u < BN * (rank + 1) / n; u += MM_THREADS / 32) {
    const int line = u * LINES + lane / GROUPS, at = lane % GROUPS * 4;
    const long long row = SWAP ? b0 + line : a0 + line, col = SWAP ? a0 + at : b0 + at;
    MmTail t;
    mm_tail_load<T>(g, row, col, t);
    const uint32_t where = base + 4u * (uint32_t)(line * mm_pitch(BN, SWAP) + at);
    float4 s;
    if (SPLIT) {
      float4 v[8];
#pragma unroll
      for (int r = 0; r < 8; ++r)
        if (r < n) v[r] = ld_cluster4(cluster_addr(where, (uint32_t)r));
      s = v[0];
#pragma unroll
      for (int r = 1; r < 8; ++r)
        if (r < n) { s.x += v[r].x; s.y += v[r].y; s.z += v[r].z; s.w += v[r].w; }
    } else {
      s = *reinterpret_cast<const float4*>(base_p + (where - base));
    }
    float v[4] = {s.x, s.y, s.z, s.w};
    mm_tail<T>(g, row, col, v, t);
  }
  if (SPLIT) cluster_sync_all();          // nobody leaves while its partial sums may still be read
  if (warp == 1) tc_dealloc(tmem, TMEM_COLS);
}

// ---- two multiprocessors on a 256 x 256 tile -----------------------------------------------------------------------------------------
//   warp 0      TMA loads (leader's barrier): each block its 128 rows of A and its half of B's
//   warp 1      tensor memory; in the leader one lane issues the MMAs for both
//   warps 2-9   the tail: a warp takes 32 rows x 128 columns, 32 columns at a time through its own 4 KB of shared memory, so that every access
//               to memory is of neighbours
// Two sets of accumulators (2 x 256 columns of tensor memory): a tile's tail runs beside the next one's MMAs.
constexpr int MMP_THREADS = 320, MMP_STAGES = 6, MMP_HALF = 128 * 128, MMP_STAGE = 2 * MMP_HALF;
constexpr int MMP_OFF_STORE = MMP_STAGES * MMP_STAGE;
constexpr int MMP_OFF_BARS = MMP_OFF_STORE + 8 * 4096;
constexpr int MMP_SMEM = MMP_OFF_BARS + 8 * (2 * MMP_STAGES + 4) + 16 + 1024;
static_assert(MMP_SMEM <= 227 * 1024, "the ring and the tail's patches must fit");

template <int T>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(MMP_THREADS, 1)
mm_pair_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ MmArgs g) {
  extern __shared__ unsigned char smem_raw[];
  const uint32_t raw = smem_addr(smem_raw), base = (raw + 1023u) & ~1023u;      // the same offset in both blocks
  unsigned char* base_p = smem_raw + (base - raw);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
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
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();                                                           // barriers of both blocks are set up
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  const int n_tiles = g.tiles_a * g.tiles_b, pairs = (int)gridDim.x >> 1;
  bool failed = false;

  // tiles in bands of eight of A: pairs that run together share rows of both operands in L2
  auto tile_at = [&](int tile, int& a0, int& b0) {
    const int band = tile / (8 * g.tiles_b), in_band = tile % (8 * g.tiles_b), band_rows = min(8, g.tiles_a - band * 8);
    a0 = (band * 8 + in_band % band_rows) * 256 + (int)rank * 128;
    b0 = in_band / band_rows * 256;
  };

  if (warp == 0) {
    if (lane == 0) {
      Ring r(1);
      for (int tile = (int)blockIdx.x >> 1; tile < n_tiles && !failed; tile += pairs) {
        int a0, b0;
        tile_at(tile, a0, b0);
        b0 += (int)rank * 128;
        for (int it = 0; it < g.kb; ++it, r.step<MMP_STAGES>()) {
          if (!mbar_wait(empty(r.s), r.phase)) { failed = true; break; }
          const uint32_t at = base + (uint32_t)r.s * MMP_STAGE, to_b = at + MMP_HALF, bar = cluster_addr(full(r.s), 0);
          const int k0 = it * 64;
          if (rank == 0) mbar_arrive_expect_tx(full(r.s), 2u * MMP_STAGE);
          if (g.a_t) {
            tma_load_2d_pair(at, &map_a, a0, k0, bar);
            tma_load_2d_pair(at + 8192, &map_a, a0 + 64, k0, bar);
          } else {
            tma_load_2d_pair(at, &map_a, k0, a0, bar);
          }
          if (g.b_t) {
            tma_load_2d_pair(to_b, &map_b, b0, k0, bar);
            tma_load_2d_pair(to_b + 8192, &map_b, b0 + 64, k0, bar);
          } else {
            tma_load_2d_pair(to_b, &map_b, k0, b0, bar);
          }
        }
      }
      if (failed)
        for (int i = 0; i < 1000; ++i) __nanosleep(1000);                       // let what is in flight land
    }
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
        if (!mbar_wait_warp(acc_empty(buf), acc_phase)) { failed = true; break; }
        tc_fence_after();
        const uint32_t d = tmem + 256u * buf;
        for (int it = 0; it < g.kb; ++it) {
          if (!there && !mbar_wait_warp(full(r.s), r.phase)) { failed = true; break; }
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
    unsigned char* st = base_p + MMP_OFF_STORE + (warp - 2) * 4096;
    int buf = 0;
    uint32_t phase = 0;
    for (int tile = (int)blockIdx.x >> 1; tile < n_tiles; tile += pairs) {
      int a0, b0;
      tile_at(tile, a0, b0);
      const long long row0 = a0 + 32 * q + (lane >> 3), col0 = b0 + 128 * half + (lane & 7) * 4;
      const uint32_t trow = tmem + ((uint32_t)(32 * q) << 16) + 256u * buf + 128 * half, done = cluster_addr(acc_empty(buf), 0);
      if (!failed && !mbar_wait_warp_long(acc_full(buf), phase)) failed = true;           // from then on every tile of this block is NaN
      tc_fence_after();
#pragma unroll 1
      for (int ch = 0; ch < 4; ++ch) {
        uint32_t v[32];
        tc_ld32_async(trow + 32 * ch, v);
        tc_ld_wait();
        if (ch == 3) {                                                          // the accumulators are read: the tile after the next may start
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive_cluster(done);
        }
        if (failed) {
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] = 0x7FC00000u;
        }
        __syncwarp();
#pragma unroll
        for (int p = 0; p < 8; ++p)
          *reinterpret_cast<uint4*>(st + lane * 128 + ((p ^ (lane & 7)) << 4)) = make_uint4(v[4 * p], v[4 * p + 1], v[4 * p + 2], v[4 * p + 3]);
        __syncwarp();
        const long long col = col0 + 32 * ch;
#pragma unroll 1
        for (int h = 0; h < 2; ++h) {                                           // four accesses of four rows each in flight
          MmTail t[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) mm_tail_load<T>(g, row0 + 16 * h + 4 * i, col, t[i]);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int r = 16 * h + 4 * i + (lane >> 3);
            const float4 s = *reinterpret_cast<const float4*>(st + r * 128 + (((lane & 7) ^ (r & 7)) << 4));
            float x[4] = {s.x, s.y, s.z, s.w};
            mm_tail<T>(g, row0 + 16 * h + 4 * i, col, x, t[i]);
          }
        }
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
// Rows that do not start on 16-byte boundaries are copied to rows that do (cols rounded up to eight elements) before the product: one read
// and one write more of an operand that the tiles read many times.
__global__ void __launch_bounds__(256) mm_repack_kernel(const uint16_t* x, long long rows, long long cols, long long ld, uint16_t* out) {
  const uint32_t pieces = (uint32_t)((cols + 7) / 8);
  for (PieceWalk at((long long)blockIdx.x * 256 + threadIdx.x, (long long)gridDim.x * 256, pieces); at.row < rows; at.next()) {
    const long long c = 8ll * at.at;
    const uint16_t* src = x + at.row * ld + c;
    uint32_t v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = c + e < cols ? src[e] : 0u;
    *reinterpret_cast<uint4*>(out + (at.row * pieces + at.at) * 8) = make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
  }
}

}  // namespace ssim
