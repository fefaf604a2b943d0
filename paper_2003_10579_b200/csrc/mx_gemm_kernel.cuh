// Product of MXFP4 operands on the tensor cores: D[i, j] = sum_k A[i, k] B[j, k], fp32 accumulators, one rounding at the end.
//
// tcgen05.mma kind::mxf4 multiplies 4-bit operands with a scale per 32 elements of k; one instruction takes 128 rows of A, BN rows
// of B and 64 elements of k.  A stage holds 256 elements of k: 128 bytes a row, one swizzle atom, loaded by TMA; the rows'
// scales come as whole 512-byte tiles (128 rows x 128 elements of k, mx_kernel.cuh) by bulk copies and go from shared into tensor
// memory with tcgen05.cp, into columns of their own for each stage of the ring, so that a stage's release also frees them.
//
//   warp 0     producer: TMA loads and bulk copies into the ring
//   warp 1     allocates tensor memory; one lane issues the copies of the scales and the MMAs
//   warps 2-5  epilogue: accumulators from tensor memory to D
//
// SWAP: the caller's product has few rows; its weights are A (128 rows an instruction, whatever BN is) and its few rows are B,
// so an instruction wastes nothing on rows that do not exist, and D is written transposed (a lane holds one of 32 consecutive columns).
// Few tiles: the blocks of a cluster share one, each takes a range of k, and the partial sums meet in distributed shared
// memory, added in block order - the same bits each time, no workspace.
// Waits are bounded; where one runs out the tile is written as NaN.
#pragma once
#include "lowbits.cuh"
#include "ptx_util.cuh"

namespace ssim {

constexpr int MXG_THREADS = 192;
constexpr int MXG_A_BYTES = 128 * 128;

template <int BN>
struct MxgShape {
  static constexpr int NT = BN > 128 ? BN / 128 : 1;                 // scale tiles of B
  static constexpr int B_BYTES = BN * 128;
  static constexpr int SCALE_BYTES = 1024 * (1 + NT);                // two tiles of A, two of each 128 rows of B
  static constexpr int STAGE_BYTES = MXG_A_BYTES + B_BYTES + SCALE_BYTES;
  static constexpr int STAGES = BN == 256 ? 4 : BN == 128 ? 3 : BN == 16 ? 5 : 4;
  static constexpr int SCALE_COLS = 8 + 8 * NT;                      // tensor-memory columns of a stage's scales
  static constexpr int USED_COLS = BN + STAGES * SCALE_COLS;
  static constexpr int TMEM_COLS = USED_COLS <= 128 ? 128 : USED_COLS <= 256 ? 256 : 512;
  static constexpr int OFF_BARS = STAGES * STAGE_BYTES;
  static constexpr int SMEM = OFF_BARS + 8 * (2 * STAGES + 1) + 16 + 1024;   // slack for the alignment to 1024 bytes
};

struct MxgArgs {
  const uint8_t* a_scales;
  const uint8_t* b_scales;
  long long rows_a, rows_b;
  int kb;                  // 128-element blocks of k
  int kb_split;            // of them for each block of the cluster (even)
  int tiles_a, tiles_b;
  void* d;
  long long ldd;
  int vec;                 // D's rows allow 16-byte stores
};

__device__ __forceinline__ void mxg_mma(uint32_t d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
      ::"r"(d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory");
}
// 512 bytes of shared memory, 32 rows of 16, to four tensor-memory columns of every quarter of the lanes
__device__ __forceinline__ void mxg_copy_scales(uint32_t taddr, uint32_t saddr) {
  const uint64_t desc = (uint64_t)((saddr & 0x3FFFFu) >> 4) | ((uint64_t)(128 >> 4) << 32) | ((uint64_t)1 << 46);   // 8-row groups 128 B apart, no swizzle
  asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}
// A and B E2M1, scales E8M0, M = 128, N = n; id: which half of a column's four scale bytes (0 or 2)
__device__ __forceinline__ uint32_t mxg_idesc(int n, uint32_t id) {
  return (id << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | (1u << 23) | (1u << 27) | (id << 29);
}
__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ void cluster_sync_all() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ float ld_cluster(uint32_t addr, uint32_t rank) {
  uint32_t p;
  float v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(p) : "r"(addr), "r"(rank));
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(p) : "memory");
  return v;
}

template <int T>
__device__ __forceinline__ void mxg_store(void* d, long long i, float v) { Elem<T>::put(d, i, v); }

template <int BN, int T, bool SWAP, bool SPLIT>
__global__ void __launch_bounds__(MXG_THREADS) mx_gemm_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, MxgArgs g) {
  using S = MxgShape<BN>;
  extern __shared__ unsigned char smem_raw[];
  const uint32_t raw = smem_addr(smem_raw), base = (raw + 1023u) & ~1023u;
  unsigned char* base_p = smem_raw + (base - raw);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t bars = base + S::OFF_BARS;
  auto full = [&](int s) { return bars + 8u * s; };
  auto empty = [&](int s) { return bars + 8u * (S::STAGES + s); };
  const uint32_t acc_bar = bars + 16u * S::STAGES;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(base_p + S::OFF_BARS + 8 * (2 * S::STAGES + 1));

  // tiles in bands of eight of A: neighbouring blocks share rows of both operands in L2
  const int tile = blockIdx.x, band = tile / (8 * g.tiles_b), in_band = tile % (8 * g.tiles_b);
  const int band_rows = min(8, g.tiles_a - band * 8);
  const int ta = band * 8 + in_band % band_rows, tb = in_band / band_rows;
  const int a0 = ta * 128, b0 = tb * BN;
  const int k_begin = SPLIT ? (int)blockIdx.y * g.kb_split : 0, k_end = SPLIT ? min(g.kb, k_begin + g.kb_split) : g.kb;
  const int stages = (k_end - k_begin + 1) / 2;               // >= 1: the host gives every block of a cluster a part

  if (tid == 0) {
    for (int s = 0; s < S::STAGES; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
    mbar_init(acc_bar, 1);
    mbar_fence_init();
  }
  if (warp == 1) tc_alloc(smem_addr(tmem_slot), S::TMEM_COLS);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  bool failed = false;

  if (warp == 0) {
    if (lane == 0) {
      const int b_tile0 = b0 >> 7, b_tiles = min(S::NT, (int)((g.rows_b + 127) >> 7) - b_tile0);
      int issued = 0;
      for (int it = 0; it < stages; ++it) {
        const int s = it % S::STAGES, k0 = k_begin + 2 * it, nk = min(2, k_end - k0);
        if (!mbar_wait(empty(s), (uint32_t)(((it / S::STAGES) & 1) ^ 1))) { failed = true; break; }
        const uint32_t at = base + (uint32_t)s * S::STAGE_BYTES, sc = at + MXG_A_BYTES + S::B_BYTES;
        mbar_arrive_expect_tx(full(s), (uint32_t)(MXG_A_BYTES + S::B_BYTES + 512 * nk * (1 + b_tiles)));
        tma_load_2d(at, &map_a, k0 * 64, a0, full(s));
        tma_load_2d(at + MXG_A_BYTES, &map_b, k0 * 64, b0, full(s));
        bulk_g2s(sc, g.a_scales + ((long long)(a0 >> 7) * g.kb + k0) * 512, (uint32_t)(512 * nk), full(s));
        for (int t = 0; t < b_tiles; ++t)
          bulk_g2s(sc + 1024u * (1 + t), g.b_scales + ((long long)(b_tile0 + t) * g.kb + k0) * 512, (uint32_t)(512 * nk), full(s));
        issued = it + 1;
      }
      if (failed)     // let what is in flight land (a bounded time) before the block gives up its shared memory
        for (int it = max(0, issued - S::STAGES); it < issued; ++it) mbar_wait(full(it % S::STAGES), (uint32_t)((it / S::STAGES) & 1), 1u << 14);
    }
    __syncwarp();
  } else if (warp == 1) {
    const uint32_t sf_base = tmem + BN, b_col = (uint32_t)((b0 & 127) >> 5);
    for (int it = 0; it < stages; ++it) {
      const int s = it % S::STAGES, nk = min(2, k_end - (k_begin + 2 * it));
      if (!mbar_wait(full(s), (uint32_t)((it / S::STAGES) & 1))) { failed = true; break; }
      tc_fence_after();
      if (lane == 0) {
        const uint32_t at = base + (uint32_t)s * S::STAGE_BYTES, bt = at + MXG_A_BYTES, sc = bt + S::B_BYTES;
        const uint32_t sfa = sf_base + (uint32_t)(s * S::SCALE_COLS), sfb = sfa + 8;
        for (int k = 0; k < nk; ++k) {
          mxg_copy_scales(sfa + 4 * k, sc + 512 * k);
#pragma unroll
          for (int t = 0; t < S::NT; ++t) mxg_copy_scales(sfb + 4 * (S::NT * k + t), sc + 1024 * (1 + t) + 512 * k);
        }
        for (int k = 0; k < nk; ++k) {
#pragma unroll
          for (int h = 0; h < 2; ++h)
            mxg_mma(tmem, tc_desc_kmajor(at + 64 * k + 32 * h), tc_desc_kmajor(bt + 64 * k + 32 * h), mxg_idesc(BN, 2 * h), sfa + 4 * k,
                    sfb + 4 * S::NT * k + b_col, (it > 0 || k > 0 || h > 0) ? 1u : 0u);
        }
        tc_commit(empty(s));
        if (it == stages - 1) tc_commit(acc_bar);
      }
      __syncwarp();
    }
  } else {
    if (!mbar_wait(acc_bar, 0)) failed = true;
    tc_fence_after();
    const int q = warp & 3, row = 32 * q + lane;
    const uint32_t trow = tmem + ((uint32_t)(32 * q) << 16);
    float* part = reinterpret_cast<float*>(base_p);            // the ring's bytes: every MMA has read them
    constexpr int CH = BN < 32 ? 16 : 32;
    for (int ch = 0; ch < BN / CH; ++ch) {
      uint32_t v[32];
      if (CH == 32) {
        tc_ld32(trow + ch * 32, v);
      } else {
        asm volatile(
            "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
            : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
              "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]) : "r"(trow));
        asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
      }
      if (failed) {
#pragma unroll
        for (int j = 0; j < CH; ++j) v[j] = 0x7FC00000u;
      }
      if (SPLIT) {
#pragma unroll
        for (int j = 0; j < CH; ++j) part[SWAP ? (ch * CH + j) * 128 + row : row * (BN + 1) + ch * CH + j] = __uint_as_float(v[j]);
      } else if (SWAP) {
#pragma unroll
        for (int j = 0; j < CH; ++j)
          if (b0 + ch * CH + j < g.rows_b && a0 + row < g.rows_a) mxg_store<T>(g.d, (long long)(b0 + ch * CH + j) * g.ldd + a0 + row, __uint_as_float(v[j]));
      } else {
        // 32 x CH values through the warp's own patch of shared memory: rows leave as consecutive elements
        float* patch = part + q * 32 * (CH + 1);
        __syncwarp();
#pragma unroll
        for (int j = 0; j < CH; ++j) patch[lane * (CH + 1) + j] = __uint_as_float(v[j]);
        __syncwarp();
        const int col = b0 + ch * CH + lane;
        if (lane < CH && col < g.rows_b)
          for (int r = 0; r < 32; ++r)
            if (a0 + 32 * q + r < g.rows_a) mxg_store<T>(g.d, (long long)(a0 + 32 * q + r) * g.ldd + col, patch[r * (CH + 1) + lane]);
      }
    }
  }

  if (SPLIT) {
    __syncthreads();
    cluster_sync_all();
    const uint32_t rank = cluster_rank(), n = gridDim.y;
    const uint32_t part = base;
    constexpr int W = BN + 1;
    if (SWAP) {      // columns of A's rows side by side: block `rank` adds columns rank, rank + n, ... of B's rows
      for (int i = tid; i < 128 * BN; i += MXG_THREADS) {
        const int j = i >> 7, row = i & 127;
        if (j % (int)n != (int)rank || b0 + j >= g.rows_b || a0 + row >= g.rows_a) continue;
        float s = 0.f;
        for (uint32_t r = 0; r < n; ++r) s += ld_cluster(part + 4u * (uint32_t)(j * 128 + row), r);
        mxg_store<T>(g.d, (long long)(b0 + j) * g.ldd + a0 + row, s);
      }
    } else {
      for (int i = tid; i < 128 * BN; i += MXG_THREADS) {
        const int row = i / BN, j = i % BN;
        if (row % (int)n != (int)rank || b0 + j >= g.rows_b || a0 + row >= g.rows_a) continue;
        float s = 0.f;
        for (uint32_t r = 0; r < n; ++r) s += ld_cluster(part + 4u * (uint32_t)(row * W + j), r);
        mxg_store<T>(g.d, (long long)(a0 + row) * g.ldd + b0 + j, s);
      }
    }
    cluster_sync_all();          // nobody leaves while its partial sums may still be read
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) tc_dealloc(tmem, S::TMEM_COLS);
}

}  // namespace ssim
