// Product of MXFP4 operands on the tensor cores: D[i, j] = sum_k A[i, k] B[j, k], fp32 accumulators, one rounding at the end.
//
// tcgen05.mma kind::mxf4 multiplies 4-bit operands with a scale per 32 elements of k; one instruction takes 128 rows of A, BN rows
// of B and 64 elements of k.  A stage holds 256 elements of k: 128 bytes a row, one swizzle atom, loaded by TMA; the rows'
// scales come as whole 512-byte tiles (128 rows x 128 elements of k, mx_kernel.cuh), two to a TMA box (plain bulk copies of 512 or 1024
// bytes were far slower), and go from shared into tensor memory with tcgen05.cp, into columns of their own for each stage of the
// ring, so that a stage's release also frees them.  This kernel takes products with few tiles or few rows; it is bound by latencies: launch,
// first loads, the chain of its stages (1 x 12288 x 4096: 10.4 us, 26.7 MB; 1024 x 1024 x 1024: 7.4 us).
//
//   warp 0     producer: TMA loads into the ring
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

template <int BN>      // 16, 32, 64 or 128 rows of B
struct MxgShape {
  static constexpr int B_BYTES = BN * 128;
  static constexpr int SCALE_BYTES = 2 * 1024;                       // two tiles of A's scales, two of B's
  static constexpr int STAGE_BYTES = MXG_A_BYTES + B_BYTES + SCALE_BYTES;
  static constexpr int STAGES = BN == 128 ? 3 : BN == 16 ? 5 : 4;    // about 100 KB: two blocks to a multiprocessor
  static constexpr int SCALE_COLS = 16;                              // tensor-memory columns of a stage's scales
  static constexpr int USED_COLS = BN + STAGES * SCALE_COLS;
  static constexpr int TMEM_COLS = USED_COLS <= 128 ? 128 : 256;
  static constexpr int OFF_BARS = STAGES * STAGE_BYTES;
  static constexpr int SMEM = OFF_BARS + 8 * (2 * STAGES + 1) + 16 + 1024;   // slack for the alignment to 1024 bytes
};

struct MxgArgs {
  long long rows_a, rows_b;
  int kb;                  // 128-element blocks of k
  int kb_split;            // of them for each block of the cluster (even)
  int tiles_a, tiles_b;
  void* d;
  long long ldd;
  int vec;                 // D's rows allow 16-byte stores
};

// Issued by one elected lane of a converged warp: with the whole warp in step the operands stay in uniform registers, where the
// instruction wants them.
__device__ __forceinline__ void mxg_mma(uint32_t d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %6, 0;\n\telect.sync _|q, 0xFFFFFFFF;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
      ::"r"(d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void mxg_commit(uint32_t bar) {
  asm volatile(
      "{\n\t.reg .pred q;\n\telect.sync _|q, 0xFFFFFFFF;\n\t"
      "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar) : "memory");
}
// 512 bytes of shared memory, 32 rows of 16, to four tensor-memory columns of every quarter of the lanes
__device__ __forceinline__ void mxg_copy_scales(uint32_t taddr, uint32_t saddr) {
  const uint64_t desc = (uint64_t)((saddr & 0x3FFFFu) >> 4) | ((uint64_t)(128 >> 4) << 32) | ((uint64_t)1 << 46);   // 8-row groups 128 B apart, no swizzle
  asm volatile("{\n\t.reg .pred q;\n\telect.sync _|q, 0xFFFFFFFF;\n\t@q tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;\n\t}" ::"r"(taddr), "l"(desc) : "memory");
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }
// The warp's wait: one lane polls.
__device__ __forceinline__ bool mbar_wait_warp(uint32_t bar, uint32_t parity) {
  bool ok = false;
  if ((threadIdx.x & 31) == 0) ok = mbar_wait(bar, parity);
  ok = __any_sync(0xFFFFFFFFu, ok);
  __syncwarp();            // what the polling lane has seen is ordered before the others' accesses
  return ok;
}
// A and B E2M1, scales E8M0, M = 128, N = n; id: which half of a column's four scale bytes (0 or 2)
__device__ __forceinline__ uint32_t mxg_idesc(int n, uint32_t id) {
  return (id << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | (1u << 23) | (1u << 27) | (id << 29);
}
__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ void cluster_sync_all() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t cluster_addr(uint32_t addr, uint32_t rank) {
  uint32_t p;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(p) : "r"(addr), "r"(rank));
  return p;
}
__device__ __forceinline__ float4 ld_cluster4(uint32_t cluster_ptr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(cluster_ptr) : "memory");
  return v;
}

template <int T>
__device__ __forceinline__ void mxg_store(void* d, long long i, float v) { Elem<T>::put(d, i, v); }

// A warp's 32 rows x 128 bytes of D: each lane leaves its row in the warp's 4 KB of shared memory, the eight 16-byte pieces XOR-swizzled
// with the row, and the rows leave as whole 128-byte lines (or as pairs or single elements where D's alignment allows no more).
__device__ __forceinline__ void mxg_stage(unsigned char* st, int lane, const uint32_t* w) {
#pragma unroll
  for (int p = 0; p < 8; ++p)
    *reinterpret_cast<uint4*>(st + lane * 128 + ((p ^ (lane & 7)) << 4)) = make_uint4(w[4 * p], w[4 * p + 1], w[4 * p + 2], w[4 * p + 3]);
}
// n accumulators as the words of D's type, in place
template <int T, int N>
__device__ __forceinline__ void mxg_pack(const uint32_t* v, uint32_t* w) {
#pragma unroll
  for (int j = 0; j < N * Elem<T>::bytes / 4; ++j) w[j] = T == T_F32 ? v[j] : float_to_bf16x2(__uint_as_float(v[2 * j]), __uint_as_float(v[2 * j + 1]));
}
template <int T>
__device__ __forceinline__ void mxg_write_rows(const unsigned char* st, int lane, void* d, long long ldd, long long row0, int rows, long long col0, int cols, int vec) {
  constexpr int EB = Elem<T>::bytes;
  if (rows <= 0 || cols <= 0) return;
  char* out = static_cast<char*>(d) + (row0 * ldd + col0) * EB;
  const long long pitch = ldd * EB;
  if (vec && cols * EB >= 128) {
    const int r0 = lane >> 3, piece = lane & 7;
    char* at = out + r0 * pitch + piece * 16;
#pragma unroll
    for (int it = 0; it < 8; ++it, at += 4 * pitch) {
      const int r = it * 4 + r0;
      if (r < rows) *reinterpret_cast<uint4*>(at) = *reinterpret_cast<const uint4*>(st + r * 128 + ((piece ^ (r & 7)) << 4));
    }
    return;
  }
  const bool pairs = EB == 2 && ((reinterpret_cast<uintptr_t>(out) | (uintptr_t)pitch) & 3) == 0;
#pragma unroll 4
  for (int r = 0; r < 32; ++r, out += pitch) {
    if (r >= rows) break;
    const unsigned char* row = st + r * 128;
    const int sw = r & 7;
    if (EB == 4) {
      if (lane < cols) reinterpret_cast<uint32_t*>(out)[lane] = *reinterpret_cast<const uint32_t*>(row + (((lane >> 2) ^ sw) << 4) + (lane & 3) * 4);
    } else if (pairs) {
      const uint32_t w = *reinterpret_cast<const uint32_t*>(row + (((lane >> 2) ^ sw) << 4) + (lane & 3) * 4);
      if (2 * lane + 1 < cols) reinterpret_cast<uint32_t*>(out)[lane] = w;
      else if (2 * lane < cols) reinterpret_cast<uint16_t*>(out)[2 * lane] = (uint16_t)w;
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int e = lane + 32 * h;
        if (e < cols) reinterpret_cast<uint16_t*>(out)[e] = *reinterpret_cast<const uint16_t*>(row + (((e >> 3) ^ sw) << 4) + (e & 7) * 2);
      }
    }
  }
}
// 32 columns of the accumulators, without waiting for them
__device__ __forceinline__ void mxg_ld32(uint32_t taddr, uint32_t* v) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
        "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]), "=r"(v[17]), "=r"(v[18]),
        "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]),
        "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
      : "r"(taddr));
}
__device__ __forceinline__ void mxg_ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

template <int BN, int T, bool SWAP, bool SPLIT>
__global__ void __launch_bounds__(MXG_THREADS) mx_gemm_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                                                              const __grid_constant__ CUtensorMap map_sa, const __grid_constant__ CUtensorMap map_sb, MxgArgs g) {
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
    prefetch_map(&map_a); prefetch_map(&map_b); prefetch_map(&map_sa); prefetch_map(&map_sb);
  }
  if (warp == 1) tc_alloc(smem_addr(tmem_slot), S::TMEM_COLS);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  bool failed = false;

  if (warp == 0) {
    if (lane == 0) {
      const int sa_row = (a0 >> 7) * g.kb, sb_row = (b0 >> 7) * g.kb;      // rows of the scales' tensors: tiles (zeros outside)
      int issued = 0;
      for (int it = 0; it < stages; ++it) {
        const int s = it % S::STAGES, k0 = k_begin + 2 * it;
        if (!mbar_wait(empty(s), (uint32_t)(((it / S::STAGES) & 1) ^ 1))) { failed = true; break; }
        const uint32_t at = base + (uint32_t)s * S::STAGE_BYTES, sc = at + MXG_A_BYTES + S::B_BYTES;
        mbar_arrive_expect_tx(full(s), (uint32_t)S::STAGE_BYTES);
        tma_load_2d(at, &map_a, k0 * 64, a0, full(s));
        tma_load_2d(at + MXG_A_BYTES, &map_b, k0 * 64, b0, full(s));
        tma_load_2d(sc, &map_sa, 0, sa_row + k0, full(s));
        tma_load_2d(sc + 1024, &map_sb, 0, sb_row + k0, full(s));
        issued = it + 1;
      }
      if (failed)     // let what is in flight land (a bounded time) before the block gives up its shared memory
        for (int it = max(0, issued - S::STAGES); it < issued; ++it) mbar_wait(full(it % S::STAGES), (uint32_t)((it / S::STAGES) & 1), 1u << 14);
    }
    __syncwarp();
  } else if (warp == 1) {
    const uint32_t sf_base = tmem + BN;                        // b0 is a multiple of 128 (BN < 128: zero, the host gives one tile): B's scales start with their tile
    const uint64_t adesc0 = tc_desc_kmajor(base), bdesc0 = tc_desc_kmajor(base + MXG_A_BYTES);
    int s = 0;
    uint32_t phase = 0;
    for (int it = 0; it < stages; ++it) {
      const int nk = min(2, k_end - (k_begin + 2 * it));
      if (!mbar_wait_warp(full(s), phase)) { failed = true; break; }
      tc_fence_after();
      const uint32_t sc = base + (uint32_t)s * S::STAGE_BYTES + MXG_A_BYTES + S::B_BYTES;
      const uint32_t sfa = sf_base + (uint32_t)(s * S::SCALE_COLS), sfb = sfa + 8;
      const uint64_t ad = adesc0 + (uint32_t)(s * (S::STAGE_BYTES / 16)), bd = bdesc0 + (uint32_t)(s * (S::STAGE_BYTES / 16));
      for (int k = 0; k < nk; ++k) {
        mxg_copy_scales(sfa + 4 * k, sc + 512 * k);
        mxg_copy_scales(sfb + 4 * k, sc + 1024 + 512 * k);
      }
      for (int k = 0; k < nk; ++k) {
        mxg_mma(tmem, ad + 4 * k, bd + 4 * k, mxg_idesc(BN, 0), sfa + 4 * k, sfb + 4 * k, (it > 0 || k > 0) ? 1u : 0u);
        mxg_mma(tmem, ad + 4 * k + 2, bd + 4 * k + 2, mxg_idesc(BN, 2), sfa + 4 * k, sfb + 4 * k, 1u);
      }
      mxg_commit(empty(s));
      if (it == stages - 1) mxg_commit(acc_bar);
      if (++s == S::STAGES) { s = 0; phase ^= 1u; }
    }
  } else {
    if (!mbar_wait_warp(acc_bar, 0)) failed = true;
    tc_fence_after();
    const int q = warp & 3, row = 32 * q + lane;
    const uint32_t trow = tmem + ((uint32_t)(32 * q) << 16);
    float* part = reinterpret_cast<float*>(base_p);            // the ring's bytes: every MMA has read them
    constexpr int CH = BN < 32 ? 16 : 32;
    // columns in 32s; 16-bit rows that leave through shared memory take two of them for a line
    constexpr int STEP = !SPLIT && !SWAP && CH == 32 && Elem<T>::bytes == 2 && BN >= 64 ? 2 : 1;
    for (int ch = 0; ch < BN / CH; ch += STEP) {
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
        if (SWAP) {
#pragma unroll
          for (int j = 0; j < CH; ++j) part[(ch * CH + j) * 128 + row] = __uint_as_float(v[j]);
        } else {
#pragma unroll
          for (int j = 0; j < CH; j += 4)
            *reinterpret_cast<uint4*>(part + row * (BN + 4) + ch * CH + j) = make_uint4(v[j], v[j + 1], v[j + 2], v[j + 3]);
        }
      } else if (SWAP) {
#pragma unroll
        for (int j = 0; j < CH; ++j)
          if (b0 + ch * CH + j < g.rows_b && a0 + row < g.rows_a) mxg_store<T>(g.d, (long long)(b0 + ch * CH + j) * g.ldd + a0 + row, __uint_as_float(v[j]));
      } else {
        // rows leave through the warp's patch of shared memory; 16-bit results gather two loads of 32 columns for a line
        constexpr int EB = Elem<T>::bytes, CC = 128 / EB;
        if constexpr (CH == 32 && BN * EB >= 128) {
          if constexpr (EB == 2) {
            uint32_t w[64];
#pragma unroll
            for (int j = 0; j < 32; ++j) w[j] = v[j];
            mxg_ld32(trow + (ch + 1) * 32, w + 32);
            mxg_ld_wait();
            if (failed) {
#pragma unroll
              for (int j = 32; j < 64; ++j) w[j] = 0x7FC00000u;
            }
            unsigned char* st = base_p + q * 4096;
            __syncwarp();
            uint32_t packed[32];
            mxg_pack<T, 64>(w, packed);
            mxg_stage(st, lane, packed);
            __syncwarp();
            mxg_write_rows<T>(st, lane, g.d, g.ldd, a0 + 32 * q, (int)min(32ll, g.rows_a - a0 - 32 * q), b0 + ch * 32, (int)min((long long)CC, g.rows_b - b0 - ch * 32), g.vec);
          } else {
            unsigned char* st = base_p + q * 4096;
            __syncwarp();
            mxg_stage(st, lane, v);
            __syncwarp();
            mxg_write_rows<T>(st, lane, g.d, g.ldd, a0 + 32 * q, (int)min(32ll, g.rows_a - a0 - 32 * q), b0 + ch * 32, (int)min(32ll, g.rows_b - b0 - ch * 32), g.vec);
          }
        } else {     // fewer columns than a line
#pragma unroll
          for (int j = 0; j < CH; ++j)
            if (b0 + ch * CH + j < g.rows_b && a0 + row < g.rows_a) mxg_store<T>(g.d, (long long)(a0 + row) * g.ldd + b0 + ch * CH + j, __uint_as_float(v[j]));
        }
      }
    }
  }

  if (SPLIT) {
    __syncthreads();
    cluster_sync_all();
    // the block of rank r adds the r-th part of the tile, four neighbours of a line at a time, over the blocks in their order
    const int rank = (int)cluster_rank(), n = (int)gridDim.y;
    constexpr int ITEMS = 128 * BN / 4, LINE = SWAP ? 32 : BN / 4, PITCH = SWAP ? 128 : BN + 4;
    for (int i = ITEMS * rank / n + tid; i < ITEMS * (rank + 1) / n; i += MXG_THREADS) {
      const int line = i / LINE, at = i % LINE * 4;
      const uint32_t where = base + 4u * (uint32_t)(line * PITCH + at);
      float4 v[8];
#pragma unroll
      for (int r = 0; r < 8; ++r)
        if (r < n) v[r] = ld_cluster4(cluster_addr(where, (uint32_t)r));
      float4 t = v[0];
#pragma unroll
      for (int r = 1; r < 8; ++r)
        if (r < n) { t.x += v[r].x; t.y += v[r].y; t.z += v[r].z; t.w += v[r].w; }
      const long long out_row = SWAP ? b0 + line : a0 + line, out_col = SWAP ? a0 + at : b0 + at;
      const long long rows = SWAP ? g.rows_b : g.rows_a, cols = SWAP ? g.rows_a : g.rows_b;
      if (out_row >= rows) continue;
      const long long to = out_row * g.ldd + out_col;
      if (g.vec && out_col + 4 <= cols) {
        if (T == T_F32) *reinterpret_cast<float4*>(static_cast<float*>(g.d) + to) = t;
        else *reinterpret_cast<uint2*>(static_cast<uint16_t*>(g.d) + to) = make_uint2(float_to_bf16x2(t.x, t.y), float_to_bf16x2(t.z, t.w));
      } else {
        const float e[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (out_col + j < cols) mxg_store<T>(g.d, to + j, e[j]);
      }
    }
    cluster_sync_all();          // nobody leaves while its partial sums may still be read
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) tc_dealloc(tmem, S::TMEM_COLS);
}

// ---- two multiprocessors on one tile ---------------------------------------------------------------------------------------
// Large products.  A 128 x 256 tile a multiprocessor needs 51 KB of operands for 512 cycles of MMA, more than L2 delivers to all of
// them at once (measured: 35 KB in 523 cycles); the pair of a cluster works on 256 x 256 with cta_group::2, each block holding its 128
// rows of A and half of B's rows.  Both load their own parts and count them on the leader's barrier; the leader issues the MMAs for
// both; its commits release the slots of both.  Each block keeps its 128 x 256 accumulators and the scales of all 256 rows of B.
//
// A slot of codes comes back about 1.4 us after its release, so the scales, whose way is longer, have rings of their own that run
// further ahead, and nothing else sits in the codes' ring.  Measured at 4096 x 8192 x 8192 (bf16 result): 113 us, 4.8 PFLOP/s; the issuing
// warp then finds codes and scales ready (no waits on either), an MMA takes about 200 cycles where the same MMA issued again on the same
// operands takes 100: what bounds the main loop is the MMAs' own operand traffic through shared memory beside the 35 KB of loads a
// stage.  Between tiles 1.5 to 3 us are exposed (last MMA, reading the accumulators, first MMA): with 256 accumulator columns
// and the scales there is no room for a second set.
//
//   warp 0      codes: TMA loads (leader's barrier)
//   warp 1      tensor memory; in the leader one lane issues the MMAs
//   warps 2-5   scales from shared to tensor memory with plain stores.  (tcgen05.cp by the issuing lane puts their latency into
//               the codes' ring: 1190 cycles a stage instead of 784 without copies.  Their arrivals at the leader are relaxed: the stores are
//               ordered by tcgen05.wait::st and the fence, and a release at cluster scope took about a microsecond each.)
//   warps 6-13  epilogue: a warp takes 32 rows x 128 columns into registers (half of an fp32 result into shared memory), frees the
//               accumulators, and writes through shared memory while the next tile's MMAs run, two rows of 256 bytes at a time
//               (8192 x 8192 x 1024: 44 to 49 us by the clock; 32 bytes of its own row a lane: 58 us)
//   warp 14     scales: TMA loads (own barrier), 512 elements of k at a time
// Persistent: the producers run ahead of the epilogue into the next tile.
constexpr int MXP_THREADS = 480;
constexpr int MXP_SF_STAGES = 4, MXP_SFT_STAGES = 4;                  // scales of 512 elements of k: in shared memory, in tensor memory
constexpr int MXP_HALF = 128 * 128;                                   // 128 rows x 128 bytes: A's rows, and this block's half of B's
constexpr int MXP_SF_BYTES = 3 * 2048;                                // of 128 rows of A and 256 of B: four tiles of each 128 rows
constexpr int MXP_STAGES = 4;                                         // codes: 256 elements of k (five: 1 % less at k = 8192 at most)
constexpr int MXP_OFF_SF = MXP_STAGES * 2 * MXP_HALF;
constexpr int MXP_OFF_STORE = MXP_OFF_SF + MXP_SF_STAGES * MXP_SF_BYTES;    // 8 KB for each epilogue warp: 32 rows of 256 bytes
constexpr int MXP_OFF_BARS = MXP_OFF_STORE + 8 * 8192;
constexpr int MXP_BARS = 2 * (MXP_STAGES + MXP_SF_STAGES + MXP_SFT_STAGES) + 2;
constexpr int MXP_SMEM = MXP_OFF_BARS + 8 * MXP_BARS + 16 + 1024;
constexpr int MXP_SCALE_COLS = 48;                                    // four tiles: 16 columns of A's scales, 32 of B's
constexpr int MXP_TMEM_COLS = 512;
static_assert(256 + MXP_SFT_STAGES * MXP_SCALE_COLS <= MXP_TMEM_COLS && MXP_SMEM <= 227 * 1024, "accumulators, scales and rings must fit");

__device__ __forceinline__ void mbar_arrive_cluster(uint32_t cluster_bar) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}
__device__ __forceinline__ void tma_load_2d_pair(uint32_t dst, const CUtensorMap* map, int c0, int c1, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
      ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(bar) : "memory");
}
// Issued by one elected lane of a converged warp: with the whole warp in step the operands stay in uniform registers, where the
// instruction wants them (4096 x 8192 x 8192: 121 us issued by one lane alone, 116 us so).
__device__ __forceinline__ void mxp_commit(uint32_t bar) {            // to the barrier at this address in both blocks
  asm volatile(
      "{\n\t.reg .pred q;\n\telect.sync _|q, 0xFFFFFFFF;\n\t"
      "@q tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n\t}" ::"r"(bar), "h"((uint16_t)3) : "memory");
}
__device__ __forceinline__ void mxp_mma(uint32_t d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %6, 0;\n\telect.sync _|q, 0xFFFFFFFF;\n\t"
      "@q tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
      ::"r"(d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory");
}
__device__ __forceinline__ uint32_t mxp_idesc(uint32_t id) {          // M = 256, N = 256
  return (id << 4) | (1u << 7) | (1u << 10) | ((256u >> 3) << 17) | (1u << 23) | (2u << 27) | (id << 29);
}
__device__ __forceinline__ void mxp_st8(uint32_t taddr, const uint4 a, const uint4 b) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
               ::"r"(taddr), "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b.x), "r"(b.y), "r"(b.z), "r"(b.w) : "memory");
}

__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity) {   // a look, without waiting
  uint32_t ok;
  asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}

// The warp's wait for a whole tile: one lane sleeps instead of polling, which leaves the issue slots to the others (4096 x 8192 x 8192: 128 us
// polling, 113 us).  The limit is four seconds; the longest tile whose operands fit the memory takes 0.2 s.
__device__ __forceinline__ bool mbar_wait_warp_long(uint32_t bar, uint32_t parity) {
  bool ok = false;
  if ((threadIdx.x & 31) == 0) ok = mbar_wait_asleep(bar, parity, 4000000000ull);
  ok = __any_sync(0xFFFFFFFFu, ok);
  __syncwarp();
  return ok;
}

// slot and parity of a ring, stepped
struct MxpRing {
  int s = 0;
  uint32_t phase;
  __device__ __forceinline__ explicit MxpRing(uint32_t first) : phase(first) {}
  template <int N> __device__ __forceinline__ void step() { if (++s == N) { s = 0; phase ^= 1u; } }
};

// Up to sixteen rows of 256 bytes from shared memory (16-byte pieces XOR-swizzled with the row) to rows of D at any alignment of the
// element type: a lane writes an aligned 16-byte piece of its row, put together from five words of shared memory, and at most one of the
// elements before the first or behind the last such piece.
template <int EB>
__device__ __forceinline__ void mxp_write_rows(const unsigned char* st, int lane, void* d, long long ldd, long long row0, int rows, long long col0, int cols) {
  if (rows <= 0 || cols <= 0) return;
  const int j = lane & 15, bytes = cols * EB;
  char* out = static_cast<char*>(d) + ((row0 + (lane >> 4)) * ldd + col0) * EB;
  const long long pitch2 = 2 * ldd * EB;
#pragma unroll
  for (int it = 0; it < 8; ++it, out += pitch2) {
    const int r = 2 * it + (lane >> 4);
    if (r >= rows) continue;
    const unsigned char* row = st + r * 256;
    const int sw = r & 7;
    const int head = min(bytes, (int)(-(intptr_t)out & 15)), pieces = (bytes - head) >> 4, tail = head + 16 * pieces;
    if (j < pieces) {
      const int o = head + 16 * j, first = o >> 2, shift = (o & 3) * 8;          // EB == 4: shift is 0
      uint32_t w[5];
#pragma unroll
      for (int k = 0; k < 5; ++k) {
        const int wi = min(first + k, 63);
        if (k < 4 || EB == 2) w[k] = *reinterpret_cast<const uint32_t*>(row + (((wi >> 2) ^ sw) << 4) + (wi & 3) * 4);
      }
      if (EB == 2) {
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = __funnelshift_r(w[k], w[k + 1], shift);
      }
      *reinterpret_cast<uint4*>(out + o) = make_uint4(w[0], w[1], w[2], w[3]);
    }
    const int e = j < 8 ? j * EB : tail + (j - 8) * EB;                          // before the first piece, behind the last
    if (j < 8 ? e < head : e < bytes) {
      const unsigned char* at = row + (((e >> 4) ^ sw) << 4) + (e & 15);
      if (EB == 2) *reinterpret_cast<uint16_t*>(out + e) = *reinterpret_cast<const uint16_t*>(at);
      else *reinterpret_cast<uint32_t*>(out + e) = *reinterpret_cast<const uint32_t*>(at);
    }
  }
}

template <int T>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(MXP_THREADS, 1)
mx_gemm_pair_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_sa,
                    const __grid_constant__ CUtensorMap map_sb, MxgArgs g) {
  extern __shared__ unsigned char smem_raw[];
  const uint32_t raw = smem_addr(smem_raw), base = (raw + 1023u) & ~1023u;      // the same offset in both blocks
  unsigned char* base_p = smem_raw + (base - raw);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t rank = cluster_rank();
  const uint32_t bars = base + MXP_OFF_BARS;
  constexpr int B_SF = 2 * MXP_STAGES, B_SFT = B_SF + 2 * MXP_SF_STAGES, B_ACC = B_SFT + 2 * MXP_SFT_STAGES;
  auto full = [&](int s) { return bars + 8u * s; };                             // codes of both blocks have landed: the leader's count
  auto empty = [&](int s) { return bars + 8u * (MXP_STAGES + s); };
  auto sf_full = [&](int s) { return bars + 8u * (B_SF + s); };                 // this block's scales have landed in shared memory
  auto sf_empty = [&](int s) { return bars + 8u * (B_SF + MXP_SF_STAGES + s); };
  auto sft_full = [&](int s) { return bars + 8u * (B_SFT + s); };               // both blocks' scales are in tensor memory: the leader's count
  auto sft_empty = [&](int s) { return bars + 8u * (B_SFT + MXP_SFT_STAGES + s); };
  const uint32_t acc_full = bars + 8u * B_ACC, acc_empty = acc_full + 8;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(base_p + MXP_OFF_BARS + 8 * MXP_BARS);

  if (tid == 0) {
    for (int s = 0; s < MXP_STAGES; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
    for (int s = 0; s < MXP_SF_STAGES; ++s) { mbar_init(sf_full(s), 1); mbar_init(sf_empty(s), 4); }
    for (int s = 0; s < MXP_SFT_STAGES; ++s) { mbar_init(sft_full(s), 8); mbar_init(sft_empty(s), 1); }
    mbar_init(acc_full, 1);
    mbar_init(acc_empty, 16);                                                   // eight epilogue warps of each block
    mbar_fence_init();
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(tmem_slot)), "r"(MXP_TMEM_COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();                                                           // barriers of both blocks are set up
  tc_fence_after();
  const uint32_t tmem = *tmem_slot, sf_cols = tmem + 256;
  const int stages = (g.kb + 1) / 2, sf_stages = (g.kb + 3) / 4, n_tiles = g.tiles_a * g.tiles_b, pairs = (int)gridDim.x >> 1;
  bool failed = false;

  // tiles in bands of eight of A: pairs that run together share rows of both operands in L2
  auto tile_at = [&](int tile, int& a0, int& b0) {
    const int band = tile / (8 * g.tiles_b), in_band = tile % (8 * g.tiles_b), band_rows = min(8, g.tiles_a - band * 8);
    a0 = (band * 8 + in_band % band_rows) * 256 + (int)rank * 128;
    b0 = in_band / band_rows * 256;
  };

  if (warp == 0) {
    if (lane == 0) {
      MxpRing r(1);
      for (int tile = (int)blockIdx.x >> 1; tile < n_tiles && !failed; tile += pairs) {
        int a0, b0;
        tile_at(tile, a0, b0);
        for (int it = 0; it < stages; ++it, r.step<MXP_STAGES>()) {
          if (!mbar_wait(empty(r.s), r.phase)) { failed = true; break; }
          const uint32_t at = base + (uint32_t)r.s * (2 * MXP_HALF), bar = cluster_addr(full(r.s), 0);
          if (rank == 0) mbar_arrive_expect_tx(full(r.s), 4u * MXP_HALF);
          tma_load_2d_pair(at, &map_a, it * 128, a0, bar);
          tma_load_2d_pair(at + MXP_HALF, &map_b, it * 128, b0 + (int)rank * 128, bar);
        }
      }
      if (failed)
        for (int i = 0; i < 1000; ++i) __nanosleep(1000);                       // let what is in flight land
    }
    __syncwarp();
  } else if (warp == 14) {
    if (lane == 0) {
      MxpRing r(1);
      for (int tile = (int)blockIdx.x >> 1; tile < n_tiles && !failed; tile += pairs) {
        int a0, b0;
        tile_at(tile, a0, b0);
        const int sa_row = (a0 >> 7) * g.kb, sb_row = (b0 >> 7) * g.kb;         // rows of the scales' tensors: tiles (zeros outside)
        for (int it = 0; it < sf_stages; ++it, r.step<MXP_SF_STAGES>()) {
          if (!mbar_wait(sf_empty(r.s), r.phase)) { failed = true; break; }
          const uint32_t sc = base + MXP_OFF_SF + (uint32_t)r.s * MXP_SF_BYTES;
          mbar_arrive_expect_tx(sf_full(r.s), MXP_SF_BYTES);
          tma_load_2d(sc, &map_sa, 0, sa_row + 4 * it, sf_full(r.s));
          tma_load_2d(sc + 2048, &map_sb, 0, sb_row + 4 * it, sf_full(r.s));
          tma_load_2d(sc + 4096, &map_sb, 0, sb_row + g.kb + 4 * it, sf_full(r.s));
        }
      }
      if (failed)
        for (int i = 0; i < 1000; ++i) __nanosleep(1000);
    }
    __syncwarp();
  } else if (warp == 1) {
    if (rank == 0) {
      // The MMA pipe queues about two instructions, 270 cycles of work.  What the thread does between the last MMA of a stage and the
      // first of the next has to be shorter, so the next stage's barriers are looked at while this one's MMAs are queued.
      const uint64_t adesc0 = tc_desc_kmajor(base), bdesc0 = tc_desc_kmajor(base + MXP_HALF);
      MxpRing r(0), rs(0);
      uint32_t acc_phase = 1;
      bool codes = false, scales = false;                                       // known to be there
      for (int tile = (int)blockIdx.x >> 1; tile < n_tiles && !failed; tile += pairs, acc_phase ^= 1u) {
        if (!mbar_wait_warp(acc_empty, acc_phase)) { failed = true; break; }    // both blocks have read the last tile's accumulators
        for (int it = 0; it < stages; ++it) {
          const bool first = (it & 1) == 0, last = !first || it == stages - 1;  // of the two stages that share a slot of scales
          if (first && !scales && !mbar_wait_warp(sft_full(rs.s), rs.phase)) { failed = true; break; }
          if (!codes && !mbar_wait_warp(full(r.s), r.phase)) { failed = true; break; }
          tc_fence_after();
          const uint64_t ad = adesc0 + (uint32_t)(r.s * (2 * MXP_HALF / 16)), bd = bdesc0 + (uint32_t)(r.s * (2 * MXP_HALF / 16));
          const uint32_t sf = sf_cols + (uint32_t)(rs.s * MXP_SCALE_COLS), sfa = sf + (first ? 0u : 8u), sfb = sf + (first ? 16u : 32u);
          mxp_mma(tmem, ad, bd, mxp_idesc(0), sfa, sfb, it > 0 ? 1u : 0u);
          mxp_mma(tmem, ad + 2, bd + 2, mxp_idesc(2), sfa, sfb, 1u);
          const int s_now = r.s, rs_now = rs.s;
          r.step<MXP_STAGES>();
          codes = __all_sync(0xFFFFFFFFu, mbar_test(full(r.s), r.phase));
          if (last) {
            rs.step<MXP_SFT_STAGES>();
            scales = __all_sync(0xFFFFFFFFu, mbar_test(sft_full(rs.s), rs.phase));
          }
          if (2 * it + 1 < g.kb) {
            mxp_mma(tmem, ad + 4, bd + 4, mxp_idesc(0), sfa + 4, sfb + 8, 1u);
            mxp_mma(tmem, ad + 6, bd + 6, mxp_idesc(2), sfa + 4, sfb + 8, 1u);
          }
          mxp_commit(empty(s_now));
          if (last) mxp_commit(sft_empty(rs_now));
          if (it == stages - 1) mxp_commit(acc_full);
        }
      }
    }
    __syncwarp();
  } else if (warp < 6) {
    // a lane holds rows l, 32 + l, 64 + l, 96 + l of each 512-byte tile: four columns of its tensor-memory lane; the four warps
    // write the same to their quarters of the lanes
    const uint32_t trow = sf_cols + ((uint32_t)(32 * (warp & 3)) << 16);
    MxpRing r(0), rs(1);
    for (int tile = (int)blockIdx.x >> 1; tile < n_tiles && !failed; tile += pairs) {
      for (int it = 0; it < sf_stages; ++it, r.step<MXP_SF_STAGES>(), rs.step<MXP_SFT_STAGES>()) {
        if (!mbar_wait_warp(sf_full(r.s), r.phase) || !mbar_wait_warp(sft_empty(rs.s), rs.phase)) { failed = true; break; }
        tc_fence_after();
        const uint4* t = reinterpret_cast<const uint4*>(base_p + MXP_OFF_SF + r.s * MXP_SF_BYTES) + lane;
        uint4 a[4], b[2][4];                                                    // [128 rows of B][k]
#pragma unroll
        for (int k = 0; k < 4; ++k) { a[k] = t[32 * k]; b[0][k] = t[128 + 32 * k]; b[1][k] = t[256 + 32 * k]; }
        const uint32_t at = trow + (uint32_t)(rs.s * MXP_SCALE_COLS);
        mxp_st8(at, a[0], a[1]);
        mxp_st8(at + 8, a[2], a[3]);
#pragma unroll
        for (int k = 0; k < 4; ++k) mxp_st8(at + 16 + 8 * k, b[0][k], b[1][k]);
        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive_cluster(cluster_addr(sft_full(rs.s), 0));
          // Only here may the slot in shared memory be refilled: the stores have taken the loads' values.  An arrival right after the
          // loads let a slow warp read the next round's scales (the loads need not have been performed by then).
          mbar_arrive(sf_empty(r.s));
        }
      }
    }
  } else {
    const int q = warp & 3, half = (warp - 6) >> 2;
    const uint32_t trow = tmem + ((uint32_t)(32 * q) << 16) + 128 * half, done = cluster_addr(acc_empty, 0);
    unsigned char* st = base_p + MXP_OFF_STORE + (warp - 6) * 8192;
    uint32_t phase = 0;
    for (int tile = (int)blockIdx.x >> 1; tile < n_tiles; tile += pairs, phase ^= 1u) {
      int a0, b0;
      tile_at(tile, a0, b0);
      a0 += 32 * q;
      b0 += 128 * half;
      if (!failed && !mbar_wait_warp_long(acc_full, phase)) failed = true;                // from then on every tile of this block is NaN
      tc_fence_after();
      const int rows = (int)max(0ll, min(32ll, g.rows_a - a0));
      constexpr int EB = Elem<T>::bytes, GROUP = 256 / EB;                      // columns taken into registers at a time: 256 bytes of a row
      const long long cols = g.rows_b - b0;                                     // columns that exist from here on
      uint32_t w[64];
      auto to_rows = [&]() {                                                    // the lane's 256 bytes as a row of shared memory
        if (failed) {
#pragma unroll
          for (int j = 0; j < 64; ++j) w[j] = EB == 2 ? 0x7FC07FC0u : 0x7FC00000u;
        }
        __syncwarp();
#pragma unroll
        for (int p = 0; p < 16; ++p)
          *reinterpret_cast<uint4*>(st + lane * 256 + ((p ^ (lane & 7)) << 4)) = make_uint4(w[4 * p], w[4 * p + 1], w[4 * p + 2], w[4 * p + 3]);
      };
      auto write = [&](int c0) {                                                // to D's columns from b0 + c0 on, sixteen lanes a row
        __syncwarp();
        if (g.vec && cols >= c0 + GROUP && rows == 32) {
          char* out = static_cast<char*>(g.d) + ((long long)(a0 + (lane >> 4)) * g.ldd + b0 + c0) * EB + (lane & 15) * 16;
          const unsigned char* row = st + (lane >> 4) * 256;
#pragma unroll
          for (int it = 0; it < 16; ++it, out += 2 * g.ldd * EB)
            *reinterpret_cast<uint4*>(out) = *reinterpret_cast<const uint4*>(row + it * 512 + (((lane & 15) ^ ((2 * it + (lane >> 4)) & 7)) << 4));
        } else {
#pragma unroll 1
          for (int h = 0; h < 2; ++h)
            mxp_write_rows<EB>(st + 4096 * h, lane, g.d, g.ldd, a0 + 16 * h, min(16, rows - 16 * h), b0 + c0, (int)max(0ll, min((long long)GROUP, cols - c0)));
        }
      };
      if constexpr (EB == 2) {
#pragma unroll
        for (int h = 0; h < 4; ++h) {
          uint32_t v[32];
          mxg_ld32(trow + 32 * h, v);
          mxg_ld_wait();
          mxg_pack<T, 32>(v, w + 16 * h);
        }
      } else {
        // the first half of the columns waits in shared memory, so that the accumulators are free before anything is written
        mxg_ld32(trow, w);
        mxg_ld32(trow + 32, w + 32);
        mxg_ld_wait();
        to_rows();
        mxg_ld32(trow + 64, w);
        mxg_ld32(trow + 96, w + 32);
        mxg_ld_wait();
      }
      tc_fence_before();                                                        // the accumulators are read: the next tile may start
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster(done);
      if (EB == 4) write(0);
      to_rows();
      write(128 - GROUP);
    }
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();                        // nobody leaves while the other may still load, commit or arrive here
  if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(MXP_TMEM_COLS) : "memory");
}

}  // namespace ssim
