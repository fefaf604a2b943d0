// Activations kept in 8 bits between the forward and the backward pass, and what the backward pass makes of them.
//
// A kept matrix [rows][cols] has E4M3 codes in rows of 32 ceil(cols / 32) bytes (the tail of a row zero) and one scale byte per block of
// 32 elements of a row, [rows][ceil(cols / 32)]: 2^(byte - 127), the smallest power of two, at least 2^-127, for which no magnitude of
// the block exceeds 448 times it; elements are rounded to nearest even (lowbits.cuh).  33/32 of a byte an element.
//
// Each of the three kernels is one pass whose floor is HBM: what it reads and writes once.  Rows that start on 16-byte boundaries move in
// whole 32-byte sectors, a thread a block; others go a warp to a block of 32, a lane an element, which still reads and writes neighbours together.
// Measured at 16384 x 11264 bf16 (floors 86, 86, 143 us): written in 82 us, read through gelu in 124 (two special-function instructions an element keep that
// unit 61 % busy), dz and its sums through gelu in 218 (issue slots 60 %, 26 instructions an element; HBM 50 %); without an activation 22 us for 33 M
// elements read and 42 us for 92 M summed.
#pragma once
#include "act_math.cuh"
#include "lowbits.cuh"
#include "ptx_util.cuh"

namespace ssim {

__host__ __device__ inline long long ckpt_pitch(long long cols) { return (cols + 31) / 32 * 32; }

struct CkptArgs {
  const void* x;              // write: the matrix; act_backward: dy (rows ld apart)
  long long rows, cols, ld;
  uint8_t* codes;
  uint8_t* scales;
  void* out;                  // read: the values; act_backward: dz
  long long ldo;
  int vec;                    // rows of x and out on 16-byte boundaries
  float* partial;             // act_backward: column sums [splits][cols], or null
  void* db;                   // act_backward: column sums [cols] of db_type, where the splits are the blocks of a cluster, or null
  int db_type, split_rows;
};

__device__ __forceinline__ void put_as(int type, void* p, long long i, float v) {
  if (type == T_F32) Elem<T_F32>::put(p, i, v);
  else if (type == T_BF16) Elem<T_BF16>::put(p, i, v);
  else Elem<T_F16>::put(p, i, v);
}

// Row and piece of the pieces first, first + step, ... of a matrix with `pieces` to a row, without a division each time
struct PieceWalk {
  long long row, drow;
  uint32_t at, dat, pieces;
  __device__ __forceinline__ PieceWalk(long long first, long long step, uint32_t pieces_) : pieces(pieces_) {
    row = first / pieces; at = (uint32_t)(first - row * pieces);
    drow = step / pieces; dat = (uint32_t)(step - drow * pieces);
  }
  __device__ __forceinline__ void next() {
    row += drow;
    at += dat;
    if (at >= pieces) { at -= pieces; ++row; }
  }
};

template <int T>
__global__ void __launch_bounds__(256) ckpt_write_kernel(const __grid_constant__ CkptArgs a) {
  constexpr int EB = Elem<T>::bytes;
  const uint32_t blocks = (uint32_t)((a.cols + 31) / 32);
  const long long pitch = 32ll * blocks;
  if (a.vec) {
    for (PieceWalk at((long long)blockIdx.x * 256 + threadIdx.x, (long long)gridDim.x * 256, blocks); at.row < a.rows; at.next()) {
      const long long c = 32ll * at.at;
      const char* src = static_cast<const char*>(a.x) + at.row * a.ld * EB;
      Raw8<T> x[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (c + 32 <= a.cols) x[q].load(src, c + 8 * q);
        else x[q].load_some(src, c + 8 * q, (int)max(0ll, min(8ll, a.cols - c - 8 * q)));
      }
      const uint32_t code = scale_code_e4m3(max(max(x[0].amax(), x[1].amax()), max(x[2].amax(), x[3].amax())));
      const float inv = scale_inverse(code);
      uint32_t o[8];
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const Raw8<T>& r = x[q >> 1];
        const int e = 4 * (q & 1);
        o[q] = to_e4m3x4(r.value(e) * inv, r.value(e + 1) * inv, r.value(e + 2) * inv, r.value(e + 3) * inv);
      }
      uint4* to = reinterpret_cast<uint4*>(a.codes + at.row * pitch + c);
      to[0] = make_uint4(o[0], o[1], o[2], o[3]);
      to[1] = make_uint4(o[4], o[5], o[6], o[7]);
      a.scales[at.row * blocks + at.at] = (uint8_t)code;
    }
  } else {
    const int lane = threadIdx.x & 31;
    for (PieceWalk at((long long)blockIdx.x * 8 + (threadIdx.x >> 5), (long long)gridDim.x * 8, blocks); at.row < a.rows; at.next()) {
      const long long c = 32ll * at.at + lane;
      const float v = c < a.cols ? Elem<T>::get(static_cast<const char*>(a.x) + at.row * a.ld * EB, c) : 0.f;
      const uint32_t code = scale_code_e4m3(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(v) & ABS_MASK));
      a.codes[at.row * pitch + c] = (uint8_t)to_e4m3x2(v * scale_inverse(code), 0.f);
      if (lane == 0) a.scales[at.row * blocks + at.at] = (uint8_t)code;
    }
  }
}

// four codes of a block and its scale -> values
__device__ __forceinline__ void ckpt_values4(uint32_t w, float scale, float* v) {
  const float2 lo = from_e4m3x2(w & 0xFFFFu), hi = from_e4m3x2(w >> 16);
  v[0] = lo.x * scale; v[1] = lo.y * scale; v[2] = hi.x * scale; v[3] = hi.y * scale;
}

template <int T, int ACT>
__global__ void __launch_bounds__(256) ckpt_read_kernel(const __grid_constant__ CkptArgs a) {
  constexpr int EB = Elem<T>::bytes;
  const uint32_t blocks = (uint32_t)((a.cols + 31) / 32);
  const long long pitch = 32ll * blocks;
  if (a.vec) {
    for (PieceWalk at((long long)blockIdx.x * 256 + threadIdx.x, (long long)gridDim.x * 256, blocks); at.row < a.rows; at.next()) {
      const long long c = 32ll * at.at;
      const uint4* from = reinterpret_cast<const uint4*>(a.codes + at.row * pitch + c);
      const uint4 w0 = from[0], w1 = from[1];
      const float scale = scale_value(a.scales[at.row * blocks + at.at]);
      const uint32_t w[8] = {w0.x, w0.y, w0.z, w0.w, w1.x, w1.y, w1.z, w1.w};
      char* row = static_cast<char*>(a.out) + at.row * a.ldo * EB;
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        float v[8];
        ckpt_values4(w[2 * h], scale, v);
        ckpt_values4(w[2 * h + 1], scale, v + 4);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = act_value<ACT>(v[e]);
        if (c + 8 * h + 8 <= a.cols) Elem<T>::put8(row, c + 8 * h, v);
        else
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (c + 8 * h + e < a.cols) Elem<T>::put(row, c + 8 * h + e, v[e]);
      }
    }
  } else {
    const int lane = threadIdx.x & 31;
    for (PieceWalk at((long long)blockIdx.x * 8 + (threadIdx.x >> 5), (long long)gridDim.x * 8, blocks); at.row < a.rows; at.next()) {
      const long long c = 32ll * at.at + lane;
      const float v = from_e4m3x2(a.codes[at.row * pitch + c]).x * scale_value(a.scales[at.row * blocks + at.at]);
      if (c < a.cols) Elem<T>::put(static_cast<char*>(a.out) + at.row * a.ldo * EB, c, act_value<ACT>(v));
    }
  }
}

// dz = dy act'(z) and the sums of dz (before it is rounded) over the rows.  A block takes 256 columns and split_rows rows, a warp every
// eighth of these, a lane eight columns.  What a lane reads stays packed until its row's turn, so that the loads of two rows are
// in flight and three blocks fit a multiprocessor (four rows, or two worked on while the next two load, spill: 351 us; at two blocks 311).  The eight warps' sums meet in shared memory in the order of the warps; the blocks' in
// the order of the splits, where there are at most eight in the distributed shared memory of a cluster, else in a second kernel: the same
// bits every time.  KEPT = false: no z, only the sums of dy, and dz (if there is one) is a copy of dy.
template <int T, int ACT, bool KEPT, bool VEC>
__global__ void __launch_bounds__(256, 3) act_backward_kernel(const __grid_constant__ CkptArgs a) {
  constexpr int EB = Elem<T>::bytes, AHEAD = VEC || !KEPT ? 2 : 1, STEP = VEC ? 1 : 32;      // STEP: between a lane's eight columns
  __shared__ float sums[8][256];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t blocks = (uint32_t)((a.cols + 31) / 32);
  const long long pitch = 32ll * blocks, c0 = 256ll * blockIdx.x;
  const long long r0 = (long long)blockIdx.y * a.split_rows, r1 = min(a.rows, r0 + a.split_rows);
  const long long c = c0 + (VEC ? 8 * lane : lane);
  const int n = (int)max(0ll, min(8ll, VEC ? a.cols - c : (a.cols - c + 31) / 32));                 // of the eight that exist
  float acc[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = 0.f;

#pragma unroll 1
  for (long long r = r0 + warp; r < r1; r += 8 * AHEAD) {
    Raw8<T> g[AHEAD];
    uint2 code[AHEAD];
    uint32_t scale[AHEAD][VEC ? 1 : 8];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const long long row = r + 8 * k;
      const int m = row < r1 ? n : 0;
      const char* src = static_cast<const char*>(a.x) + row * a.ld * EB;
      if (VEC && m == 8) g[k].load(src, c);
      else if (VEC) g[k].load_some(src, c, m);
      else g[k].load_apart(src, c, 32, m);
      if constexpr (KEPT) {
        code[k] = make_uint2(0u, 0u);
        const uint8_t* from = a.codes + row * pitch + c;
        const uint8_t* sc = a.scales + row * blocks + (c >> 5);
        if (VEC) {
          scale[k][0] = 0u;
          if (m > 0) { code[k] = *reinterpret_cast<const uint2*>(from); scale[k][0] = *sc; }        // c is in the row, and a row of codes has whole blocks
        } else {
          uint32_t w[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            w[e] = e < m ? from[32 * e] : 0u;
            scale[k][e] = e < m ? sc[e] : 0u;
          }
          code[k] = make_uint2(w[0] | w[1] << 8 | w[2] << 16 | w[3] << 24, w[4] | w[5] << 8 | w[6] << 16 | w[7] << 24);
        }
      }
    }
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const long long row = r + 8 * k;
      const int m = row < r1 ? n : 0;
      float d[8];                                                          // what does not exist was read as zeros
#pragma unroll
      for (int e = 0; e < 8; ++e) d[e] = g[k].value(e);
      if constexpr (KEPT) {
        float z[8];
        bool lost = false;                                                 // a NaN block
        if (VEC) {
          const float s = scale_value(scale[k][0]);
          ckpt_values4(code[k].x, s, z);
          ckpt_values4(code[k].y, s, z + 4);
          lost = scale[k][0] == 255u;
        } else {
          ckpt_values4(code[k].x, 1.f, z);
          ckpt_values4(code[k].y, 1.f, z + 4);
#pragma unroll
          for (int e = 0; e < 8; ++e) { z[e] *= scale_value(scale[k][VEC ? 0 : e]); lost |= scale[k][VEC ? 0 : e] == 255u; }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) d[e] *= act_slope<ACT>(z[e]);
        if (lost) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (scale[k][VEC ? 0 : e] == 255u) d[e] = __uint_as_float(0x7FC00000u);
        }
      }
      if (KEPT || a.out) {
        char* to = static_cast<char*>(a.out) + row * a.ldo * EB;
        if (VEC && m == 8) Elem<T>::put8(to, c, d);
        else
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (e < m) Elem<T>::put(to, c + e * STEP, d[e]);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] += d[e];                          // zeros (or, of a tail, columns that are not there) add nothing that counts
    }
  }
  if (!a.partial && !a.db) return;
#pragma unroll
  for (int e = 0; e < 8; ++e) sums[warp][(VEC ? 8 * lane : lane) + e * STEP] = acc[e];
  __syncthreads();
  const long long at = c0 + threadIdx.x;
  float s = sums[0][threadIdx.x];
#pragma unroll
  for (int w = 1; w < 8; ++w) s += sums[w][threadIdx.x];
  if (a.partial) {
    if (at < a.cols) a.partial[(long long)blockIdx.y * a.cols + at] = s;
    return;
  }
  if (gridDim.y > 1) {
    sums[0][threadIdx.x] = s;                                            // read by this thread alone so far
    cluster_sync_all();
    if (blockIdx.y == 0)
      for (int r = 1; r < (int)gridDim.y; ++r) s += ld_cluster1(cluster_addr(smem_addr(&sums[0][threadIdx.x]), (uint32_t)r));
    cluster_sync_all();                                                  // nobody leaves while its sums may still be read
  }
  if (blockIdx.y == 0 && at < a.cols) put_as(a.db_type, a.db, at, s);
}

// Sums [splits][cols] -> out [cols].  A block takes 32 columns, a warp every eighth split.
__global__ void __launch_bounds__(256) column_sum_finish_kernel(const float* partial, int splits, long long cols, void* out, int type) {
  __shared__ float sums[8][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long c = 32ll * blockIdx.x + lane;
  float s = 0.f;
  if (c < cols)
#pragma unroll 4
    for (int k = warp; k < splits; k += 8) s += partial[(long long)k * cols + c];
  sums[warp][lane] = s;
  __syncthreads();
  if (warp == 0 && c < cols) {
#pragma unroll
    for (int w = 1; w < 8; ++w) s += sums[w][lane];
    put_as(type, out, c, s);
  }
}

}  // namespace ssim
