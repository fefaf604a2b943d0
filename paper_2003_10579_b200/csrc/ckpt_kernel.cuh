// Activations kept in 8 bits between the forward and the backward pass, and what the backward pass makes of them.
//
// A kept matrix [rows][cols] has E4M3 codes in rows of 32 ceil(cols / 32) bytes (the tail of a row zero) and one scale byte per block of
// 32 elements of a row, [rows][ceil(cols / 32)]: 2^(byte - 127), the smallest power of two, at least 2^-127, for which no magnitude of
// the block exceeds 448 times it; elements are rounded to nearest even (lowbits.cuh).  33/32 of a byte an element.
//
// Each of the three kernels is one pass whose floor is HBM: what it reads and writes once.  Rows that start on 16-byte boundaries move in
// whole 32-byte sectors, a thread a block or half a block; others go a warp to a block of 32, a lane an element, which still reads and
// writes neighbours together.
#pragma once
#include "act_math.cuh"
#include "lowbits.cuh"

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
  int split_rows;
};

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

// sixteen codes of a block and its scale -> values
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
    for (PieceWalk at((long long)blockIdx.x * 256 + threadIdx.x, (long long)gridDim.x * 256, 2 * blocks); at.row < a.rows; at.next()) {   // halves of blocks
      const long long c = 16ll * at.at;
      if (c >= a.cols) continue;
      const uint4 w = *reinterpret_cast<const uint4*>(a.codes + at.row * pitch + c);
      const float scale = scale_value(a.scales[at.row * blocks + (at.at >> 1)]);
      float v[2][8];
      ckpt_values4(w.x, scale, v[0]); ckpt_values4(w.y, scale, v[0] + 4); ckpt_values4(w.z, scale, v[1]); ckpt_values4(w.w, scale, v[1] + 4);
      char* row = static_cast<char*>(a.out) + at.row * a.ldo * EB;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[h][e] = act_value<ACT>(v[h][e]);
        if (c + 8 * h + 8 <= a.cols) Elem<T>::put8(row, c + 8 * h, v[h]);
        else
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (c + 8 * h + e < a.cols) Elem<T>::put(row, c + 8 * h + e, v[h][e]);
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
// eighth of these, a lane eight columns, four rows at a time so that loads of four rows are in flight.  The eight warps' sums meet in
// shared memory in the order of the warps, the blocks' in a second kernel in the order of the splits: the same bits every time.
// KEPT = false: no z, only the sums of dy.
template <int T, int ACT, bool KEPT>
__global__ void __launch_bounds__(256) act_backward_kernel(const __grid_constant__ CkptArgs a) {
  constexpr int EB = Elem<T>::bytes;
  __shared__ float sums[8][256];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t blocks = (uint32_t)((a.cols + 31) / 32);
  const long long pitch = 32ll * blocks, c0 = 256ll * blockIdx.x;
  const long long r0 = (long long)blockIdx.y * a.split_rows, r1 = min(a.rows, r0 + a.split_rows);
  const int step = a.vec ? 1 : 32;                                       // a lane's eight columns: neighbours, or 32 apart
  const long long c = c0 + (a.vec ? 8 * lane : lane);
  const bool whole = a.vec && c + 8 <= a.cols;
  float acc[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = 0.f;

  for (long long r = r0 + warp; r < r1; r += 32) {
    float g[4][8], z[4][8];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const long long row = r + 8 * k;
      const char* src = static_cast<const char*>(a.x) + row * a.ld * EB;
      if (row < r1 && whole) Elem<T>::get8(src, c, g[k]);
      else
#pragma unroll
        for (int e = 0; e < 8; ++e) g[k][e] = row < r1 && c + e * step < a.cols ? Elem<T>::get(src, c + e * step) : 0.f;
      if constexpr (KEPT) {
        const uint8_t* code = a.codes + row * pitch;
        const uint8_t* scale = a.scales + row * blocks;
        if (a.vec) {
          if (row < r1 && c < pitch) {
            const uint2 w = *reinterpret_cast<const uint2*>(code + c);
            const float s = scale_value(scale[c >> 5]);
            ckpt_values4(w.x, s, z[k]); ckpt_values4(w.y, s, z[k] + 4);
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) z[k][e] = 0.f;
          }
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const long long at = c + 32 * e;
            z[k][e] = row < r1 && at < pitch ? from_e4m3x2(code[at]).x * scale_value(scale[at >> 5]) : 0.f;
          }
        }
      }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const long long row = r + 8 * k;
      if constexpr (KEPT) {
#pragma unroll
        for (int e = 0; e < 8; ++e) g[k][e] *= act_slope<ACT>(z[k][e]);
        if (row < r1) {
          char* to = static_cast<char*>(a.out) + row * a.ldo * EB;
          if (whole) Elem<T>::put8(to, c, g[k]);
          else
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (c + e * step < a.cols) Elem<T>::put(to, c + e * step, g[k][e]);
        }
      }
      if (row < r1)
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] += g[k][e];
    }
  }
  if (!a.partial) return;
#pragma unroll
  for (int e = 0; e < 8; ++e) sums[warp][(a.vec ? 8 * lane : lane) + e * step] = acc[e];
  __syncthreads();
  const long long at = c0 + threadIdx.x;
  if (at < a.cols) {
    float s = sums[0][threadIdx.x];
#pragma unroll
    for (int w = 1; w < 8; ++w) s += sums[w][threadIdx.x];
    a.partial[(long long)blockIdx.y * a.cols + at] = s;
  }
}

// Sums [splits][cols] -> out [cols].  A block takes 32 columns, a warp every eighth split.
template <int T>
__global__ void __launch_bounds__(256) column_sum_finish_kernel(const float* partial, int splits, long long cols, void* out) {
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
    Elem<T>::put(out, c, s);
  }
}

}  // namespace ssim
