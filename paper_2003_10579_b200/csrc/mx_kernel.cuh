// MXFP4 quantisation and reading back (formats and rounding: lowbits.cuh).
//
// A matrix [rows][cols] has its codes in rows of 64 ceil(cols / 128) bytes (two codes a byte, the tail of a row zero), and one
// scale byte per block of 32 along the row, in one of two orders:
//   linear  [rows][ceil(cols / 32)]
//   tiles   the order the block-scaled tensor-core products read: tiles of 128 rows x 4 blocks, 512 bytes, tiles of one row group
//           one behind the other; row r of a tile at byte 16 (r % 32) + 4 (r / 32), its four blocks side by side.
// Both kernels are bound by HBM: 4 or 2 bytes an element in, 17/32 out per orientation.
#pragma once
#include "lowbits.cuh"

namespace ssim {

constexpr uint32_t MX_TAG_ROWS = 3, MX_TAG_COLS = 4;     // counter tags of the random numbers of the two orientations

__host__ __device__ inline long long mx_pitch(long long cols) { return 64 * ((cols + 127) / 128); }
__host__ __device__ inline long long mx_scale_at(long long row, long long block, long long blocks, long long kb, bool tiles) {
  return tiles ? ((row >> 7) * kb + (block >> 2)) * 512 + (row & 31) * 16 + ((row & 127) >> 5) * 4 + (block & 3) : row * blocks + block;
}

struct MxQuantArgs {
  const void* x;
  long long rows, cols, ld;
  uint8_t* codes;        // of the rows, or null
  uint8_t* scales;
  uint8_t* codes_t;      // of the columns (the transpose's rows), or null
  uint8_t* scales_t;
  int tiles, stochastic, vec;
  uint64_t seed;
};

__device__ __forceinline__ U4 mx_random(uint64_t seed, uint32_t tag, unsigned long long group, unsigned long long row) {
  return philox4x32_10((uint32_t)seed, (uint32_t)(seed >> 32), (uint32_t)group, (tag << 24) | (uint32_t)(group >> 32), (uint32_t)row, (uint32_t)(row >> 32));
}

// eight values -> eight codes; inv = 1 / scale
template <bool SR>
__device__ __forceinline__ uint32_t encode_e2m1(const float (&x)[8], float inv, const U4& u) {
  uint32_t w = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    float a = x[2 * k] * inv, b = x[2 * k + 1] * inv;
    if (SR) {
      a = round_stochastic<1, 0>(a, half_word(u, 2 * k));
      b = round_stochastic<1, 0>(b, half_word(u, 2 * k + 1));
    }
    w |= to_e2m1x2(a, b) << (8 * k);
  }
  return w;
}

// Rows only.  A thread takes eight elements, four neighbouring lanes a block; rows are padded to 128 elements, so a block of lanes
// never spans two rows.
template <int T, bool SR>
__global__ void __launch_bounds__(256) mx_quantize_rows_kernel(MxQuantArgs a) {
  const long long kb = (a.cols + 127) / 128, groups = kb * 16, blocks = (a.cols + 31) / 32, pitch = kb * 64;
  const long long step = (long long)gridDim.x * blockDim.x, first = (long long)blockIdx.x * blockDim.x + threadIdx.x;
  const long long drow = step / groups, dgrp = step % groups;
  long long row = first / groups, grp = first % groups;
  // all four lanes of a block run the same number of rounds: their groups differ only in the last two bits
  for (; row < a.rows; row += drow, grp += dgrp, row += grp >= groups, grp -= grp >= groups ? groups : 0) {
    const long long c = grp * 8;
    const char* src = static_cast<const char*>(a.x) + (row * a.ld) * Elem<T>::bytes;
    float x[8];
    if (a.vec && c + 8 <= a.cols) {
      Elem<T>::get8(src, c, x);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = c + e < a.cols ? Elem<T>::get(src, c + e) : 0.f;
    }
    uint32_t amax = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) amax = max(amax, __float_as_uint(x[e]) & ABS_MASK);
    const uint32_t team = 0xFu << (threadIdx.x & 28);
    amax = max(amax, __shfl_xor_sync(team, amax, 1));
    amax = max(amax, __shfl_xor_sync(team, amax, 2));
    const uint32_t code = scale_code_e2m1(amax);
    const uint32_t w = encode_e2m1<SR>(x, scale_inverse(code), SR ? mx_random(a.seed, MX_TAG_ROWS, grp, row) : U4{0, 0, 0, 0});
    *reinterpret_cast<uint32_t*>(a.codes + row * pitch + grp * 4) = w;
    const long long block = grp >> 2;
    if ((threadIdx.x & 3) == 0 && (a.tiles || block < blocks)) a.scales[mx_scale_at(row, block, blocks, kb, a.tiles)] = (uint8_t)code;
  }
}

// Columns, and rows from the same read: a block takes 128 x 128 elements through shared memory.  First every thread quantises eight
// neighbours of a row as above and leaves the raw elements in the tile; then a thread takes 32 elements of a column (two
// columns of 16-bit elements: one word a row) - whole blocks of the transpose, no exchange between lanes.  Codes of the
// transpose leave through shared memory, 64 consecutive bytes a column, scales as whole 512-byte tiles.
template <int T, bool SR>
__global__ void __launch_bounds__(256) mx_quantize_tile_kernel(MxQuantArgs a) {
  constexpr int EB = Elem<T>::bytes, CT = EB == 2 ? 2 : 1;     // columns a thread reads with one word
  extern __shared__ __align__(16) unsigned char tile[];        // [128][128] raw elements | codes_t [128][80] | scales [512] | scales_t [512]
  unsigned char* ct_s = tile + 128 * 128 * EB;
  unsigned char* sc_s = ct_s + 128 * 80;
  unsigned char* sct_s = sc_s + 512;
  const int tid = threadIdx.x;
  const long long row_tiles = (a.rows + 127) / 128, col_tiles = (a.cols + 127) / 128;
  const long long blocks = (a.cols + 31) / 32, blocks_t = (a.rows + 31) / 32;
  for (long long t = blockIdx.x; t < row_tiles * col_tiles; t += gridDim.x) {
    const long long rt = t / col_tiles, c_t = t % col_tiles, r0 = rt * 128, c0 = c_t * 128;
#pragma unroll
    for (int it = 0; it < 8; ++it) {
      const int r = it * 16 + (tid >> 4), g = tid & 15;
      const long long row = r0 + r, c = c0 + 8 * g;
      const char* src = static_cast<const char*>(a.x) + row * a.ld * EB;
      float x[8];
      if (row < a.rows && a.vec && c + 8 <= a.cols) {
        Elem<T>::get8(src, c, x);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = row < a.rows && c + e < a.cols ? Elem<T>::get(src, c + e) : 0.f;
      }
      Elem<T>::put8(tile, r * 128 + 8 * g, x);                  // exact: the values came from this type
      if (a.codes) {
        uint32_t amax = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) amax = max(amax, __float_as_uint(x[e]) & ABS_MASK);
        amax = max(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, 1));
        amax = max(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, 2));
        const uint32_t code = scale_code_e2m1(amax);
        const uint32_t w = encode_e2m1<SR>(x, scale_inverse(code), SR ? mx_random(a.seed, MX_TAG_ROWS, (c0 >> 3) + g, row) : U4{0, 0, 0, 0});
        if (row < a.rows) *reinterpret_cast<uint32_t*>(a.codes + row * (col_tiles * 64) + c0 / 2 + g * 4) = w;
        if ((g & 3) == 0) {
          if (a.tiles) sc_s[(r & 31) * 16 + (r >> 5) * 4 + (g >> 2)] = (unsigned char)code;
          else if (row < a.rows && (c0 >> 5) + (g >> 2) < blocks) a.scales[row * blocks + (c0 >> 5) + (g >> 2)] = (uint8_t)code;
        }
      }
    }
    __syncthreads();
    if (a.codes && a.tiles && tid < 128)
      reinterpret_cast<uint32_t*>(a.scales + (rt * col_tiles + c_t) * 512)[tid] = reinterpret_cast<const uint32_t*>(sc_s)[tid];
    for (int task = tid; task < 4 * 128 / CT; task += 256) {
      const int cp = task % (128 / CT), rb = task / (128 / CT);
      uint32_t raw[32];
#pragma unroll
      for (int i = 0; i < 32; ++i) raw[i] = *reinterpret_cast<const uint32_t*>(tile + ((rb * 32 + i) * 128 + cp * CT) * EB);
#pragma unroll
      for (int h = 0; h < CT; ++h) {
        const int col = cp * CT + h;
        auto value = [&](int i) -> float {
          if (T == T_F32) return __uint_as_float(raw[i]);
          if (T == T_BF16) return h ? __uint_as_float(raw[i] & 0xFFFF0000u) : __uint_as_float(raw[i] << 16);
          return f16_to_float(h ? raw[i] >> 16 : raw[i] & 0xFFFFu);
        };
        uint32_t amax = 0;
#pragma unroll
        for (int i = 0; i < 32; ++i) amax = max(amax, __float_as_uint(value(i)) & ABS_MASK);
        const uint32_t code = scale_code_e2m1(amax);
        const float inv = scale_inverse(code);
        uint32_t w[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          float x[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = value(8 * q + e);
          w[q] = encode_e2m1<SR>(x, inv, SR ? mx_random(a.seed, MX_TAG_COLS, (r0 >> 3) + rb * 4 + q, c0 + col) : U4{0, 0, 0, 0});
        }
        *reinterpret_cast<uint4*>(ct_s + col * 80 + rb * 16) = make_uint4(w[0], w[1], w[2], w[3]);
        if (a.tiles) sct_s[(col & 31) * 16 + (col >> 5) * 4 + rb] = (unsigned char)code;
        else if (c0 + col < a.cols && (r0 >> 5) + rb < blocks_t) a.scales_t[(c0 + col) * blocks_t + (r0 >> 5) + rb] = (uint8_t)code;
      }
    }
    __syncthreads();
    for (int i = tid; i < 512; i += 256) {
      const int col = i >> 2, piece = i & 3;
      if (c0 + col < a.cols)
        *reinterpret_cast<uint4*>(a.codes_t + (c0 + col) * (row_tiles * 64) + r0 / 2 + piece * 16) = *reinterpret_cast<const uint4*>(ct_s + col * 80 + piece * 16);
    }
    if (a.tiles && tid < 128)
      reinterpret_cast<uint32_t*>(a.scales_t + (c_t * row_tiles + rt) * 512)[tid] = reinterpret_cast<const uint32_t*>(sct_s)[tid];
    __syncthreads();
  }
}
template <int T>
constexpr int mx_tile_smem() { return 128 * 128 * Elem<T>::bytes + 128 * 80 + 1024; }

struct MxReadArgs {
  const uint8_t* codes;
  const uint8_t* scales;
  long long rows, cols, ld;
  void* out;
  int tiles, vec;
  int word;            // codes rows may be read as words (a single row of a pushed gradient may end in mid-word)
};

template <int T>
__global__ void __launch_bounds__(256) mx_dequantize_kernel(MxReadArgs a) {
  const long long kb = (a.cols + 127) / 128, groups = (a.cols + 7) / 8, blocks = (a.cols + 31) / 32, pitch = kb * 64;
  const long long step = (long long)gridDim.x * blockDim.x, first = (long long)blockIdx.x * blockDim.x + threadIdx.x;
  const long long drow = step / groups, dgrp = step % groups;
  long long row = first / groups, grp = first % groups;
  for (; row < a.rows; row += drow, grp += dgrp, row += grp >= groups, grp -= grp >= groups ? groups : 0) {
    const long long c = grp * 8;
    const int n8 = (int)min(8ll, a.cols - c);
    const uint8_t* src = a.codes + row * pitch + grp * 4;
    uint32_t w = 0;
    if (a.word && n8 == 8) {
      w = *reinterpret_cast<const uint32_t*>(src);
    } else {
      for (int b = 0; 2 * b < n8; ++b) w |= (uint32_t)src[b] << (8 * b);
    }
    const float s = scale_value(a.scales[mx_scale_at(row, grp >> 2, blocks, kb, a.tiles)]);
    float x[8];
    e2m1x8(w, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] *= s;
    char* dst = static_cast<char*>(a.out) + row * a.ld * Elem<T>::bytes;
    if (a.vec && n8 == 8) {
      Elem<T>::put8(dst, c, x);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < n8) Elem<T>::put(dst, c + e, x[e]);
    }
  }
}

}  // namespace ssim
