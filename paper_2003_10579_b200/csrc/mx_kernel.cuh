// MXFP4 quantisation and reading back (formats and rounding: lowbits.cuh).
//
// A matrix [rows][cols] has its codes in rows of 64 ceil(cols / 128) bytes (two codes a byte, the tail of a row zero), and one
// scale byte per block of 32 along the row, in one of two orders:
//   linear  [rows][ceil(cols / 32)]
//   tiles   the order the block-scaled tensor-core products read: tiles of 128 rows x 4 blocks, 512 bytes, tiles of one row group
//           one behind the other; row r of a tile at byte 16 (r % 32) + 4 (r / 32), its four blocks side by side.
// The floor of each is HBM: 4 or 2 bytes an element in, 17/32 out per orientation.  Measured: 8192 x 5120 bf16 along rows 18.6 us (5.7 TB/s),
// along both axes 37 us (3.5 TB/s; 69 % of the issue slots: a block's three phases wait for one another; stochastically 78 us), read back 19.6 us (5.4 TB/s); 30 M fp32 along one row 26.7
// us, stochastically 31 us (4.4 TB/s), read back 26.6 us.
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
  PhiloxKeys keys;
};

__device__ __forceinline__ U4 mx_random(const PhiloxKeys& keys, uint32_t tag, unsigned long long group, unsigned long long row) {
  return philox_keyed(keys, (uint32_t)group, (tag << 24) | (uint32_t)(group >> 32), (uint32_t)row, (uint32_t)(row >> 32));
}

// eight values times inv = 1 / scale -> eight codes
template <bool SR>
__device__ __forceinline__ uint32_t encode_e2m1(float (&x)[8], float inv, const U4& u) {
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] *= inv;
  if (SR) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = round_stochastic<1, 0>(x[e], half_word(u, e));
  }
  return to_e2m1x8(x);
}

// Where a thread stands in a matrix whose rows are `units` pieces long, stepped by the size of the grid without a division each time
struct RowWalk {
  long long row, drow;
  uint32_t unit, dunit, units;
  __device__ __forceinline__ RowWalk(long long units_) : units((uint32_t)units_) {
    const long long step = (long long)gridDim.x * blockDim.x, first = (long long)blockIdx.x * blockDim.x + threadIdx.x;
    row = first / units_; unit = (uint32_t)(first % units_);
    drow = step / units_; dunit = (uint32_t)(step % units_);
  }
  __device__ __forceinline__ void next() {
    row += drow;
    unit += dunit;
    if (unit >= units) { unit -= units; ++row; }
  }
};

// Rows only.  A thread takes a block of 32 elements, in whole 32-byte sectors where the rows allow it.
template <int T, bool SR>
__global__ void __launch_bounds__(256) mx_quantize_rows_kernel(const __grid_constant__ MxQuantArgs a) {
  constexpr int EB = Elem<T>::bytes;
  const long long kb = (a.cols + 127) / 128, blocks = (a.cols + 31) / 32, pitch = kb * 64;
  for (RowWalk w(kb * 4); w.row < a.rows; w.next()) {
    const long long c = (long long)w.unit * 32;
    const char* src = static_cast<const char*>(a.x) + w.row * a.ld * EB;
    Raw8<T> x[4];
    if (a.vec == 2 && c + 32 <= a.cols) {
      if constexpr (EB == 4) {
#pragma unroll
        for (int q = 0; q < 4; ++q) load32(src + (c + 8 * q) * 4, x[q].w);
      } else {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          uint32_t t[8];
          load32(src + (c + 16 * q) * 2, t);
#pragma unroll
          for (int k = 0; k < 4; ++k) { x[2 * q].w[k] = t[k]; x[2 * q + 1].w[k] = t[4 + k]; }
        }
      }
    } else if (a.vec && c + 32 <= a.cols) {
#pragma unroll
      for (int q = 0; q < 4; ++q) x[q].load(src, c + 8 * q);
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q) x[q].load_some(src, c + 8 * q, (int)max(0ll, min(8ll, a.cols - c - 8 * q)));
    }
    const uint32_t code = scale_code_e2m1(max(max(x[0].amax(), x[1].amax()), max(x[2].amax(), x[3].amax())));
    const float inv = scale_inverse(code);
    uint32_t o[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = x[q].value(e);
      o[q] = encode_e2m1<SR>(v, inv, SR ? mx_random(a.keys, MX_TAG_ROWS, 4ull * w.unit + q, w.row) : U4{0, 0, 0, 0});
    }
    *reinterpret_cast<uint4*>(a.codes + w.row * pitch + 16ll * w.unit) = make_uint4(o[0], o[1], o[2], o[3]);
    if (a.tiles || w.unit < blocks) a.scales[mx_scale_at(w.row, w.unit, blocks, kb, a.tiles)] = (uint8_t)code;
  }
}

// Columns, and rows from the same read: a block takes 128 x 128 elements through shared memory.  First every thread quantises eight
// neighbours of a row as above and leaves the raw elements in the tile; then a thread takes 32 elements of a column (two
// columns of 16-bit elements: one word a row) - whole blocks of the transpose, no exchange between lanes.  Codes of the
// transpose leave through shared memory, 64 consecutive bytes a column, scales as whole 512-byte tiles.
template <int T, bool SR>
__global__ void __launch_bounds__(256, 4) mx_quantize_tile_kernel(const __grid_constant__ MxQuantArgs a) {
  constexpr int EB = Elem<T>::bytes, CT = EB == 2 ? 2 : 1;     // columns a thread reads with one word
  extern __shared__ __align__(16) unsigned char tile[];        // [128][128] raw elements | codes_t [128][80] | scales [512] | scales_t [512]
  unsigned char* ct_s = tile + 128 * 128 * EB;
  unsigned char* sc_s = ct_s + 128 * 80;
  unsigned char* sct_s = sc_s + 512;
  const int tid = threadIdx.x;
  const long long row_tiles = (a.rows + 127) / 128, col_tiles = (a.cols + 127) / 128;
  const long long blocks = (a.cols + 31) / 32, blocks_t = (a.rows + 31) / 32;
  const long long t = blockIdx.x;
  const long long rt = t / col_tiles, c_t = t % col_tiles, r0 = rt * 128, c0 = c_t * 128;
  const int r_first = tid >> 4, g = tid & 15;
  const long long c = c0 + 8 * g;
  const bool wide = a.vec && c + 8 <= a.cols;
  const char* src = static_cast<const char*>(a.x) + (r0 + r_first) * a.ld * EB;
#pragma unroll
  for (int batch = 0; batch < 2; ++batch) {
    Raw8<T> x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = (4 * batch + i) * 16 + r_first;
      const char* from = src + (long long)(4 * batch + i) * 16 * a.ld * EB;
      if (r0 + r < a.rows && wide) x[i].load(from, c);
      else x[i].load_some(from, c, r0 + r < a.rows ? (int)max(0ll, min(8ll, a.cols - c)) : 0);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = (4 * batch + i) * 16 + r_first;
      uint4* to = reinterpret_cast<uint4*>(tile + (r * 128 + 8 * g) * EB);
      to[0] = make_uint4(x[i].w[0], x[i].w[1], x[i].w[2], x[i].w[3]);
      if constexpr (EB == 4) to[1] = make_uint4(x[i].w[4], x[i].w[5], x[i].w[6], x[i].w[7]);
      if (a.codes) {
        uint32_t amax = x[i].amax();
        amax = max(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, 1));
        amax = max(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, 2));
        const uint32_t code = scale_code_e2m1(amax);
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = x[i].value(e);
        const uint32_t w = encode_e2m1<SR>(v, scale_inverse(code), SR ? mx_random(a.keys, MX_TAG_ROWS, (c0 >> 3) + g, r0 + r) : U4{0, 0, 0, 0});
        if (r0 + r < a.rows) *reinterpret_cast<uint32_t*>(a.codes + (r0 + r) * (col_tiles * 64) + c0 / 2 + g * 4) = w;
        if ((g & 3) == 0) {
          if (a.tiles) sc_s[(r & 31) * 16 + (r >> 5) * 4 + (g >> 2)] = (unsigned char)code;
          else if (r0 + r < a.rows && (c0 >> 5) + (g >> 2) < blocks) a.scales[(r0 + r) * blocks + (c0 >> 5) + (g >> 2)] = (uint8_t)code;
        }
      }
    }
  }
  __syncthreads();
  if (a.codes && a.tiles && tid < 128)
    reinterpret_cast<uint32_t*>(a.scales + (rt * col_tiles + c_t) * 512)[tid] = reinterpret_cast<const uint32_t*>(sc_s)[tid];
#pragma unroll 1
  for (int task = tid; task < 4 * 128 / CT; task += 256) {
    const int cp = task % (128 / CT), rb = task / (128 / CT);
    const unsigned char* col_s = tile + (rb * 32 * 128 + cp * CT) * EB;
    // largest magnitudes of the column (of both columns side by side)
    uint32_t top = 0;
    float topf = 0.f;
#pragma unroll
    for (int i = 0; i < 32; i += 2) {
      const uint32_t p = *reinterpret_cast<const uint32_t*>(col_s + i * 128 * EB), q = *reinterpret_cast<const uint32_t*>(col_s + (i + 1) * 128 * EB);
      if (EB == 2) top = max_u16x2(top, max_u16x2(p & 0x7FFF7FFFu, q & 0x7FFF7FFFu));
      else topf = max3_abs(topf, __uint_as_float(p), __uint_as_float(q));
    }
    uint32_t code[CT];
    float inv[CT];
#pragma unroll
    for (int h = 0; h < CT; ++h) {
      uint32_t amax;
      if constexpr (EB == 2) amax = Raw8<T>::widen(h ? top >> 16 : top & 0xFFFFu);
      else amax = __float_as_uint(topf) & ABS_MASK;
      code[h] = scale_code_e2m1(amax);
      inv[h] = scale_inverse(code[h]);
    }
    uint32_t w[CT][4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      uint32_t raw[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) raw[i] = *reinterpret_cast<const uint32_t*>(col_s + (8 * q + i) * 128 * EB);
#pragma unroll
      for (int h = 0; h < CT; ++h) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (T == T_F32) v[i] = __uint_as_float(raw[i]);
          else if (T == T_BF16) v[i] = __uint_as_float(h ? raw[i] & 0xFFFF0000u : raw[i] << 16);
          else v[i] = f16_to_float(h ? raw[i] >> 16 : raw[i] & 0xFFFFu);
        }
        w[h][q] = encode_e2m1<SR>(v, inv[h], SR ? mx_random(a.keys, MX_TAG_COLS, (r0 >> 3) + rb * 4 + q, c0 + cp * CT + h) : U4{0, 0, 0, 0});
      }
    }
#pragma unroll
    for (int h = 0; h < CT; ++h) {
      const int col = cp * CT + h;
      *reinterpret_cast<uint4*>(ct_s + col * 80 + rb * 16) = make_uint4(w[h][0], w[h][1], w[h][2], w[h][3]);
      if (a.tiles) sct_s[(col & 31) * 16 + (col >> 5) * 4 + rb] = (unsigned char)code[h];
      else if (c0 + col < a.cols && (r0 >> 5) + rb < blocks_t) a.scales_t[(c0 + col) * blocks_t + (r0 >> 5) + rb] = (uint8_t)code[h];
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
}
template <int T>
constexpr int mx_tile_smem() { return 128 * 128 * Elem<T>::bytes + 128 * 80 + 1024; }

struct MxReadArgs {
  const uint8_t* codes;
  const uint8_t* scales;
  long long rows, cols, ld;
  void* out;
  int tiles, vec;
  int word;            // rows of codes may be read sixteen bytes at a time
};

// 64 bytes of stored elements a thread (32 of 16 bits, 16 of fp32: 128 bytes a thread took 31 us instead of 27 for 30 M), in whole
// 32-byte sectors where the rows allow it
template <int T>
__host__ __device__ constexpr int mx_read_unit() { return 64 / Elem<T>::bytes; }

template <int T>
__global__ void __launch_bounds__(256) mx_dequantize_kernel(const __grid_constant__ MxReadArgs a) {
  constexpr int EB = Elem<T>::bytes, UNIT = mx_read_unit<T>(), WORDS = UNIT / 8;
  const long long kb = (a.cols + 127) / 128, blocks = (a.cols + 31) / 32, pitch = kb * 64;
  for (RowWalk w((a.cols + UNIT - 1) / UNIT); w.row < a.rows; w.next()) {
    const long long c = (long long)w.unit * UNIT;
    const int n = (int)min((long long)UNIT, a.cols - c);
    const uint8_t* src = a.codes + w.row * pitch + c / 2;
    uint32_t q[WORDS];
    if (a.word && n == UNIT) {
      if constexpr (WORDS == 4) {
        const uint4 x = *reinterpret_cast<const uint4*>(src);
        q[0] = x.x; q[1] = x.y; q[2] = x.z; q[3] = x.w;
      } else {
        const uint2 x = *reinterpret_cast<const uint2*>(src);
        q[0] = x.x; q[1] = x.y;
      }
    } else {
#pragma unroll
      for (int k = 0; k < WORDS; ++k) q[k] = 0u;
#pragma unroll
      for (int b = 0; b < UNIT / 2; ++b)
        if (2 * b < n) q[b >> 2] |= (uint32_t)src[b] << (8 * (b & 3));
    }
    const float s = scale_value(a.scales[mx_scale_at(w.row, c >> 5, blocks, kb, a.tiles)]);
    char* dst = static_cast<char*>(a.out) + (w.row * a.ld + c) * EB;
#pragma unroll
    for (int h = 0; h < 2; ++h) {                // 32 bytes of the result
      constexpr int E = 32 / EB;
      float x[E / 8][8];
#pragma unroll
      for (int k = 0; k < E / 8; ++k) {
        e2m1x8(q[h * (E / 8) + k], x[k]);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[k][e] *= s;
      }
      if (a.vec && n == UNIT) {
        uint32_t o[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          if constexpr (EB == 4) o[k] = __float_as_uint(x[0][k]);
          else o[k] = T == T_BF16 ? float_to_bf16x2(x[k >> 2][2 * (k & 3)], x[k >> 2][2 * (k & 3) + 1]) : float_to_f16x2(x[k >> 2][2 * (k & 3)], x[k >> 2][2 * (k & 3) + 1]);
        }
        store32(dst + 32 * h, o);
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (E * h + e < n) Elem<T>::put(dst, E * h + e, x[e >> 3][e & 7]);
      }
    }
  }
}

}  // namespace ssim
