// C entry points of MXFP4 quantisation, reading back and products (mx_kernel.cuh, mx_gemm_kernel.cuh).
#include <atomic>
#include <cstdio>

#include "error.cuh"
#include "mx_gemm_kernel.cuh"
#include "mx_kernel.cuh"

using namespace ssim;

namespace {

sim_status cuda_failed(const char* where, cudaError_t e) {
  char msg[200];
  std::snprintf(msg, sizeof msg, "%s: %s", where, cudaGetErrorString(e));
  return record_error(e == cudaErrorMemoryAllocation ? SIM_ERR_ALLOC : SIM_ERR_CUDA, msg);
}
bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
bool bad_size(int64_t rows, int64_t cols) { return rows < 1 || cols < 1 || rows > (int64_t)1 << 35 || cols > (int64_t)1 << 35 || rows > ((int64_t)1 << 48) / cols; }
int elem_bytes(sim_dtype t) { return t == SIM_F32 ? 4 : 2; }

int sm_count() {
  int dev = 0, sms = 148;
  if (cudaGetDevice(&dev) == cudaSuccess) cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  return sms;
}
// Dynamic shared memory of a kernel, asked for once a device (the call costs a microsecond)
template <typename K>
cudaError_t allow_smem(K kern, int bytes, std::atomic<unsigned long long>& done) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess || (dev < 64 && (done.load(std::memory_order_relaxed) >> dev & 1))) return e;
  e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess && dev < 64) done.fetch_or(1ull << dev, std::memory_order_relaxed);
  return e;
}
unsigned grid_for(long long threads) {
  const long long blocks = (threads + 255) / 256, full = 16ll * sm_count();
  return (unsigned)(blocks < full ? blocks : full);
}

template <int T, bool SR>
cudaError_t quantize(const MxQuantArgs& a, cudaStream_t st) {
  if (!a.codes_t) {
    mx_quantize_rows_kernel<T, SR><<<grid_for(a.rows * ((a.cols + 127) / 128) * 4), 256, 0, st>>>(a);
    return cudaGetLastError();
  }
  constexpr int smem = mx_tile_smem<T>();
  static std::atomic<unsigned long long> done{0};
  cudaError_t e = allow_smem(mx_quantize_tile_kernel<T, SR>, smem, done);
  if (e != cudaSuccess) return e;
  // a block a tile: the hardware's dealing beats a grid that stays (8192 x 5120 bf16: 37 against 41 us)
  const long long tiles = ((a.rows + 127) / 128) * ((a.cols + 127) / 128);
  if (tiles > 0x7FFFFFFFll) return cudaErrorInvalidValue;
  mx_quantize_tile_kernel<T, SR><<<(unsigned)tiles, 256, smem, st>>>(a);
  return cudaGetLastError();
}
template <int T>
cudaError_t quantize_sr(const MxQuantArgs& a, cudaStream_t st) { return a.stochastic ? quantize<T, true>(a, st) : quantize<T, false>(a, st); }

// rows of codes as a 2-D byte tensor; box: 128 bytes (256 elements of k) x box_rows, 128-byte swizzle, zeros outside
bool make_map(CUtensorMap* map, const uint8_t* codes, int64_t rows, int64_t cols, uint32_t box_rows) {
  PFN_encodeTiled fn = tc_encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)mx_pitch(cols), (cuuint64_t)rows};
  const cuuint64_t strides[1] = {dims[0]};
  const cuuint32_t box[2] = {128, box_rows}, one[2] = {1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<uint8_t*>(codes), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// scale tiles as a 2-D tensor of 512-byte rows; box: `tiles` that follow one another along k
bool make_scale_map(CUtensorMap* map, const uint8_t* scales, int64_t rows, int64_t kb, uint32_t tiles) {
  PFN_encodeTiled fn = tc_encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[2] = {128, (cuuint64_t)((rows + 127) / 128 * kb)};
  const cuuint64_t strides[1] = {512};
  const cuuint32_t box[2] = {128, tiles}, one[2] = {1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT32, 2, const_cast<uint8_t*>(scales), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct MxgMaps { CUtensorMap a, b, sa, sb; };

template <int T>
cudaError_t launch_pair(const MxgMaps& m, const MxgArgs& g, int sms, cudaStream_t st) {
  static std::atomic<unsigned long long> done{0};
  cudaError_t e = allow_smem(mx_gemm_pair_kernel<T>, MXP_SMEM, done);
  if (e != cudaSuccess) return e;
  const long long tiles = (long long)g.tiles_a * g.tiles_b, pairs = sms / 2;
  mx_gemm_pair_kernel<T><<<(unsigned)(2 * (tiles < pairs ? tiles : pairs)), MXP_THREADS, MXP_SMEM, st>>>(m.a, m.b, m.sa, m.sb, g);
  return cudaGetLastError();
}

template <int BN, int T, bool SWAP, bool SPLIT>
cudaError_t launch(const MxgMaps& m, const MxgArgs& g, int split, cudaStream_t st) {
  auto kern = mx_gemm_kernel<BN, T, SWAP, SPLIT>;
  // partial sums of a split tile lie in the ring's bytes
  static_assert(!SPLIT || 128 * (BN + 4) * 4 <= MxgShape<BN>::OFF_BARS, "the partial sums must fit the ring");
  static std::atomic<unsigned long long> done{0};
  cudaError_t e = allow_smem(kern, MxgShape<BN>::SMEM, done);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(g.tiles_a * g.tiles_b), (unsigned)split, 1);
  cfg.blockDim = dim3(MXG_THREADS, 1, 1);
  cfg.dynamicSmemBytes = MxgShape<BN>::SMEM;
  cfg.stream = st;
  cudaLaunchAttribute attr{};
  if (SPLIT) {
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = 1; attr.val.clusterDim.y = (unsigned)split; attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
  }
  return cudaLaunchKernelEx(&cfg, kern, m.a, m.b, m.sa, m.sb, g);
}
template <int BN, int T, bool SWAP>
cudaError_t launch_split(const MxgMaps& m, const MxgArgs& g, int split, cudaStream_t st) {
  return split > 1 ? launch<BN, T, SWAP, true>(m, g, split, st) : launch<BN, T, SWAP, false>(m, g, split, st);
}
template <int T, bool SWAP>
cudaError_t launch_bn(int bn, const MxgMaps& m, const MxgArgs& g, int split, cudaStream_t st) {
  switch (bn) {
    case 16: return launch_split<16, T, SWAP>(m, g, split, st);
    case 32: return launch_split<32, T, SWAP>(m, g, split, st);
    case 64: return launch_split<64, T, SWAP>(m, g, split, st);
    default:
      if constexpr (!SWAP) return launch_split<128, T, false>(m, g, split, st);
      return cudaErrorInvalidValue;      // at most 64 rows are swapped
  }
}

}  // namespace

extern "C" {

int64_t sim_mx_codes_bytes(int64_t rows, int64_t cols) { return bad_size(rows, cols) ? 0 : rows * mx_pitch(cols); }
int64_t sim_mx_scales_bytes(int64_t rows, int64_t cols, int32_t tiles) {
  if (bad_size(rows, cols)) return 0;
  return tiles ? (rows + 127) / 128 * ((cols + 127) / 128) * 512 : rows * ((cols + 31) / 32);
}

sim_status sim_mx_quantize(const void* x, sim_dtype type, int64_t rows, int64_t cols, int64_t ld, int32_t tiles, int32_t stochastic,
                           uint64_t seed, uint8_t* codes, uint8_t* scales, uint8_t* codes_t, uint8_t* scales_t, void* cuda_stream) {
  if (bad_size(rows, cols)) return record_error(SIM_ERR_ARG, "sim_mx_quantize: rows and cols must be in [1, 2^35], and their product at most 2^48");
  if (type != SIM_F32 && type != SIM_BF16 && type != SIM_F16) return record_error(SIM_ERR_ARG, "sim_mx_quantize: type must be SIM_F32, SIM_BF16 or SIM_F16");
  if (codes_t && (rows + 127) / 128 * ((cols + 127) / 128) > 0x7FFFFFFFll) return record_error(SIM_ERR_ARG, "sim_mx_quantize: at most 2^31 - 1 tiles of 128 x 128 along the columns");
  if (ld < cols || ld > ((int64_t)1 << 50) / rows) return record_error(SIM_ERR_ARG, "sim_mx_quantize: ld must be at least cols");
  if (!x || !aligned(x, elem_bytes(type))) return record_error(SIM_ERR_ARG, "sim_mx_quantize: x must be aligned to its type");
  if (!codes != !scales || !codes_t != !scales_t || (!codes && !codes_t))
    return record_error(SIM_ERR_ARG, "sim_mx_quantize: codes and scales of the rows, of the columns, or of both are required");
  if (!aligned(codes, 16) || !aligned(codes_t, 16) || (tiles && (!aligned(scales, 16) || !aligned(scales_t, 16))))
    return record_error(SIM_ERR_ARG, "sim_mx_quantize: codes and tiled scales must be 16-byte aligned");
  MxQuantArgs a{};
  a.x = x; a.rows = rows; a.cols = cols; a.ld = ld; a.codes = codes; a.scales = scales; a.codes_t = codes_t; a.scales_t = scales_t;
  a.tiles = tiles ? 1 : 0; a.stochastic = stochastic ? 1 : 0; a.keys = philox_keys(seed);
  for (int to = 16; to <= 32; to += 16)       // rows on 16-byte, on 32-byte boundaries
    if (aligned(x, to) && (rows == 1 || ld * elem_bytes(type) % to == 0)) a.vec = to / 16;
  const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const cudaError_t e = type == SIM_F32 ? quantize_sr<T_F32>(a, st) : type == SIM_BF16 ? quantize_sr<T_BF16>(a, st) : quantize_sr<T_F16>(a, st);
  return e == cudaSuccess ? SIM_OK : cuda_failed("sim_mx_quantize", e);
}

sim_status sim_mx_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t cols, int32_t tiles, sim_dtype type, void* out,
                             int64_t ld, void* cuda_stream) {
  if (bad_size(rows, cols)) return record_error(SIM_ERR_ARG, "sim_mx_dequantize: rows and cols must be in [1, 2^35], and their product at most 2^48");
  if (type != SIM_F32 && type != SIM_BF16 && type != SIM_F16) return record_error(SIM_ERR_ARG, "sim_mx_dequantize: type must be SIM_F32, SIM_BF16 or SIM_F16");
  if (ld < cols || ld > ((int64_t)1 << 50) / rows) return record_error(SIM_ERR_ARG, "sim_mx_dequantize: ld must be at least cols");
  if (!codes || !scales || !out || !aligned(out, elem_bytes(type))) return record_error(SIM_ERR_ARG, "sim_mx_dequantize: codes, scales and out (aligned to its type) are required");
  MxReadArgs a{};
  a.codes = codes; a.scales = scales; a.rows = rows; a.cols = cols; a.ld = ld; a.out = out; a.tiles = tiles ? 1 : 0;
  a.vec = aligned(out, 32) && (rows == 1 || ld * elem_bytes(type) % 32 == 0) ? 1 : 0;
  a.word = aligned(codes, 16) ? 1 : 0;
  const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const int unit = type == SIM_F32 ? mx_read_unit<T_F32>() : mx_read_unit<T_BF16>();
  const unsigned grid = grid_for(rows * ((cols + unit - 1) / unit));
  if (type == SIM_F32) mx_dequantize_kernel<T_F32><<<grid, 256, 0, st>>>(a);
  else if (type == SIM_BF16) mx_dequantize_kernel<T_BF16><<<grid, 256, 0, st>>>(a);
  else mx_dequantize_kernel<T_F16><<<grid, 256, 0, st>>>(a);
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? SIM_OK : cuda_failed("sim_mx_dequantize", e);
}

sim_status sim_mx_matmul(const uint8_t* a_codes, const uint8_t* a_scales, const uint8_t* b_codes, const uint8_t* b_scales, int64_t M, int64_t N,
                         int64_t K, sim_dtype type, void* c, int64_t ldc, void* cuda_stream) {
  const int64_t top = (int64_t)1 << 30;
  if (M < 1 || N < 1 || K < 1 || M > top || N > top || K > top) return record_error(SIM_ERR_ARG, "sim_mx_matmul: M, N and K must be in [1, 2^30]");
  if (type != SIM_F32 && type != SIM_BF16) return record_error(SIM_ERR_ARG, "sim_mx_matmul: the result is SIM_F32 or SIM_BF16");
  if (ldc < N || ldc > ((int64_t)1 << 50) / M) return record_error(SIM_ERR_ARG, "sim_mx_matmul: ldc must be at least N");
  if (!a_codes || !a_scales || !b_codes || !b_scales || !c || !aligned(c, elem_bytes(type)))
    return record_error(SIM_ERR_ARG, "sim_mx_matmul: operands and result (aligned to its type) are required");
  if (!aligned(a_codes, 16) || !aligned(a_scales, 16) || !aligned(b_codes, 16) || !aligned(b_scales, 16))
    return record_error(SIM_ERR_ARG, "sim_mx_matmul: codes and scales must be 16-byte aligned");
  // few rows: they become the B operand of the instruction (16, 32 or 64 wide), the other matrix its 128-row A operand
  const bool swap = M <= 64 && M <= N;
  const int64_t ra = swap ? N : M, rb = swap ? M : N;
  const int kb = (int)((K + 127) / 128), sms = sm_count();
  const int64_t tiles_a = (ra + 127) / 128;
  int bn = rb <= 16 ? 16 : rb <= 32 ? 32 : rb <= 64 ? 64 : 128;
  // Pairs of multiprocessors on 256 x 256 tiles: from a tile for every second pair on (256 x 4096 x 4096, 16 tiles: 14.6 us against 13.6),
  // and, while single multiprocessors finish in one wave, for long sums only (1280 x 2048 x 1024, 40 tiles: 10.5 against 8.5 us; 1024 x 4096 x
  // 4096, 64 tiles: 15.7 against 15.9; 1024 x 1280 x 8192: 20.8 against 21.4; 2048 x 4096 x 1024, 128 tiles: 12.6 against 14.6)
  const int64_t tiles_256 = (ra + 255) / 256 * ((rb + 255) / 256);
  const bool pair = ra > 128 && rb > 128 && tiles_256 >= sms / 4 && (tiles_256 > sms / 2 || kb >= 32);
  const int64_t tiles_b = (rb + bn - 1) / bn;
  if (tiles_a * tiles_b > (int64_t)1 << 30) return record_error(SIM_ERR_ARG, "sim_mx_matmul: the result has too many tiles");
  // Few tiles: k is split over a cluster.  Narrow tiles add little to the end of the kernel, so down to 512 elements of k a block and up to
  // two blocks a multiprocessor (1 x 4096 x 4096: 12.5 -> 8.4 us); 128 x 128 partial sums cost as much as 2048 elements of k
  // (512 x 512 x 8192: 20.7 -> 12.5 us, but 1024 x 1024 x 1024: 7.4 -> 10.4 us).
  int split = 1;
  const int least = bn < 128 ? 4 : 16, blocks = bn < 128 ? 2 * sms : sms;
  while (!pair && split < 8 && tiles_a * tiles_b * split * 2 <= blocks && kb >= split * 2 * least) split *= 2;
  MxgArgs g{};
  g.rows_a = ra; g.rows_b = rb; g.kb = kb;
  g.kb_split = ((kb + split - 1) / split + 1) / 2 * 2;
  split = (kb + g.kb_split - 1) / g.kb_split;          // every block of a cluster has a part
  g.tiles_a = (int)tiles_a; g.tiles_b = (int)tiles_b;
  g.d = c; g.ldd = ldc;
  g.vec = aligned(c, 16) && ldc * elem_bytes(type) % 16 == 0 ? 1 : 0;
  MxgMaps m;
  const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  cudaError_t e;
  if (pair) {
    g.rows_a = M; g.rows_b = N;
    g.tiles_a = (int)((M + 255) / 256); g.tiles_b = (int)((N + 255) / 256);
    if (!make_map(&m.a, a_codes, M, K, 128) || !make_map(&m.b, b_codes, N, K, 128) || !make_scale_map(&m.sa, a_scales, M, kb, 4) || !make_scale_map(&m.sb, b_scales, N, kb, 4))
      return record_error(SIM_ERR_CUDA, "sim_mx_matmul: the driver refused a tensor map");
    e = type == SIM_F32 ? launch_pair<T_F32>(m, g, sms, st) : launch_pair<T_BF16>(m, g, sms, st);
    return e == cudaSuccess ? SIM_OK : cuda_failed("sim_mx_matmul", e);
  }
  if (!make_map(&m.a, swap ? b_codes : a_codes, ra, K, 128) || !make_map(&m.b, swap ? a_codes : b_codes, rb, K, (uint32_t)bn) ||
      !make_scale_map(&m.sa, swap ? b_scales : a_scales, ra, kb, 2) || !make_scale_map(&m.sb, swap ? a_scales : b_scales, rb, kb, 2))
    return record_error(SIM_ERR_CUDA, "sim_mx_matmul: the driver refused a tensor map");
  if (type == SIM_F32) e = swap ? launch_bn<T_F32, true>(bn, m, g, split, st) : launch_bn<T_F32, false>(bn, m, g, split, st);
  else e = swap ? launch_bn<T_BF16, true>(bn, m, g, split, st) : launch_bn<T_BF16, false>(bn, m, g, split, st);
  return e == cudaSuccess ? SIM_OK : cuda_failed("sim_mx_matmul", e);
}

}  // extern "C"
