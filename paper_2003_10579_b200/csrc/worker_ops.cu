// C entry points of a worker's operators: products with their tails (matmul_kernel.cuh), activations in 8 bits (ckpt_kernel.cuh),
// log probabilities (logprob_kernel.cuh).
#include <atomic>
#include <cmath>
#include <cstdio>

#include "ckpt_kernel.cuh"
#include "error.cuh"
#include "logprob_kernel.cuh"
#include "matmul_kernel.cuh"

using namespace ssim;

namespace {

sim_status cuda_failed(const char* where, cudaError_t e) {
  char msg[200];
  std::snprintf(msg, sizeof msg, "%s: %s", where, cudaGetErrorString(e));
  return record_error(e == cudaErrorMemoryAllocation ? SIM_ERR_ALLOC : SIM_ERR_CUDA, msg);
}
sim_status bad(const char* msg) { return record_error(SIM_ERR_ARG, msg); }
bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
int elem_bytes(sim_dtype t) { return t == SIM_F32 ? 4 : 2; }
bool plain_type(sim_dtype t) { return t == SIM_F32 || t == SIM_BF16 || t == SIM_F16; }
bool known_act(sim_act a) { return a >= SIM_ACT_NONE && a <= SIM_ACT_SILU; }
// rows of `cols` elements, ld apart: sizes that the kernels' arithmetic holds
bool bad_matrix(int64_t rows, int64_t cols, int64_t ld) {
  return rows < 0 || cols < 0 || rows > (int64_t)1 << 31 || cols > (int64_t)1 << 31 || ld < cols || (rows > 1 && ld > ((int64_t)1 << 48) / rows);
}
// rows on boundaries of `to` bytes
bool rows_aligned(const void* p, int64_t rows, int64_t ld, sim_dtype t, int to) { return aligned(p, to) && (rows <= 1 || ld * elem_bytes(t) % to == 0); }
// A matrix in memory, first byte to behind the last, rows of `width` bytes `pitch` apart; and whether two share a byte.  Rows as far apart in both, as of
// column slices of one buffer, may lie between one another.
struct Range { uintptr_t from, to, pitch, width; };
Range range_of(const void* p, int64_t rows, int64_t cols, int64_t ld, int bytes) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p);
  if (!p || rows < 1 || cols < 1) return Range{a, a, 0, 0};
  return Range{a, a + (uintptr_t)(((rows - 1) * ld + cols) * bytes), (uintptr_t)(ld * bytes), (uintptr_t)(cols * bytes)};
}
bool overlap(const Range& a, const Range& b) {
  if (!(a.from < b.to && b.from < a.to)) return false;
  if (a.from == a.to || b.from == b.to) return false;
  if (a.pitch != b.pitch) return true;
  const uintptr_t P = a.pitch, apart = b.from >= a.from ? (b.from - a.from) % P : (P - (a.from - b.from) % P) % P;      // of b's rows behind a's
  return apart < a.width || apart + b.width > P;
}

int sm_count() {
  int dev = 0, sms = 148;
  if (cudaGetDevice(&dev) == cudaSuccess) cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  return sms;
}
// Dynamic shared memory of a kernel, asked for once a device
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

// ---- activations in 8 bits ------------------------------------------------------------------------------------------------
template <int T>
cudaError_t ckpt_read(const CkptArgs& a, sim_act act, unsigned grid, cudaStream_t st) {
  switch (act) {
    case SIM_ACT_RELU: ckpt_read_kernel<T, ACT_RELU><<<grid, 256, 0, st>>>(a); break;
    case SIM_ACT_GELU: ckpt_read_kernel<T, ACT_GELU><<<grid, 256, 0, st>>>(a); break;
    case SIM_ACT_SILU: ckpt_read_kernel<T, ACT_SILU><<<grid, 256, 0, st>>>(a); break;
    default: ckpt_read_kernel<T, ACT_NONE><<<grid, 256, 0, st>>>(a);
  }
  return cudaGetLastError();
}
template <int T, int ACT, bool KEPT, bool VEC>
cudaError_t launch_act_backward(const CkptArgs& a, dim3 grid, cudaStream_t st) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(256, 1, 1);
  cfg.stream = st;
  cudaLaunchAttribute attr{};
  if (a.db && grid.y > 1) {
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = 1; attr.val.clusterDim.y = grid.y; attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
  }
  return cudaLaunchKernelEx(&cfg, act_backward_kernel<T, ACT, KEPT, VEC>, a);
}
template <int T, bool VEC>
cudaError_t act_backward_kept(const CkptArgs& a, sim_act act, dim3 grid, cudaStream_t st) {
  switch (act) {
    case SIM_ACT_RELU: return launch_act_backward<T, ACT_RELU, true, VEC>(a, grid, st);
    case SIM_ACT_GELU: return launch_act_backward<T, ACT_GELU, true, VEC>(a, grid, st);
    case SIM_ACT_SILU: return launch_act_backward<T, ACT_SILU, true, VEC>(a, grid, st);
    default: return launch_act_backward<T, ACT_NONE, true, VEC>(a, grid, st);
  }
}
template <int T>
cudaError_t act_backward(const CkptArgs& a, sim_act act, dim3 grid, cudaStream_t st) {
  if (a.codes) return a.vec ? act_backward_kept<T, true>(a, act, grid, st) : act_backward_kept<T, false>(a, act, grid, st);
  return a.vec ? launch_act_backward<T, ACT_NONE, false, true>(a, grid, st) : launch_act_backward<T, ACT_NONE, false, false>(a, grid, st);
}
// Blocks along the rows: one for every 32 rows begun, rounded up to a power of two (so that each has 17 rows or more) up to the eight of a cluster, where three or
// seven blocks ran slower than half as many; and from there no more than fill a B200's 148 multiprocessors a few times over (a constant: the workspace is asked
// for without a device)
int64_t sum_splits(int64_t rows, int64_t cols) {
  const int64_t strips = (cols + 255) / 256, most = (rows + 31) / 32, want = (8 * 148 + strips - 1) / strips;
  const int64_t s = most < want ? most : want;
  return s <= 1 ? 1 : s <= 2 ? 2 : s <= 4 ? 4 : s <= 8 ? 8 : s > 65535 ? 65535 : s;
}

// ---- products ----------------------------------------------------------------------------------------------------------------
// An operand as TMA reads it: [rows][cols] with rows on 16-byte boundaries, a box of 64 columns (128 bytes) x box_rows, 128-byte swizzle,
// zeros outside
bool make_map(CUtensorMap* map, const void* p, sim_dtype type, int64_t rows, int64_t cols, int64_t ld, uint32_t box_rows) {
  PFN_encodeTiled fn = tc_encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {rows > 1 ? (cuuint64_t)ld * 2 : ((cuuint64_t)cols * 2 + 15) / 16 * 16};
  const cuuint32_t box[2] = {64, box_rows}, one[2] = {1, 1};
  return fn(map, type == SIM_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, const_cast<void*>(p), dims, strides, box, one,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct Operand {
  const void* p;
  int64_t rows, cols, ld;      // as it lies in memory
  int64_t along;               // rows of c's side: what a tile counts
  int t;
  bool fits;                   // TMA can read it
  // of a copy: rows of more than a line of memory start on lines (2300 x 5000 x 900 with its rows on 16-byte
  // boundaries 37 us, on lines 23.4; 1531 x 2736 x 1001 16.8 and 15.2: a box's rows else take parts of two lines each)
  int64_t pitch() const { return cols <= 64 ? (cols + 7) / 8 * 8 : (cols + 63) / 64 * 64; }
  int64_t copy_bytes() const { return fits ? 0 : rows * pitch() * 2; }
};
Operand operand(const void* p, int64_t ld, int t, int64_t along, int64_t k) {
  Operand o{p, t ? k : along, t ? along : k, ld, along, t ? 1 : 0, true};
  o.fits = rows_aligned(p, o.rows, ld, SIM_BF16, 16);
  return o;
}
// Copies of the operands that do not fit, in one launch
cudaError_t repack(Operand& a, Operand& b, char* room, cudaStream_t st) {
  MmRepack r{};
  int64_t pieces = 0;
  Operand* const both[2] = {&a, &b};
  for (int i = 0; i < 2; ++i) {
    Operand& o = *both[i];
    if (o.fits) continue;
    MmRepack::One& one = r.of[r.n++];
    one.x = static_cast<const uint16_t*>(o.p); one.out = reinterpret_cast<uint16_t*>(room); one.rows = o.rows; one.cols = o.cols; one.ld = o.ld; one.pitch = o.pitch();
    pieces += o.rows * ((o.cols + 7) / 8);
    room += (o.copy_bytes() + 255) / 256 * 256;
    o.p = one.out;
    o.ld = one.pitch;
  }
  if (r.n == 0) return cudaSuccess;
  mm_repack_kernel<<<grid_for(pieces), 256, 0, st>>>(r);
  return cudaGetLastError();
}

// Launches a product; `copied`: behind copies of its operands, which it awaits itself
template <typename K>
cudaError_t launch_mm(K kern, dim3 grid, int threads, size_t smem, int cluster_x, int cluster_y, bool copied, const CUtensorMap& ma, const CUtensorMap& mb, const MmArgs& g, cudaStream_t st) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)threads, 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2] = {};
  unsigned n = 0;
  if (cluster_x * cluster_y > 1) {
    attr[n].id = cudaLaunchAttributeClusterDimension;
    attr[n].val.clusterDim.x = (unsigned)cluster_x; attr[n].val.clusterDim.y = (unsigned)cluster_y; attr[n].val.clusterDim.z = 1;
    ++n;
  }
  if (copied) {
    attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[n].val.programmaticStreamSerializationAllowed = 1;
    ++n;
  }
  cfg.attrs = attr;
  cfg.numAttrs = n;
  return cudaLaunchKernelEx(&cfg, kern, ma, mb, g);
}
template <int T>
cudaError_t launch_pair(const CUtensorMap& ma, const CUtensorMap& mb, const MmArgs& g, int sms, bool copied, cudaStream_t st) {
  static std::atomic<unsigned long long> done{0};
  cudaError_t e = allow_smem(mm_pair_kernel<T>, MMP_SMEM, done);
  if (e != cudaSuccess) return e;
  const long long tiles = (long long)g.tiles_a * g.tiles_b, pairs = sms / 2;
  return launch_mm(mm_pair_kernel<T>, dim3((unsigned)(2 * (tiles < pairs ? tiles : pairs)), 1, 1), MMP_THREADS, MMP_SMEM, 1, 1, copied, ma, mb, g, st);    // in clusters of two, as declared
}
template <int BN, int T, bool SWAP, bool SPLIT>
cudaError_t launch_tile(const CUtensorMap& ma, const CUtensorMap& mb, const MmArgs& g, int split, bool copied, cudaStream_t st) {
  auto kern = mm_tile_kernel<BN, T, SWAP, SPLIT>;
  static_assert(mm_part_bytes(BN, SWAP) <= (SWAP ? MM_RING_NARROW : MM_OFF_PATCH), "the sums and the patches lie in the ring's bytes");
  static std::atomic<unsigned long long> done{0};
  cudaError_t e = allow_smem(kern, MM_RING_WIDE + 1024, done);
  if (e != cudaSuccess) return e;
  const int ring = SWAP ? g.stages * g.stage_bytes : g.stages * g.stage_bytes > MM_RING ? MM_RING_WIDE : MM_RING;
  return launch_mm(kern, dim3((unsigned)(g.tiles_a * g.tiles_b), (unsigned)split, 1), MM_THREADS, (size_t)ring + 1024, 1, split, copied, ma, mb, g, st);
}
template <int BN, int T, bool SWAP>
cudaError_t launch_split(const CUtensorMap& ma, const CUtensorMap& mb, const MmArgs& g, int split, bool copied, cudaStream_t st) {
  return split > 1 ? launch_tile<BN, T, SWAP, true>(ma, mb, g, split, copied, st) : launch_tile<BN, T, SWAP, false>(ma, mb, g, split, copied, st);
}
template <int T>
cudaError_t launch_product(bool pair, bool swap, int bn, const CUtensorMap& ma, const CUtensorMap& mb, const MmArgs& g, int split, int sms, bool copied, cudaStream_t st) {
  if (pair) return launch_pair<T>(ma, mb, g, sms, copied, st);
  if (swap) return bn == 16 ? launch_split<16, T, true>(ma, mb, g, split, copied, st) : bn == 32 ? launch_split<32, T, true>(ma, mb, g, split, copied, st) : launch_split<64, T, true>(ma, mb, g, split, copied, st);
  return bn == 32 ? launch_split<32, T, false>(ma, mb, g, split, copied, st) : bn == 64 ? launch_split<64, T, false>(ma, mb, g, split, copied, st) : launch_split<128, T, false>(ma, mb, g, split, copied, st);
}

const char* product_refusal(const sim_product* p) {
  const int64_t top = (int64_t)1 << 30;
  if (!p) return "sim_matmul: no product";
  if (p->M < 0 || p->N < 0 || p->K < 0 || p->M > top || p->N > top || p->K > top) return "sim_matmul: M, N and K must be in [0, 2^30]";
  if (p->type != SIM_BF16 && p->type != SIM_F16) return "sim_matmul: the operands are SIM_BF16 or SIM_F16";
  if (p->c_type != SIM_F32 && p->c_type != p->type) return "sim_matmul: the result is SIM_F32 or of the operands' type";
  if (p->bias && p->bias_type != SIM_F32 && p->bias_type != p->type) return "sim_matmul: bias is SIM_F32 or of the operands' type";
  if (!known_act(p->act)) return "sim_matmul: unknown activation";
  if (!p->z_codes != !p->z_scales) return "sim_matmul: codes and scales of z go together";
  if (p->act_grad && (!p->z_codes || p->bias)) return "sim_matmul: act_grad takes z and no bias";
  if (p->M == 0 || p->N == 0) return nullptr;
  if (p->K > 0 && (!p->a || !p->b || !aligned(p->a, 2) || !aligned(p->b, 2))) return "sim_matmul: operands (aligned to their type) are required";
  if (p->K > 0 && (bad_matrix(p->a_t ? p->K : p->M, p->a_t ? p->M : p->K, p->lda) || bad_matrix(p->b_t ? p->K : p->N, p->b_t ? p->N : p->K, p->ldb)))
    return "sim_matmul: lda and ldb must be at least the rows' lengths";
  if (!p->c || !aligned(p->c, elem_bytes(p->c_type)) || bad_matrix(p->M, p->N, p->ldc)) return "sim_matmul: c (aligned to its type) with ldc of at least N is required";
  if (p->residual && (!aligned(p->residual, elem_bytes(p->c_type)) || bad_matrix(p->M, p->N, p->ldr))) return "sim_matmul: the residual is of c's type, with ldr of at least N";
  if (p->bias && !aligned(p->bias, elem_bytes(p->bias_type))) return "sim_matmul: bias must be aligned to its type";
  if (p->z_codes && !aligned(p->z_codes, 16)) return "sim_matmul: z's codes must be 16-byte aligned";
  const Range c = range_of(p->c, p->M, p->N, p->ldc, elem_bytes(p->c_type));
  const Range zc = range_of(p->z_codes, p->M, ckpt_pitch(p->N), ckpt_pitch(p->N), 1), zs = range_of(p->z_scales, p->M, ckpt_pitch(p->N) / 32, ckpt_pitch(p->N) / 32, 1);
  const Range in[4] = {range_of(p->a, p->a_t ? p->K : p->M, p->a_t ? p->M : p->K, p->lda, 2), range_of(p->b, p->b_t ? p->K : p->N, p->b_t ? p->N : p->K, p->ldb, 2),
                       range_of(p->bias, 1, p->N, p->N, p->bias ? elem_bytes(p->bias_type) : 1), range_of(p->residual, p->M, p->N, p->ldr, elem_bytes(p->c_type))};
  for (int i = 0; i < 4; ++i) {
    const bool in_place = i == 3 && p->residual == p->c && p->ldr == p->ldc;
    if (overlap(c, in[i]) && !in_place) return "sim_matmul: c overlaps an operand (the residual may be c itself, with the same rows)";
    if (!p->act_grad && (overlap(zc, in[i]) || overlap(zs, in[i]))) return "sim_matmul: z overlaps an operand";
  }
  if (overlap(c, zc) || overlap(c, zs) || overlap(zc, zs)) return "sim_matmul: c and z overlap";
  return nullptr;
}

// Which kernel, which of the two is the instruction's 128-row operand, how wide the other's tile is, and how many blocks share a tile along k.
struct Plan { bool pair, swap; int bn, split; };
Plan plan_of(int64_t M, int64_t N, int64_t K, int sms) {
  Plan q{};
  q.swap = M <= 64 && M <= N;
  const int64_t ra = q.swap ? N : M, rb = q.swap ? M : N;
  const int kb = (int)((K + 63) / 64);
  // Pairs of multiprocessors where tiles of 128 x 128 would take turns (1008 x 1531 x 2736, 176 such tiles: 13.9 us against 18.1; 2048 x 2048 x 1200, 160:
  // 16.1 against 16.0; 1536 x 8192 x 1664, 156: 42.7 against 44.1; 1531 x 1008 x 2736, 264: 11.8 against 13.8; 4000 x 64 x 4000, 1024: 15.0 against 15.9; 3000 x
  // 128 x 3000, 576: 11.5 against 12.2).  The count of tiles alone is too coarse where k is short: 1800 x 64 x 1400, 165 tiles, 7.5 us against 7.0; 1800 x 512 x
  // 1400 9.7 against 9.4; 1800 x 128 x 2500, 300 tiles, 80 of the pairs' 256 x 256 in two turns, 14.6 against 10.9.  Where each tile has a multiprocessor, not
  // (640 x 8192 x 3000, 120 tiles: 43 against 33; 300 x 4096 x 4096, 96: 24.6 against 18.5; 700 x 1024 x 3000, 144: 12.1 against 8.9)
  q.pair = kb > 0 && ra > 128 && rb > 128 && (ra + 127) / 128 * ((rb + 127) / 128) > sms;
  q.split = 1;
  if (q.pair) return q;
  // Else the time of each tile width and split, estimated (us).  64 elements of k cost a block 0.25 (few rows, whose weights come from memory: 0.3), more
  // blocks than multiprocessors take turns, the tail costs 0.6 for each 64 columns, meeting in distributed shared memory what is listed.
  // (512 x 2048 x 2048: 13.5, 11.8 and 16 us for 1, 2 and 4 blocks a tile of 128 x 128, 12.1 in tiles of 128 x 64; 2048 x 1024 x 512: 9.2, and 7.9
  // in tiles of 128 x 64; 2000 x 2000 x 704: 13.5, and 16.4; 16 x 4096 x 4096: 24.5, 16.7, 12.6, and 13.6 for 8.)
  const double meet[4] = {0.0, q.swap ? 1.5 : 2.5, q.swap ? 2.5 : 4.5, q.swap ? 4.5 : 9.0}, step = q.swap ? 0.3 : 0.25;
  const int widest = q.swap ? (rb <= 16 ? 16 : rb <= 32 ? 32 : 64) : rb <= 32 ? 32 : rb <= 64 ? 64 : 128;
  double best = 0.0;
  for (int bn = widest; bn >= (q.swap ? widest : 32); bn /= 2) {
    const double tiles = (double)((ra + 127) / 128) * (double)((rb + bn - 1) / bn);
    // (few rows, a tile for each multiprocessor: memory is busy without a split; 1 x 1024 x 50000 in four parts 37.3 us, whole 22.3)
    const int most = q.swap && tiles >= sms ? 1 : 8;
    for (int i = 0, split = 1; split <= most && (split == 1 || split <= kb); ++i, split *= 2) {
      const double t = std::ceil(tiles * split / (q.swap ? 1.3 * sms : sms)) * (((kb + split - 1) / split) * step + (q.swap ? 0.0 : bn / 64 * 0.6)) + meet[i];
      if (q.bn == 0 || t < best) { best = t; q.split = split; q.bn = bn; }
    }
  }
  return q;
}

}  // namespace

extern "C" {

int64_t sim_ckpt_codes_bytes(int64_t rows, int64_t cols) { return rows < 1 || cols < 1 || bad_matrix(rows, cols, cols) ? 0 : rows * ckpt_pitch(cols); }
int64_t sim_ckpt_scales_bytes(int64_t rows, int64_t cols) { return rows < 1 || cols < 1 || bad_matrix(rows, cols, cols) ? 0 : rows * (ckpt_pitch(cols) / 32); }

sim_status sim_ckpt_write(const void* x, sim_dtype type, int64_t rows, int64_t cols, int64_t ld, uint8_t* codes, uint8_t* scales, void* cuda_stream) {
  if (!plain_type(type)) return bad("sim_ckpt_write: type must be SIM_F32, SIM_BF16 or SIM_F16");
  if (bad_matrix(rows, cols, ld)) return bad("sim_ckpt_write: rows and cols must be in [0, 2^31], ld at least cols");
  if (rows == 0 || cols == 0) return SIM_OK;
  if (!x || !aligned(x, elem_bytes(type)) || !codes || !scales || !aligned(codes, 16)) return bad("sim_ckpt_write: x (aligned to its type), codes (16-byte aligned) and scales are required");
  const Range in = range_of(x, rows, cols, ld, elem_bytes(type)), c = range_of(codes, rows, ckpt_pitch(cols), ckpt_pitch(cols), 1), s = range_of(scales, rows, ckpt_pitch(cols) / 32, ckpt_pitch(cols) / 32, 1);
  if (overlap(in, c) || overlap(in, s) || overlap(c, s)) return bad("sim_ckpt_write: the buffers overlap");
  CkptArgs a{};
  a.x = x; a.rows = rows; a.cols = cols; a.ld = ld; a.codes = codes; a.scales = scales;
  a.vec = rows_aligned(x, rows, ld, type, 16);
  const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const unsigned grid = grid_for(rows * ((cols + 31) / 32) * (a.vec ? 1 : 32));
  if (type == SIM_F32) ckpt_write_kernel<T_F32><<<grid, 256, 0, st>>>(a);
  else if (type == SIM_BF16) ckpt_write_kernel<T_BF16><<<grid, 256, 0, st>>>(a);
  else ckpt_write_kernel<T_F16><<<grid, 256, 0, st>>>(a);
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? SIM_OK : cuda_failed("sim_ckpt_write", e);
}

sim_status sim_ckpt_read(const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t cols, sim_act act, sim_dtype type, void* out, int64_t ld, void* cuda_stream) {
  if (!plain_type(type)) return bad("sim_ckpt_read: type must be SIM_F32, SIM_BF16 or SIM_F16");
  if (!known_act(act)) return bad("sim_ckpt_read: unknown activation");
  if (bad_matrix(rows, cols, ld)) return bad("sim_ckpt_read: rows and cols must be in [0, 2^31], ld at least cols");
  if (rows == 0 || cols == 0) return SIM_OK;
  if (!out || !aligned(out, elem_bytes(type)) || !codes || !scales || !aligned(codes, 16)) return bad("sim_ckpt_read: codes (16-byte aligned), scales and out (aligned to its type) are required");
  const Range o = range_of(out, rows, cols, ld, elem_bytes(type)), c = range_of(codes, rows, ckpt_pitch(cols), ckpt_pitch(cols), 1), s = range_of(scales, rows, ckpt_pitch(cols) / 32, ckpt_pitch(cols) / 32, 1);
  if (overlap(o, c) || overlap(o, s)) return bad("sim_ckpt_read: the buffers overlap");
  CkptArgs a{};
  a.rows = rows; a.cols = cols; a.codes = const_cast<uint8_t*>(codes); a.scales = const_cast<uint8_t*>(scales); a.out = out; a.ldo = ld;
  a.vec = rows_aligned(out, rows, ld, type, 16);
  const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const unsigned grid = grid_for(rows * ((cols + 31) / 32) * (a.vec ? 1 : 32));
  const cudaError_t e = type == SIM_F32 ? ckpt_read<T_F32>(a, act, grid, st) : type == SIM_BF16 ? ckpt_read<T_BF16>(a, act, grid, st) : ckpt_read<T_F16>(a, act, grid, st);
  return e == cudaSuccess ? SIM_OK : cuda_failed("sim_ckpt_read", e);
}

int64_t sim_act_backward_workspace(int64_t rows, int64_t cols) { return rows < 1 || cols < 1 || bad_matrix(rows, cols, cols) || sum_splits(rows, cols) <= 8 ? 0 : sum_splits(rows, cols) * cols * 4; }

sim_status sim_act_backward(const void* dy, sim_dtype type, int64_t rows, int64_t cols, int64_t ld, const uint8_t* codes, const uint8_t* scales, sim_act act, void* dz, int64_t lddz,
                            void* db, sim_dtype db_type, void* workspace, int64_t workspace_bytes, void* cuda_stream) {
  if (!plain_type(type) || (db && !plain_type(db_type))) return bad("sim_act_backward: types must be SIM_F32, SIM_BF16 or SIM_F16");
  if (!known_act(act)) return bad("sim_act_backward: unknown activation");
  if (bad_matrix(rows, cols, ld) || (dz && bad_matrix(rows, cols, lddz))) return bad("sim_act_backward: rows and cols must be in [0, 2^31], ld and lddz at least cols");
  if (!codes != !scales || (codes && !dz)) return bad("sim_act_backward: codes and scales go together, and with dz");
  if (!dz && !db) return bad("sim_act_backward: nothing to compute");
  if (cols == 0) return SIM_OK;
  if (db && !aligned(db, elem_bytes(db_type))) return bad("sim_act_backward: db must be aligned to its type");
  const int64_t need = db ? sim_act_backward_workspace(rows, cols) : 0;
  if (need > 0 && (!workspace || !aligned(workspace, 4) || workspace_bytes < need))
    return bad("sim_act_backward: sums need a workspace of sim_act_backward_workspace bytes");
  const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  cudaError_t e = cudaSuccess;
  const int eb = elem_bytes(type);
  int64_t splits = 0;
  if (rows > 0) {
    if (!dy || !aligned(dy, eb) || !aligned(codes, 16) || !aligned(dz, eb)) return bad("sim_act_backward: dy and dz (aligned to their type) and codes (16-byte aligned) are required");
    const int64_t pitch = ckpt_pitch(cols);
    const Range in[3] = {range_of(dy, rows, cols, ld, eb), range_of(codes, rows, pitch, pitch, 1), range_of(scales, rows, pitch / 32, pitch / 32, 1)};
    const Range out[3] = {range_of(dz, rows, cols, lddz, eb), range_of(db, 1, cols, cols, db ? elem_bytes(db_type) : 1), range_of(need > 0 ? workspace : nullptr, 1, need, need, 1)};
    for (int i = 0; i < 3; ++i)
      for (int o = 0; o < 3; ++o)
        if (overlap(in[i], out[o]) && !(i == 0 && o == 0 && dy == dz && ld == lddz)) return bad("sim_act_backward: the buffers overlap (dz may be dy itself, with the same rows)");
    if (overlap(out[0], out[1]) || overlap(out[0], out[2]) || overlap(out[1], out[2])) return bad("sim_act_backward: the buffers overlap");
    splits = sum_splits(rows, cols);
    CkptArgs a{};
    a.x = dy; a.rows = rows; a.cols = cols; a.ld = ld; a.codes = const_cast<uint8_t*>(codes); a.scales = const_cast<uint8_t*>(scales); a.out = dz; a.ldo = lddz;
    a.vec = rows_aligned(dy, rows, ld, type, 16) && (!dz || rows_aligned(dz, rows, lddz, type, 16));
    a.partial = need > 0 ? static_cast<float*>(workspace) : nullptr;
    a.db = need > 0 ? nullptr : db; a.db_type = db_type;
    a.split_rows = (int)((rows + splits - 1) / splits);
    const dim3 grid((unsigned)((cols + 255) / 256), (unsigned)splits, 1);
    e = type == SIM_F32 ? act_backward<T_F32>(a, act, grid, st) : type == SIM_BF16 ? act_backward<T_BF16>(a, act, grid, st) : act_backward<T_F16>(a, act, grid, st);
    if (e != cudaSuccess) return cuda_failed("sim_act_backward", e);
  }
  if (db && (need > 0 || rows == 0)) {
    column_sum_finish_kernel<<<(unsigned)((cols + 31) / 32), 256, 0, st>>>(static_cast<const float*>(workspace), (int)splits, cols, db, db_type);
    e = cudaGetLastError();
  }
  return e == cudaSuccess ? SIM_OK : cuda_failed("sim_act_backward", e);
}

int64_t sim_matmul_workspace(const sim_product* p) {
  if (product_refusal(p) || p->M == 0 || p->N == 0 || p->K == 0) return 0;
  const Operand a = operand(p->a, p->lda, p->a_t, p->M, p->K), b = operand(p->b, p->ldb, p->b_t, p->N, p->K);
  return (a.copy_bytes() + 255) / 256 * 256 + (b.copy_bytes() + 255) / 256 * 256;
}

sim_status sim_matmul(const sim_product* p, void* workspace, int64_t workspace_bytes, void* cuda_stream) {
  if (const char* why = product_refusal(p)) return bad(why);
  const int64_t M = p->M, N = p->N, K = p->K;
  if (M == 0 || N == 0) return SIM_OK;
  const int64_t need = sim_matmul_workspace(p);
  if (need > 0) {
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < need) return bad("sim_matmul: operands whose rows do not start on 16-byte boundaries need a workspace of sim_matmul_workspace bytes, 256-byte aligned");
    const Range w = range_of(workspace, 1, need, need, 1);
    if (overlap(w, range_of(p->c, M, N, p->ldc, elem_bytes(p->c_type))) || overlap(w, range_of(p->a, p->a_t ? K : M, p->a_t ? M : K, p->lda, 2)) ||
        overlap(w, range_of(p->b, p->b_t ? K : N, p->b_t ? N : K, p->ldb, 2)) || overlap(w, range_of(p->residual, M, N, p->ldr, elem_bytes(p->c_type))) ||
        overlap(w, range_of(p->bias, 1, N, N, p->bias ? elem_bytes(p->bias_type) : 1)) || overlap(w, range_of(p->z_codes, M, ckpt_pitch(N), ckpt_pitch(N), 1)) ||
        overlap(w, range_of(p->z_scales, M, ckpt_pitch(N) / 32, ckpt_pitch(N) / 32, 1)))
      return bad("sim_matmul: the workspace overlaps another buffer");
  }
  const int sms = sm_count();
  const Plan q = plan_of(M, N, K, sms);
  Operand a = operand(p->a, p->lda, p->a_t, M, K), b = operand(p->b, p->ldb, p->b_t, N, K);
  const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  cudaError_t e = need > 0 ? repack(a, b, static_cast<char*>(workspace), st) : cudaSuccess;
  if (e != cudaSuccess) return cuda_failed("sim_matmul", e);
  if (q.swap) { const Operand t = a; a = b; b = t; }

  MmArgs g{};
  g.M = M; g.N = N;
  g.kb = (int)((K + 63) / 64);
  g.kb_split = (g.kb + q.split - 1) / q.split;
  const int split = g.kb_split > 0 ? (g.kb + g.kb_split - 1) / g.kb_split : 1;        // every block of a cluster has a part
  const int tile_a = q.pair ? 256 : 128, tile_b = q.pair ? 256 : q.bn;
  const int64_t ta = (a.along + tile_a - 1) / tile_a, tb = (b.along + tile_b - 1) / tile_b;
  if (ta * tb > (int64_t)1 << 30) return bad("sim_matmul: the result has too many tiles");
  g.tiles_a = (int)ta; g.tiles_b = (int)tb;
  g.a_t = a.t; g.b_t = b.t;
  g.stage_bytes = MM_A_BYTES + (b.t ? (q.bn < 64 ? 64 : q.bn) : q.bn) * 128;
  // One block to a multiprocessor: its ring may take all shared memory (2048 x 1024 x 512: 10.4 -> 9.2 us).  Few rows and more blocks than two to a
  // multiprocessor hold: rings for three (1 x 4096 x 50000, 391 blocks: 102 -> 71 us with the tiles whole).
  const int64_t blocks = ta * tb * split;
  const int ring = blocks <= sms ? MM_RING_WIDE : q.swap && blocks > 2 * sms ? MM_RING_NARROW : MM_RING;
  g.stages = ring / g.stage_bytes;
  if (g.stages > MM_MAX_STAGES) g.stages = MM_MAX_STAGES;
  g.idesc = mm_idesc(q.pair ? 256 : 128, q.pair ? 256 : q.bn, p->type == SIM_BF16, a.t, b.t);
  g.act = p->act; g.grad = p->act_grad ? 1 : 0; g.bias = p->bias; g.bias_type = p->bias_type;
  g.z_codes = p->z_codes; g.z_scales = p->z_scales; g.res = p->residual; g.ldr = p->ldr; g.c = p->c; g.ldc = p->ldc;
  g.vec_c = rows_aligned(p->c, M, p->ldc, p->c_type, 32) ? 2 : rows_aligned(p->c, M, p->ldc, p->c_type, 16) ? 1 : 0;
  g.vec_r = p->residual && rows_aligned(p->residual, M, p->ldr, p->c_type, 16);
  CUtensorMap ma{}, mb{};
  if (K > 0 && (!make_map(&ma, a.p, p->type, a.rows, a.cols, a.ld, a.t ? 64 : 128) ||
                !make_map(&mb, b.p, p->type, b.rows, b.cols, b.ld, b.t ? 64 : q.pair ? 128 : (uint32_t)q.bn)))
    return record_error(SIM_ERR_CUDA, "sim_matmul: the driver refused a tensor map");
  e = p->c_type == SIM_F32 ? launch_product<T_F32>(q.pair, q.swap, q.bn, ma, mb, g, split, sms, need > 0, st)
      : p->c_type == SIM_BF16 ? launch_product<T_BF16>(q.pair, q.swap, q.bn, ma, mb, g, split, sms, need > 0, st) : launch_product<T_F16>(q.pair, q.swap, q.bn, ma, mb, g, split, sms, need > 0, st);
  return e == cudaSuccess ? SIM_OK : cuda_failed("sim_matmul", e);
}

}  // extern "C"

// ---- log probabilities -----------------------------------------------------------------------------------------------------------
namespace {

template <int T, int G, int E>
cudaError_t launch_short(const LogpArgs& a, cudaStream_t st) {
  logp_short_kernel<T, G, E><<<(unsigned)((a.rows + 128 / G - 1) / (128 / G)), 128, 0, st>>>(a);
  return cudaGetLastError();
}
template <int T, int NT>
cudaError_t launch_rows(const LogpArgs& a, int slices, int slice_len, cudaStream_t st) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(a.rows * slices), 1, 1);
  cfg.blockDim = dim3(NT, 1, 1);
  cfg.stream = st;
  cudaLaunchAttribute attr{};
  if (slices > 1) {
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = (unsigned)slices; attr.val.clusterDim.y = 1; attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
  }
  return cudaLaunchKernelEx(&cfg, logp_row_kernel<T, NT>, a, slices, slice_len);
}
template <int T>
cudaError_t log_probs(const LogpArgs& a, cudaStream_t st) {
  if (a.vocab <= 16) return launch_short<T, 1, 16>(a, st);
  if (a.vocab <= 128) return launch_short<T, 8, 16>(a, st);
  if (a.vocab <= 1024) return launch_short<T, 32, 32>(a, st);
  if (a.vocab <= 8192) return launch_rows<T, 128>(a, 1, (int)a.vocab, st);
  // few rows: a cluster of blocks for each, as long as a thread of a slice still has a group of eight or so
  const int64_t sms = sm_count();
  int slices = 1;
  while (slices < 8 && a.rows * slices * 2 <= 2 * sms && a.vocab >= slices * 2 * 4096) slices *= 2;
  const int len = (int)(((a.vocab + slices - 1) / slices + 7) / 8 * 8);
  // Many rows: blocks of 256 threads, six to a multiprocessor, whose phases mix (4096 x 131072 bf16 with eight alternatives: 220 us against 243 in blocks of
  // 512; with the gradient, rows of 20, 100 and 256 KB: 245, 361 and 541 us against 341, 366 and 525).  Few: a thread's share is what a row takes.
  return slices == 1 ? launch_rows<T, 256>(a, slices, len, st) : launch_rows<T, 512>(a, slices, len, st);
}

}  // namespace

extern "C" sim_status sim_log_probs(const void* logits, sim_dtype type, int64_t rows, int64_t vocab, int64_t ld, const void* tokens, int32_t token_bytes, float temperature, int32_t top,
                                    float* logp, float* entropy, float* lse, int32_t* top_ids, float* top_logp, const float* d_logp, const float* d_entropy, void* d_logits, int64_t ldd,
                                    void* cuda_stream) {
  if (!plain_type(type)) return bad("sim_log_probs: type must be SIM_F32, SIM_BF16 or SIM_F16");
  if (rows < 0 || rows > (int64_t)1 << 27 || vocab < 1 || vocab > (int64_t)1 << 30) return bad("sim_log_probs: rows must be in [0, 2^27], vocab in [1, 2^30]");
  if (bad_matrix(rows, vocab, ld) || (d_logits && bad_matrix(rows, vocab, ldd))) return bad("sim_log_probs: ld and ldd must be at least vocab");
  if (!(temperature >= 1e-3f && temperature <= 1e3f)) return bad("sim_log_probs: temperature must be in [0.001, 1000]");
  if (top < 0 || top > LP_MAX_TOP || top > vocab) return bad("sim_log_probs: top must be in [0, 32] and at most vocab");
  if (rows == 0) return SIM_OK;
  if (tokens && token_bytes != 4 && token_bytes != 8) return bad("sim_log_probs: tokens have 4 or 8 bytes");
  if (top > 0 && !top_ids && !top_logp) return bad("sim_log_probs: top needs top_ids or top_logp");
  if (top == 0 && (top_ids || top_logp)) return bad("sim_log_probs: top_ids and top_logp need top");
  if (!tokens && (logp || d_logp)) return bad("sim_log_probs: logp and d_logp need tokens");
  if (!d_logits && (d_logp || d_entropy)) return bad("sim_log_probs: d_logp and d_entropy need d_logits");
  if (!logits || !aligned(logits, elem_bytes(type)) || !aligned(d_logits, elem_bytes(type)) || (tokens && !aligned(tokens, token_bytes)))
    return bad("sim_log_probs: logits, d_logits and tokens must be there and aligned to their types");
  for (const void* p : {(const void*)logp, (const void*)entropy, (const void*)lse, (const void*)top_ids, (const void*)top_logp, (const void*)d_logp, (const void*)d_entropy})
    if (!aligned(p, 4)) return bad("sim_log_probs: results and derivatives must be 4-byte aligned");
  const int eb = elem_bytes(type);
  const Range out[6] = {range_of(d_logits, rows, vocab, ldd, eb), range_of(logp, 1, rows, rows, 4), range_of(entropy, 1, rows, rows, 4), range_of(lse, 1, rows, rows, 4),
                        range_of(top_ids, rows, top, top, 4), range_of(top_logp, rows, top, top, 4)};
  const Range in[4] = {range_of(logits, rows, vocab, ld, eb), range_of(tokens, 1, rows, rows, token_bytes), range_of(d_logp, 1, rows, rows, 4), range_of(d_entropy, 1, rows, rows, 4)};
  for (int o = 0; o < 6; ++o) {
    for (int i = 0; i < 4; ++i)
      if (overlap(out[o], in[i]) && !(o == 0 && i == 0 && d_logits == logits && ldd == ld)) return bad("sim_log_probs: the buffers overlap (d_logits may be logits itself, with the same rows)");
    for (int i = 0; i < o; ++i)
      if (overlap(out[o], out[i])) return bad("sim_log_probs: the results overlap");
  }
  LogpArgs a{};
  a.x = logits; a.rows = rows; a.vocab = vocab; a.ld = ld; a.tokens = tokens; a.token64 = token_bytes == 8;
  a.c = (float)(1.4426950408889634 / (double)temperature); a.c4 = 0.25f * a.c; a.inv_t = (float)(1.0 / (double)temperature);
  a.top = top; a.logp = logp; a.entropy = entropy; a.lse = lse; a.top_ids = top_ids; a.top_logp = top_logp;
  a.d_logp = d_logp; a.d_entropy = d_entropy; a.out = d_logits; a.ldo = ldd;
  const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const cudaError_t e = type == SIM_F32 ? log_probs<T_F32>(a, st) : type == SIM_BF16 ? log_probs<T_BF16>(a, st) : log_probs<T_F16>(a, st);
  return e == cudaSuccess ? SIM_OK : cuda_failed("sim_log_probs", e);
}
