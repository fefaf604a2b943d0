// C entry points of the AdamW step over a list of tensors (adamw_kernel.cuh): argument checks, tables, launches.
#include <algorithm>
#include <cmath>
#include <cstdio>
#include <new>
#include <vector>

#include "adamw_kernel.cuh"
#include "error.cuh"

using namespace ssim;

namespace {

struct Group { int pt, gt; uint32_t first, count, grid[2]; };   // chunks of tensors with the same parameter and gradient types

struct DeviceGuard {   // the handle's device for the duration of a call
  int before = -1;
  cudaError_t err;
  explicit DeviceGuard(int device) {
    err = cudaGetDevice(&before);
    if (err == cudaSuccess && before != device) err = cudaSetDevice(device);
  }
  ~DeviceGuard() { if (before >= 0) cudaSetDevice(before); }
};

using Kernel = void (*)(AdamwArgs);

template <int PT, int BITS, bool MULTI>
Kernel pick_g(int gt) {
  switch (gt) {
    case T_F32: return adamw_kernel<PT, T_F32, BITS, MULTI>;
    case T_BF16: return adamw_kernel<PT, T_BF16, BITS, MULTI>;
    case T_F16: return adamw_kernel<PT, T_F16, BITS, MULTI>;
    default: return adamw_kernel<PT, T_MXFP4, BITS, MULTI>;
  }
}
template <bool MULTI>
Kernel pick_p(int bits, int pt, int gt) {
  if (bits == 32) return pt == T_F32 ? pick_g<T_F32, 32, MULTI>(gt) : pick_g<T_BF16, 32, MULTI>(gt);
  return pt == T_F32 ? pick_g<T_F32, 8, MULTI>(gt) : pick_g<T_BF16, 8, MULTI>(gt);
}
Kernel pick(int bits, int pt, int gt, int K) { return K > 1 ? pick_p<true>(bits, pt, gt) : pick_p<false>(bits, pt, gt); }

bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

}  // namespace

struct sim_adamw {
  int device = 0, n_tensors = 0, n_grads = 0, bits = 32;
  double beta1 = 0, beta2 = 0;
  float eps = 0;
  uint64_t seed = 0;
  std::vector<Group> groups;
  void* tables = nullptr;      // one allocation: tensors, chunks, gradient pointers, their scale pointers
  const AdamwTensor* tensors = nullptr;
  const AdamwChunk* chunks = nullptr;
  const void* const* g = nullptr;
  const uint8_t* const* g_scale = nullptr;
};

namespace {

sim_status bad(const char* fmt, long long i) {
  char msg[200];
  std::snprintf(msg, sizeof msg, fmt, i);
  return record_error(SIM_ERR_ARG, msg);
}
sim_status cuda_failed(const char* where, cudaError_t e) {
  char msg[200];
  std::snprintf(msg, sizeof msg, "%s: %s", where, cudaGetErrorString(e));
  return record_error(e == cudaErrorMemoryAllocation ? SIM_ERR_ALLOC : SIM_ERR_CUDA, msg);
}

sim_status check_tensor(const sim_adamw_tensor& t, int i, int n_grads, int bits) {
  if (t.n < 0 || t.n > (int64_t)1 << 40) return bad("sim_adamw_create: tensor %lld: n must be in [0, 2^40]", i);
  if (t.p_type != SIM_F32 && t.p_type != SIM_BF16) return bad("sim_adamw_create: tensor %lld: parameters are SIM_F32 or SIM_BF16", i);
  if ((int)t.g_type < 0 || (int)t.g_type > (int)SIM_MXFP4) return bad("sim_adamw_create: tensor %lld: unknown gradient type", i);
  if (!(t.weight_decay >= 0.f) || std::isinf(t.weight_decay)) return bad("sim_adamw_create: tensor %lld: weight_decay must be finite and >= 0", i);
  if (t.shadow && t.p_type != SIM_F32) return bad("sim_adamw_create: tensor %lld: a bf16 copy is written beside fp32 parameters only", i);
  if (t.n == 0) return SIM_OK;
  const size_t pb = t.p_type == SIM_F32 ? 4 : 2, gb = t.g_type == SIM_F32 ? 4 : t.g_type == SIM_MXFP4 ? 1 : 2, sb = bits == 32 ? 4 : 1;
  if (!t.p || !t.m || !t.v || !t.g) return bad("sim_adamw_create: tensor %lld: p, g, m and v are required", i);
  if (bits == 8 && (!t.m_scale || !t.v_scale)) return bad("sim_adamw_create: tensor %lld: 8-bit states need m_scale and v_scale", i);
  if (t.g_type == SIM_MXFP4 && !t.g_scale) return bad("sim_adamw_create: tensor %lld: MXFP4 gradients need g_scale", i);
  if (!aligned(t.p, pb) || !aligned(t.m, sb) || !aligned(t.v, sb) || !aligned(t.shadow, 2))
    return bad("sim_adamw_create: tensor %lld: a pointer is not aligned to its element type", i);
  for (int l = 0; l < n_grads; ++l) {
    if (!t.g[l] || !aligned(t.g[l], gb)) return bad("sim_adamw_create: tensor %lld: a gradient pointer is NULL or not aligned to its type", i);
    if (t.g_type == SIM_MXFP4 && !t.g_scale[l]) return bad("sim_adamw_create: tensor %lld: a gradient's scale pointer is NULL", i);
  }
  return SIM_OK;
}

// A buffer that a step writes must not overlap any other buffer of the list: blocks run in any order.
bool overlaps(const sim_adamw_tensor* ts, int n_tensors, int n_grads, int bits) {
  struct Range { uintptr_t begin, end; bool written; };
  std::vector<Range> all;
  auto add = [&](const void* p, int64_t bytes, bool written) {
    if (p && bytes > 0) all.push_back(Range{reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + (uintptr_t)bytes, written});
  };
  for (int i = 0; i < n_tensors; ++i) {
    const sim_adamw_tensor& t = ts[i];
    if (t.n == 0) continue;
    const int64_t blocks = (t.n + 31) / 32, state = bits == 32 ? 4 * t.n : t.n;
    add(t.p, t.n * (t.p_type == SIM_F32 ? 4 : 2), true);
    add(t.m, state, true);
    add(t.v, state, true);
    if (bits == 8) { add(t.m_scale, blocks, true); add(t.v_scale, blocks, true); }
    add(t.shadow, 2 * t.n, true);
    for (int l = 0; l < n_grads; ++l) {
      add(t.g[l], t.g_type == SIM_MXFP4 ? (t.n + 1) / 2 : t.n * (t.g_type == SIM_F32 ? 4 : 2), false);
      if (t.g_type == SIM_MXFP4) add(t.g_scale[l], blocks, false);
    }
  }
  std::sort(all.begin(), all.end(), [](const Range& a, const Range& b) { return a.begin < b.begin; });
  uintptr_t end = 0, end_written = 0;
  for (const Range& r : all) {
    if (r.begin < (r.written ? end : end_written)) return true;
    end = std::max(end, r.end);
    if (r.written) end_written = std::max(end_written, r.end);
  }
  return false;
}

sim_status create(const sim_adamw_tensor* ts, int n_tensors, int n_grads, int bits, double beta1, double beta2, double eps, uint64_t seed,
                  sim_adamw** out) {
  if (!ts || n_tensors < 1) return record_error(SIM_ERR_ARG, "sim_adamw_create: at least one tensor is required");
  if (n_grads < 1 || n_grads > SIM_MAX_P) return record_error(SIM_ERR_ARG, "sim_adamw_create: n_grads must be in [1, SIM_MAX_P]");
  if (bits != 32 && bits != 8) return record_error(SIM_ERR_ARG, "sim_adamw_create: state_bits must be 32 or 8");
  if (!(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0)) return record_error(SIM_ERR_ARG, "sim_adamw_create: betas must be in [0, 1)");
  if (!adamw_eps_ok((float)eps)) return record_error(SIM_ERR_ARG, "sim_adamw_create: eps must be in [2^-126, 2^125]");
  long long total_chunks = 0;
  for (int i = 0; i < n_tensors; ++i) {
    const sim_status st = check_tensor(ts[i], i, n_grads, bits);
    if (st != SIM_OK) return st;
    total_chunks += (ts[i].n + ADAMW_CHUNK - 1) / ADAMW_CHUNK;
  }
  if (overlaps(ts, n_tensors, n_grads, bits)) return record_error(SIM_ERR_ARG, "sim_adamw_create: a buffer that the step writes overlaps another one");
  if (total_chunks >= (1ll << 31)) return record_error(SIM_ERR_ARG, "sim_adamw_create: more than 2^42 elements in all");

  std::vector<AdamwTensor> tensors((size_t)n_tensors);
  std::vector<AdamwChunk> chunks;
  chunks.reserve((size_t)total_chunks);
  std::vector<const void*> g((size_t)n_tensors * n_grads, nullptr);
  std::vector<const uint8_t*> gs((size_t)n_tensors * n_grads, nullptr);
  std::vector<Group> groups;
  for (int i = 0; i < n_tensors; ++i) {
    const sim_adamw_tensor& t = ts[i];
    const size_t sv = bits == 32 ? 16 : 8, gv = t.g_type == SIM_MXFP4 ? 4 : 16;
    bool vec = aligned(t.p, 16) && aligned(t.m, sv) && aligned(t.v, sv) && aligned(t.shadow, 16);
    for (int l = 0; l < n_grads && t.n > 0; ++l) {
      g[(size_t)l * n_tensors + i] = t.g[l];
      if (t.g_type == SIM_MXFP4) gs[(size_t)l * n_tensors + i] = t.g_scale[l];
      vec = vec && aligned(t.g[l], gv);
    }
    tensors[i] = AdamwTensor{t.p, t.m, t.v, t.m_scale, t.v_scale, static_cast<uint16_t*>(t.shadow), g[i], gs[i], t.n, t.weight_decay, vec ? 1 : 0};
  }
  for (int pt = 0; pt < 2; ++pt)
    for (int gt = 0; gt < 4; ++gt) {
      Group grp{pt, gt, (uint32_t)chunks.size(), 0, {0, 0}};
      for (int i = 0; i < n_tensors; ++i)
        if ((int)ts[i].p_type == pt && (int)ts[i].g_type == gt)
          for (long long c = 0; c < (ts[i].n + ADAMW_CHUNK - 1) / ADAMW_CHUNK; ++c) chunks.push_back(AdamwChunk{(uint32_t)i, (uint32_t)c});
      grp.count = (uint32_t)chunks.size() - grp.first;
      if (grp.count) groups.push_back(grp);
    }

  sim_adamw* h = new sim_adamw();
  h->n_tensors = n_tensors; h->n_grads = n_grads; h->bits = bits; h->beta1 = beta1; h->beta2 = beta2; h->eps = (float)eps; h->seed = seed;
  const size_t nb_t = tensors.size() * sizeof(AdamwTensor), nb_c = chunks.size() * sizeof(AdamwChunk), nb_g = g.size() * sizeof(void*);
  char* d = nullptr;
  cudaError_t e = cudaGetDevice(&h->device);
  int sms = 0;
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, h->device);
  for (Group& grp : groups)       // 8-bit states: as many blocks as the machine holds at once; 32-bit: one for each chunk
    for (int multi = 0; multi < 2; ++multi) {
      int per_sm = 0;
      if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, pick(bits, grp.pt, grp.gt, 1 + multi), ADAMW_THREADS, 0);
      const uint32_t full = (uint32_t)(per_sm > 0 ? per_sm : 1) * (uint32_t)sms;
      grp.grid[multi] = bits == 32 || grp.count < full ? grp.count : full;
    }
  h->groups.swap(groups);
  if (e == cudaSuccess) e = cudaMalloc(&h->tables, nb_t + nb_c + 2 * nb_g);
  if (e == cudaSuccess) {
    d = static_cast<char*>(h->tables);
    e = cudaMemcpy(d, tensors.data(), nb_t, cudaMemcpyHostToDevice);
  }
  if (e == cudaSuccess && nb_c) e = cudaMemcpy(d + nb_t, chunks.data(), nb_c, cudaMemcpyHostToDevice);
  if (e == cudaSuccess) e = cudaMemcpy(d + nb_t + nb_c, g.data(), nb_g, cudaMemcpyHostToDevice);
  if (e == cudaSuccess) e = cudaMemcpy(d + nb_t + nb_c + nb_g, gs.data(), nb_g, cudaMemcpyHostToDevice);
  if (e == cudaSuccess) e = cudaStreamSynchronize(cudaStreamLegacy);   // a copy from pageable memory may return before it has arrived; other streams do not wait for it
  if (e != cudaSuccess) {
    cudaFree(h->tables);
    delete h;
    cudaGetLastError();
    return cuda_failed("sim_adamw_create", e);
  }
  h->tensors = reinterpret_cast<const AdamwTensor*>(d);
  h->chunks = reinterpret_cast<const AdamwChunk*>(d + nb_t);
  h->g = reinterpret_cast<const void* const*>(d + nb_t + nb_c);
  h->g_scale = reinterpret_cast<const uint8_t* const*>(d + nb_t + nb_c + nb_g);
  *out = h;
  return SIM_OK;
}

sim_status step(const sim_adamw* h, int64_t t, const int64_t* t_dev, float lr, const float* lr_dev, float grad_scale, int K, void* stream) {
  if (!h) return record_error(SIM_ERR_ARG, "sim_adamw_step: the handle is NULL");
  if (K < 1 || K > h->n_grads) return record_error(SIM_ERR_ARG, "sim_adamw_step: K must be in [1, n_grads]");
  if (!std::isfinite(grad_scale)) return record_error(SIM_ERR_ARG, "sim_adamw_step: grad_scale must be finite");
  if (!t_dev && (t < 1 || t > 0xFFFFFFFFll)) return record_error(SIM_ERR_ARG, "sim_adamw_step: step must be in [1, 2^32)");
  if (!lr_dev && !(std::isfinite(lr) && lr >= 0.f)) return record_error(SIM_ERR_ARG, "sim_adamw_step: lr must be finite and >= 0");
  DeviceGuard guard(h->device);
  if (guard.err != cudaSuccess) return cuda_failed("sim_adamw_step", guard.err);
  AdamwArgs a{};
  a.tensors = h->tensors; a.g = h->g; a.g_scale = h->g_scale; a.n_tensors = h->n_tensors; a.K = K;
  a.beta1 = h->beta1; a.beta2 = h->beta2; a.mean = (double)grad_scale / K;
  a.coef = adamw_coef(h->beta1, h->beta2, h->eps, a.mean, lr, t_dev ? 1 : t);
  a.step32 = (uint32_t)t; a.lr_dev = lr_dev; a.step_dev = reinterpret_cast<const long long*>(t_dev); a.keys = philox_keys(h->seed);
  for (const Group& grp : h->groups) {
    a.chunks = h->chunks + grp.first;
    a.n_chunks = grp.count;
    pick(h->bits, grp.pt, grp.gt, K)<<<grp.grid[K > 1], ADAMW_THREADS, 0, static_cast<cudaStream_t>(stream)>>>(a);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return cuda_failed("sim_adamw_step", e);
  }
  return SIM_OK;
}

}  // namespace

extern "C" {

sim_status sim_adamw_create(const sim_adamw_tensor* tensors, int32_t n_tensors, int32_t n_grads, int32_t state_bits, double beta1,
                            double beta2, double eps, uint64_t seed, sim_adamw** out) {
  if (!out) return record_error(SIM_ERR_ARG, "sim_adamw_create: out is NULL");
  *out = nullptr;
  try {
    return create(tensors, n_tensors, n_grads, state_bits, beta1, beta2, eps, seed, out);
  } catch (const std::bad_alloc&) {
    return record_error(SIM_ERR_ALLOC, "sim_adamw_create: host allocation failed");
  }
}

sim_status sim_adamw_step(const sim_adamw* h, int64_t t, float lr, float grad_scale, int32_t K, void* cuda_stream) {
  return step(h, t, nullptr, lr, nullptr, grad_scale, K, cuda_stream);
}

sim_status sim_adamw_step_device(const sim_adamw* h, const int64_t* t, const float* lr, float grad_scale, int32_t K, void* cuda_stream) {
  if (!t || !lr) return record_error(SIM_ERR_ARG, "sim_adamw_step_device: t and lr are required");
  return step(h, 0, t, 0.f, lr, grad_scale, K, cuda_stream);
}

void sim_adamw_destroy(sim_adamw* h) {
  if (!h) return;
  DeviceGuard guard(h->device);
  cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;   // a handle may be dropped while some stream captures: that must not end the capture
  cudaThreadExchangeStreamCaptureMode(&mode);
  cudaFree(h->tables);          // waits for the device: no step can still be reading the tables
  cudaThreadExchangeStreamCaptureMode(&mode);
  delete h;
}

}  // extern "C"
