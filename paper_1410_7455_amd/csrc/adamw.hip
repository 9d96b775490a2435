// C ABI of AdamW over many tensors: argument checks, tables, launches.  Declarations and contracts are in include/ngsgd.h.
#include "adamw.h"

#include <algorithm>
#include <cmath>
#include <new>
#include <utility>
#include <vector>

#include "host.h"

using namespace ngsgd;

struct ngsgd_adamw {
  int n_tensors = 0, n_chunks = 0, param_type = 0, grad_type = 0, bits = 32;
  bool master = false;
  double beta1 = 0.0, beta2 = 0.0;
  float eps = 0.f;
  int64_t elements = 0;              // of the flat arrays
  std::vector<int> first_chunk;      // of each tensor, and behind the last
  AdamState s{};
};

namespace {

// Fewer chunks than this are split into quarters (a wavefront then takes one block instead of four: 1 M elements in 61 tensors 9.8 us, else 13.2).
// Steps of so few workgroups count themselves: with 52 a step takes the host 11.9 us instead of 14.6 and the GPU 5.3 instead of 4.6 (with 100
// 15.3 instead of 18.3, and 7.5 instead of 4.6).
constexpr int kAdamFewChunks = 512, kAdamCounting = 64;
constexpr int64_t kAdamMostChunks = (1 << 24) - 1;   // (a launch has less than 2^32 threads)

int check_config(const ngsgd_adamw_config* cfg) {
  if (cfg == nullptr || cfg->n_tensors < 1 || cfg->dev_params == nullptr || cfg->sizes == nullptr) return NGSGD_EINVAL;
  if (!known_type(cfg->param_type) || !known_type(cfg->grad_type)) return NGSGD_EINVAL;
  // gradients: of the parameters' type, in fp32, or in 16 bits for fp32 parameters
  if (cfg->grad_type != cfg->param_type && cfg->grad_type != NGSGD_FLOAT32 && cfg->param_type != NGSGD_FLOAT32) return NGSGD_EINVAL;
  if (cfg->state_bits != 8 && cfg->state_bits != 32) return NGSGD_EINVAL;
  if (cfg->master != 0 && (cfg->master != 1 || cfg->param_type == NGSGD_FLOAT32)) return NGSGD_EINVAL;
  if (!(cfg->beta1 >= 0.0 && cfg->beta1 < 1.0) || !(cfg->beta2 >= 0.0 && cfg->beta2 < 1.0)) return NGSGD_EINVAL;
  if (!(cfg->epsilon == 0.f || std::isnormal(cfg->epsilon)) || cfg->epsilon < 0.f) return NGSGD_EINVAL;
  int64_t elements = 0, chunks = 0;
  const int64_t bytes = type_bytes(cfg->param_type);
  std::vector<std::pair<uintptr_t, uintptr_t>> spans;
  for (int i = 0; i < cfg->n_tensors; ++i) {
    const int64_t n = cfg->sizes[i];
    if (n < 0 || n > (int64_t)1 << 40) return NGSGD_EINVAL;
    if (n > 0 && (cfg->dev_params[i] == nullptr || !on_element(cfg->dev_params[i], cfg->param_type))) return NGSGD_EINVAL;
    if (cfg->weight_decay != nullptr && !std::isfinite(cfg->weight_decay[i])) return NGSGD_EINVAL;
    if (cfg->rate != nullptr && !std::isfinite(cfg->rate[i])) return NGSGD_EINVAL;
    elements += (n + kAdamBlock - 1) / kAdamBlock * kAdamBlock;
    chunks += (n + kAdamChunk - 1) / kAdamChunk;
    if (chunks > kAdamMostChunks) return NGSGD_EINVAL;
    if (n > 0) {
      const uintptr_t p = reinterpret_cast<uintptr_t>(cfg->dev_params[i]);
      spans.emplace_back(p, p + (uintptr_t)(n * bytes));
    }
  }
  // two workgroups would update an element that two tensors share
  std::sort(spans.begin(), spans.end());
  for (size_t i = 1; i < spans.size(); ++i)
    if (spans[i].first < spans[i - 1].second) return NGSGD_EINVAL;
  return NGSGD_OK;
}

void layout(ngsgd_adamw& h, const ngsgd_adamw_config* cfg, Carver& c) {
  h.n_tensors = cfg->n_tensors;
  h.param_type = cfg->param_type;
  h.grad_type = cfg->grad_type;
  h.bits = cfg->state_bits;
  h.master = cfg->master != 0;
  h.beta1 = cfg->beta1;
  h.beta2 = cfg->beta2;
  h.eps = cfg->epsilon;
  h.first_chunk.assign(1, 0);
  h.elements = 0;
  for (int i = 0; i < cfg->n_tensors; ++i) {
    h.elements += (cfg->sizes[i] + kAdamBlock - 1) / kAdamBlock * kAdamBlock;
    h.first_chunk.push_back(h.first_chunk.back() + (int)((cfg->sizes[i] + kAdamChunk - 1) / kAdamChunk));
  }
  h.n_chunks = h.first_chunk.back();
  const size_t n = (size_t)h.elements;
  if (h.bits == 32) {
    h.s.m32 = c.take<float>(n);
    h.s.v32 = c.take<float>(n);
  } else {
    h.s.m8 = c.take<uint8_t>(n);
    h.s.v8 = c.take<uint8_t>(n);
    h.s.exps = c.take<AdamExponents>(n / kAdamBlock);
  }
  if (h.master) h.s.master = c.take<float>(n);
  h.s.scalars = c.take<AdamScalars>(1);
  h.s.chunks = c.take<AdamChunk>((size_t)h.n_chunks);
}

unsigned blocks_grid(const int64_t blocks) {
  return (unsigned)std::max<int64_t>(1, std::min<int64_t>(1 << 20, (blocks + kAdamThreads / 64 - 1) / (kAdamThreads / 64)));
}

int set_state(const ngsgd_adamw* h, const float* m, const float* v, const int64_t t, hipStream_t s) {
  const AdamScalars scalars{t, std::pow(h->beta1, (double)t), std::pow(h->beta2, (double)t), 0.f, 0.f, 0, 0};
  const int64_t blocks = h->elements / kAdamBlock;
  hipLaunchKernelGGL(adamw_set_state_kernel, dim3(blocks_grid(blocks)), dim3(kAdamThreads), 0, s, h->s, h->bits, blocks, m, v, scalars);
  LAUNCH_CHECK();
  return NGSGD_OK;
}

int set_master(const ngsgd_adamw* h, const float* in, hipStream_t s) {
  if (!h->master || h->n_chunks == 0) return NGSGD_OK;
  const dim3 grid((unsigned)h->n_chunks);
  if (h->param_type == NGSGD_BFLOAT16)
    hipLaunchKernelGGL(adamw_set_master_kernel<bf16>, grid, dim3(kAdamThreads), 0, s, h->s, in);
  else
    hipLaunchKernelGGL(adamw_set_master_kernel<fp16>, grid, dim3(kAdamThreads), 0, s, h->s, in);
  LAUNCH_CHECK();
  return NGSGD_OK;
}

int fill_workspace(ngsgd_adamw& h, const ngsgd_adamw_config* cfg, void* dev_workspace, const size_t bytes) {
  Carver c(dev_workspace);
  layout(h, cfg, c);
  std::vector<AdamChunk> chunks;
  chunks.reserve((size_t)h.n_chunks);
  int64_t offset = 0;
  for (int i = 0; i < cfg->n_tensors; ++i) {
    const int64_t n = cfg->sizes[i];
    for (int64_t at = 0; at < n; at += kAdamChunk)
      chunks.push_back(AdamChunk{static_cast<char*>(cfg->dev_params[i]) + at * type_bytes(h.param_type), offset + at, i, (int)(at / kAdamChunk),
                                 (int)std::min<int64_t>(kAdamChunk, n - at), cfg->rate != nullptr ? cfg->rate[i] : 1.f,
                                 cfg->weight_decay != nullptr ? cfg->weight_decay[i] : 0.f, 0});
    offset += (n + kAdamBlock - 1) / kAdamBlock * kAdamBlock;
  }
  HIP_TRY(hipDeviceSynchronize());   // whatever writes the parameters
  HIP_TRY(hipMemset(dev_workspace, 0, bytes));
  if (!chunks.empty())
    HIP_TRY(hipMemcpy(const_cast<AdamChunk*>(h.s.chunks), chunks.data(), chunks.size() * sizeof(AdamChunk), hipMemcpyHostToDevice));
  NG_TRY(set_state(&h, nullptr, nullptr, 0, nullptr));
  NG_TRY(set_master(&h, nullptr, nullptr));
  HIP_TRY(hipDeviceSynchronize());
  return NGSGD_OK;
}

template <typename P, typename G>
void launch_step(const ngsgd_adamw* h, const AdamStep& a, const unsigned grid, hipStream_t s) {
  constexpr bool half = sizeof(P) == 2;   // fp32 parameters need no copy
  if (h->bits == 32) {
    if (half && h->master)
      hipLaunchKernelGGL((adamw_kernel<P, G, 32, half>), dim3(grid), dim3(kAdamThreads), 0, s, a);
    else
      hipLaunchKernelGGL((adamw_kernel<P, G, 32, false>), dim3(grid), dim3(kAdamThreads), 0, s, a);
  } else {
    if (half && h->master)
      hipLaunchKernelGGL((adamw_kernel<P, G, 8, half>), dim3(grid), dim3(kAdamThreads), 0, s, a);
    else
      hipLaunchKernelGGL((adamw_kernel<P, G, 8, false>), dim3(grid), dim3(kAdamThreads), 0, s, a);
  }
}

}  // namespace

extern "C" int ngsgd_adamw_workspace_bytes(const ngsgd_adamw_config* cfg, size_t* out_bytes) {
  if (out_bytes == nullptr) return NGSGD_EINVAL;
  try {
    NG_TRY(check_config(cfg));
    ngsgd_adamw h;
    Carver c(nullptr);
    layout(h, cfg, c);
    *out_bytes = align_up(c.off, 256);
    return NGSGD_OK;
  } catch (const std::bad_alloc&) {   // no host memory for the tables
    return NGSGD_ENOMEM;
  }
}

extern "C" int ngsgd_adamw_create(const ngsgd_adamw_config* cfg, void* dev_workspace, size_t workspace_bytes, ngsgd_adamw** out) {
  if (out == nullptr || dev_workspace == nullptr || (reinterpret_cast<uintptr_t>(dev_workspace) & 255u)) return NGSGD_EINVAL;
  size_t need = 0;
  NG_TRY(ngsgd_adamw_workspace_bytes(cfg, &need));
  if (workspace_bytes < need) return NGSGD_ENOMEM;
  ngsgd_adamw* h = new (std::nothrow) ngsgd_adamw();
  if (h == nullptr) return NGSGD_ENOMEM;
  int rc = NGSGD_ENOMEM;
  try {
    rc = fill_workspace(*h, cfg, dev_workspace, need);
  } catch (const std::bad_alloc&) {   // no host memory for the tables
  }
  if (rc != NGSGD_OK) {
    delete h;
    return rc;
  }
  *out = h;
  return NGSGD_OK;
}

extern "C" int ngsgd_adamw_destroy(ngsgd_adamw* h) {
  if (h == nullptr) return NGSGD_EINVAL;
  delete h;
  return NGSGD_OK;
}

extern "C" int ngsgd_adamw_step(ngsgd_adamw* h, const void* const* dev_grads, float lr, const float* dev_lr, float grad_scale,
                                const float* dev_grad_scale, void* hip_stream) {
  if (h == nullptr || dev_grads == nullptr) return NGSGD_EINVAL;
  if (!on_element(dev_lr, NGSGD_FLOAT32) || !on_element(dev_grad_scale, NGSGD_FLOAT32)) return NGSGD_EINVAL;
  for (int i = 0; i < h->n_tensors; ++i)
    if (!on_element(dev_grads[i], h->grad_type)) return NGSGD_EINVAL;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  AdamStep a;
  a.s = h->s;
  a.lr = lr;
  a.scale = grad_scale;
  a.eps = h->eps;
  a.beta1 = h->beta1;
  a.beta2 = h->beta2;
  a.dev_lr = dev_lr;
  a.dev_scale = dev_grad_scale;
  a.part_bits = h->n_chunks < kAdamFewChunks ? 2 : 0;
  a.counts = h->n_tensors <= kAdamGrads && h->n_chunks << a.part_bits <= kAdamCounting && h->n_chunks > 0;
  if (!a.counts) {
    hipLaunchKernelGGL(adamw_count_kernel, dim3(1), dim3(1), 0, s, h->s.scalars, h->beta1, h->beta2);
    LAUNCH_CHECK();
  }
  for (int first = 0; first < h->n_tensors; first += kAdamGrads) {
    const int end = std::min(first + kAdamGrads, h->n_tensors);
    a.first_tensor = first;
    a.first_chunk = h->first_chunk[first];
    const int n_chunks = h->first_chunk[end] - a.first_chunk;
    for (int i = 0; i < kAdamGrads; ++i) a.grads[i] = first + i < end ? dev_grads[first + i] : nullptr;
    if (n_chunks == 0) continue;
    const unsigned grid = (unsigned)n_chunks << a.part_bits;
    if (h->param_type == NGSGD_FLOAT32) {
      if (h->grad_type == NGSGD_FLOAT32) launch_step<float, float>(h, a, grid, s);
      if (h->grad_type == NGSGD_BFLOAT16) launch_step<float, bf16>(h, a, grid, s);
      if (h->grad_type == NGSGD_FLOAT16) launch_step<float, fp16>(h, a, grid, s);
    } else if (h->param_type == NGSGD_BFLOAT16) {
      if (h->grad_type == NGSGD_FLOAT32) launch_step<bf16, float>(h, a, grid, s);
      else launch_step<bf16, bf16>(h, a, grid, s);
    } else {
      if (h->grad_type == NGSGD_FLOAT32) launch_step<fp16, float>(h, a, grid, s);
      else launch_step<fp16, fp16>(h, a, grid, s);
    }
    LAUNCH_CHECK();
  }
  return NGSGD_OK;
}

extern "C" int ngsgd_adamw_arrays(const ngsgd_adamw* h, int64_t* elements, float** dev_m, float** dev_v, float** dev_master) {
  if (h == nullptr) return NGSGD_EINVAL;
  if (elements != nullptr) *elements = h->elements;
  if (dev_m != nullptr) *dev_m = h->s.m32;
  if (dev_v != nullptr) *dev_v = h->s.v32;
  if (dev_master != nullptr) *dev_master = h->s.master;
  return NGSGD_OK;
}

extern "C" int ngsgd_adamw_get_state(const ngsgd_adamw* h, void* dev_m, void* dev_v, int32_t type, int64_t* dev_t, void* hip_stream) {
  if (h == nullptr || (type != NGSGD_FLOAT32 && type != NGSGD_BFLOAT16)) return NGSGD_EINVAL;
  if (!aligned16(dev_m) || !aligned16(dev_v) || (reinterpret_cast<uintptr_t>(dev_t) & 7u)) return NGSGD_EINVAL;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const int64_t blocks = h->elements / kAdamBlock;
  if ((dev_m != nullptr || dev_v != nullptr) && blocks > 0) {
    const dim3 grid(blocks_grid(blocks));
    if (type == NGSGD_FLOAT32)
      hipLaunchKernelGGL(adamw_get_state_kernel<float>, grid, dim3(kAdamThreads), 0, s, h->s, h->bits, blocks, static_cast<float*>(dev_m),
                         static_cast<float*>(dev_v));
    else
      hipLaunchKernelGGL(adamw_get_state_kernel<bf16>, grid, dim3(kAdamThreads), 0, s, h->s, h->bits, blocks, static_cast<bf16*>(dev_m),
                         static_cast<bf16*>(dev_v));
    LAUNCH_CHECK();
  }
  if (dev_t != nullptr) HIP_TRY(hipMemcpyAsync(dev_t, &h->s.scalars->t, sizeof(int64_t), hipMemcpyDeviceToDevice, s));
  return NGSGD_OK;
}

extern "C" int ngsgd_adamw_set_state(ngsgd_adamw* h, const float* dev_m, const float* dev_v, const float* dev_master, int64_t t,
                                     void* hip_stream) {
  if (h == nullptr || t < 0 || !aligned16(dev_m) || !aligned16(dev_v) || !aligned16(dev_master)) return NGSGD_EINVAL;
  if (dev_master != nullptr && !h->master) return NGSGD_EINVAL;
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  NG_TRY(set_state(h, dev_m, dev_v, t, s));
  return set_master(h, dev_master, s);
}
