// C ABI of the gradients' norm and of clipping: argument checks, launches.  Declarations and contracts are in include/ngsgd.h.
#include "grad_norm.h"

#include <algorithm>
#include <new>
#include <vector>

#include "host.h"

using namespace ngsgd;

namespace {

constexpr int32_t kMostTensors = 1 << 20;
constexpr int64_t kMostElements = (int64_t)1 << 40;

size_t most_parts(const int32_t n_tensors) { return (size_t)((n_tensors + kNormTensors - 1) / kNormTensors) * kNormParts; }

struct Workspace {
  NormResult* result;
  double* parts;
};
Workspace layout(Carver& c, const int32_t n_tensors) {
  Workspace w;
  w.result = c.take<NormResult>(1);
  w.parts = c.take<double>(most_parts(n_tensors));
  return w;
}

// The tensors from `first` on that one launch takes; returns where the next one goes on.  Empty ones are left out.
int fill(NormTensors& a, int first, const int32_t n_tensors, const int64_t* sizes, const void* const* grads, void* const* out) {
  int count = 0;
  int64_t total = 0;
  for (; first < n_tensors && count < kNormTensors; ++first) {
    if (sizes[first] == 0 || grads[first] == nullptr) continue;
    a.g[count] = grads[first];
    a.out[count] = out != nullptr ? out[first] : const_cast<void*>(grads[first]);
    a.n[count++] = sizes[first];
    total += sizes[first];
  }
  const int64_t share = (total + kNormPieces - 1) / kNormPieces;
  a.piece = std::max<int64_t>(kNormLeast, (share + kNormThreads * 8 - 1) / (kNormThreads * 8) * (kNormThreads * 8));
  a.pieces = 0;
  for (int i = 0; i < count; ++i) {
    a.first[i] = a.pieces;
    a.pieces += (int)((a.n[i] + a.piece - 1) / a.piece);
  }
  for (int i = count; i < kNormTensors; ++i) a.first[i] = INT32_MAX;
  return first;
}

// Outputs share memory with nothing but their own gradients: otherwise a factor would be applied twice, or to what another workgroup has written.
bool outputs_apart(const int32_t n_tensors, const int64_t* sizes, const void* const* grads, const int type, void* const* out) {
  struct Span {
    uintptr_t from, to;
    int index;
  };
  const auto span = [&](const void* p, const int i) {
    const uintptr_t from = reinterpret_cast<uintptr_t>(p);
    return Span{from, from + (uintptr_t)(sizes[i] * type_bytes(type)), i};
  };
  std::vector<Span> outs;
  for (int i = 0; i < n_tensors; ++i)
    if (sizes[i] > 0 && grads[i] != nullptr) outs.push_back(span(out != nullptr ? out[i] : grads[i], i));
  std::sort(outs.begin(), outs.end(), [](const Span& a, const Span& b) { return a.from < b.from; });
  for (size_t k = 1; k < outs.size(); ++k)
    if (outs[k].from < outs[k - 1].to) return false;
  for (int i = 0; out != nullptr && i < n_tensors; ++i) {
    if (sizes[i] == 0 || grads[i] == nullptr) continue;
    const Span g = span(grads[i], i);
    for (auto o = std::upper_bound(outs.begin(), outs.end(), g.from, [](const uintptr_t at, const Span& b) { return at < b.to; });
         o != outs.end() && o->from < g.to; ++o)
      if (o->index != i || o->from != g.from) return false;
  }
  return true;
}

template <typename F>
int with_type(const int type, F f) { return type == NGSGD_FLOAT32 ? f(float()) : type == NGSGD_BFLOAT16 ? f(bf16()) : f(fp16()); }

int run(int32_t n_tensors, const int64_t* sizes, const void* const* grads, int32_t type, double max_norm, bool clip, void* const* out, float* dev_norm,
        float* dev_factor, void* dev_workspace, size_t workspace_bytes, hipStream_t s) {
  size_t need = 0;
  NG_TRY(ngsgd_grad_norm_workspace_bytes(n_tensors, &need));
  if (!known_type(type) || sizes == nullptr || grads == nullptr || !(max_norm >= 0.0)) return NGSGD_EINVAL;
  if (!on_element(dev_norm, NGSGD_FLOAT32) || !on_element(dev_factor, NGSGD_FLOAT32)) return NGSGD_EINVAL;
  for (int i = 0; i < n_tensors; ++i) {
    if (sizes[i] < 0 || sizes[i] > kMostElements || !on_element(grads[i], type)) return NGSGD_EINVAL;
    if (out != nullptr && sizes[i] > 0 && grads[i] != nullptr && (out[i] == nullptr || !on_element(out[i], type))) return NGSGD_EINVAL;
  }
  NG_TRY(check_workspace(dev_workspace, workspace_bytes, need));
  if (clip) {
    try {
      if (!outputs_apart(n_tensors, sizes, grads, type, out)) return NGSGD_EINVAL;
    } catch (const std::bad_alloc&) {   // no host memory for the addresses
      return NGSGD_ENOMEM;
    }
  }
  Carver c(dev_workspace);
  const Workspace w = layout(c, n_tensors);
  const NormOut to{dev_norm, dev_factor};
  NormTensors a;
  int parts = 0, launches = 0;
  for (int first = 0; first < n_tensors;) {
    first = fill(a, first, n_tensors, sizes, grads, out);
    if (first == n_tensors && launches == 0 && a.pieces <= kNormSmallPieces)
      return with_type(type, [&](auto t) {
        hipLaunchKernelGGL(grad_small_kernel<decltype(t)>, dim3(1), dim3(kNormSmallThreads), 0, s, a, clip, max_norm, to);
        LAUNCH_CHECK();
        return NGSGD_OK;
      });
    if (a.pieces == 0) continue;
    NG_TRY(with_type(type, [&](auto t) {
      hipLaunchKernelGGL(grad_norm_kernel<decltype(t)>, dim3(a.pieces), dim3(kNormThreads), 0, s, a, w.parts + parts);
      LAUNCH_CHECK();
      return NGSGD_OK;
    }));
    parts += a.pieces;
    ++launches;
  }
  // the sums of one launch are joined by every workgroup that clips (2048 of them: 2 us, a launch for it 4)
  const bool join = clip && launches == 1;
  if (!join) {
    hipLaunchKernelGGL(grad_norm_finish_kernel, dim3(1), dim3(1024), 0, s, w.parts, parts, max_norm, w.result, to);
    LAUNCH_CHECK();
  }
  for (int first = 0; clip && first < n_tensors;) {
    first = fill(a, first, n_tensors, sizes, grads, out);
    if (a.pieces == 0) continue;
    NG_TRY(with_type(type, [&](auto t) {
      hipLaunchKernelGGL(grad_clip_kernel<decltype(t)>, dim3(a.pieces), dim3(kNormThreads), 0, s, a, w.parts, join ? parts : 0, max_norm, w.result, to);
      LAUNCH_CHECK();
      return NGSGD_OK;
    }));
  }
  return NGSGD_OK;
}

}  // namespace

extern "C" int ngsgd_grad_norm_workspace_bytes(int32_t n_tensors, size_t* out_bytes) {
  if (out_bytes == nullptr || n_tensors < 1 || n_tensors > kMostTensors) return NGSGD_EINVAL;
  Carver c(nullptr);
  (void)layout(c, n_tensors);
  *out_bytes = align_up(c.off, 256);
  return NGSGD_OK;
}

extern "C" int ngsgd_grad_norm(int32_t n_tensors, const int64_t* sizes, const void* const* dev_grads, int32_t type, double max_norm, float* dev_norm,
                               float* dev_factor, void* dev_workspace, size_t workspace_bytes, void* hip_stream) {
  return run(n_tensors, sizes, dev_grads, type, max_norm, false, nullptr, dev_norm, dev_factor, dev_workspace, workspace_bytes,
             static_cast<hipStream_t>(hip_stream));
}

extern "C" int ngsgd_grad_clip(int32_t n_tensors, const int64_t* sizes, const void* const* dev_grads, int32_t type, double max_norm, void* const* dev_out,
                               float* dev_norm, float* dev_factor, void* dev_workspace, size_t workspace_bytes, void* hip_stream) {
  return run(n_tensors, sizes, dev_grads, type, max_norm, true, dev_out, dev_norm, dev_factor, dev_workspace, workspace_bytes,
             static_cast<hipStream_t>(hip_stream));
}
