// Declarations shared by the translation units of the fine-tuning operators (not installed).
#pragma once

#include <initializer_list>
#include <utility>

#include "internal.h"
#include "slidedp_ops.h"

namespace slidedp {
namespace host {

constexpr int kMaxHeadDim = 256;

constexpr int64_t kMaxTokens = 1ll << 30;  // row indices and lane arithmetic stay in 32 bits

// A heads view is usable when it has data and its strides are not negative. The element alignment
// of the base is the caller's language's; only the vector paths ask for more.
inline bool heads_ok(const slidedp_heads* v, int64_t elem_bytes) {
  return v && v->data && v->stride_token >= 0 && v->stride_head >= 0 &&
         reinterpret_cast<uintptr_t>(v->data) % (uintptr_t)elem_bytes == 0;
}
// Base and strides are multiples of `bytes` (strides of an axis of length 1 do not matter).
inline bool heads_aligned(const slidedp_heads* v, int64_t elem_bytes, int64_t bytes, int64_t tokens, int heads) {
  return reinterpret_cast<uintptr_t>(v->data) % (uintptr_t)bytes == 0 &&
         (tokens <= 1 || v->stride_token * elem_bytes % bytes == 0) &&
         (heads <= 1 || v->stride_head * elem_bytes % bytes == 0);
}
inline bool is_finite(double x) { return x - x == 0.0; }
// The kernels compute with FP32 factors: a number that FP32 turns into infinity, or a positive one that it turns into zero,
// would silently be another.
inline bool fits_f32(double x) { return is_finite((double)(float)x); }
inline bool positive_f32(double x) { return fits_f32(x) && (float)x > 0.0f; }

inline bool rows_ok(const slidedp_rows* r, int elem, int64_t rows, int64_t columns, bool output) {
  return r && r->data && r->stride >= 0 && reinterpret_cast<uintptr_t>(r->data) % elem == 0 && (!output || rows <= 1 || r->stride >= columns);
}
inline int elem_bytes(int32_t dtype) { return dtype == SLIDEDP_F32 ? 4 : 2; }

// Values per thread and row that all tensors' alignment allows.
inline int vector_width(int64_t hidden, int elem, std::initializer_list<std::pair<const slidedp_rows*, int>> all) {
  const auto fits = [&](int v) {
    if (hidden % v != 0) return false;
    for (const auto& r : all) {
      if (!r.first) continue;
      const int64_t bytes = v * r.second < 16 ? v * r.second : 16;
      if (reinterpret_cast<uintptr_t>(r.first->data) % bytes != 0 || r.first->stride * r.second % bytes != 0) return false;
    }
    return true;
  };
  if (fits(16 / elem)) return 16 / elem;
  return elem == 2 && fits(2) ? 2 : 1;
}

// Launches a kernel of the operators, in clusters of `cluster` blocks if that is above one. It may be set up while the
// kernel before it in the stream ends: every block of it waits for that kernel before its first access to memory (where it
// does not, its comment says why). Calls back to back, before and after: norm of one token 6.5 -> 5.9 us, its training pass on
// 1537 tokens 22.5 -> 18.4, attention of 77 tokens 8.2 -> 6.3.
template <typename... P, typename... A>
void launch_after(void (*kernel)(P...), dim3 grid, unsigned threads, size_t smem, unsigned cluster, cudaStream_t st, A&&... args) {
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  (void)cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);   // the caller asks for the error
}

}  // namespace host
}  // namespace slidedp
