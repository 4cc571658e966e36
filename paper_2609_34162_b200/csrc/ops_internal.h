// Declarations shared by the translation units of the fine-tuning operators (not installed).
#pragma once

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

// A wait inside an earlier kernel of the context ran out.
inline int check_kernel_error(slidedp_ctx* ctx) {
  volatile int* e = ctx->kernel_error;
  if (*e == 0) return SLIDEDP_OK;
  *e = 0;
  return SLIDEDP_ERR_TIMEOUT;
}

}  // namespace host
}  // namespace slidedp
