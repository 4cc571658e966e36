// Parameters and host checks shared by the attention kernels.
#pragma once

#include "ops_internal.h"

namespace slidedp {

// Which keys a query sees. Documents are contiguous, so the visible keys of a query are ONE interval,
// and so are the queries that see a key; both intervals' ends never decrease along the sequence,
// which is what lets a tile of rows find the range of its partners from its first and last row.
struct DocMask {
  const int32_t* cu;       // null: one document
  const int32_t* prefix;   // null: none
  int docs, tokens, causal;

#ifdef __CUDACC__
  // Document of token i as [s, e) and its index; false (and an empty range that keeps the order)
  // when no document holds it. Bounds are clamped to the sequence whatever the array holds.
  __device__ __forceinline__ bool find(int i, int* s, int* e, int* d) const {
    if (!cu) { *s = 0; *e = tokens; *d = 0; return true; }
    int lo = 0, hi = docs + 1;       // first index whose offset is above i
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (cu[mid] <= i) lo = mid + 1; else hi = mid;
    }
    *d = lo - 1;
    if (lo == 0 || lo == docs + 1) {
      *s = *e = clamp(cu[lo == 0 ? 0 : docs]);
      return false;
    }
    *s = clamp(cu[lo - 1]);
    *e = clamp(cu[lo]);
    return true;
  }
  __device__ __forceinline__ int clamp(int x) const { return x < 0 ? 0 : x > tokens ? tokens : x; }
  __device__ __forceinline__ int seen_by_all(int s, int e, int d) const {   // end of the prefix
    if (!causal) return e;
    if (!prefix) return s;
    const int n = prefix[d];
    return n <= 0 ? s : n >= e - s ? e : s + n;
  }
  __device__ __forceinline__ void keys_of(int i, int* lo, int* hi) const {
    int e, d;
    if (!find(i, lo, &e, &d)) { *hi = *lo; return; }
    const int all = seen_by_all(*lo, e, d);
    *hi = i + 1 > all ? i + 1 : all;
  }
  __device__ __forceinline__ void queries_of(int j, int* lo, int* hi) const {
    int s, d;
    if (!find(j, &s, hi, &d)) { *lo = *hi; return; }
    *lo = j < seen_by_all(s, *hi, d) ? s : j;
  }
#endif
};

struct AttnView {
  uint16_t* p;
  int64_t t, h;   // strides in elements
};

struct AttnParams {
  AttnView q, k, v, o, dout, dq, dk, dv;
  float* lse;          // [heads_q][tokens]
  float* row_lse;      // backward: lse * log2 e as [heads_q][pitch], zeros past tokens
  float* row_delta;    // backward: sum_d dout * out, likewise
  int64_t pitch;
  int* error;          // pinned host word that a wait which runs out sets
  const float* slopes;
  DocMask mask;
  int tokens, heads_q, heads_kv, group, head_dim;
  float scale;         // of the scores
  float softcap;       // 0: none
  float scale_log2;    // scale * log2 e
};

namespace host {

// attention_mma.cu: the tensor-core kernels; head_dim a multiple of 8 up to 128, 16-byte aligned views.
int attention_forward_mma(slidedp_ctx* ctx, const AttnParams& p, cudaStream_t st);
int attention_backward_mma(slidedp_ctx* ctx, const AttnParams& p, cudaStream_t st);

}  // namespace host
}  // namespace slidedp
