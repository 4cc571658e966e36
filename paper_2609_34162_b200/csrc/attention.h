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
  // First index whose offset is above i, known to lie in [from, to]; 0 and 0 without offsets.
  __device__ __forceinline__ int above(int i, int from, int to) const {
    while (from < to) {
      const int mid = (from + to) >> 1;
      if (cu[mid] <= i) from = mid + 1; else to = mid;
    }
    return from;
  }
  __device__ __forceinline__ int above(int i) const { return cu ? above(i, 0, docs + 1) : 0; }
  // The document before that index as [s, e); false (and an empty range that keeps the order) when there is
  // none. Bounds are clamped to the sequence whatever the array holds.
  __device__ __forceinline__ bool document(int index, int* s, int* e) const {
    if (!cu) { *s = 0; *e = tokens; return true; }
    if (index == 0 || index == docs + 1) {
      *s = *e = clamp(cu[index == 0 ? 0 : docs]);
      return false;
    }
    *s = clamp(cu[index - 1]);
    *e = clamp(cu[index]);
    return true;
  }
  __device__ __forceinline__ int clamp(int x) const { return x < 0 ? 0 : x > tokens ? tokens : x; }
  __device__ __forceinline__ int seen_by_all(int s, int e, int index) const {   // end of the prefix
    if (!causal) return e;
    if (!prefix) return s;
    const int n = prefix[index - 1];
    return n <= 0 ? s : n >= e - s ? e : s + n;
  }
  // The keys that query i sees and the queries that see key j, as [lo, hi), from above(i) or above(j).
  __device__ __forceinline__ void keys_of(int i, int index, int* lo, int* hi) const {
    int e;
    if (!document(index, lo, &e)) { *hi = *lo; return; }
    const int all = seen_by_all(*lo, e, index);
    *hi = i + 1 > all ? i + 1 : all;
  }
  __device__ __forceinline__ void queries_of(int j, int index, int* lo, int* hi) const {
    int s;
    if (!document(index, &s, hi)) { *lo = *hi; return; }
    *lo = j < seen_by_all(s, *hi, index) ? s : j;
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
  uint32_t polls;      // and how long it polls
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
