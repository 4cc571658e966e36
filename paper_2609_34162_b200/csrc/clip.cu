// libslidedp: clipping by the norm over many tensors. See include/slidedp_ops.h for the contract.
//
// norm = sqrt(sum (scale x)^2), out = x scale min(1, max / (norm + 1e-6)).
// Bound: HBM; everything is read twice, once for the norm and once to be scaled, unless it stays in L2 in between (keeping part of it
// there on purpose gained 2 % for FP32 and lost for BF16). 193M values, FP32 to BF16: 310 us, 1.93 GB at 6.2 TB/s; BF16 to BF16: 206. Two kernels: sums
// of tiles by a grid that does not depend on anything but the number of tiles, a partial sum per block; then every block adds up
// those partial sums in the same order, so that no third kernel and no hand-over between blocks is needed.
#include "ops_internal.h"
#include "device_utils.cuh"

namespace slidedp {

constexpr int kClipThreads = 256;
constexpr int kClipBlocks = 148 * 4;
constexpr int kClipUnroll = 4;           // 16-byte loads per thread under way
// A launch has its tensors' addresses and sizes among its parameters, which replays of a captured call keep. Few tensors
// are 2 KB of them, many 32 KB.
constexpr int kFewTensors = 64, kManyTensors = 960;

// Sizes hold the types in their two top bits.
constexpr int kInF32 = 62, kOutF32 = 63;

template <int CAP>
struct TensorTable {
  const void* in[CAP];
  void* out[CAP];
  uint64_t n[CAP];
  int32_t first_tile[CAP + 1];
  int32_t count;
  int32_t tile;      // elements
  __device__ int64_t size(int i) const { return (int64_t)(n[i] & ((1ull << kInF32) - 1)); }
  __device__ bool in_f32(int i) const { return n[i] >> kInF32 & 1; }
  __device__ bool out_f32(int i) const { return n[i] >> kOutF32 & 1; }
  // The tensor that a tile belongs to: the last one whose first tile is not behind it (empty tensors have none).
  __device__ int find(int t) const {
    int lo = 0, hi = count;
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (first_tile[mid] <= t) lo = mid; else hi = mid;
    }
    return lo;
  }
};

__device__ __forceinline__ double block_sum(double x) {
  __shared__ double warp[kClipThreads / 32];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  if (threadIdx.x % 32 == 0) warp[threadIdx.x / 32] = x;
  __syncthreads();
  x = warp[0];
#pragma unroll
  for (int w = 1; w < kClipThreads / 32; ++w) x += warp[w];
  return x;
}

template <typename T> struct Element;
template <> struct Element<float> {
  static constexpr int kPer = 4;
  static __device__ float get(const float* p) { return __ldcs(p); }
  static __device__ void unpack(uint4 a, float* v) {
    v[0] = __uint_as_float(a.x); v[1] = __uint_as_float(a.y); v[2] = __uint_as_float(a.z); v[3] = __uint_as_float(a.w);
  }
};
template <> struct Element<uint16_t> {
  static constexpr int kPer = 8;
  static __device__ float get(const uint16_t* p) { return __uint_as_float((uint32_t)__ldcs(p) << 16); }
  static __device__ void unpack(uint4 a, float* v) {
    v[0] = bf16_lo(a.x); v[1] = bf16_hi(a.x); v[2] = bf16_lo(a.y); v[3] = bf16_hi(a.y);
    v[4] = bf16_lo(a.z); v[5] = bf16_hi(a.z); v[6] = bf16_lo(a.w); v[7] = bf16_hi(a.w);
  }
};

__device__ __forceinline__ void put(float* p, float v) { __stcs(p, v); }
__device__ __forceinline__ void put(uint16_t* p, float v) { __stcs(p, (uint16_t)f32_to_bf16_bits(v)); }

// Sum of squares of n values by the block's threads, this thread's share.
template <typename T>
__device__ __forceinline__ double sum_squares(const T* x, int n) {
  constexpr int P = Element<T>::kPer;
  double acc = 0.0;
  const auto add = [&](float v) { acc = fma((double)v, (double)v, acc); };
  const int head = min(n, (int)((16 - (reinterpret_cast<uintptr_t>(x) & 15u)) % 16 / sizeof(T)));
  const int whole = (n - head) / P;
  if ((int)threadIdx.x < head) add(Element<T>::get(x + threadIdx.x));
  const uint4* mid = reinterpret_cast<const uint4*>(x + head);
  for (int i0 = threadIdx.x; i0 < whole; i0 += kClipThreads * kClipUnroll) {
    uint4 a[kClipUnroll];
#pragma unroll
    for (int u = 0; u < kClipUnroll; ++u) {
      const int i = i0 + u * kClipThreads;
      a[u] = i < whole ? __ldg(mid + i) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int u = 0; u < kClipUnroll; ++u) {
      float v[P];
      Element<T>::unpack(a[u], v);
#pragma unroll
      for (int e = 0; e < P; ++e) add(v[e]);
    }
  }
  const int tail = head + whole * P + threadIdx.x;
  if (tail < n) add(Element<T>::get(x + tail));
  return acc;
}

template <int CAP>
__global__ void __launch_bounds__(kClipThreads, 4) tensors_sumsq_kernel(const __grid_constant__ TensorTable<CAP> t, double* sums) {
  start_after_previous_kernel();
  double acc = 0.0;
  for (int tile = blockIdx.x; tile < t.first_tile[t.count]; tile += gridDim.x) {
    const int i = t.find(tile);
    const int64_t from = (int64_t)(tile - t.first_tile[i]) * t.tile;
    const int n = (int)min((int64_t)t.tile, t.size(i) - from);
    acc += t.in_f32(i) ? sum_squares(static_cast<const float*>(t.in[i]) + from, n) : sum_squares(static_cast<const uint16_t*>(t.in[i]) + from, n);
  }
  acc = block_sum(acc);
  if (threadIdx.x == 0) sums[blockIdx.x] = acc;
}

template <typename I, typename O>
__device__ __forceinline__ void scale_tile(const I* x, O* y, int n, float f) {
  constexpr int P = Element<I>::kPer, U = kClipUnroll;
  if (((reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(y)) & 15u) == 0) {
    const int whole = n / P;
    const uint4* from = reinterpret_cast<const uint4*>(x);
    for (int i0 = threadIdx.x; i0 < whole; i0 += kClipThreads * U) {
      uint4 a[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (i0 + u * kClipThreads < whole) a[u] = ld_stream(from + i0 + u * kClipThreads);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = i0 + u * kClipThreads;
        if (i >= whole) continue;
        float v[P];
        Element<I>::unpack(a[u], v);
#pragma unroll
        for (int e = 0; e < P; ++e) v[e] *= f;
        if constexpr (sizeof(O) == 4) {
#pragma unroll
          for (int e = 0; e < P; e += 4)
            st_stream(y + (int64_t)i * P + e, make_uint4(__float_as_uint(v[e]), __float_as_uint(v[e + 1]), __float_as_uint(v[e + 2]), __float_as_uint(v[e + 3])));
        } else if constexpr (P == 8) {
          st_stream(y + (int64_t)i * P, make_uint4(f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3]), f32x2_to_bf16x2(v[4], v[5]), f32x2_to_bf16x2(v[6], v[7])));
        } else {
          __stcs(reinterpret_cast<uint2*>(y + (int64_t)i * P), make_uint2(f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3])));
        }
      }
    }
    const int i = whole * P + threadIdx.x;
    if (i < n) put(y + i, Element<I>::get(x + i) * f);
  } else {   // one value per lane: no alignment to share
    constexpr int V = 8;
    for (int i0 = threadIdx.x; i0 < n; i0 += kClipThreads * V) {
      float v[V];
#pragma unroll
      for (int u = 0; u < V; ++u)
        if (i0 + u * kClipThreads < n) v[u] = Element<I>::get(x + i0 + u * kClipThreads);
#pragma unroll
      for (int u = 0; u < V; ++u)
        if (i0 + u * kClipThreads < n) put(y + i0 + u * kClipThreads, v[u] * f);
    }
  }
}

// The norm from `count` partial sums, by every block alike; then the tiles, the last ones first: they were read last and may
// still be in L2.
template <int CAP>
__global__ void __launch_bounds__(kClipThreads, 4) tensors_scale_kernel(const __grid_constant__ TensorTable<CAP> t, const double* sums, int count,
                                                                     double scale, double max_norm, double* result) {
  start_after_previous_kernel();
  double acc = 0.0;
  for (int i = threadIdx.x; i < count; i += kClipThreads) acc += sums[i];
  const double total = block_sum(acc) * scale * scale, norm = sqrt(total);
  double c = 1.0;
  if (max_norm > 0.0) {
    c = max_norm / (norm + 1e-6);
    if (c > 1.0) c = 1.0;      // a NaN coefficient stays NaN
  }
  if (result && blockIdx.x == 0 && threadIdx.x == 0) {
    result[0] = total;
    result[1] = norm;
    result[2] = c;
    result[3] = norm - norm == 0.0 ? 0.0 : 1.0;
  }
  const float f = (float)(scale * c);
  const int tiles = t.first_tile[t.count];
  for (int k = blockIdx.x; k < tiles; k += gridDim.x) {
    const int tile = tiles - 1 - k, i = t.find(tile);
    const int64_t from = (int64_t)(tile - t.first_tile[i]) * t.tile;
    const int n = (int)min((int64_t)t.tile, t.size(i) - from);
    const float *xf = static_cast<const float*>(t.in[i]) + from;
    const uint16_t* xb = static_cast<const uint16_t*>(t.in[i]) + from;
    float* yf = static_cast<float*>(t.out[i]) + from;
    uint16_t* yb = static_cast<uint16_t*>(t.out[i]) + from;
    if (f == 1.0f && t.in[i] == t.out[i]) continue;
    if (t.in_f32(i)) {
      if (t.out_f32(i)) scale_tile(xf, yf, n, f); else scale_tile(xf, yb, n, f);
    } else {
      if (t.out_f32(i)) scale_tile(xb, yf, n, f); else scale_tile(xb, yb, n, f);
    }
  }
}

}  // namespace slidedp

using namespace slidedp;
using namespace slidedp::host;

namespace {

constexpr int64_t kMaxElements = 1ll << 44;   // per tensor: tiles are counted in 32 bits
// Elements per tile: small ones where that is needed to give every SM something to do.
constexpr int kTile = 16384, kSmallTile = 4096;

int check_tensors(const slidedp_tensor* t, int32_t count, int64_t* total) {
  if (count < 0 || (count > 0 && !t)) return SLIDEDP_ERR_INVALID_ARG;
  *total = 0;
  for (int32_t i = 0; i < count; ++i) {
    if (t[i].count < 0 || t[i].count > kMaxElements || (t[i].dtype != SLIDEDP_BF16 && t[i].dtype != SLIDEDP_F32)) return SLIDEDP_ERR_INVALID_ARG;
    const uintptr_t a = reinterpret_cast<uintptr_t>(t[i].data);
    if (t[i].count > 0 && (!a || a % (t[i].dtype == SLIDEDP_F32 ? 4 : 2) != 0)) return SLIDEDP_ERR_INVALID_ARG;
    *total += t[i].count;
    if (*total > kMaxElements) return SLIDEDP_ERR_INVALID_ARG;
  }
  return SLIDEDP_OK;
}

int64_t launches_for(int32_t count) { return count <= kFewTensors ? 1 : (count + kManyTensors - 1) / kManyTensors; }

template <int CAP>
void fill_table(TensorTable<CAP>* t, const slidedp_tensor* in, const slidedp_tensor* out, int32_t count, int tile) {
  t->count = count;
  t->tile = tile;
  int32_t at = 0;
  for (int32_t i = 0; i < count; ++i) {
    t->in[i] = in[i].data;
    t->out[i] = out ? out[i].data : nullptr;
    t->n[i] = (uint64_t)in[i].count | (uint64_t)(in[i].dtype == SLIDEDP_F32) << kInF32 | (uint64_t)(out && out[i].dtype == SLIDEDP_F32) << kOutF32;
    t->first_tile[i] = at;
    at += (int32_t)((in[i].count + tile - 1) / tile);
  }
  t->first_tile[count] = at;
}

template <int CAP>
int run_clip(slidedp_ctx* ctx, const slidedp_tensor* in, const slidedp_tensor* out, int32_t count, int tile, double scale, double max_norm,
             double* result, double* sums, cudaStream_t st) {
  TensorTable<CAP> t;
  t.count = 0;
  t.first_tile[0] = 0;
  int partials = 0;
  const auto part = [&](int32_t from) { return count - from < CAP ? count - from : CAP; };
  const auto blocks = [&] {
    const int tiles = t.first_tile[t.count];
    return tiles < 1 ? 1 : tiles < kClipBlocks ? tiles : kClipBlocks;
  };
  for (int32_t from = 0; from == 0 || from < count; from += CAP) {
    fill_table<CAP>(&t, in + from, nullptr, part(from), tile);
    FAULT_POINT();
    launch_after(tensors_sumsq_kernel<CAP>, dim3(blocks()), kClipThreads, 0, 1, st, t, sums + partials);
    ctx->launches += 1;
    CU_AFTER_LAUNCH();
    partials += blocks();
  }
  for (int32_t from = 0; from == 0 || (out && from < count); from += CAP) {
    fill_table<CAP>(&t, in + from, out ? out + from : nullptr, out ? part(from) : 0, tile);
    FAULT_POINT();
    launch_after(tensors_scale_kernel<CAP>, dim3(blocks()), kClipThreads, 0, 1, st, t, sums, partials, scale, max_norm, from == 0 ? result : nullptr);
    ctx->launches += 1;
    CU_AFTER_LAUNCH();
  }
  return SLIDEDP_OK;
}

}  // namespace

extern "C" {

size_t slidedp_clip_grad_norm_workspace(const slidedp_tensor* grads, int32_t count) {
  int64_t total;
  if (check_tensors(grads, count, &total) != SLIDEDP_OK) return 0;
  return (size_t)((count ? launches_for(count) : 1) * kClipBlocks) * sizeof(double);
}

int slidedp_clip_grad_norm(slidedp_ctx* ctx, const slidedp_tensor* grads, const slidedp_tensor* outs, int32_t count, double scale,
                           double max_norm, double* result, void* workspace, void* cuda_stream) {
  int64_t total, unused;
  if (!ctx || check_tensors(grads, count, &total) != SLIDEDP_OK || (outs && check_tensors(outs, count, &unused) != SLIDEDP_OK) ||
      !fits_f32(scale) || max_norm != max_norm || !result || reinterpret_cast<uintptr_t>(result) % 8 != 0 || !workspace)
    return SLIDEDP_ERR_INVALID_ARG;
  for (int32_t i = 0; outs && i < count; ++i)
    if (outs[i].count != grads[i].count || (outs[i].count > 0 && outs[i].data == grads[i].data && outs[i].dtype != grads[i].dtype))
      return SLIDEDP_ERR_INVALID_ARG;
  if (!aligned16(workspace)) return SLIDEDP_ERR_MISALIGNED;
  const int rc = check_kernel_error(ctx);
  if (rc != SLIDEDP_OK) return rc;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return cuda_fail(ctx, cudaGetLastError());
  const int tile = total >= (int64_t)kClipBlocks * kTile ? kTile : kSmallTile;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  double* sums = static_cast<double*>(workspace);
  return count <= kFewTensors ? run_clip<kFewTensors>(ctx, grads, outs, count, tile, scale, max_norm, result, sums, st)
                              : run_clip<kManyTensors>(ctx, grads, outs, count, tile, scale, max_norm, result, sums, st);
}

}  // extern "C"
