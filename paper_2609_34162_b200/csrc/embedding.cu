// libslidedp: token embedding with scaling, and the table's gradient by sorted tokens. See include/slidedp_ops.h for the contract.
//
// out[t] = s table[id t];  d_table[v] = s sum of d_out[t] over id t = v.  Bound: HBM.
// The gradient is two kernels. The first sorts the tokens by id, stably, so that each id's tokens stand together in their
// order. The second cuts the sorted list into pieces of equal length, however often an id occurs, and sums each piece's rows; an id
// whose tokens lie in several pieces has a partial sum per piece, added in the pieces' order by the block that comes last. No
// floating-point atomics: the order of every sum follows from the ids alone.
#include "ops_internal.h"
#include "rows.cuh"
#include "tcgen05.cuh"

namespace slidedp {

// ---- forward ------------------------------------------------------------------------------------------------

constexpr int kEmbedThreads = 128;
constexpr int kEmbedTokens = 4;     // per block: as many rows under way per thread

struct EmbedParams {
  const void* table;
  const int32_t* ids;
  void* out;
  int64_t table_stride, out_stride;
  int64_t tokens, vocab, hidden;
  int chunks;                       // blocks side by side that a row takes
  float scale;
};

// Bound: HBM, each row read once and written once. One vector of four tokens' rows per thread.
template <typename T, int V>
__global__ void __launch_bounds__(kEmbedThreads) embedding_kernel(const __grid_constant__ EmbedParams p) {
  start_after_previous_kernel();
  typedef typename Raw<T, V>::type R;
  const int64_t t0 = (int64_t)(blockIdx.x / p.chunks) * kEmbedTokens;
  const int64_t col = ((int64_t)(blockIdx.x % p.chunks) * blockDim.x + threadIdx.x) * V;
  if (col >= p.hidden) return;
  int id[kEmbedTokens];
  R a[kEmbedTokens];
#pragma unroll
  for (int k = 0; k < kEmbedTokens; ++k) id[k] = t0 + k < p.tokens ? p.ids[t0 + k] : -1;
#pragma unroll
  for (int k = 0; k < kEmbedTokens; ++k)
    if (id[k] >= 0 && id[k] < p.vocab) a[k] = __ldg(reinterpret_cast<const R*>(static_cast<const T*>(p.table) + id[k] * p.table_stride + col));
#pragma unroll
  for (int k = 0; k < kEmbedTokens; ++k) {
    if (t0 + k >= p.tokens) return;
    float v[V];
    const bool has = id[k] >= 0 && id[k] < p.vocab;
    if (has) to_floats<T, V>(a[k], v);
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = has ? v[e] * p.scale : 0.0f;
    store_values<V>(static_cast<T*>(p.out) + (t0 + k) * p.out_stride + col, v);
  }
}

// ---- sort ---------------------------------------------------------------------------------------------------

constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kSortItems = 4;                  // tokens per thread and turn
constexpr int kMaxDigit = 9;                   // bits per pass
constexpr int kBins = 1 << kMaxDigit;
constexpr int kMaxSortCluster = 8;

struct SortParams {
  const int32_t* ids;
  uint32_t *key[2], *pos[2];     // sorted ids (vocab: absent) and their tokens, the result in [passes % 2]
  uint32_t* used;                // a bit per row of the table
  int32_t* arrived;              // counters of the blocks that have a part of an id's sum
  int64_t used_words, arrived_words;
  int32_t tokens, vocab, per_block;
  int passes, digit;
};
struct SortShared {
  uint32_t count[kSortWarps][kBins];   // of one turn, per warp; then where its first one goes
  uint32_t total[kBins];               // of this block
  uint32_t next[kBins];                // where the next of each digit goes
  uint32_t warp[kSortWarps];
};

// Sorts by digits of up to nine bits, the lowest first, in one cluster whatever the number of tokens: each block has a contiguous
// part of the list. A pass counts the digits, exchanges the counts through distributed shared memory, and moves the tokens in
// turns of 4096: a warp finds equal digits among its lanes, and the counts per warp give every token its place. Bound: latency
// of its steps (8192 tokens, two passes: 4 MB of shared-memory counters go through their zeroing, counting and sums).
__global__ void __launch_bounds__(kSortThreads) sort_tokens_kernel(const __grid_constant__ SortParams p, int cluster) {
  extern __shared__ uint4 dynamic[];
  SortShared& sh = *reinterpret_cast<SortShared*>(dynamic);
  start_after_previous_kernel();
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, rank = blockIdx.x;
  const int from = min((int64_t)rank * p.per_block, (int64_t)p.tokens), to = min((int64_t)from + p.per_block, (int64_t)p.tokens);
  for (int64_t i = (int64_t)rank * kSortThreads + tid; i < p.used_words; i += (int64_t)cluster * kSortThreads) p.used[i] = 0;
  for (int64_t i = (int64_t)rank * kSortThreads + tid; i < p.arrived_words; i += (int64_t)cluster * kSortThreads) p.arrived[i] = 0;
  const uint32_t mask = (1u << p.digit) - 1;
  const int bins = 1 << p.digit;
  for (int pass = 0; pass < p.passes; ++pass) {
    const int shift = pass * p.digit, dst = (pass + 1) & 1;
    const auto key_at = [&](int i) -> uint32_t {
      if (pass > 0) return __ldcg(p.key[pass & 1] + i);
      const int id = p.ids[i];
      return id >= 0 && id < p.vocab ? id : p.vocab;
    };
    for (int b = tid; b < bins; b += kSortThreads) sh.total[b] = 0;
    __syncthreads();
    for (int i0 = from; i0 < to; i0 += kSortThreads) {
      const int i = i0 + tid;
      const uint32_t d = i < to ? key_at(i) >> shift & mask : kBins;
      const uint32_t same = __match_any_sync(0xffffffffu, d);
      if (d < (uint32_t)bins && lane == __ffs(same) - 1) atomicAdd(&sh.total[d], __popc(same));
    }
    if (cluster > 1) cluster_sync(); else __syncthreads();
    // exclusive sums over the digits, and within a digit over the blocks
    uint32_t before = 0, all = 0;
    if (tid < bins) {
      for (int r = 0; r < cluster; ++r) {
        uint32_t c;
        if (cluster > 1) asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(c) : "r"(peer_addr(smem_addr(&sh.total[tid]), r)));
        else c = sh.total[tid];
        if (r < rank) before += c;
        all += c;
      }
    }
    uint32_t sum = all;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t x = __shfl_up_sync(0xffffffffu, sum, o);
      if (lane >= o) sum += x;
    }
    if (lane == 31) sh.warp[warp] = sum;
    __syncthreads();
    uint32_t ahead = 0;
    for (int w = 0; w < warp; ++w) ahead += sh.warp[w];
    if (tid < bins) sh.next[tid] = ahead + sum - all + before;
    for (int i0 = from; i0 < to; i0 += kSortThreads * kSortItems) {
      for (int b = tid; b < kSortWarps * bins; b += kSortThreads) sh.count[b / bins][b % bins] = 0;
      __syncthreads();
      uint32_t k[kSortItems], place[kSortItems];
      const int first = i0 + warp * 32 * kSortItems + lane;
#pragma unroll
      for (int j = 0; j < kSortItems; ++j) k[j] = first + 32 * j < to ? key_at(first + 32 * j) : 0;
#pragma unroll
      for (int j = 0; j < kSortItems; ++j) {
        const bool on = first + 32 * j < to;
        const uint32_t d = on ? k[j] >> shift & mask : kBins;
        const uint32_t same = __match_any_sync(0xffffffffu, d);
        const uint32_t prior = on ? sh.count[warp][d] : 0;
        __syncwarp();
        if (on && lane == __ffs(same) - 1) sh.count[warp][d] = prior + __popc(same);
        __syncwarp();
        place[j] = prior + __popc(same & ((1u << lane) - 1));
      }
      __syncthreads();
      for (int b = tid; b < bins; b += kSortThreads) {
        uint32_t at = sh.next[b];
        for (int w = 0; w < kSortWarps; ++w) {
          const uint32_t c = sh.count[w][b];
          sh.count[w][b] = at;
          at += c;
        }
        sh.next[b] = at;
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < kSortItems; ++j) {
        const int i = first + 32 * j;
        if (i >= to) continue;
        const uint32_t at = sh.count[warp][k[j] >> shift & mask] + place[j];
        p.key[dst][at] = k[j];
        p.pos[dst][at] = pass > 0 ? __ldcg(p.pos[pass & 1] + i) : i;
        if (pass == p.passes - 1 && k[j] < (uint32_t)p.vocab) atomicOr(&p.used[k[j] / 32], 1u << k[j] % 32);
      }
      __syncthreads();
    }
    // what the others have written is read in the next pass, and nobody clears counts that are still being read
    __threadfence();
    if (cluster > 1) cluster_sync(); else __syncthreads();
  }
}

// ---- sums ---------------------------------------------------------------------------------------------------

struct EmbedGradParams {
  const uint32_t *key, *pos;     // sorted
  const uint32_t* used;
  int32_t* arrived;              // [pieces][chunks]
  float* partial;                // [pieces][2][hidden]: of an id that began before the piece, of one that goes on behind it
  const void* d_out;
  void* d_table;
  int64_t d_out_stride, d_table_stride;
  int64_t vocab, hidden;
  int32_t tokens, piece, pieces, chunks;
  int accumulate;
  float scale;
};

constexpr int kMaxPiece = 128;
constexpr int kClearRows = 32;   // rows of the table that a block of the second kind looks after: a word of `used`

// The first of [lo, hi) in the sorted keys that is not below `key`, by all lanes of a warp.
__device__ __forceinline__ int first_not_below(const uint32_t* keys, int lo, int hi, uint32_t key) {
  const int lane = threadIdx.x % 32;
  while (lo < hi) {
    const int step = (hi - lo + 31) / 32, i = lo + lane * step;
    const uint32_t below = __ballot_sync(0xffffffffu, i < hi && keys[i] < key);
    const int n = __popc(below);      // probes below come first
    if (n == 0) return lo;
    const int l = lo + (n - 1) * step + 1, h = min(hi, lo + n * step);
    lo = l;
    hi = h;
  }
  return lo;
}

// The first `pieces * chunks` blocks sum pieces; the others write the zeros of rows that no token has.
template <typename T, typename G, int V>
__global__ void __launch_bounds__(kEmbedThreads) embedding_sum_kernel(const __grid_constant__ EmbedGradParams p) {
  start_after_previous_kernel();
  typedef typename Raw<T, V>::type R;
  __shared__ uint32_t key[kMaxPiece + 2], pos[kMaxPiece];
  __shared__ int last;
  G* table = static_cast<G*>(p.d_table);
  if (blockIdx.x >= (unsigned)(p.pieces * p.chunks)) {
    const int64_t w = blockIdx.x - p.pieces * p.chunks;
    const uint32_t used = p.used[w];
    const float zero[V] = {};
    for (int r = 0; r < kClearRows && w * kClearRows + r < p.vocab; ++r)
      if (!(used >> r & 1))
        for (int64_t c = threadIdx.x * V; c < p.hidden; c += blockDim.x * V) store_values<V>(table + (w * kClearRows + r) * p.d_table_stride + c, zero);
    return;
  }
  const int piece = blockIdx.x / p.chunks, chunk = blockIdx.x % p.chunks;
  const int from = piece * p.piece, n = min(p.piece, p.tokens - from);
  for (int i = threadIdx.x; i < n + 2; i += blockDim.x) {     // one on either side
    const int at = from + i - 1;
    key[i] = at >= 0 && at < p.tokens ? p.key[at] : 0xffffffffu;
    if (i >= 1 && i <= n) pos[i - 1] = p.pos[at];
  }
  __syncthreads();
  const int64_t col = ((int64_t)chunk * blockDim.x + threadIdx.x) * V;
  const bool on = col < p.hidden;
  const T* src = static_cast<const T*>(p.d_out) + (on ? col : 0);
  constexpr int U = 8;
  R a[U];
  float sum[V] = {};
  int begin = 0;                       // of the present id within the piece
  for (int i0 = 0; i0 < n && key[i0 + 1] < (uint32_t)p.vocab; i0 += U) {
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (on && i0 + u < n && key[i0 + u + 1] < (uint32_t)p.vocab) a[u] = __ldcs(reinterpret_cast<const R*>(src + pos[i0 + u] * p.d_out_stride));
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u;
      if (i >= n || key[i + 1] >= (uint32_t)p.vocab) break;
      const uint32_t id = key[i + 1];
      float v[V] = {};
      if (on) to_floats<T, V>(a[u], v);
#pragma unroll
      for (int e = 0; e < V; ++e) sum[e] += v[e];
      const bool ends = i + 1 == n;
      if (!ends && key[i + 2] == id) continue;
      const bool before = begin == 0 && key[0] == id, behind = ends && key[i + 2] == id;
      bool write = true;
      if (before || behind) {
        const int first = before ? first_not_below(p.key, 0, from, id) / p.piece : piece;
        const int final = behind ? (first_not_below(p.key, from + n, p.tokens, id + 1) - 1) / p.piece : piece;
        if (on) {
#pragma unroll
          for (int e = 0; e < V; ++e) p.partial[((int64_t)piece * 2 + (before ? 0 : 1)) * p.hidden + col + e] = sum[e];
        }
        __threadfence();
        __syncthreads();
        if (threadIdx.x == 0) last = atomicAdd(&p.arrived[(int64_t)first * p.chunks + chunk], 1) == final - first;
        __syncthreads();
        write = last;
        if (write) {
          __threadfence();
          // in its first piece the id's part is in the second place, in the others in the first
          if (on) {
#pragma unroll
            for (int e = 0; e < V; ++e) {
              const float* at = p.partial + (int64_t)first * 2 * p.hidden + col + e;
              float s = __ldcg(at + p.hidden);
              for (int k = 1; k <= final - first; ++k) s += __ldcg(at + (int64_t)k * 2 * p.hidden);
              sum[e] = s;
            }
          }
        }
      }
      if (write && on) {
        G* to = table + id * p.d_table_stride + col;
#pragma unroll
        for (int e = 0; e < V; ++e) sum[e] *= p.scale;
        if (p.accumulate) {
          float old[V];
          load_values<V>(to, old);
#pragma unroll
          for (int e = 0; e < V; ++e) sum[e] += old[e];
        }
        store_values<V>(to, sum);
      }
#pragma unroll
      for (int e = 0; e < V; ++e) sum[e] = 0.0f;
      begin = i + 1;
    }
  }
}

}  // namespace slidedp

using namespace slidedp;
using namespace slidedp::host;

namespace {

constexpr int64_t kMaxHidden = 1 << 20;

int check_embedding(const slidedp_embedding_args* a) {
  const auto type = [](int32_t t) { return t == SLIDEDP_BF16 || t == SLIDEDP_F32; };
  if (!a || a->tokens < 0 || a->tokens > kMaxTokens || a->vocab < 1 || a->vocab > kMaxTokens || a->hidden < 1 || a->hidden > kMaxHidden ||
      !type(a->dtype) || !type(a->grad_dtype) || (a->accumulate != 0 && a->accumulate != 1) || !fits_f32(a->scale))
    return SLIDEDP_ERR_INVALID_ARG;
  return SLIDEDP_OK;
}

struct Split {
  unsigned threads;
  int chunks;
};
Split split_row(int64_t hidden, int v) {
  const int64_t vectors = (hidden + v - 1) / v;
  const unsigned threads = vectors >= kEmbedThreads ? kEmbedThreads : (unsigned)((vectors + 31) / 32 * 32);
  return Split{threads, (int)((vectors + threads - 1) / threads)};
}

// Tokens per piece: short ones where there are few tokens, so that they fill the SMs; the partial sums are at most 2 / piece of the
// tokens' rows in FP32.
int piece_length(int64_t tokens) { return tokens <= 16384 ? 16 : tokens <= 131072 ? 32 : kMaxPiece; }

// The workspace: sorted keys and tokens twice, the used rows' bits, counters, partial sums.
struct Layout {
  int64_t keys, used_words, arrived_words, pieces, bytes;
  int64_t used_at, arrived_at, partial_at;
};
Layout layout(const slidedp_embedding_args* a) {
  Layout l;
  const int piece = piece_length(a->tokens);
  const auto up = [](int64_t b) { return (b + 15) / 16 * 16; };
  l.keys = up(a->tokens * 4);
  l.pieces = (a->tokens + piece - 1) / piece;
  l.used_words = (a->vocab + 31) / 32;
  l.arrived_words = l.pieces * split_row(a->hidden, 1).chunks;
  l.used_at = 4 * l.keys;
  l.arrived_at = l.used_at + up(l.used_words * 4);
  l.partial_at = l.arrived_at + up(l.arrived_words * 4);
  l.bytes = l.partial_at + l.pieces * 2 * a->hidden * 4;
  return l;
}

int sort_tokens(slidedp_ctx* ctx, const slidedp_embedding_args* a, const int32_t* ids, const Layout& l, char* ws, int* result, cudaStream_t st) {
  SortParams p = {};
  p.ids = ids;
  for (int i = 0; i < 2; ++i) {
    p.key[i] = reinterpret_cast<uint32_t*>(ws + i * l.keys);
    p.pos[i] = reinterpret_cast<uint32_t*>(ws + (2 + i) * l.keys);
  }
  p.used = reinterpret_cast<uint32_t*>(ws + l.used_at);
  p.arrived = reinterpret_cast<int32_t*>(ws + l.arrived_at);
  p.used_words = l.used_words;
  p.arrived_words = l.arrived_words;
  p.tokens = (int32_t)a->tokens;
  p.vocab = (int32_t)a->vocab;
  int bits = 1;
  while (a->vocab >> bits) ++bits;       // the absent ones' key is vocab
  p.passes = (bits + kMaxDigit - 1) / kMaxDigit;
  p.digit = (bits + p.passes - 1) / p.passes;
  int cluster = 1;
  while (cluster < kMaxSortCluster && a->tokens > (int64_t)cluster * kSortThreads) cluster *= 2;
  p.per_block = (int32_t)((a->tokens + cluster - 1) / cluster);
  CU(cudaFuncSetAttribute(sort_tokens_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(SortShared)));
  FAULT_POINT();
  launch_after(sort_tokens_kernel, dim3(cluster), kSortThreads, sizeof(SortShared), cluster, st, p, cluster);
  ctx->launches += 1;
  CU_AFTER_LAUNCH();
  *result = p.passes & 1;
  return SLIDEDP_OK;
}

}  // namespace

extern "C" {

int slidedp_embedding(slidedp_ctx* ctx, const slidedp_embedding_args* a, const slidedp_rows* table, const int32_t* ids, const slidedp_rows* out,
                      void* cuda_stream) {
  if (!ctx || check_embedding(a) != SLIDEDP_OK) return SLIDEDP_ERR_INVALID_ARG;
  if (a->tokens == 0) return SLIDEDP_OK;
  const int elem = elem_bytes(a->dtype);
  if (!rows_ok(table, elem, a->vocab, a->hidden, false) || !rows_ok(out, elem, a->tokens, a->hidden, true) || !ids ||
      reinterpret_cast<uintptr_t>(ids) % 4 != 0 || out->data == table->data)
    return SLIDEDP_ERR_INVALID_ARG;
  const int v = vector_width(a->hidden, elem, {{table, elem}, {out, elem}});
  const Split s = split_row(a->hidden, v);
  const int64_t blocks = (a->tokens + kEmbedTokens - 1) / kEmbedTokens * s.chunks;
  if (blocks > 0x7fffffff) return SLIDEDP_ERR_INVALID_ARG;
  const EmbedParams p = {table->data, ids, out->data, table->stride, out->stride, a->tokens, a->vocab, a->hidden, s.chunks, (float)a->scale};
  const int rc = check_kernel_error(ctx);
  if (rc != SLIDEDP_OK) return rc;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return cuda_fail(ctx, cudaGetLastError());
  FAULT_POINT();
  const auto run = [&](auto kernel) { launch_after(kernel, dim3((unsigned)blocks), s.threads, 0, 1, static_cast<cudaStream_t>(cuda_stream), p); };
  if (elem == 4) v == 4 ? run(embedding_kernel<float, 4>) : run(embedding_kernel<float, 1>);
  else v == 8 ? run(embedding_kernel<uint16_t, 8>) : v == 2 ? run(embedding_kernel<uint16_t, 2>) : run(embedding_kernel<uint16_t, 1>);
  ctx->launches += 1;
  CU_AFTER_LAUNCH();
  return SLIDEDP_OK;
}

size_t slidedp_embedding_workspace(const slidedp_embedding_args* a) {
  return check_embedding(a) == SLIDEDP_OK ? (size_t)layout(a).bytes + 16 : 0;
}

int slidedp_embedding_backward(slidedp_ctx* ctx, const slidedp_embedding_args* a, const int32_t* ids, const slidedp_rows* d_out,
                               const slidedp_rows* d_table, void* workspace, void* cuda_stream) {
  if (!ctx || check_embedding(a) != SLIDEDP_OK) return SLIDEDP_ERR_INVALID_ARG;
  const int elem = elem_bytes(a->dtype), grad = elem_bytes(a->grad_dtype);
  if (!rows_ok(d_table, grad, a->vocab, a->hidden, true) || !workspace ||
      (a->tokens > 0 && (!rows_ok(d_out, elem, a->tokens, a->hidden, false) || !ids || reinterpret_cast<uintptr_t>(ids) % 4 != 0 ||
                         d_out->data == d_table->data)))
    return SLIDEDP_ERR_INVALID_ARG;
  if (!aligned16(workspace)) return SLIDEDP_ERR_MISALIGNED;
  if (a->tokens == 0 && a->accumulate) return SLIDEDP_OK;
  const slidedp_rows none = {nullptr, 0};
  if (a->tokens == 0) d_out = &none;
  const int v = vector_width(a->hidden, elem, {{d_out, elem}, {d_table, grad}});
  const Split s = split_row(a->hidden, v);
  const Layout l = layout(a);
  const int64_t sums = l.pieces * s.chunks, blocks = sums + (a->accumulate ? 0 : l.used_words);
  if (blocks > 0x7fffffff) return SLIDEDP_ERR_INVALID_ARG;
  int rc = check_kernel_error(ctx);
  if (rc != SLIDEDP_OK) return rc;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return cuda_fail(ctx, cudaGetLastError());
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  char* ws = static_cast<char*>(workspace);
  int sorted;
  rc = sort_tokens(ctx, a, ids, l, ws, &sorted, st);
  if (rc != SLIDEDP_OK) return rc;
  EmbedGradParams p = {};
  p.key = reinterpret_cast<uint32_t*>(ws + sorted * l.keys);
  p.pos = reinterpret_cast<uint32_t*>(ws + (2 + sorted) * l.keys);
  p.used = reinterpret_cast<uint32_t*>(ws + l.used_at);
  p.arrived = reinterpret_cast<int32_t*>(ws + l.arrived_at);
  p.partial = reinterpret_cast<float*>(ws + l.partial_at);
  p.d_out = d_out->data;
  p.d_table = d_table->data;
  p.d_out_stride = d_out->stride;
  p.d_table_stride = d_table->stride;
  p.vocab = a->vocab;
  p.hidden = a->hidden;
  p.tokens = (int32_t)a->tokens;
  p.piece = piece_length(a->tokens);
  p.pieces = (int32_t)l.pieces;
  p.chunks = s.chunks;
  p.accumulate = a->accumulate;
  p.scale = (float)a->scale;
  FAULT_POINT();
  const auto run = [&](auto kernel) { launch_after(kernel, dim3((unsigned)blocks), s.threads, 0, 1, st, p); };
  if (elem == 4) {
    if (grad == 4) v == 4 ? run(embedding_sum_kernel<float, float, 4>) : run(embedding_sum_kernel<float, float, 1>);
    else v == 4 ? run(embedding_sum_kernel<float, uint16_t, 4>) : run(embedding_sum_kernel<float, uint16_t, 1>);
  } else if (grad == 4) {
    v == 8 ? run(embedding_sum_kernel<uint16_t, float, 8>) : v == 2 ? run(embedding_sum_kernel<uint16_t, float, 2>) : run(embedding_sum_kernel<uint16_t, float, 1>);
  } else {
    v == 8 ? run(embedding_sum_kernel<uint16_t, uint16_t, 8>) : v == 2 ? run(embedding_sum_kernel<uint16_t, uint16_t, 2>) : run(embedding_sum_kernel<uint16_t, uint16_t, 1>);
  }
  ctx->launches += 1;
  CU_AFTER_LAUNCH();
  return SLIDEDP_OK;
}

}  // extern "C"
