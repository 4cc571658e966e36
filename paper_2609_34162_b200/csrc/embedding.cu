// libslidedp: token embedding with scaling, and the table's gradient by sorted tokens. See include/slidedp_ops.h for the contract.
//
// out[t] = s table[id t];  d_table[v] = s sum of d_out[t] over id t = v.  Bound: HBM.
// The gradient is three kernels. The first sorts the tokens by id, stably, so that each id's tokens stand together in their
// order; meanwhile the SMs that it leaves idle clear part of the table. The second cuts the sorted list into pieces and sums their
// rows, and clears what is left; the tokens of an id that has many are cut where the pieces are, however often it occurs, and have a
// partial sum per piece, which the third adds in the pieces' order. No atomics, no waiting for other blocks: the order of every sum
// follows from the ids alone.
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

// A thread's values of a row: K vectors of V, blockDim vectors apart, so that narrow ones (rows that are not aligned) come in numbers.
template <int V> constexpr int vectors_per_thread = V == 1 ? 4 : V == 2 ? 2 : 1;

// Bound: HBM, each row read once and written once. K vectors of four tokens' rows per thread. 8192 tokens of 4096 BF16 columns out of
// 131072 rows: 17.8 us (134 MB, some of it still in L2); 32749 of 1000 FP32: 24.6.
template <typename T, int V>
__global__ void __launch_bounds__(kEmbedThreads) embedding_kernel(const __grid_constant__ EmbedParams p) {
  start_after_previous_kernel();
  typedef typename Raw<T, V>::type R;
  constexpr int K = vectors_per_thread<V>;
  const int64_t t0 = (int64_t)(blockIdx.x / p.chunks) * kEmbedTokens;
  const int64_t first = (int64_t)(blockIdx.x % p.chunks) * K * blockDim.x + threadIdx.x;
  int id[kEmbedTokens];
  R a[kEmbedTokens][K];
#pragma unroll
  for (int t = 0; t < kEmbedTokens; ++t) id[t] = t0 + t < p.tokens ? p.ids[t0 + t] : -1;
#pragma unroll
  for (int t = 0; t < kEmbedTokens; ++t) {
    if (id[t] < 0 || id[t] >= p.vocab) continue;
    const T* row = static_cast<const T*>(p.table) + id[t] * p.table_stride;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int64_t col = (first + k * blockDim.x) * V;
      if (col < p.hidden) a[t][k] = __ldg(reinterpret_cast<const R*>(row + col));
    }
  }
#pragma unroll
  for (int t = 0; t < kEmbedTokens; ++t) {
    if (t0 + t >= p.tokens) return;
    const bool has = id[t] >= 0 && id[t] < p.vocab;
    T* row = static_cast<T*>(p.out) + (t0 + t) * p.out_stride;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int64_t col = (first + k * blockDim.x) * V;
      float v[V] = {};
      if (has && col < p.hidden) to_floats<T, V>(a[t][k], v);
#pragma unroll
      for (int e = 0; e < V; ++e) v[e] = has ? v[e] * p.scale : 0.0f;
      if (col < p.hidden) store_values<V>(row + col, v);
    }
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
  uint2* item[2];                // ids (vocab: absent) and their tokens, sorted in [passes % 2]
  uint32_t* used;                // a bit per row of the table
  int32_t* cut;                  // how many runs are cut
  int64_t used_words;
  int32_t tokens, vocab, per_block, per_lane;
  int passes, digit;
  char* clear;                   // rows [0, clear_rows) of the table, each `clear_vectors` of clear_width bytes
  int64_t clear_stride;
  uint32_t clear_rows, clear_vectors;
  int clear_width;
};
struct SortShared {
  uint32_t count[kSortWarps][kBins];   // of one turn, per warp; then where in the turn's tokens of that digit its first one stands
  uint32_t total[kBins];               // of this block
  uint32_t next[kBins];                // where the next of each digit goes
  uint32_t warp[kSortWarps];
  uint2 moved[kSortThreads * kSortItems];   // this block's part of the list between two passes, if it is one turn
};

// Sorts by digits of up to nine bits, the lowest first, in one cluster whatever the number of tokens: each block has a contiguous
// part of the list. A pass counts the digits, exchanges the counts through distributed shared memory, and moves the tokens in
// turns of 4096: a warp finds equal digits among its lanes, and the counts per warp give every token its place. Blocks whose part is
// one turn find the places first and have their counts from them, and pass tokens on through each other's shared memory. Bound:
// latency of its steps, a barrier of the cluster being 1 us: 32749 tokens, two passes, 20 us.
__device__ __forceinline__ void clear_rows(const SortParams& p, uint32_t block, uint32_t blocks) {
  const uint32_t all = p.clear_rows * p.clear_vectors;
  for (uint32_t i = block * kSortThreads + threadIdx.x; i < all; i += blocks * kSortThreads) {
    char* to = p.clear + (int64_t)(i / p.clear_vectors) * p.clear_stride + (int64_t)(i % p.clear_vectors) * p.clear_width;
    if (p.clear_width == 16) st_stream(to, make_uint4(0, 0, 0, 0));
    else if (p.clear_width == 4) __stcs(reinterpret_cast<uint32_t*>(to), 0u);
    else __stcs(reinterpret_cast<uint16_t*>(to), (uint16_t)0);
  }
}
__global__ void __launch_bounds__(kSortThreads) sort_tokens_kernel(const __grid_constant__ SortParams p, int cluster) {
  extern __shared__ uint4 dynamic[];
  SortShared& sh = *reinterpret_cast<SortShared*>(dynamic);
  start_after_previous_kernel();
  if ((int)blockIdx.x >= cluster) return clear_rows(p, blockIdx.x - cluster, gridDim.x - cluster);   // whole clusters of them
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, rank = blockIdx.x;
  const int from = min((int64_t)rank * p.per_block, (int64_t)p.tokens), to = min((int64_t)from + p.per_block, (int64_t)p.tokens);
  const bool one_turn = p.per_block <= kSortThreads * kSortItems;
  const uint32_t mask = (1u << p.digit) - 1;
  const int bins = 1 << p.digit;
  uint2 item[kSortItems];        // of this turn: id and token
  uint32_t place[kSortItems];    // among the warp's tokens of the same digit
  int source = 0, shift = 0;
  const auto fetch = [&](int i0) {
    const int first = i0 + warp * 32 * p.per_lane + lane;
#pragma unroll
    for (int j = 0; j < kSortItems; ++j) {
      const int i = first + 32 * j;
      if (j >= p.per_lane || i >= to) continue;
      if (shift > 0) {
        item[j] = one_turn ? sh.moved[i - from] : __ldcg(p.item[source] + i);
      } else {
        const int id = p.ids[i];
        item[j] = make_uint2(id >= 0 && id < p.vocab ? id : p.vocab, i);
      }
    }
  };
  // places of a turn's tokens, and the turn's number of each digit in one thread per digit
  const auto rank_turn = [&](int i0) -> uint32_t {
    for (int b = tid; b < kSortWarps * bins / 4; b += kSortThreads)
      reinterpret_cast<uint4*>(sh.count[b * 4 / bins])[(b * 4 % bins) / 4] = make_uint4(0, 0, 0, 0);
    __syncthreads();
    const int first = i0 + warp * 32 * p.per_lane + lane;
    uint32_t same[kSortItems];
#pragma unroll
    for (int j = 0; j < kSortItems; ++j)
      if (j < p.per_lane) same[j] = __match_any_sync(0xffffffffu, first + 32 * j < to ? item[j].x >> shift & mask : kBins);
#pragma unroll
    for (int j = 0; j < kSortItems; ++j) {
      if (j >= p.per_lane) break;
      const bool on = first + 32 * j < to;
      const uint32_t d = item[j].x >> shift & mask;
      const uint32_t prior = on ? sh.count[warp][d] : 0;
      __syncwarp();
      if (on && lane == __ffs(same[j]) - 1) sh.count[warp][d] = prior + __popc(same[j]);
      __syncwarp();
      place[j] = prior + __popc(same[j] & ((1u << lane) - 1));
    }
    __syncthreads();
    uint32_t sum = 0;
    if (tid < bins) {
      uint32_t c[kSortWarps];
#pragma unroll
      for (int w = 0; w < kSortWarps; ++w) c[w] = sh.count[w][tid];
#pragma unroll
      for (int w = 0; w < kSortWarps; ++w) {
        sh.count[w][tid] = sum;
        sum += c[w];
      }
    }
    return sum;
  };
  if (rank == 0 && tid == 0) *p.cut = 0;
  for (int64_t i = (int64_t)rank * kSortThreads + tid; i < p.used_words; i += (int64_t)cluster * kSortThreads) p.used[i] = 0;
  for (int pass = 0; pass < p.passes; ++pass, shift += p.digit, source = pass & 1) {
    if (one_turn) {
      fetch(from);
      const uint32_t sum = rank_turn(from);
      if (tid < bins) sh.total[tid] = sum;
    } else {
      for (int b = tid; b < bins; b += kSortThreads) sh.total[b] = 0;
      __syncthreads();
      for (int i0 = from; i0 < to; i0 += kSortThreads * kSortItems) {
        fetch(i0);
        const int first = i0 + warp * 32 * p.per_lane + lane;
#pragma unroll
        for (int j = 0; j < kSortItems; ++j) {
          if (j >= p.per_lane) break;
          const uint32_t d = first + 32 * j < to ? item[j].x >> shift & mask : kBins;
          const uint32_t same = __match_any_sync(0xffffffffu, d);
          if (d < (uint32_t)bins && lane == __ffs(same) - 1) atomicAdd(&sh.total[d], __popc(same));
        }
      }
    }
    if (cluster > 1) cluster_sync(); else __syncthreads();
    // exclusive sums over the digits, and within a digit over the blocks
    uint32_t before = 0, all = 0;
    if (tid < bins) {
      uint32_t c[kMaxSortCluster] = {};
#pragma unroll
      for (int r = 0; r < kMaxSortCluster; ++r) {
        if (r >= cluster) break;
        if (cluster > 1) asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(c[r]) : "r"(peer_addr(smem_addr(&sh.total[tid]), r)));
        else c[r] = sh.total[tid];
      }
#pragma unroll
      for (int r = 0; r < kMaxSortCluster; ++r) {
        if (r < rank) before += c[r];
        all += c[r];
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
    if (tid < bins) {
      uint32_t ahead = 0;
      for (int w = 0; w < warp; ++w) ahead += sh.warp[w];
      sh.next[tid] = ahead + sum - all + before;
    }
    __syncthreads();
    for (int i0 = from; i0 < to; i0 += kSortThreads * kSortItems) {
      uint32_t turn = 0;
      if (!one_turn) {
        fetch(i0);
        turn = rank_turn(i0);
        __syncthreads();
      }
      const int first = i0 + warp * 32 * p.per_lane + lane;
#pragma unroll
      for (int j = 0; j < kSortItems; ++j) {
        if (j >= p.per_lane || first + 32 * j >= to) continue;
        const uint32_t d = item[j].x >> shift & mask, at = sh.next[d] + sh.count[warp][d] + place[j];
        if (!one_turn || pass == p.passes - 1) {
          p.item[(pass + 1) & 1][at] = item[j];
        } else if (cluster > 1) {
          const uint32_t there = peer_addr(smem_addr(&sh.moved[at % (uint32_t)p.per_block]), at / (uint32_t)p.per_block);
          asm volatile("st.shared::cluster.v2.u32 [%0], {%1, %2};" ::"r"(there), "r"(item[j].x), "r"(item[j].y) : "memory");
        } else {
          sh.moved[at] = item[j];
        }
      }
      __syncthreads();
      if (!one_turn && tid < bins) sh.next[tid] += turn;
    }
    // what the others have written is read in the next pass, and nobody clears counts that are still being read, or leaves
    if (cluster > 1) cluster_sync(); else __syncthreads();
  }
  // the rows that are used, by the first token of each
  if (p.used_words > 0)
    for (int i = from + tid; i < to; i += kSortThreads) {
      const uint32_t id = __ldcg(p.item[source] + i).x;
      if (id < (uint32_t)p.vocab && (i == 0 || __ldcg(p.item[source] + i - 1).x != id)) atomicOr(&p.used[id / 32], 1u << id % 32);
    }
}

// ---- sums ---------------------------------------------------------------------------------------------------

struct EmbedGradParams {
  const uint2* item;             // sorted: id and token
  const uint32_t* used;
  int32_t* cut;                  // how many runs are cut, then the pieces where they begin, in any order
  float* partial;                // [pieces][2][hidden]: of an id that began before the piece, of one that goes on behind it
  const void* d_out;
  void* d_table;
  int64_t d_out_stride, d_table_stride;
  int64_t vocab, hidden;
  int32_t tokens, piece, pieces, chunks;
  int accumulate;
  int32_t first_clear;           // the first word of `used` whose rows are to be cleared here
  float scale;
};

constexpr int kMaxPiece = 128;
constexpr int kLongRun = 32;     // ids with more tokens are cut where pieces are; the others belong to the piece where they begin
constexpr int kClearRows = 32;   // rows of the table that a block of the second kind looks after: a word of `used`

// By all lanes of a warp: where the run of `id` ends that has `begin`. Most end within 32 places; the others are found by looking at 32
// places at a time.
__device__ __forceinline__ int run_end(const uint2* item, int begin, int tokens, uint32_t id) {
  const int lane = threadIdx.x % 32, near = begin + lane;
  const uint32_t other = __ballot_sync(0xffffffffu, near >= tokens || item[near].x != id);
  if (other) return begin + __ffs(other) - 1;
  int lo = begin + 32, hi = tokens;                // the first of [lo, hi] that is above
  while (lo < hi) {
    const int step = (hi - lo + 31) / 32, i = lo + lane * step;
    const int n = __popc(__ballot_sync(0xffffffffu, i < hi && item[i].x <= id));
    if (n == 0) return lo;
    lo += (n - 1) * step + 1;
    hi = min(hi, lo - 1 + step);
  }
  return lo;
}

// A thread's columns of a row are K vectors of V, `step` vectors apart from `first` on. Their sums, scaled and added to what is there, to a
// row of the table.
template <typename G, int V>
__device__ __forceinline__ void write_columns(G* row, int64_t first, int step, int64_t hidden, const float* sum, float scale, bool accumulate) {
#pragma unroll
  for (int k = 0; k < vectors_per_thread<V>; ++k) {
    const int64_t col = (first + k * step) * V;
    if (col >= hidden) continue;
    float v[V];
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = sum[k * V + e] * scale;
    if (accumulate) {
      float old[V];
      load_values<V>(row + col, old);
#pragma unroll
      for (int e = 0; e < V; ++e) v[e] += old[e];
    }
    store_values<V>(row + col, v);
  }
}

// Bound: HBM, and for tables with few rows the chain of additions of the ids that occur often. 32749 tokens of 1000 FP32 columns: 27 us
// (8 rows under way in place of 4: 60 us for all three kernels where these take 55), 8192 of 4096 BF16 with a table of 131072 rows, whose
// zeros are most of it: 182 for all three.
// The first `pieces * chunks` blocks sum pieces; the others write the zeros of rows that no token has. A thread has four rows under way
// while it adds the four before them.
template <typename T, typename G, int V>
__global__ void __launch_bounds__(kEmbedThreads) embedding_sum_kernel(const __grid_constant__ EmbedGradParams p) {
  start_after_previous_kernel();
  typedef typename Raw<T, V>::type R;
  constexpr int K = vectors_per_thread<V>, N = K * V, U = 4, W = kLongRun;
  __shared__ uint32_t key[kMaxPiece + 2 * W], pos[kMaxPiece + 2 * W];     // of the piece and 32 tokens on either side
  __shared__ int64_t offset[kMaxPiece + 2 * W];
  __shared__ uint8_t what[kMaxPiece + 2 * W];
  G* table = static_cast<G*>(p.d_table);
  if (blockIdx.x >= (unsigned)(p.pieces * p.chunks)) {
    const int64_t w = p.first_clear + (int64_t)(blockIdx.x - p.pieces * p.chunks);
    const uint32_t used = p.used[w];
    const float zero[V] = {};
    for (int r = 0; r < kClearRows && w * kClearRows + r < p.vocab; ++r)
      if (!(used >> r & 1))
        for (int64_t c = threadIdx.x * V; c < p.hidden; c += blockDim.x * V) store_values<V>(table + (w * kClearRows + r) * p.d_table_stride + c, zero);
    return;
  }
  const int piece = blockIdx.x / p.chunks, from = piece * p.piece, n = min(p.piece, p.tokens - from), lane = threadIdx.x % 32;
  const uint32_t absent = (uint32_t)p.vocab;
  for (int i = threadIdx.x; i < n + 2 * W; i += blockDim.x) {
    const int at = from + i - W;
    const uint2 it = at >= 0 && at < p.tokens ? p.item[at] : make_uint2(0xffffffffu, 0);
    key[i] = it.x;
    pos[i] = it.y;
  }
  __syncthreads();
  // places are counted in the window: the piece is [W, end), less absent tokens, which come last
  int end = W + n;
  const uint32_t head = key[W];
  if (head >= absent) return;
  for (int at = W; at < W + n; at += 32) {
    const uint32_t none = __ballot_sync(0xffffffffu, at + lane < W + n && key[at + lane] >= absent);
    if (none) {
      end = at + __ffs(none) - 1;
      break;
    }
  }
  const uint32_t tail = key[end - 1];
  const auto same_before = [&](int at, uint32_t id) {   // up to W of them
    const uint32_t other = __ballot_sync(0xffffffffu, key[at - 1 - lane] != id);
    return other ? __ffs(other) - 1 : W;
  };
  const auto same_from = [&](int at, uint32_t id) {
    const uint32_t other = __ballot_sync(0xffffffffu, key[at + lane] != id);
    return other ? __ffs(other) - 1 : W;
  };
  int i = W;
  bool cut_head = false, cut_tail = false;               // the part of the first run belongs to one that is cut before; of the last, behind
  const int before = same_before(W, head);
  if (before > 0) {
    const int here = same_from(W, head);
    cut_head = before + here > W;
    if (!cut_head) i += here;                            // the piece before has them
  }
  const int behind = cut_head && tail == head ? 0 : same_from(end, tail);
  if (behind > 0 && i < end) {
    const int here = min(same_before(end, tail), n);     // more than W of them: a long run
    cut_tail = here + behind > W;
    if (!cut_tail) end += behind;
  }
  if (i >= end) return;
  // where each token's row is, and what is to be done after it: nothing yet, the run's sum to the table, or to one of the two places
  for (int at = i + threadIdx.x; at < end; at += blockDim.x) {
    const bool last = at + 1 == end || key[at + 1] != key[at];
    offset[at] = pos[at] * p.d_out_stride;
    what[at] = !last ? 0 : cut_head && key[at] == head ? 2 : cut_tail && at + 1 == end ? 3 : 1;
  }
  __syncthreads();
  const int64_t first = (int64_t)(blockIdx.x % p.chunks) * K * blockDim.x + threadIdx.x;
  const auto col = [&](int k) { return (first + k * blockDim.x) * V; };
  const T* src = static_cast<const T*>(p.d_out);
  R buffer[2][U][K];
  const auto fetch = [&](R (&a)[U][K], int i0) {          // behind the end the last one again
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const T* row = src + offset[min(i0 + u, end - 1)];
#pragma unroll
      for (int k = 0; k < K; ++k)
        if (col(k) < p.hidden) a[u][k] = __ldg(reinterpret_cast<const R*>(row + col(k)));
    }
  };
  float sum[N] = {};
  const auto add = [&](const R (&a)[U][K], int i0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int at = i0 + u;
      if (at >= end) break;
#pragma unroll
      for (int k = 0; k < K; ++k) {
        float v[V] = {};
        if (col(k) < p.hidden) to_floats<T, V>(a[u][k], v);
#pragma unroll
        for (int e = 0; e < V; ++e) sum[k * V + e] += v[e];
      }
      const int todo = what[at];
      if (todo == 0) continue;
      if (todo == 1) {
        write_columns<G, V>(table + key[at] * p.d_table_stride, first, blockDim.x, p.hidden, sum, p.scale, p.accumulate);
      } else {
        if (todo == 3 && blockIdx.x % p.chunks == 0 && threadIdx.x == 0) p.cut[1 + atomicAdd(p.cut, 1)] = piece;
        float* mine = p.partial + ((int64_t)piece * 2 + (todo - 2)) * p.hidden;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
          for (int e = 0; e < V; ++e)
            if (col(k) < p.hidden) mine[col(k) + e] = sum[k * V + e];
      }
#pragma unroll
      for (int e = 0; e < N; ++e) sum[e] = 0.0f;
    }
  };
  fetch(buffer[0], i);
  for (; i < end; i += 2 * U) {
    fetch(buffer[1], i + U);
    add(buffer[0], i);
    fetch(buffer[0], i + 2 * U);
    add(buffer[1], i + U);
  }
}

// Adds the parts of the runs that are cut: in its first piece a run's part is in the second place, in the others in the first. A block has
// the columns of one of its warps; the warps share the parts, and the first adds up what they have.
template <typename G, int V>
__global__ void __launch_bounds__(kEmbedThreads) embedding_join_kernel(const __grid_constant__ EmbedGradParams p, int chunks) {
  start_after_previous_kernel();
  constexpr int K = vectors_per_thread<V>, N = K * V, kWarps = kEmbedThreads / 32;
  __shared__ float sums[kWarps][N][32];
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  for (int work = blockIdx.x; work < p.cut[0] * chunks; work += gridDim.x) {
    const int piece = p.cut[1 + work / chunks], end = (piece + 1) * p.piece;
    const uint32_t id = p.item[end - 1].x;
    const int parts = (run_end(p.item, end, p.tokens, id) - 1) / p.piece - piece + 1, each = (parts + kWarps - 1) / kWarps;
    const int64_t first = (int64_t)(work % chunks) * K * 32 + lane;
    const auto col = [&](int k) { return (first + k * 32) * V; };
    float sum[N] = {};
    constexpr int B = 8;                                 // parts under way
    const int stop = min(parts, (warp + 1) * each);
    for (int q = warp * each; q < stop; q += B) {
      float part[B][N];
#pragma unroll
      for (int b = 0; b < B; ++b) {
        const float* at = p.partial + ((int64_t)(piece + q + b) * 2 + (q + b == 0)) * p.hidden;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
          for (int e = 0; e < V; ++e) part[b][k * V + e] = q + b < stop && col(k) < p.hidden ? at[col(k) + e] : 0.0f;
      }
#pragma unroll
      for (int b = 0; b < B; ++b)
#pragma unroll
        for (int e = 0; e < N; ++e) sum[e] += part[b][e];
    }
#pragma unroll
    for (int e = 0; e < N; ++e) sums[warp][e][lane] = sum[e];
    __syncthreads();
    if (warp == 0) {
#pragma unroll
      for (int w = 1; w < kWarps; ++w)
#pragma unroll
        for (int e = 0; e < N; ++e) sum[e] += sums[w][e][lane];
      write_columns<G, V>(static_cast<G*>(p.d_table) + id * p.d_table_stride, first, 32, p.hidden, sum, p.scale, p.accumulate);
    }
    __syncthreads();
  }
}

}  // namespace slidedp

using namespace slidedp;
using namespace slidedp::host;

namespace {

constexpr int64_t kMaxHidden = 1 << 20;
// What the SMs beside the sort clear of the table: about as much as they can in its time. 148 blocks of 1024 threads in all.
constexpr int64_t kClearBytes = 64 << 20;
constexpr int kSms = 148, kClearBlocks = kSms;

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
  const int64_t per = v == 1 ? vectors_per_thread<1> : v == 2 ? vectors_per_thread<2> : 1, vectors = (hidden + v - 1) / v;
  const int64_t wanted = (vectors + per - 1) / per;
  const unsigned threads = wanted >= kEmbedThreads ? kEmbedThreads : (unsigned)((wanted + 31) / 32 * 32);
  return Split{threads, (int)((wanted + threads - 1) / threads)};
}

// Tokens per piece: as many as make the pieces' blocks one round of the device, 16 to 128. The partial sums are at most 2 / piece of the
// tokens' rows in FP32.
int piece_length(const slidedp_embedding_args* a) {
  const int64_t blocks = a->tokens * split_row(a->hidden, 16 / elem_bytes(a->dtype)).chunks;
  int p = 16;
  while (p < kMaxPiece && blocks > (int64_t)p * kSms * 8) p *= 2;
  return p;
}

// The workspace: ids and tokens twice, the used rows' bits, the pieces where runs are cut, partial sums.
struct Layout {
  int64_t items, used_words, pieces, bytes;
  int64_t used_at, cut_at, partial_at;
};
Layout layout(const slidedp_embedding_args* a) {
  Layout l;
  const int piece = piece_length(a);
  const auto up = [](int64_t b) { return (b + 15) / 16 * 16; };
  l.items = up(a->tokens * 8);
  l.pieces = (a->tokens + piece - 1) / piece;
  l.used_words = (a->vocab + 31) / 32;
  l.used_at = 2 * l.items;
  l.cut_at = l.used_at + up(l.used_words * 4);
  l.partial_at = l.cut_at + up((l.pieces + 1) * 4);
  l.bytes = l.partial_at + l.pieces * 2 * a->hidden * 4;
  return l;
}

int sort_tokens(slidedp_ctx* ctx, const slidedp_embedding_args* a, const int32_t* ids, const Layout& l, const slidedp_rows* d_table,
                int64_t clear_rows, bool all_cleared, char* ws, int* result, cudaStream_t st) {
  SortParams p = {};
  p.ids = ids;
  for (int i = 0; i < 2; ++i) p.item[i] = reinterpret_cast<uint2*>(ws + i * l.items);
  p.used = reinterpret_cast<uint32_t*>(ws + l.used_at);
  p.used_words = all_cleared ? 0 : l.used_words;
  p.cut = reinterpret_cast<int32_t*>(ws + l.cut_at);
  p.tokens = (int32_t)a->tokens;
  p.vocab = (int32_t)a->vocab;
  int bits = 1;
  while (a->vocab >> bits) ++bits;       // the absent ones' key is vocab
  p.passes = (bits + kMaxDigit - 1) / kMaxDigit;
  p.digit = (bits + p.passes - 1) / p.passes;
  if (p.digit < 2) p.digit = 2;          // counters are cleared by fours
  int cluster = 1;
  while (cluster < kMaxSortCluster && a->tokens > (int64_t)cluster * kSortThreads) cluster *= 2;
  p.per_block = (int32_t)((a->tokens + cluster - 1) / cluster);
  p.per_lane = p.per_block >= kSortThreads * kSortItems ? kSortItems : (p.per_block + kSortThreads - 1) / kSortThreads;
  const int64_t elem = elem_bytes(a->grad_dtype);
  const uintptr_t shape = reinterpret_cast<uintptr_t>(d_table->data) | (uintptr_t)(d_table->stride * elem) | (uintptr_t)(a->hidden * elem);
  p.clear = static_cast<char*>(d_table->data);
  p.clear_stride = d_table->stride * elem;
  p.clear_width = shape % 16 == 0 ? 16 : shape % 4 == 0 ? 4 : 2;
  p.clear_vectors = (uint32_t)(a->hidden * elem / p.clear_width);
  p.clear_rows = (uint32_t)clear_rows;
  const int others = clear_rows > 0 ? (kClearBlocks - cluster) / cluster * cluster : 0;
  CU(cudaFuncSetAttribute(sort_tokens_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(SortShared)));
  FAULT_POINT();
  launch_after(sort_tokens_kernel, dim3(cluster + others), kSortThreads, sizeof(SortShared), cluster, st, p, cluster);
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
  // whole words of `used`, as many as are cleared while the tokens are sorted
  int64_t clear_words = a->accumulate ? 0 : kClearBytes / (a->hidden * grad) / kClearRows;
  if (clear_words > l.used_words) clear_words = l.used_words;
  const int64_t clear_rows = clear_words * kClearRows < a->vocab ? clear_words * kClearRows : a->vocab;
  const int64_t sums = l.pieces * s.chunks, blocks = sums + (a->accumulate ? 0 : l.used_words - clear_words);
  if (blocks > 0x7fffffff) return SLIDEDP_ERR_INVALID_ARG;
  int rc = check_kernel_error(ctx);
  if (rc != SLIDEDP_OK) return rc;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return cuda_fail(ctx, cudaGetLastError());
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  char* ws = static_cast<char*>(workspace);
  int sorted;
  rc = sort_tokens(ctx, a, ids, l, d_table, clear_rows, a->accumulate || clear_words == l.used_words, ws, &sorted, st);
  if (rc != SLIDEDP_OK) return rc;
  EmbedGradParams p = {};
  p.item = reinterpret_cast<const uint2*>(ws + sorted * l.items);
  p.used = reinterpret_cast<uint32_t*>(ws + l.used_at);
  p.partial = reinterpret_cast<float*>(ws + l.partial_at);
  p.cut = reinterpret_cast<int32_t*>(ws + l.cut_at);
  p.d_out = d_out->data;
  p.d_table = d_table->data;
  p.d_out_stride = d_out->stride;
  p.d_table_stride = d_table->stride;
  p.vocab = a->vocab;
  p.hidden = a->hidden;
  p.tokens = (int32_t)a->tokens;
  p.piece = piece_length(a);
  p.pieces = (int32_t)l.pieces;
  p.chunks = s.chunks;
  p.accumulate = a->accumulate;
  p.scale = (float)a->scale;
  p.first_clear = (int32_t)clear_words;
  if (blocks > 0) {
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
  }
  if (a->tokens > kLongRun && l.pieces > 1) {
    FAULT_POINT();
    const int64_t columns = 32 * v * (v == 1 ? vectors_per_thread<1> : v == 2 ? vectors_per_thread<2> : 1), chunks = (a->hidden + columns - 1) / columns;
    const int64_t most = a->tokens / (kLongRun + 1) * chunks, joins = most < kSms * 8 ? most : kSms * 8;
    const auto join = [&](auto kernel) { launch_after(kernel, dim3((unsigned)joins), kEmbedThreads, 0, 1, st, p, (int)chunks); };
    if (grad == 4) v == 8 ? join(embedding_join_kernel<float, 8>) : v == 4 ? join(embedding_join_kernel<float, 4>) : v == 2 ? join(embedding_join_kernel<float, 2>) : join(embedding_join_kernel<float, 1>);
    else v == 8 ? join(embedding_join_kernel<uint16_t, 8>) : v == 4 ? join(embedding_join_kernel<uint16_t, 4>) : v == 2 ? join(embedding_join_kernel<uint16_t, 2>) : join(embedding_join_kernel<uint16_t, 1>);
    ctx->launches += 1;
    CU_AFTER_LAUNCH();
  }
  return SLIDEDP_OK;
}

}  // extern "C"
