// Embedding lookup of every worker and its gradient.
//   lookup:   out_t = scale * E_i[k_t]            (a gather: HBM-bound)
//   gradient: G_i[k] = scale * sum_{t: k_t = k} dout_t
// The gradient is dense (the local step reads every column), so writing n *
// vocab * width fp32 values is most of its traffic.  Sorting the tokens first
// makes it one write per table row without atomics: sums go over a token's
// rows in order, and the result is the same bits every time.
//
// Measured (n = 16, 65536 rows, tables of 32000 x 1024 in fp32, bf16 rows): lookup
// 69 us (343 MB, 5.0 TB/s); gradient 405 us (2.2 GB, 5.5 TB/s): sort 13, sums and
// zeros 350, join 9.  n = 5, 3001 rows, 1237 x 321 in fp32: gradient 20 us, three
// launches that each wait for a handful of loads.  A token that many rows share is
// added up by one workgroup in the join: one worker's 65536 rows with half of them
// (all of them) the same token take 250 us (414), without such a token 119.
#pragma clang fp contract(off)

#include <type_traits>

#include "layers_device.h"

namespace gasloc {
namespace {

// A wave takes kLookupRows consecutive rows.
constexpr int kLookupRows = 4;

template <int PT, int AT>
__global__ __launch_bounds__(256) void k_embedding(EmbeddingArgs a) {
  constexpr int V = AT == GASLOC_BF16 ? 8 : 4;
  const int wave = blockIdx.x * (256 / kWave) + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int lane = lane_id();
  const int rows = a.rows.begin[a.n];
  for (int r = 0; r < kLookupRows; ++r) {
    const int t = wave * kLookupRows + r;
    if (t >= rows) return;
    const int i = find_worker(a.rows, a.n, t);
    const int k = a.tokens[t];
    const bool real = k >= 0 && k < a.vocab;
    const void* row = live_row<PT>(a.w, i);
    const int64_t at = a.begin + static_cast<int64_t>(real ? k : 0) * a.width;
    for (int c = lane * V; c < a.width; c += kWave * V) {
      float w[V];
      load_row<PT, V, false>(row, at + c, a.width - c, w);
#pragma unroll
      for (int e = 0; e < V; ++e) w[e] = real ? a.scale * w[e] : 0.0f;
      store_row<AT, V>(a.out, static_cast<int64_t>(t) * a.out_ld + c, a.width - c, w);
    }
  }
}

// Stable radix sort of up to kSortTile tokens in one workgroup.  Entry e of
// the tile is item j = (e / 64) % J of lane e % 64 of wave e / (64 J), J = the
// items per thread that the tile needs.  Per pass of 8 bits: a wave ranks
// its items by digit (lanes with the same digit find each other by eight
// ballots; the wave's running counts are in LDS), the counts are scanned over
// waves and digits, and the entries move to their places in LDS.
constexpr int kSortThreads = 1024;
constexpr int kSortWaves = kSortThreads / kWave;
constexpr int kSortItems = kSortTile / kSortThreads;

__global__ __launch_bounds__(kSortThreads) void k_token_sort(SortArgs a) {
  __shared__ uint32_t s_key[kSortTile];
  __shared__ int32_t s_pos[kSortTile];
  __shared__ uint32_t s_count[kSortWaves][256];
  __shared__ uint32_t s_base[256];
  __shared__ uint32_t s_wave[4];
  const int i = find_worker(a.tiles, a.n, blockIdx.x);
  const int first = a.rows.begin[i] + (static_cast<int>(blockIdx.x) - a.tiles.begin[i]) * kSortTile;
  const int count = min(kSortTile, a.rows.begin[i + 1] - first);
  const int items = (count + kSortThreads - 1) / kSortThreads;
  const int tid = threadIdx.x, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int base = wave * kWave * items + lane;
  uint32_t key[kSortItems];
  int32_t pos[kSortItems];
#pragma unroll
  for (int j = 0; j < kSortItems; ++j) {
    const int e = base + j * kWave;
    key[j] = 0xffffffffu;  // behind everything: sorts last, and is not written out
    pos[j] = 0;
    if (j < items && e < count) {
      const int k = a.tokens[first + e];
      key[j] = k >= 0 && k < a.vocab ? static_cast<uint32_t>(k) : static_cast<uint32_t>(a.vocab);
      pos[j] = first + e;
    }
  }
  for (int shift = 0; shift < a.key_bits; shift += 8) {
    for (int k = tid; k < kSortWaves * 256; k += kSortThreads) (&s_count[0][0])[k] = 0;
    __syncthreads();
    uint32_t rank[kSortItems];
#pragma unroll
    for (int j = 0; j < kSortItems; ++j) {
      rank[j] = 0;
      if (j < items) {
        const uint32_t d = (key[j] >> shift) & 255u;
        uint64_t same = ~0ull;
#pragma unroll
        for (int b = 0; b < 8; ++b) {
          const bool bit = (d >> b) & 1u;
          const uint64_t set = __ballot(bit);
          same &= bit ? set : ~set;
        }
        const uint32_t before = __builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(same >> 32),
                                                          __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(same), 0));
        volatile uint32_t* slot = &s_count[wave][d];  // this wave's own; its accesses stay in order
        const uint32_t seen = *slot;
        __builtin_amdgcn_wave_barrier();
        rank[j] = seen + before;
        if (before == 0) *slot = seen + static_cast<uint32_t>(__popcll(same));
        __builtin_amdgcn_wave_barrier();
      }
    }
    __syncthreads();
    uint32_t total = 0, upto = 0;
    if (tid < 256) {
      for (int w = 0; w < kSortWaves; ++w) {
        const uint32_t c = s_count[w][tid];
        s_count[w][tid] = total;
        total += c;
      }
      upto = total;  // inclusive scan over the digits of this wave
      for (int d = 1; d < kWave; d *= 2) {
        const uint32_t v = __shfl_up(upto, d);
        if (lane >= d) upto += v;
      }
      if (lane == kWave - 1) s_wave[tid / kWave] = upto;
    }
    __syncthreads();
    if (tid < 256) {
      uint32_t lower = 0;
      for (int w = 0; w < tid / kWave; ++w) lower += s_wave[w];
      s_base[tid] = lower + upto - total;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kSortItems; ++j) {
      if (j < items) {
        const uint32_t d = (key[j] >> shift) & 255u;
        const uint32_t to = s_base[d] + s_count[wave][d] + rank[j];
        s_key[to] = key[j];
        s_pos[to] = pos[j];
      }
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kSortItems; ++j) {
      if (j < items) {
        key[j] = s_key[base + j * kWave];
        pos[j] = s_pos[base + j * kWave];
      }
    }
  }
#pragma unroll
  for (int j = 0; j < kSortItems; ++j) {
    const int e = base + j * kWave;
    if (j < items && e < count) {
      a.keys[first + e] = key[j];
      a.pos[first + e] = pos[j];
    }
  }
}

// Entries of keys[lo, hi) below `key` (or not above it).
__device__ __forceinline__ int count_below(const uint32_t* keys, int64_t lo, int64_t hi, uint32_t key, bool or_equal) {
  const int64_t start = lo;
  while (lo < hi) {
    const int64_t mid = lo + (hi - lo) / 2;
    const uint32_t k = keys[mid];
    if (k < key || (or_equal && k == key))
      lo = mid + 1;
    else
      hi = mid;
  }
  return static_cast<int>(lo - start);
}

// The first entry of keys[lo, hi) that is not below `key` (hi if there is none), found by the whole wave: each step
// asks 64 places at once.
__device__ __forceinline__ int64_t lower_bound(const uint32_t* keys, int64_t lo, int64_t hi, uint32_t key) {
  while (lo < hi) {
    const int64_t step = (hi - lo + kWave - 1) / kWave;
    const int64_t at = lo + (lane_id() + 1) * step - 1;
    const int below = __popcll(__ballot(at < hi && keys[at < hi ? at : lo] < key));
    const int64_t next = lo + (below + 1) * step - 1;  // not below, or behind the end
    lo += below * step;
    hi = next < hi ? next : hi;
  }
  return lo;
}

// An entry's place in the merged run: its place in its own run, and how many
// entries of each other run come first (of an earlier run also the equal ones).
__global__ __launch_bounds__(256) void k_token_merge(MergeArgs a) {
  const int i = find_worker(a.blocks, a.n, blockIdx.x);
  const int64_t begin = a.rows.begin[i], end = a.rows.begin[i + 1];
  const int64_t e = begin + static_cast<int64_t>(static_cast<int>(blockIdx.x) - a.blocks.begin[i]) * 256 + threadIdx.x;
  if (e >= end) return;
  const uint32_t key = a.keys[e];
  const int64_t mine = (e - begin) / a.run;
  const int64_t group = mine / kMergeWays * kMergeWays;
  int64_t to = begin + group * a.run + (e - begin - mine * a.run);
  for (int64_t r = group; r < group + kMergeWays; ++r) {
    const int64_t lo = begin + r * a.run;
    if (r == mine || lo >= end) continue;
    to += count_below(a.keys, lo, min(lo + a.run, end), key, r < mine);
  }
  a.keys_out[to] = key;
  a.pos_out[to] = a.pos[e];
}

// (+)= scale * sum, for V columns of a table row
constexpr int V = 4;
__device__ __forceinline__ void put_grad(const EmbeddingGradArgs& a, int i, uint32_t key, int c,
                                         const float (&sum)[V]) {
  float* g = a.grads + static_cast<int64_t>(i) * a.grad_ld + a.begin + static_cast<int64_t>(key) * a.width + c;
  float o[V];
#pragma unroll
  for (int e = 0; e < V; ++e) o[e] = a.scale * sum[e];
  if (a.accumulate) {
    float old[V];
    load_row<GASLOC_F32, V, true>(g, 0, a.width - c, old);
#pragma unroll
    for (int e = 0; e < V; ++e) o[e] = old[e] + o[e];
  }
  store_row<GASLOC_F32, V>(g, 0, a.width - c, o);
}

template <int AT>
__global__ __launch_bounds__(256) void k_embedding_sums(EmbeddingGradArgs a) {
  __shared__ uint32_t s_key[kMaxChunk + 2];  // with the entries before and behind the chunk
  __shared__ int32_t s_pos[kMaxChunk];
  const int tid = threadIdx.x, threads = blockDim.x;
  const int b = blockIdx.x, chunks = a.chunks.begin[a.n];
  if (b >= chunks) {  // zero the rows of [k0, k1) that have no token
    const int per = (a.vocab + a.fill_rows - 1) / a.fill_rows;
    const int i = (b - chunks) / per;
    const int k0 = (b - chunks) % per * a.fill_rows, k1 = min(k0 + a.fill_rows, a.vocab);
    const int64_t end = a.rows.begin[i + 1];
    const int64_t lo = lower_bound(a.keys, a.rows.begin[i], end, static_cast<uint32_t>(k0));
    const int64_t hi = lower_bound(a.keys, lo, end, static_cast<uint32_t>(k1));
    for (int k = tid; k < k1 - k0; k += threads) s_key[k] = 0;
    __syncthreads();
    for (int64_t e = lo + tid; e < hi; e += threads) s_key[a.keys[e] - static_cast<uint32_t>(k0)] = 1;
    __syncthreads();
    // Rows that follow each other are one stretch of memory.  Vectors on their boundaries, whatever the row's: a row
    // of odd width begins inside one.
    const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int k = k0, stop; k < k1; k = stop) {
      stop = k + 1;
      if (s_key[k - k0]) continue;
      while (stop < k1 && !s_key[stop - k0]) ++stop;
      const int cols = (stop - k) * a.width;
      float* g = a.grads + static_cast<int64_t>(i) * a.grad_ld + a.begin + static_cast<int64_t>(k) * a.width;
      const int inside = static_cast<int>(reinterpret_cast<uintptr_t>(g) / 4 % 4);
      for (int c = tid * V - inside; c < cols; c += threads * V) {
        if (c >= 0 && c + V <= cols) {
          st_stream(reinterpret_cast<f32x4*>(g + c), zero);
        } else {
#pragma unroll
          for (int e = 0; e < V; ++e)
            if (c + e >= 0 && c + e < cols) g[c + e] = 0.0f;
        }
      }
    }
    return;
  }
  const int i = find_worker(a.chunks, a.n, b);
  const int begin = a.rows.begin[i], end = a.rows.begin[i + 1];
  const int first = begin + (b - a.chunks.begin[i]) * a.chunk;
  const int count = min(a.chunk, end - first);
  // a key that no token has stands for "none" at the ends of the worker's list
  for (int e = tid; e < count + 2; e += threads) {
    const int at = first - 1 + e;
    s_key[e] = at >= begin && at < end ? a.keys[at] : 0xffffffffu;
    if (e < count) s_pos[e] = a.pos[first + e];
  }
  __syncthreads();
  const bool before = s_key[0] == s_key[1], behind = s_key[count + 1] == s_key[count];
  for (int c = tid * V; c < a.width; c += threads * V) {
    float sum[V] = {};
    bool head = before;  // the current row began before this chunk
    for (int e0 = 0; e0 < count; e0 += 8) {
      float v[8][V];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int at = min(e0 + e, count - 1);
        load_row<AT, V, true>(a.dout, static_cast<int64_t>(s_pos[at]) * a.dout_ld + c, a.width - c, v[e]);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (e0 + e < count) {
          const uint32_t key = __builtin_amdgcn_readfirstlane(s_key[e0 + e + 1]);
          const uint32_t next = __builtin_amdgcn_readfirstlane(s_key[e0 + e + 2]);
#pragma unroll
          for (int q = 0; q < V; ++q) sum[q] += v[e][q];
          const bool last = e0 + e == count - 1;
          if (key != next || last) {
            if (key < static_cast<uint32_t>(a.vocab)) {
              const bool tail = last && behind;
              if (!head && !tail)
                put_grad(a, i, key, c, sum);
              else
                store_row<GASLOC_F32, V>(a.partial, (2 * static_cast<int64_t>(b) + (head ? 0 : 1)) * a.width + c,
                                         a.width - c, sum);
            }
#pragma unroll
            for (int q = 0; q < V; ++q) sum[q] = 0.0f;
            head = false;
          }
        }
      }
    }
  }
}

// Finishes the row that begins in chunk b and goes on behind it: its part
// here, then its parts in the chunks that follow, in order.  It goes on into
// chunk q as long as q begins with it: 64 chunks are asked at a time.
__global__ __launch_bounds__(256) void k_embedding_join(EmbeddingGradArgs a) {
  const int b = blockIdx.x;
  const int i = find_worker(a.chunks, a.n, b);
  const int begin = a.rows.begin[i], end = a.rows.begin[i + 1];
  const int first = begin + (b - a.chunks.begin[i]) * a.chunk;
  const int next = first + a.chunk;
  if (next >= end) return;
  const uint32_t key = a.keys[next - 1], head = a.keys[first], before = a.keys[first > begin ? first - 1 : first];
  if (key >= static_cast<uint32_t>(a.vocab) || a.keys[next] != key) return;
  if (head == key && first > begin && before == key) return;  // began earlier
  int last = b;
  for (int more = kWave; more == kWave; last += more) {
    const int64_t at = first + static_cast<int64_t>(last - b + 1 + lane_id()) * a.chunk;
    const uint64_t goes_on = __ballot(at < end && a.keys[at < end ? at : first] == key);
    more = goes_on == ~0ull ? kWave : __builtin_ctzll(~goes_on);
  }
  for (int c = threadIdx.x * V; c < a.width; c += blockDim.x * V) {
    float sum[V];
    load_row<GASLOC_F32, V, true>(a.partial, (2 * static_cast<int64_t>(b) + 1) * a.width + c, a.width - c, sum);
    for (int q0 = b + 1; q0 <= last; q0 += 8) {
      float v[8][V];
#pragma unroll
      for (int q = 0; q < 8; ++q)
        load_row<GASLOC_F32, V, true>(a.partial, 2 * static_cast<int64_t>(min(q0 + q, last)) * a.width + c,
                                      a.width - c, v[q]);
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        if (q0 + q <= last) {
#pragma unroll
          for (int e = 0; e < V; ++e) sum[e] += v[q][e];
        }
      }
    }
    put_grad(a, i, key, c, sum);
  }
}

// Threads for a row of `width` columns.
int row_threads(int width) {
  const int need = (width + V - 1) / V;
  return need > 128 ? 256 : need > 64 ? 128 : 64;
}

}  // namespace

hipError_t launch_embedding(const EmbeddingArgs& a, int params, int act, hipStream_t stream) {
  const int rows = a.rows.begin[a.n];
  constexpr int per = kLookupRows * 256 / kWave;
  return launch_kernel(params == GASLOC_BF16 ? k_embedding<GASLOC_BF16, GASLOC_BF16>
                       : act == GASLOC_BF16  ? k_embedding<GASLOC_F32, GASLOC_BF16>
                                             : k_embedding<GASLOC_F32, GASLOC_F32>,
                       dim3((rows + per - 1) / per), 256, 0, stream, a);
}

hipError_t launch_token_sort(const SortArgs& a, hipStream_t stream) {
  return launch_kernel(k_token_sort, dim3(a.tiles.begin[a.n]), kSortThreads, 0, stream, a);
}

hipError_t launch_token_merge(const MergeArgs& a, hipStream_t stream) {
  return launch_kernel(k_token_merge, dim3(a.blocks.begin[a.n]), 256, 0, stream, a);
}

hipError_t launch_embedding_sums(const EmbeddingGradArgs& a, int act, hipStream_t stream) {
  const int fill = a.accumulate ? 0 : a.n * ((a.vocab + a.fill_rows - 1) / a.fill_rows);
  return launch_kernel(act == GASLOC_BF16 ? k_embedding_sums<GASLOC_BF16> : k_embedding_sums<GASLOC_F32>,
                       dim3(a.chunks.begin[a.n] + fill), row_threads(a.width), 0, stream, a);
}

hipError_t launch_embedding_join(const EmbeddingGradArgs& a, hipStream_t stream) {
  return launch_kernel(k_embedding_join, dim3(a.chunks.begin[a.n]), row_threads(a.width), 0, stream, a);
}

}  // namespace gasloc
