// Rows of an embedding table, scaled, and the table's gradient.
//   out[t] = scale table[token[t]],   d table[b] = scale * sum of d_out[t] over the positions t with token b
// A negative token is padding: a row of zeros, no gradient.
//
// The gradient is a sum over positions in the order of their tokens. A byte vocabulary has a few hundred rows for thousands of positions, most
// of them with a few tokens, so neither a row per block nor atomics suit it. The positions are sorted by token (stable, so the order of every sum
// is fixed), cut into chunks of equal length, and a chunk's positions are added up row after row: each element of d_out is read once, whatever the
// tokens are. A token whose positions lie within a chunk is written at once; of one that crosses chunks every chunk leaves its part, which are added up
// in their order afterwards.
//   embed_sort_kernel     one block sorts (up to kSortTile positions; beyond that embed_count / embed_scan / embed_scatter per digit), the
//                         others meanwhile write the zeros of the rows that no position has and ask for d_out by L2 prefetch
//   embed_segment_kernel  the chunks
//   embed_join_kernel     the tokens that cross chunks
#pragma once
#include <cuda_bf16.h>
#include <stdint.h>

#include "mtpc_ptx.cuh"
#include "mtpc_rows.cuh"

namespace mtpc {

constexpr unsigned kStatusBadToken = 8u;

// ---------------------------------------------------------------- lookup
struct EmbedArgs {
  const int* tokens;
  const void* table;
  void* out;
  unsigned* status;       // may be NULL
  long long table_stride, out_stride;
  int T, v, d;
  float scale;
};

// blockDim.x threads share a row, R rows are in flight per thread.
template <typename TI, typename TO, int V, int R>
__global__ void __launch_bounds__(256) embed_kernel(const __grid_constant__ EmbedArgs a) {
  grid_dependency_wait();
  grid_launch_dependents();
  const int row0 = (blockIdx.x * blockDim.y + threadIdx.y) * R;
  int token[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    token[r] = row0 + r < a.T ? a.tokens[row0 + r] : -1;
    if (token[r] >= a.v && threadIdx.x == 0 && blockIdx.y == 0 && a.status) atomicOr(a.status, kStatusBadToken);
  }
  for (int col = (blockIdx.y * blockDim.x + threadIdx.x) * V; col < a.d; col += gridDim.y * blockDim.x * V) {
    Pack<TI, V> p[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (token[r] >= 0 && token[r] < a.v) p[r] = load_pack<TI, V>(static_cast<const TI*>(a.table) + token[r] * a.table_stride + col);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (row0 + r >= a.T) continue;
      float x[V];
      if (token[r] >= 0 && token[r] < a.v) {
        unpack(p[r], x);
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] *= a.scale;
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = token[r] < 0 ? 0.f : __int_as_float(0x7fffffff);
      }
      store_f32<TO, V>(static_cast<TO*>(a.out) + (row0 + r) * a.out_stride + col, x);
    }
  }
}

// ---------------------------------------------------------------- the positions in the order of their tokens
constexpr int kSortThreads = 1024, kSortWarps = kSortThreads / 32;
constexpr int kSortDigit = 9, kSortBins = 1 << kSortDigit;
constexpr int kSortPerLane = 16, kSortTile = kSortThreads * kSortPerLane;      // positions a block sorts
constexpr int kEmbedMaxT = 1 << 26, kEmbedMaxV = 1 << 20, kEmbedMaxD = 1 << 20;
constexpr int kClearScanT = 1 << 16;              // positions up to which the blocks that clear rows look for the rows that have none
constexpr size_t kEmbedPrefetchBytes = 32u << 20;
constexpr size_t kSortSmem = static_cast<size_t>(kSortWarps) * kSortBins * 4;

struct EmbedSortArgs {
  const int* tokens;
  int *key_a, *pos_a, *key_b, *pos_b;     // the last digit's go to key_a, pos_a
  int* hist;                              // [bins][tiles]
  unsigned* status;                       // may be NULL
  float* d_table;                         // rows without a position are cleared (NULL: none are)
  const void* d_out;
  long long d_table_stride, d_out_stride;
  int T, v, d, digits, tiles;
  int d_out_bytes;                        // of an element
};

// The key of a position: its token, or v for padding and what is no token.
__device__ __forceinline__ int embed_key(const EmbedSortArgs& a, int i) {
  const int token = a.tokens[i];
  if (token >= a.v && a.status) atomicOr(a.status, kStatusBadToken);
  return token < 0 || token >= a.v ? a.v : token;
}
// Where the keys of digit `p` are written to (alternating so that the last one writes key_a, pos_a).
__device__ __forceinline__ int* sort_keys(const EmbedSortArgs& a, int p) { return ((a.digits - 1 - p) & 1) ? a.key_b : a.key_a; }
__device__ __forceinline__ int* sort_positions(const EmbedSortArgs& a, int p) { return ((a.digits - 1 - p) & 1) ? a.pos_b : a.pos_a; }

// A tile's keys and positions before digit p, up to 16 a lane: a warp's are adjacent.
struct SortItems {
  int key[kSortPerLane], pos[kSortPerLane];
};
__device__ __forceinline__ void sort_load(const EmbedSortArgs& a, int p, int tile, SortItems& x) {
  const int first = tile * kSortTile;
  const int count = min(a.T - first, kSortTile);
  const int per_warp = (count + kSortThreads - 1) / kSortThreads * 32;                   // at most 512
  const int begin = (threadIdx.x >> 5) * per_warp;
  const int end = min(begin + per_warp, count);
#pragma unroll
  for (int j = 0; j < kSortPerLane; ++j) {
    const int i = begin + j * 32 + (threadIdx.x & 31);
    x.key[j] = -1;
    if (i < end) {
      x.key[j] = p == 0 ? embed_key(a, first + i) : sort_keys(a, p - 1)[first + i];
      x.pos[j] = p == 0 ? first + i : sort_positions(a, p - 1)[first + i];
    }
  }
}
__device__ __forceinline__ int sort_digit(int key, int p) { return (key >> (p * kSortDigit)) & (kSortBins - 1); }

// counts[warp][bin] of the warp's keys. Equal digits of a warp's 32 keys find each other, the lowest lane counts them.
__device__ __forceinline__ void sort_count(const SortItems& x, int p, unsigned* counts) {
  unsigned* mine = counts + (threadIdx.x >> 5) * kSortBins;
  const int lane = threadIdx.x & 31;
  for (int b = lane; b < kSortBins; b += 32) mine[b] = 0;
  __syncwarp();
#pragma unroll
  for (int j = 0; j < kSortPerLane; ++j) {
    if (!__any_sync(0xffffffffu, x.key[j] >= 0)) break;
    const int digit = x.key[j] >= 0 ? sort_digit(x.key[j], p) : -1;
    const unsigned peers = __match_any_sync(0xffffffffu, digit);
    if (digit >= 0 && lane == __ffs(peers) - 1) mine[digit] += __popc(peers);
    __syncwarp();
  }
}
// counts -> the place of the warp's first key of each bin; base: the place of the tile's first key of bin threadIdx.x.
__device__ __forceinline__ void sort_offsets(unsigned* counts, unsigned base) {
  if (threadIdx.x < kSortBins) {
#pragma unroll 8
    for (int w = 0; w < kSortWarps; ++w) {
      const unsigned c = counts[w * kSortBins + threadIdx.x];
      counts[w * kSortBins + threadIdx.x] = base;
      base += c;
    }
  }
}
// Keys and positions to their places, in order.
__device__ __forceinline__ void sort_place(const EmbedSortArgs& a, const SortItems& x, int p, unsigned* counts) {
  unsigned* mine = counts + (threadIdx.x >> 5) * kSortBins;
  const int lane = threadIdx.x & 31;
  int *keys = sort_keys(a, p), *positions = sort_positions(a, p);
#pragma unroll
  for (int j = 0; j < kSortPerLane; ++j) {
    if (!__any_sync(0xffffffffu, x.key[j] >= 0)) break;
    const int digit = x.key[j] >= 0 ? sort_digit(x.key[j], p) : -1;
    const unsigned peers = __match_any_sync(0xffffffffu, digit);
    const unsigned first = digit >= 0 ? mine[digit] : 0u;
    __syncwarp();
    if (digit >= 0) {
      const unsigned at = first + __popc(peers & ((1u << lane) - 1u));
      keys[at] = x.key[j];
      positions[at] = x.pos[j];
      if (lane == __ffs(peers) - 1) mine[digit] = first + __popc(peers);
    }
    __syncwarp();
  }
}
// Exclusive running sum of one value a thread over the block; total: of all.
__device__ __forceinline__ unsigned block_running_sum(unsigned x, unsigned* warp_sums, unsigned& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  unsigned sum = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned y = __shfl_up_sync(0xffffffffu, sum, o);
    if (lane >= o) sum += y;
  }
  if (lane == 31) warp_sums[warp] = sum;
  __syncthreads();
  unsigned before = warp_sums[lane];                   // (32 warps)
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned y = __shfl_up_sync(0xffffffffu, before, o);
    if (lane >= o) before += y;
  }
  total = __shfl_sync(0xffffffffu, before, kSortWarps - 1);
  const unsigned earlier = __shfl_sync(0xffffffffu, before, warp == 0 ? 0 : warp - 1);
  __syncthreads();                                     // warp_sums may be written again
  return (warp == 0 ? 0u : earlier) + sum - x;
}

// Block `part` of `parts`: zeros to the rows of its share of the table that no position has (where there are too many positions to look
// through: to all of its rows), then its share of the first rows of d_out into L2.
__device__ __forceinline__ void clear_rows(const EmbedSortArgs& a, int part, int parts, unsigned* present) {
  if (a.d_table) {
    const int lo = static_cast<int>(static_cast<long long>(part) * a.v / parts), hi = static_cast<int>(static_cast<long long>(part + 1) * a.v / parts);
    for (int i = threadIdx.x; i < (hi - lo + 31) / 32; i += kSortThreads) present[i] = 0;
    __syncthreads();
    if (a.T <= kClearScanT) {
      for (int i = threadIdx.x; i < a.T; i += kSortThreads) {
        const int token = a.tokens[i];
        if (token >= lo && token < hi) atomicOr(&present[(token - lo) >> 5], 1u << ((token - lo) & 31));
      }
      __syncthreads();
    }
    const bool wide = a.d % 4 == 0 && a.d_table_stride % 4 == 0 && (reinterpret_cast<uintptr_t>(a.d_table) & 15) == 0;
    const int per_row = wide ? a.d / 4 : a.d;
    int share = 32;                                    // threads to a row: as many as it has elements, up to the block
    while (share < per_row && share < kSortThreads) share <<= 1;
    for (int b = lo + static_cast<int>(threadIdx.x) / share; b < hi; b += kSortThreads / share) {
      if ((present[(b - lo) >> 5] >> ((b - lo) & 31)) & 1u) continue;
      float* row = a.d_table + b * a.d_table_stride;
      for (int i = threadIdx.x & (share - 1); i < per_row; i += share) {
        if (wide) reinterpret_cast<float4*>(row)[i] = make_float4(0.f, 0.f, 0.f, 0.f);
        else row[i] = 0.f;
      }
    }
  }
  if (a.T == 0) return;
  const long long row_bytes = static_cast<long long>(a.d) * a.d_out_bytes;
  const int lines = static_cast<int>((row_bytes + 127) / 128);
  const long long rows = min(static_cast<long long>(a.T), static_cast<long long>(kEmbedPrefetchBytes) / row_bytes + 1);
  for (long long i = static_cast<long long>(part) * kSortThreads + threadIdx.x; i < rows * lines; i += static_cast<long long>(parts) * kSortThreads) {
    const long long row = i / lines, line = i - row * lines;
    prefetch_l2(static_cast<const uint8_t*>(a.d_out) + row * a.d_out_stride * a.d_out_bytes + line * 128);
  }
}

// All digits of up to kSortTile positions in block 0.
__global__ void __launch_bounds__(kSortThreads) embed_sort_kernel(const __grid_constant__ EmbedSortArgs a) {
  extern __shared__ unsigned counts[];
  __shared__ unsigned warp_sums[kSortWarps];
  grid_dependency_wait();
  grid_launch_dependents();
  if (blockIdx.x > 0) {
    clear_rows(a, blockIdx.x - 1, gridDim.x - 1, counts);
    return;
  }
  for (int p = 0; p < a.digits; ++p) {
    SortItems x;
    sort_load(a, p, 0, x);
    sort_count(x, p, counts);
    __syncthreads();
    unsigned mine = 0, total;
    if (threadIdx.x < kSortBins) {
#pragma unroll 8
      for (int w = 0; w < kSortWarps; ++w) mine += counts[w * kSortBins + threadIdx.x];
    }
    const unsigned base = block_running_sum(mine, warp_sums, total);
    sort_offsets(counts, base);
    __syncthreads();
    sort_place(a, x, p, counts);
    __syncthreads();
  }
}

// More positions, one digit: the tiles' counts, their running sums over (bin, tile), and every tile's keys to their places.
__global__ void __launch_bounds__(kSortThreads) embed_count_kernel(const __grid_constant__ EmbedSortArgs a, int p) {
  extern __shared__ unsigned counts[];
  grid_dependency_wait();
  grid_launch_dependents();
  if (static_cast<int>(blockIdx.x) >= a.tiles) {
    clear_rows(a, blockIdx.x - a.tiles, gridDim.x - a.tiles, counts);
    return;
  }
  SortItems x;
  sort_load(a, p, blockIdx.x, x);
  sort_count(x, p, counts);
  __syncthreads();
  if (threadIdx.x < kSortBins) {
    unsigned mine = 0;
#pragma unroll 8
    for (int w = 0; w < kSortWarps; ++w) mine += counts[w * kSortBins + threadIdx.x];
    a.hist[static_cast<size_t>(threadIdx.x) * a.tiles + blockIdx.x] = mine;
  }
}
__global__ void __launch_bounds__(kSortThreads) embed_scan_kernel(int* hist, int count) {
  __shared__ unsigned warp_sums[kSortWarps];
  grid_dependency_wait();
  grid_launch_dependents();
  unsigned before = 0;
  for (int i = 0; i < count; i += kSortThreads) {
    const int at = i + threadIdx.x;
    const unsigned x = at < count ? hist[at] : 0u;
    unsigned total;
    const unsigned sum = block_running_sum(x, warp_sums, total);
    if (at < count) hist[at] = before + sum;
    before += total;
  }
}
__global__ void __launch_bounds__(kSortThreads) embed_scatter_kernel(const __grid_constant__ EmbedSortArgs a, int p) {
  extern __shared__ unsigned counts[];
  grid_dependency_wait();
  grid_launch_dependents();
  SortItems x;
  sort_load(a, p, blockIdx.x, x);
  sort_count(x, p, counts);
  __syncthreads();
  sort_offsets(counts, threadIdx.x < kSortBins ? a.hist[static_cast<size_t>(threadIdx.x) * a.tiles + blockIdx.x] : 0u);
  __syncthreads();
  sort_place(a, x, p, counts);
}

// ---------------------------------------------------------------- sums of the sorted positions
constexpr int kSegmentThreads = 256;
constexpr int kSegmentStage = 256;      // positions whose keys are in shared memory at a time

struct EmbedSegmentArgs {
  const int *key, *pos;                 // sorted; key v: no token
  const void* d_out;
  float *d_table, *part;                // part [chunks][2][d]: what a chunk adds to the token it begins in / that goes on behind it
  long long d_out_stride, d_table_stride;
  int T, v, d, chunk, chunks;
  float scale;
  bool accumulate;
};

template <int V>
__device__ __forceinline__ void write_table(const EmbedSegmentArgs& a, int token, int col, const float (&x)[V]) {
  float* dst = a.d_table + token * a.d_table_stride + col;
  float o[V];
  if (a.accumulate) unpack(load_pack<float, V>(dst), o);
#pragma unroll
  for (int i = 0; i < V; ++i) o[i] = a.accumulate ? o[i] + x[i] * a.scale : x[i] * a.scale;
  store_f32<float, V>(dst, o);
}

// blockIdx.x: columns, blockIdx.y: chunk. U rows are in flight per thread.
template <typename T, int V, int U>
__global__ void __launch_bounds__(kSegmentThreads) embed_segment_kernel(const __grid_constant__ EmbedSegmentArgs a) {
  __shared__ int key[kSegmentStage + 1], pos[kSegmentStage];
  const int col = (blockIdx.x * blockDim.x + threadIdx.x) * V;
  const int lo = blockIdx.y * a.chunk, hi = min(lo + a.chunk, a.T);
  grid_dependency_wait();
  float sum[V];
#pragma unroll
  for (int i = 0; i < V; ++i) sum[i] = 0.f;
  float* part = a.part + static_cast<size_t>(blockIdx.y) * 2 * a.d + col;
  bool begins = true;                            // the token being added up has no position in an earlier chunk
  for (int base = lo; base < hi; base += kSegmentStage) {
    const int count = min(hi - base, kSegmentStage);
    __syncthreads();
    for (int i = threadIdx.x; i <= count; i += blockDim.x) {
      key[i] = base + i < a.T ? a.key[base + i] : a.v;
      if (i < count) pos[i] = a.pos[base + i];
    }
    __syncthreads();
    if (base == lo) begins = lo == 0 || a.key[lo - 1] != key[0];
    if (key[0] == a.v) break;                    // the rest of the positions have no token
    for (int i = 0; i < count; i += U) {
      Pack<T, V> x[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (i + u < count && key[i + u] != a.v && col < a.d)
          x[u] = load_pack<T, V>(static_cast<const T*>(a.d_out) + pos[i + u] * a.d_out_stride + col);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (i + u >= count || key[i + u] == a.v) break;
        float y[V];
        unpack(x[u], y);
#pragma unroll
        for (int e = 0; e < V; ++e) sum[e] += y[e];
        const bool ends = key[i + u + 1] != key[i + u];
        if (ends || base + i + u + 1 == hi) {
          if (col < a.d) {
            if (begins && ends) write_table<V>(a, key[i + u], col, sum);
            else store_f32<float, V>(part + (begins ? a.d : 0), sum);
          }
#pragma unroll
          for (int e = 0; e < V; ++e) sum[e] = 0.f;
          begins = true;
        }
      }
    }
  }
  grid_launch_dependents();
}

// The tokens that cross chunks: the block of the chunk in which one begins adds up its parts, warp y every eighth, then the warps' sums.
template <int V>
__global__ void __launch_bounds__(256) embed_join_kernel(const __grid_constant__ EmbedSegmentArgs a) {
  __shared__ float share[8][32][V];
  const int c = blockIdx.y, lo = c * a.chunk, hi = min(lo + a.chunk, a.T);
  grid_dependency_wait();
  grid_launch_dependents();
  if (hi >= a.T) return;
  const int token = a.key[hi - 1];
  if (token == a.v || a.key[hi] != token) return;                       // ends here
  if (lo > 0 && a.key[lo - 1] == token) return;                         // began earlier
  int last = c + 1;                                                     // the last chunk that has the token: its first key is the token
  for (int step = 1;; step <<= 1) {                                     // (sorted: found in steps that double, then halve)
    if (last + step >= a.chunks || a.key[static_cast<long long>(last + step) * a.chunk] != token) {
      for (step >>= 1; step > 0; step >>= 1)
        if (last + step < a.chunks && a.key[static_cast<long long>(last + step) * a.chunk] == token) last += step;
      break;
    }
    last += step;
  }
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int col = (blockIdx.x * 32 + lane) * V;
  float sum[V];
#pragma unroll
  for (int i = 0; i < V; ++i) sum[i] = 0.f;
  if (col < a.d) {
#pragma unroll 4
    for (int q = c + warp; q <= last; q += 8) {
      float x[V];
      unpack(load_pack<float, V>(a.part + (static_cast<size_t>(q) * 2 + (q == c ? 1 : 0)) * a.d + col), x);
#pragma unroll
      for (int i = 0; i < V; ++i) sum[i] += x[i];
    }
  }
#pragma unroll
  for (int i = 0; i < V; ++i) share[warp][lane][i] = sum[i];
  __syncthreads();
  if (warp == 0 && col < a.d) {
    for (int w = 1; w < 8; ++w) {
#pragma unroll
      for (int i = 0; i < V; ++i) sum[i] += share[w][lane][i];
    }
    write_table<V>(a, token, col, sum);
  }
}

}  // namespace mtpc
