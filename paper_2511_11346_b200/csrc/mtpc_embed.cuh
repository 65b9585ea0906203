// Rows of an embedding table, scaled, and the table's gradient.
//   out[t] = scale table[token[t]],   d table[b] = scale * sum of d_out[t] over the positions t with token b
// A negative token is padding: a row of zeros, no gradient.
//
// The gradient is a sum over positions in the order of their tokens. A byte vocabulary has a few hundred rows for thousands of positions, most
// of them with a few tokens, so neither a row per block nor atomics suit it. The positions are sorted by token (stable, so the order of every sum
// is fixed), cut into chunks of equal length, and a chunk's positions are added up row after row: each element of d_out is read once, whatever the
// tokens are. A token whose positions lie within a chunk is written at once; of one that crosses chunks every chunk leaves its part, which are added up
// in their order afterwards, by a kernel of its own. (Left to whichever block comes last, found by a counter, the sums of 8192 x 4096 fp32 took 57 us, fences
// included, instead of 26 and 5 for the join.)
//   embed_order_kernel    up to kOrderMaxT positions (or half as many): every block owns a range of tokens, finds their positions among
//                         all of them and sorts those;
//                         meanwhile the device asks for d_out by L2 prefetch
//   embed_count / embed_scatter_kernel   more positions: by digits of 9 bits
//                         (embed_bounds_kernel: where each token's positions begin and end, which the one-launch sort and a single digit's know)
//   embed_segment_kernel  the chunks
//   embed_join_kernel     the tokens that cross chunks
// A step of a few positions is all launches: up to kFewT of them embed_few_kernel does it alone, row of the table after row, where the table is
// not a large one.
// Rows that no position has are zeros: written by further blocks of the last two, behind whose short chains of dependent loads that hides.
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
  int shift, pitch;       // of split rows (SplitRow)
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
    Raw<TI, V> p[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (token[r] >= 0 && token[r] < a.v) p[r].load(static_cast<const TI*>(a.table) + token[r] * a.table_stride + col);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (row0 + r >= a.T) continue;
      float x[V];
      if (token[r] >= 0 && token[r] < a.v) {
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = p[r].value(i) * a.scale;
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = token[r] < 0 ? 0.f : __int_as_float(0x7fffffff);
      }
      store_f32<TO, V>(static_cast<TO*>(a.out) + (row0 + r) * a.out_stride + col, x);
    }
  }
}

// Eight adjacent elements that start anywhere, as fp32: the two or three vectors of 16 bytes that hold them, shifted (one element after the other is
// eight loads whose lanes lie eight elements apart: 20.8 instead of 14.4 us for 16000 rows of 1001, fp32 to bf16).
template <typename T>
__device__ __forceinline__ void load8_anywhere(const T* p, float (&x)[8]) {
  constexpr int kWords = 2 * sizeof(T);
  const uintptr_t at = reinterpret_cast<uintptr_t>(p);
  const uint4* from = reinterpret_cast<const uint4*>(at & ~static_cast<uintptr_t>(15));
  Raw<T, 8> value;
  uint32_t w[kWords + 4];
#pragma unroll
  for (int g = 0; g <= kWords / 4; ++g) {
    uint4 y = make_uint4(0, 0, 0, 0);
    if (g < kWords / 4 || (at & 15) != 0) y = from[g];
    w[4 * g] = y.x, w[4 * g + 1] = y.y, w[4 * g + 2] = y.z, w[4 * g + 3] = y.w;
  }
  if (at & 4) {
#pragma unroll
    for (int i = 0; i < kWords + 3; ++i) w[i] = w[i + 1];
  }
  if (at & 8) {
#pragma unroll
    for (int i = 0; i < kWords + 1; ++i) w[i] = w[i + 2];
  }
#pragma unroll
  for (int i = 0; i < kWords; ++i) value.r[i] = at & 2 ? __funnelshift_r(w[i], w[i + 1], 16) : w[i];
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = value.value(i);
}

// The same where the table's or the output's rows do not start on vectors: the output is written as vectors all the same.
template <typename TI, typename TO>
__global__ void __launch_bounds__(256) embed_split_kernel(const __grid_constant__ EmbedArgs a) {
  grid_dependency_wait();
  grid_launch_dependents();
  const int row = blockIdx.x * blockDim.y + threadIdx.y;
  if (row >= a.T) return;
  const int token = a.tokens[row];
  const bool is = token >= 0 && token < a.v;
  if (token >= a.v && threadIdx.x == 0 && a.status) atomicOr(a.status, kStatusBadToken);
  const TI* from = static_cast<const TI*>(a.table) + (is ? token : 0) * a.table_stride;
  TO* out = static_cast<TO*>(a.out) + row * a.out_stride;
  const float none = token < 0 ? 0.f : __int_as_float(0x7fffffff);
  const SplitRow split(a.shift, a.pitch, row, a.d);
  for (int i = threadIdx.x; i < split.head + split.rest; i += blockDim.x) {
    const int col = i < split.head ? i : split.packs * 8 + i;
    out[col] = from_f32<TO>(is ? to_f32(from[col]) * a.scale : none);
  }
  for (int i = threadIdx.x; i < split.packs; i += blockDim.x) {
    float x[8];
    if (is) load8_anywhere<TI>(from + split.head + i * 8, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = is ? x[e] * a.scale : none;
    store_f32<TO, 8>(out + split.head + i * 8, x);
  }
}

// ---------------------------------------------------------------- the positions in the order of their tokens
constexpr int kEmbedMaxT = 1 << 26, kEmbedMaxV = 1 << 20, kEmbedMaxD = 1 << 20;
constexpr size_t kEmbedPrefetchBytes = 32u << 20;

struct EmbedSortArgs {
  const int* tokens;
  int *key_a, *pos_a, *key_b, *pos_b;     // the last digit's go to key_a, pos_a
  int2* bounds;                           // [v + 1]: where a token's positions begin and end in the order (equal: it has none)
  uint2* hist;                            // [tiles][bins], two bins each
  unsigned* status;                       // may be NULL
  const void* d_out;
  long long d_out_stride;
  int T, v, d;
  int range;                              // embed_order_kernel: tokens of a block
  int digits, tiles, rounds;              // else: a tile is `rounds` times kSortTile positions
  int d_out_bytes;                        // of an element
};

// The key of a position: its token, or v for padding and what is no token.
__device__ __forceinline__ int embed_key(const EmbedSortArgs& a, int token) { return token < 0 || token >= a.v ? a.v : token; }

// Block `part` of `parts`: its share of the first rows of d_out into L2.
__device__ __forceinline__ void prefetch_rows(const EmbedSortArgs& a, int part, int parts) {
  const int row_bytes = a.d * a.d_out_bytes, lines = (row_bytes + 127) / 128;           // (at most 4 MB a row)
  const int rows = min(a.T, static_cast<int>(kEmbedPrefetchBytes / row_bytes) + 1);
  for (int i = part * blockDim.x + threadIdx.x; i < rows * lines; i += parts * blockDim.x) {       // (at most 2^25 lines)
    const int row = i / lines, line = i - row * lines;
    prefetch_l2(static_cast<const uint8_t*>(a.d_out) + row * a.d_out_stride * a.d_out_bytes + line * 128);
  }
}

// The lanes of a warp whose value has the same `bits` low bits (fewer instructions than the warp's match, which looks at all 32).
__device__ __forceinline__ unsigned equal_lanes(unsigned x, int bits, unsigned among) {
  for (int b = 0; b < bits; ++b) {
    const bool one = (x >> b) & 1u;
    const unsigned ones = __ballot_sync(0xffffffffu, one);
    among &= one ? ones : ~ones;
  }
  return among;
}

// Up to kOrderMaxT positions. Every block looks through all tokens (from L2) for those of its range, lists them in order, and sorts the list by
// counting: a warp counts its part of it per token, the counts become places, the warps write their keys and positions there. One launch of a
// few microseconds where a sort by one block takes 18 (8192 positions): that one sorts them all while the device waits.
constexpr int kOrderThreads = 1024, kOrderWarps = kOrderThreads / 32, kOrderMaxT = 1 << 15, kOrderMaxRange = 512;
constexpr int kOrderAhead = 8;                     // tokens that a lane holds at a time
inline size_t order_smem_bytes(int T) { return static_cast<size_t>(T) * 4; }
__global__ void __launch_bounds__(kOrderThreads, 2) embed_order_kernel(const __grid_constant__ EmbedSortArgs a) {
  extern __shared__ unsigned list[];               // token's place in the range << 16 | position (below 2^15)
  __shared__ uint16_t counts[kOrderWarps][kOrderMaxRange];
  __shared__ unsigned found[kOrderWarps], below[kOrderWarps];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int lo = blockIdx.x * a.range, tokens = min(a.range, a.v + 1 - lo);       // (key v: what is no token)
  const int per_warp = (a.T + kOrderThreads - 1) / kOrderThreads * 32;
  const int begin = min(warp * per_warp, a.T), end = min(begin + per_warp, a.T);
  for (int b = lane; b < tokens; b += 32) counts[warp][b] = 0;
  grid_dependency_wait();
  grid_launch_dependents();

  int key[kOrderAhead];
  auto look = [&](int i) {
#pragma unroll
    for (int u = 0; u < kOrderAhead; ++u) key[u] = i + u * 32 + lane < end ? a.tokens[i + u * 32 + lane] : INT32_MIN;
  };
  unsigned mine = 0, less = 0;
  bool bad = false;
  for (int i = begin; i < end; i += kOrderAhead * 32) {
    look(i);
#pragma unroll
    for (int u = 0; u < kOrderAhead; ++u) {
      const bool is = i + u * 32 + lane < end;
      bad |= key[u] >= a.v;
      const int k = embed_key(a, key[u]);
      mine += __popc(__ballot_sync(0xffffffffu, is && k >= lo && k < lo + tokens));
      less += __popc(__ballot_sync(0xffffffffu, is && k < lo));
    }
  }
  if (lane == 0) {
    found[warp] = mine;
    below[warp] = less;
  }
  prefetch_rows(a, blockIdx.x, gridDim.x);         // (behind the tokens, which otherwise wait for it)
  if (blockIdx.x == 0 && bad && a.status) atomicOr(a.status, kStatusBadToken);
  __syncthreads();
  // of the range's positions: the first one's place, how many, those of the warps before
  const unsigned base = __reduce_add_sync(0xffffffffu, below[lane]), count = __reduce_add_sync(0xffffffffu, found[lane]);
  unsigned at = __reduce_add_sync(0xffffffffu, lane < warp ? found[lane] : 0u);
  if (mine > 0) {
    for (int i = begin; i < end; i += kOrderAhead * 32) {
      if (per_warp > kOrderAhead * 32) look(i);    // (else they are still held)
#pragma unroll
      for (int u = 0; u < kOrderAhead; ++u) {
        const int k = embed_key(a, key[u]) - lo;
        const bool is = i + u * 32 + lane < end && k >= 0 && k < tokens;
        const unsigned which = __ballot_sync(0xffffffffu, is);
        if (is) list[at + __popc(which & ((1u << lane) - 1u))] = static_cast<unsigned>(k) << 16 | static_cast<unsigned>(i + u * 32 + lane);
        at += __popc(which);
      }
    }
  }
  __syncthreads();

  const int bits = 32 - __clz(tokens - 1);
  const int share = (count + kOrderThreads - 1) / kOrderThreads * 32;
  const int from = min(warp * share, static_cast<int>(count)), to = min(from + share, static_cast<int>(count));
  for (int i = from; i < to; i += 32) {
    const bool is = i + lane < to;
    const unsigned bin = is ? list[i + lane] >> 16 : 0u;
    const unsigned peers = equal_lanes(bin, bits, __ballot_sync(0xffffffffu, is));
    if (is && lane == __ffs(peers) - 1) counts[warp][bin] += __popc(peers);
    __syncwarp();
  }
  __syncthreads();
  // the places behind the range's first: tokens in order, of each the warps in order (a thread per token; at most kOrderMaxT of them)
  const bool has = static_cast<int>(threadIdx.x) < tokens;
  unsigned sum = 0;
  if (has) {
#pragma unroll 8
    for (int w = 0; w < kOrderWarps; ++w) sum += counts[w][threadIdx.x];
  }
  unsigned before = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned y = __shfl_up_sync(0xffffffffu, before, o);
    if (lane >= o) before += y;
  }
  if (lane == 31) found[warp] = before;
  __syncthreads();
  before += __reduce_add_sync(0xffffffffu, lane < warp ? found[lane] : 0u) - sum;
  if (has) {
    a.bounds[lo + threadIdx.x] = make_int2(base + before, base + before + sum);
#pragma unroll 8
    for (int w = 0; w < kOrderWarps; ++w) {
      const unsigned c = counts[w][threadIdx.x];
      counts[w][threadIdx.x] = before;
      before += c;
    }
  }
  __syncthreads();
  for (int i = from; i < to; i += 32) {
    const bool is = i + lane < to;
    const unsigned item = is ? list[i + lane] : 0u, bin = item >> 16;
    const unsigned peers = equal_lanes(bin, bits, __ballot_sync(0xffffffffu, is));
    const unsigned first = is ? counts[warp][bin] : 0u;
    __syncwarp();
    if (is) {
      const unsigned place = base + first + __popc(peers & ((1u << lane) - 1u));
      a.key_a[place] = lo + bin;
      a.pos_a[place] = item & 0xffffu;
      if (lane == __ffs(peers) - 1) counts[warp][bin] = first + __popc(peers);
    }
    __syncwarp();
  }
}

// More positions: a stable sort by digits, from the lowest. Every block has a tile of adjacent positions, `rounds` times kSortTile of them: small ones, so
// that the usual batches are many tiles.
constexpr int kSortThreads = 256, kSortWarps = kSortThreads / 32;
constexpr int kSortDigit = 9, kSortBins = 1 << kSortDigit;
constexpr int kSortPerLane = 4, kSortTile = kSortThreads * kSortPerLane;
constexpr int kSortMaxTiles = 296;      // (two blocks an SM; every block of the second kernel reads all tiles' counts)
static_assert(kSortBins == 2 * kSortThreads, "a thread has two bins");

// Where the keys of digit `p` are written to (alternating so that the last one writes key_a, pos_a).
__device__ __forceinline__ int* sort_keys(const EmbedSortArgs& a, int p) { return ((a.digits - 1 - p) & 1) ? a.key_b : a.key_a; }
__device__ __forceinline__ int* sort_positions(const EmbedSortArgs& a, int p) { return ((a.digits - 1 - p) & 1) ? a.pos_b : a.pos_a; }

// The keys and positions before digit p of one round, a warp's adjacent.
struct SortItems {
  int key[kSortPerLane], pos[kSortPerLane];
};
__device__ __forceinline__ void sort_load(const EmbedSortArgs& a, int p, long long first, SortItems& x) {
#pragma unroll
  for (int j = 0; j < kSortPerLane; ++j) {
    const long long i = first + (threadIdx.x >> 5) * (32 * kSortPerLane) + j * 32 + (threadIdx.x & 31);
    x.key[j] = -1;
    if (i < a.T) {
      if (p == 0) {
        const int token = a.tokens[i];
        if (token >= a.v && a.status) atomicOr(a.status, kStatusBadToken);
        x.key[j] = embed_key(a, token);
        x.pos[j] = static_cast<int>(i);
      } else {
        x.key[j] = sort_keys(a, p - 1)[i];
        x.pos[j] = sort_positions(a, p - 1)[i];
      }
    }
  }
}
__device__ __forceinline__ unsigned sort_digit(int key, int p) { return (static_cast<unsigned>(key) >> (p * kSortDigit)) & (kSortBins - 1); }

// counts[warp][bin] of the warp's keys. Equal digits of a warp's 32 keys find each other, the lowest lane counts them.
__device__ __forceinline__ void sort_count(const SortItems& x, int p, unsigned* counts) {
  unsigned* mine = counts + (threadIdx.x >> 5) * kSortBins;
  const int lane = threadIdx.x & 31;
  for (int b = lane; b < kSortBins; b += 32) mine[b] = 0;
  __syncwarp();
#pragma unroll
  for (int j = 0; j < kSortPerLane; ++j) {
    const unsigned digit = sort_digit(x.key[j], p);
    const unsigned peers = equal_lanes(digit, kSortDigit, __ballot_sync(0xffffffffu, x.key[j] >= 0));
    if (x.key[j] >= 0 && lane == __ffs(peers) - 1) mine[digit] += __popc(peers);
    __syncwarp();
  }
}
// counts -> the place of the warp's first key of each bin; base: that of the block's first keys of the thread's two bins, and behind it the next round's.
__device__ __forceinline__ void sort_offsets(unsigned* counts, unsigned (&base)[2]) {
#pragma unroll
  for (int w = 0; w < kSortWarps; ++w) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const unsigned c = counts[w * kSortBins + 2 * threadIdx.x + i];
      counts[w * kSortBins + 2 * threadIdx.x + i] = base[i];
      base[i] += c;
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
    const bool is = x.key[j] >= 0;
    const unsigned digit = sort_digit(x.key[j], p);
    const unsigned peers = equal_lanes(digit, kSortDigit, __ballot_sync(0xffffffffu, is));
    const unsigned first = is ? mine[digit] : 0u;
    __syncwarp();
    if (is) {
      const unsigned at = first + __popc(peers & ((1u << lane) - 1u));
      keys[at] = x.key[j];
      positions[at] = x.pos[j];
      if (lane == __ffs(peers) - 1) mine[digit] = first + __popc(peers);
    }
    __syncwarp();
  }
}
// Exclusive running sum of one value a thread over the block.
__device__ __forceinline__ unsigned block_running_sum(unsigned x, unsigned* warp_sums) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  unsigned sum = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned y = __shfl_up_sync(0xffffffffu, sum, o);
    if (lane >= o) sum += y;
  }
  if (lane == 31) warp_sums[warp] = sum;
  __syncthreads();
  return __reduce_add_sync(0xffffffffu, lane < warp ? warp_sums[lane] : 0u) + sum - x;
}

// One digit: the tiles' counts, hist[tile][bin]; and every tile's keys to their places. Where those begin, over the bins and of each the tiles, every block adds
// up for itself (with a launch of one block between the two that did so, and tiles of 4096: the gradient of 65536 positions of 512 55 us, now 44.5). The
// blocks of the first count that have no tile prefetch, and clear the bounds if a later kernel finds them.
__global__ void __launch_bounds__(kSortThreads) embed_count_kernel(const __grid_constant__ EmbedSortArgs a, int p) {
  __shared__ unsigned counts[kSortWarps * kSortBins];
  grid_dependency_wait();
  grid_launch_dependents();
  if (static_cast<int>(blockIdx.x) >= a.tiles) {
    const int part = blockIdx.x - a.tiles, parts = gridDim.x - a.tiles;
    if (a.digits > 1)
      for (int b = part * kSortThreads + threadIdx.x; b <= a.v; b += parts * kSortThreads) a.bounds[b] = make_int2(0, 0);
    prefetch_rows(a, part, parts);
    return;
  }
  uint2 sum = make_uint2(0, 0);
  for (int r = 0; r < a.rounds; ++r) {
    SortItems x;
    sort_load(a, p, (static_cast<long long>(blockIdx.x) * a.rounds + r) * kSortTile, x);
    sort_count(x, p, counts);
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kSortWarps; ++w) {
      sum.x += counts[w * kSortBins + 2 * threadIdx.x];
      sum.y += counts[w * kSortBins + 2 * threadIdx.x + 1];
    }
    __syncthreads();
  }
  a.hist[blockIdx.x * kSortThreads + threadIdx.x] = sum;
}
__global__ void __launch_bounds__(kSortThreads) embed_scatter_kernel(const __grid_constant__ EmbedSortArgs a, int p) {
  __shared__ unsigned counts[kSortWarps * kSortBins];
  __shared__ unsigned warp_sums[kSortWarps];
  grid_dependency_wait();
  grid_launch_dependents();
  SortItems x;
  sort_load(a, p, static_cast<long long>(blockIdx.x) * a.rounds * kSortTile, x);
  uint2 all = make_uint2(0, 0), before = make_uint2(0, 0);
#pragma unroll 16
  for (int t = 0; t < a.tiles; ++t) {
    const uint2 c = a.hist[t * kSortThreads + threadIdx.x];
    all.x += c.x, all.y += c.y;
    if (t < static_cast<int>(blockIdx.x)) before.x += c.x, before.y += c.y;
  }
  const unsigned first = block_running_sum(all.x + all.y, warp_sums), second = first + all.x;
  if (a.digits == 1 && blockIdx.x == 0) {
    const int b = 2 * threadIdx.x;
    if (b <= a.v) a.bounds[b] = make_int2(first, second);
    if (b < a.v) a.bounds[b + 1] = make_int2(second, second + all.y);
  }
  unsigned base[2] = {first + before.x, second + before.y};
  for (int r = 0; r < a.rounds; ++r) {
    if (r > 0) sort_load(a, p, (static_cast<long long>(blockIdx.x) * a.rounds + r) * kSortTile, x);
    sort_count(x, p, counts);
    __syncthreads();
    sort_offsets(counts, base);
    __syncthreads();
    sort_place(a, x, p, counts);
    __syncthreads();
  }
}

__global__ void __launch_bounds__(256) embed_bounds_kernel(const __grid_constant__ EmbedSortArgs a) {
  grid_dependency_wait();
  grid_launch_dependents();
  for (int i = blockIdx.x * 256 + threadIdx.x; i < a.T; i += gridDim.x * 256) {
    const int key = a.key_a[i];
    if (i == 0 || a.key_a[i - 1] != key) a.bounds[key].x = i;
    if (i == a.T - 1 || a.key_a[i + 1] != key) a.bounds[key].y = i + 1;
  }
}

// ---------------------------------------------------------------- sums of the sorted positions
constexpr int kSegmentThreads = 256;
constexpr int kSegmentStage = 256;      // positions whose keys are in shared memory at a time
constexpr int kClearRows = 8;           // rows that a block clears at a time

struct EmbedSegmentArgs {
  const int *key, *pos;                 // sorted; key v: no token
  const int2* bounds;
  const void* d_out;
  float *d_table, *part;                // part [chunks][2][d]: what a chunk adds to the token it begins in / that goes on behind it
  long long d_out_stride, d_table_stride;
  int T, v, d, chunk, chunks, slabs;    // slabs: of the columns
  int clear_begin, clear_end;           // the rows that this launch's further blocks look at
  float scale;
  bool accumulate;
  int row_vec;                          // vectors of so many elements fit the table's rows
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

// Zeros to the rows without positions: block `part` of `parts`, kClearRows adjacent rows at a time (longer runs per block write slower:
// 256 MB by blocks of 256 threads in runs of 56 KB 41 us, warps with runs of 64 KB 47 to 75).
__device__ __forceinline__ void clear_rows(const EmbedSegmentArgs& a, int part, int parts) {
  const int lane = threadIdx.x & 31;
  const int groups = (a.clear_end - a.clear_begin + kClearRows - 1) / kClearRows;
  for (int g = part; g < groups; g += parts) {
    const int row0 = a.clear_begin + g * kClearRows;
    bool none = false;
    if (lane < kClearRows && row0 + lane < a.clear_end) {
      const int2 b = a.bounds[row0 + lane];
      none = b.x == b.y;
    }
    for (unsigned absent = __ballot_sync(0xffffffffu, none); absent; absent &= absent - 1) {
      float* row = a.d_table + (row0 + __ffs(absent) - 1) * a.d_table_stride;
      if (a.row_vec == 8) {
        const float zeros[8] = {};
        for (int i = threadIdx.x * 8; i < a.d; i += blockDim.x * 8) st_global_v8(row + i, zeros);
      } else if (a.row_vec == 4) {
        for (int i = threadIdx.x; i < a.d / 4; i += blockDim.x) reinterpret_cast<float4*>(row)[i] = make_float4(0.f, 0.f, 0.f, 0.f);
      } else {
        for (int i = threadIdx.x; i < a.d; i += blockDim.x) row[i] = 0.f;
      }
    }
  }
}

// V adjacent sums, in pairs where they are several.
template <typename T, int V>
struct RowSum {
  uint64_t pairs[V / 2 > 0 ? V / 2 : 1];
  float one;
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (uint64_t& x : pairs) x = 0;
    one = 0.f;
  }
  __device__ __forceinline__ void add(const Raw<T, V>& x) {
    if constexpr (V == 1) {
      one += x.value(0);
    } else {
#pragma unroll
      for (int i = 0; i < V / 2; ++i) pairs[i] = add2(pairs[i], x.pair(i));
    }
  }
  __device__ __forceinline__ void get(float (&x)[V]) const {
    if constexpr (V == 1) {
      x[0] = one;
    } else {
#pragma unroll
      for (int i = 0; i < V / 2; ++i) {
        const float2 y = unpack2(pairs[i]);
        x[2 * i] = y.x, x[2 * i + 1] = y.y;
      }
    }
  }
};

// A block per chunk and slab of columns (the slabs of a chunk follow each other), beside those that clear. U rows are in flight per thread. A slab is
// 4 KB of a row where rows are that long: in slabs of 1 KB, with four times as long chunks, the kernel alone takes 26 to 32 us instead of
// 25 (8192 x 4096 fp32), by registers or by a ring of cp.async.
template <typename T, int V, int U>
__global__ void __launch_bounds__(kSegmentThreads, 4) embed_segment_kernel(const __grid_constant__ EmbedSegmentArgs a) {
  static_assert(32 % U == 0 && kSegmentStage == 256, "a group's bits lie in one of eight words");
  __shared__ alignas(16) const T* row[kSegmentStage];
  __shared__ int key[kSegmentStage + 1];
  __shared__ alignas(16) unsigned valid[kSegmentStage / 32], ends[kSegmentStage / 32];      // bits: has a token; the last one of it or of the chunk
  grid_dependency_wait();
  if (static_cast<int>(blockIdx.x) >= a.chunks * a.slabs) {
    clear_rows(a, blockIdx.x - a.chunks * a.slabs, gridDim.x - a.chunks * a.slabs);
    grid_launch_dependents();
    return;
  }
  const int chunk = blockIdx.x / a.slabs, lane = threadIdx.x & 31;
  const int col = ((blockIdx.x - chunk * a.slabs) * blockDim.x + threadIdx.x) * V;
  const int lo = chunk * a.chunk, hi = min(lo + a.chunk, a.T);
  RowSum<T, V> sum;
  sum.clear();
  float* part = a.part + static_cast<size_t>(chunk) * 2 * a.d + col;
  bool begins = true;                            // the token being added up has no position in an earlier chunk
  for (int base = lo; base < hi; base += kSegmentStage) {
    const int here = min(hi - base, kSegmentStage);
    const int earlier = base == lo && lo > 0 ? a.key[lo - 1] : -1;
    __syncthreads();
    for (int i = threadIdx.x; i <= here; i += blockDim.x) {
      key[i] = base + i < a.T ? a.key[base + i] : a.v;
      if (i < here) row[i] = static_cast<const T*>(a.d_out) + a.pos[base + i] * a.d_out_stride;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < kSegmentStage; i += blockDim.x) {
      const bool is = i < here && key[i] != a.v;
      const unsigned some = __ballot_sync(0xffffffffu, is), last = __ballot_sync(0xffffffffu, is && (key[i + 1] != key[i] || base + i + 1 == hi));
      if (lane == 0) valid[i / 32] = some, ends[i / 32] = last;
    }
    __syncthreads();
    if (base == lo) begins = earlier != key[0];
    int count = 0;                               // the positions that have a token come first
#pragma unroll
    for (int w = 0; w < kSegmentStage / 32; ++w) count += __popc(valid[w]);
    if (count == 0) break;
    if (col >= a.d) continue;
    for (int i = 0; i < count; i += U) {
      Raw<T, V> x[U];
      const unsigned stops = ends[i / 32] >> (i % 32);
      if (i + U <= count) {
#pragma unroll
        for (int u = 0; u < U; ++u) x[u].load(row[i + u] + col);
      } else {
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (i + u < count) x[u].load(row[i + u] + col);
      }
      if (i + U <= count && (stops & ((1u << U) - 1u)) == 0u) {
#pragma unroll
        for (int u = 0; u < U; ++u) sum.add(x[u]);
        continue;
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (i + u >= count) break;
        sum.add(x[u]);
        if ((stops >> u) & 1u) {
          float total[V];
          sum.get(total);
          const bool over = key[i + u + 1] != key[i + u];                // the token's last position, not only the chunk's
          if (begins && over) write_table<V>(a, key[i + u], col, total);
          else store_f32<float, V>(part + (begins ? a.d : 0), total);
          sum.clear();
          begins = true;
        }
      }
    }
  }
  grid_launch_dependents();
}

// The tokens that cross chunks. A block has eight chunks and 32 V columns; the chunk in which such a token begins answers for it: a warp adds up its
// parts if they are at most eight, all warps together (every eighth part each, then the warps' sums) if they are more.
constexpr int kJoinWarps = 8;
template <int V>
__global__ void __launch_bounds__(32 * kJoinWarps) embed_join_kernel(const __grid_constant__ EmbedSegmentArgs a) {
  __shared__ float share[kJoinWarps][32][V];
  grid_dependency_wait();
  grid_launch_dependents();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int slabs = (a.d + 32 * V - 1) / (32 * V), groups = (a.chunks + kJoinWarps - 1) / kJoinWarps;
  if (static_cast<int>(blockIdx.x) >= groups * slabs) {
    clear_rows(a, blockIdx.x - groups * slabs, gridDim.x - groups * slabs);
    return;
  }
  const int c0 = blockIdx.x / slabs * kJoinWarps;
  const int col = ((blockIdx.x - blockIdx.x / slabs * slabs) * 32 + lane) * V;
  int token = a.v, last = -1;                                           // lane q: of chunk c0 + q, and the last chunk that has the token
  if (lane < kJoinWarps && c0 + lane < a.chunks) {
    const int lo = (c0 + lane) * a.chunk, hi = min(lo + a.chunk, a.T);
    token = a.key[hi - 1];
    if (token != a.v) {
      const int2 b = a.bounds[token];
      if (b.x >= lo && b.y > hi) last = (b.y - 1) / a.chunk;            // begins here and goes on
    }
  }
  auto add = [&](int begin, int end, int first, int step, float (&sum)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) sum[i] = 0.f;
    if (col >= a.d) return;
#pragma unroll 8
    for (int q = begin + first; q <= end; q += step) {
      float x[V];
      unpack(load_pack<float, V>(a.part + (static_cast<size_t>(q) * 2 + (q == begin ? 1 : 0)) * a.d + col), x);
#pragma unroll
      for (int i = 0; i < V; ++i) sum[i] += x[i];
    }
  };
  const unsigned owners = __ballot_sync(0xffffffffu, last >= 0), many = __ballot_sync(0xffffffffu, last - (c0 + lane) >= kJoinWarps);
  const int own_token = __shfl_sync(0xffffffffu, token, warp), own_last = __shfl_sync(0xffffffffu, last, warp);
  float sum[V];
  if ((owners & ~many) >> warp & 1u) {
    add(c0 + warp, own_last, 0, 1, sum);
    if (col < a.d) write_table<V>(a, own_token, col, sum);
  }
  for (unsigned left = many; left; left &= left - 1) {                  // (the same in every warp)
    const int q = __ffs(left) - 1;
    const int its_token = __shfl_sync(0xffffffffu, token, q);
    add(c0 + q, __shfl_sync(0xffffffffu, last, q), warp, kJoinWarps, sum);
#pragma unroll
    for (int i = 0; i < V; ++i) share[warp][lane][i] = sum[i];
    __syncthreads();
    if (warp == 0 && col < a.d) {
      for (int w = 1; w < kJoinWarps; ++w) {
#pragma unroll
        for (int i = 0; i < V; ++i) sum[i] += share[w][lane][i];
      }
      write_table<V>(a, its_token, col, sum);
    }
    __syncthreads();
  }
}

// Few positions: a block has its columns of every gridDim.x-th row of the table and adds up the positions that have the row's token, U on their way at a
// time, or writes zeros. (T = 128, d = 1024, bf16, 268 rows: the other kernels 14 us, this one 6.)
constexpr int kFewT = 128, kFewThreads = 256;
template <typename T, int V, int U>
__global__ void __launch_bounds__(kFewThreads) embed_few_kernel(const int* tokens, const __grid_constant__ EmbedSegmentArgs a, unsigned* status) {
  __shared__ int token[kFewT];
  __shared__ int place[kFewThreads / 32][kFewT];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int col = (blockIdx.y * blockDim.x + threadIdx.x) * V;
  grid_dependency_wait();
  grid_launch_dependents();
  for (int i = threadIdx.x; i < a.T; i += blockDim.x) {
    token[i] = tokens[i];
    if (blockIdx.x == 0 && blockIdx.y == 0 && token[i] >= a.v && status) atomicOr(status, kStatusBadToken);
  }
  __syncthreads();
  for (int b = blockIdx.x; b < a.v; b += gridDim.x) {
    int count = 0;                             // of the row's positions, in order (a warp's own list)
    for (int i = 0; i < a.T; i += 32) {
      const bool is = i + lane < a.T && token[i + lane] == b;
      const unsigned which = __ballot_sync(0xffffffffu, is);
      if (is) place[warp][count + __popc(which & ((1u << lane) - 1u))] = i + lane;
      count += __popc(which);
    }
    __syncwarp();
    if ((count > 0 || !a.accumulate) && col < a.d) {
      float sum[V];
#pragma unroll
      for (int i = 0; i < V; ++i) sum[i] = 0.f;
      for (int i = 0; i < count; i += U) {
        Raw<T, V> x[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (i + u < count) x[u].load(static_cast<const T*>(a.d_out) + place[warp][i + u] * a.d_out_stride + col);
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (i + u < count) {
#pragma unroll
            for (int e = 0; e < V; ++e) sum[e] += x[u].value(e);
          }
        }
      }
      write_table<V>(a, b, col, sum);
    }
    __syncwarp();                              // the list may be written again
  }
}

}  // namespace mtpc
