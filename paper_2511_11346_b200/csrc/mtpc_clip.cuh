// The 2-norm of many gradient tensors together, and the gradients scaled to a largest norm.
//   norm = sqrt(sum over all tensors of g^2),   out = g min(1, max_norm / norm)
// Two passes over the data, since no element can be scaled before the last one is squared. The tensors are cut into chunks of 2048 elements when the
// list is made, eight to a thread, so that a list of one large tensor and one of thousands of small ones are the same work; the chunks are dealt
// round-robin to the blocks, as many as take the same number of rounds. Where three chunks that follow each other in a block are full and fp32 on both sides, a thread
// has its elements of all three on their way at once, else of one chunk after the other (bf16 of 419 MB in place 345 us, fp32 of 671 MB 300). (Chunks of 8192
// left up to a third of the last round empty: 78 MB of fp32 48 us. A run of its own for every block writes a tenth
// slower than chunks dealt out. Hints to L2 what to keep: 2 % at best.) The second pass walks the chunks backwards: what the first one read last is still in L2
// (126 MB). Lists of fp32 after a flush of the caches, second pass alone: 40 MB 6 us, 80 MB 16, 120 MB 27, 640 MB 158, which is 12.8, 9.8, 9.0 and 8.1 TB/s of what
// it reads and writes, where a copy of 640 MB reaches 6.3.
// Squares and their sums are fp64, so that no fp32 gradient overflows or vanishes in them; the order of every sum is fixed.
#pragma once
#include <cuda_bf16.h>
#include <stdint.h>

#include "mtpc_ptx.cuh"
#include "mtpc_rows.cuh"

namespace mtpc {

constexpr int kClipThreads = 256;
constexpr int kClipChunk = 8 * kClipThreads;   // elements (the first chunk of a tensor: and those before its first vector)
constexpr int kClipAhead = 3;                  // chunks in flight, where they are full and fp32
constexpr int kClipBlocks = 148 * 4;           // of a wave
constexpr int kClipWaves = 8;                  // at most
constexpr int kClipStage = 64;                 // chunks of a block that are known ahead (the last of a full stage goes by itself)

struct alignas(16) ClipChunk {
  const void* g;
  void* out;                                   // NULL: the norm alone is wanted
  int count;
  unsigned kind;                               // kClip* bits, and from bit 8 on the elements before the first that vectors may start at
  unsigned pad[2];
};
constexpr unsigned kClipF32 = 1u, kClipOutF32 = 2u, kClipWide = 4u;     // Wide: behind those, both addresses allow vectors of eight elements
constexpr unsigned kClipFull = 8u;             // Wide, nothing before the first vector, kClipChunk elements

// What a thread has of a chunk: a vector and perhaps one of the up to fourteen elements beside the vectors, or (not Wide) eight elements apart.
struct ClipItem {
  uint32_t x[8], beside;
};
struct ClipPlace {
  bool wide, has;                              // has: a vector, at `at`
  int at, beside;                              // beside: -1: none
};
__device__ __forceinline__ ClipPlace clip_place(const ClipChunk& c) {
  ClipPlace p;
  const int tid = threadIdx.x, head = c.kind >> 8, packs = (c.count - head) / 8, rest = c.count - head - packs * 8;
  p.wide = (c.kind & kClipWide) != 0;
  p.has = p.wide && tid < packs;
  p.at = head + tid * 8;
  p.beside = !p.wide ? -1 : tid < head ? tid : tid >= 8 && tid - 8 < rest ? head + packs * 8 + tid - 8 : -1;
  return p;
}
template <typename T>
__device__ __forceinline__ uint32_t raw_element(const T* p) {
  if constexpr (sizeof(T) == 4) return *reinterpret_cast<const uint32_t*>(p);
  else return *reinterpret_cast<const uint16_t*>(p);
}
template <typename T>
__device__ __forceinline__ void clip_load(const ClipChunk& c, ClipItem& item) {
  const T* g = static_cast<const T*>(c.g);
  const ClipPlace p = clip_place(c);
  if (p.wide) {
    if (p.has) {
      const Pack<T, 8> pack = load_pack<T, 8>(g + p.at);
      const uint32_t* words = reinterpret_cast<const uint32_t*>(pack.e);
#pragma unroll
      for (int i = 0; i < static_cast<int>(2 * sizeof(T)); ++i) item.x[i] = words[i];
    }
    if (p.beside >= 0) item.beside = raw_element(g + p.beside);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int at = threadIdx.x + i * kClipThreads;
      if (at < c.count) item.x[i] = raw_element(g + at);
    }
  }
}
__device__ __forceinline__ void clip_load(const ClipChunk& c, ClipItem& item) {
#pragma unroll
  for (int i = 0; i < 8; ++i) item.x[i] = 0;
  item.beside = 0;
  if (c.kind & kClipF32) clip_load<float>(c, item);
  else clip_load<__nv_bfloat16>(c, item);
}
// The elements as fp32 (zeros where there is none).
__device__ __forceinline__ void clip_values(const ClipChunk& c, const ClipItem& item, float (&x)[8], float& beside) {
  if (c.kind & kClipF32) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(item.x[i]);
    beside = __uint_as_float(item.beside);
  } else {
    beside = __uint_as_float(item.beside << 16);
    if (c.kind & kClipWide) {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[2 * i] = __uint_as_float(item.x[i] << 16), x[2 * i + 1] = __uint_as_float(item.x[i] & 0xffff0000u);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(item.x[i] << 16);
    }
  }
}

// Sum over the block; every thread has it.
__device__ __forceinline__ double block_sum(double x, double* share) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  if ((threadIdx.x & 31) == 0) share[threadIdx.x >> 5] = x;
  __syncthreads();
  x = 0.0;
#pragma unroll
  for (int w = 0; w < kClipThreads / 32; ++w) x += share[w];
  return x;
}

// The block's chunks, in the order of `walk` (its i-th is chunks[walk(i)], of `mine` in all), kClipAhead at a time. Where all of those are full and fp32,
// as most are of most lists, whole(chunks) does them, at half of the instructions; else part(chunk, item) each that skip(chunk) does not leave out.
template <typename Walk, typename Skip, typename Whole, typename Part>
__device__ __forceinline__ void clip_walk(const ClipChunk* chunks, int mine, ClipChunk* stage, Walk walk, Skip skip, Whole whole, Part part) {
  ClipChunk next;
  const int tid = threadIdx.x;
  if (tid < kClipStage && tid < mine) next = chunks[walk(tid)];
  for (int first = 0; first < mine; first += kClipStage) {
    const int here = min(kClipStage, mine - first);
    __syncthreads();
    if (tid < here) stage[tid] = next;
    __syncthreads();
    if (tid < kClipStage && first + kClipStage + tid < mine) next = chunks[walk(first + kClipStage + tid)];
    for (int i = 0; i < here; i += kClipAhead) {
      unsigned all = i + kClipAhead <= here ? kClipFull | kClipF32 | kClipOutF32 : 0u;
#pragma unroll
      for (int u = 0; u < kClipAhead; ++u)
        if (all && skip(stage[i + u])) all = 0;
        else if (all) all &= stage[i + u].kind;
      if (all == (kClipFull | kClipF32 | kClipOutF32)) {
        whole(stage + i);
      } else {
#pragma unroll 1
        for (int u = 0; u < min(kClipAhead, here - i); ++u) {
          if (skip(stage[i + u])) continue;
          ClipItem item;
          clip_load(stage[i + u], item);
          part(stage[i + u], item);
        }
      }
    }
  }
}

__global__ void __launch_bounds__(kClipThreads, 4) gradient_square_kernel(const ClipChunk* chunks, int count, double* partial) {
  __shared__ double share[kClipThreads / 32];
  __shared__ ClipChunk stage[kClipStage];
  grid_dependency_wait();
  double sum = 0.0;
  const int block = blockIdx.x, blocks = gridDim.x;
  clip_walk(chunks, block < count ? (count - block + blocks - 1) / blocks : 0, stage, [&](int i) { return block + i * blocks; },
            [](const ClipChunk&) { return false; },
            [&](const ClipChunk* c) {
              Pack<float, 8> x[kClipAhead];
#pragma unroll
              for (int u = 0; u < kClipAhead; ++u) x[u] = load_pack<float, 8>(static_cast<const float*>(c[u].g) + threadIdx.x * 8);
#pragma unroll
              for (int u = 0; u < kClipAhead; ++u) {
#pragma unroll
                for (int i = 0; i < 8; ++i) sum += static_cast<double>(x[u].e[i]) * x[u].e[i];
              }
            },
            [&](const ClipChunk& c, const ClipItem& item) {
              float x[8], beside;
              clip_values(c, item, x, beside);
#pragma unroll
              for (int i = 0; i < 8; ++i) sum += static_cast<double>(x[i]) * x[i];
              sum += static_cast<double>(beside) * beside;
            });
  sum = block_sum(sum, share);
  if (threadIdx.x == 0) partial[blockIdx.x] = sum;
  grid_launch_dependents();
}

template <typename T>
__device__ __forceinline__ void clip_store(const ClipChunk& c, const float (&x)[8], float beside) {
  T* out = static_cast<T*>(c.out);
  const ClipPlace p = clip_place(c);
  if (p.wide) {
    if (p.has) store_f32<T, 8>(out + p.at, x);
    if (p.beside >= 0) out[p.beside] = from_f32<T>(beside);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int at = threadIdx.x + i * kClipThreads;
      if (at < c.count) out[at] = from_f32<T>(x[i]);
    }
  }
}

// blocks: of both kernels.
__global__ void __launch_bounds__(kClipThreads, 4) gradient_scale_kernel(const ClipChunk* chunks, int count, const double* partial, int blocks,
                                                                         float max_norm, float* out_norm) {
  __shared__ double share[kClipThreads / 32];
  __shared__ ClipChunk stage[kClipStage];
  grid_dependency_wait();
  double sum = 0.0;
  for (int i = threadIdx.x; i < blocks; i += kClipThreads) sum += partial[i];
  const double norm = sqrt(block_sum(sum, share));
  if (blockIdx.x == 0 && threadIdx.x == 0) out_norm[0] = static_cast<float>(norm);
  // A norm that is not finite scales nothing: the gradients stay as they are.
  const double ratio = norm > max_norm && norm <= 1.7976931348623157e308 ? max_norm / norm : 1.0;
  // A ratio below fp32's normal range is multiplied in two steps, the first a power of two that leaves the least normal number to the second: what the first step
  // takes below the range is nothing after the second.
  const float first = ratio < 0x1p-126 ? ldexpf(1.f, max(ilogb(ratio) + 126, -149)) : 1.f, by = static_cast<float>(ratio / first);
  const int block = blockIdx.x;
  clip_walk(chunks, block < count ? (count - block + blocks - 1) / blocks : 0, stage, [&](int i) { return count - 1 - block - i * blocks; },
            [&](const ClipChunk& c) { return c.out == nullptr || (c.out == c.g && ratio == 1.0); },
            [&](const ClipChunk* c) {
              Pack<float, 8> x[kClipAhead];
#pragma unroll
              for (int u = 0; u < kClipAhead; ++u) x[u] = load_pack<float, 8>(static_cast<const float*>(c[u].g) + threadIdx.x * 8);
#pragma unroll
              for (int u = 0; u < kClipAhead; ++u) {
#pragma unroll
                for (int i = 0; i < 8; ++i) x[u].e[i] = x[u].e[i] * first * by;
                store_pack<float, 8>(static_cast<float*>(c[u].out) + threadIdx.x * 8, x[u]);
              }
            },
            [&](const ClipChunk& c, const ClipItem& item) {
              float x[8], beside;
              clip_values(c, item, x, beside);
#pragma unroll
              for (int i = 0; i < 8; ++i) x[i] = x[i] * first * by;
              beside = beside * first * by;
              if (c.kind & kClipOutF32) clip_store<float>(c, x, beside);
              else clip_store<__nv_bfloat16>(c, x, beside);
            });
  grid_launch_dependents();
}

}  // namespace mtpc
