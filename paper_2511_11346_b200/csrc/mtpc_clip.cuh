// The 2-norm of many gradient tensors together, and the gradients scaled to a largest norm.
//   norm = sqrt(sum over all tensors of g^2),   out = g min(1, max_norm / norm)
// Two passes over the data, since no element can be scaled before the last one is squared. The tensors are cut into chunks when the list is made, so
// that a list of one large tensor and one of thousands of small ones are the same work, dealt evenly. The second pass walks the chunks
// backwards: what the first one read last is still in L2 (126 MB).
// Squares and their sums are fp64, so that no fp32 gradient overflows or vanishes in them; the order of every sum is fixed.
#pragma once
#include <cuda_bf16.h>
#include <stdint.h>

#include "mtpc_ptx.cuh"
#include "mtpc_rows.cuh"

namespace mtpc {

constexpr int kClipThreads = 256;
constexpr int kClipChunk = 8192;             // elements
constexpr int kClipAhead = 2;                // vectors of eight in flight per thread
constexpr int kClipMaxBlocks = 148 * 8;

struct ClipChunk {
  const void* g;
  void* out;                                 // NULL: the norm alone is wanted
  int count;
  unsigned kind;                             // kClip* bits, and from bit 8 on the elements before the first that vectors may start at
};
constexpr unsigned kClipF32 = 1u, kClipOutF32 = 2u, kClipWide = 4u;     // Wide: behind those, both addresses allow vectors of eight elements

template <typename T>
__device__ __forceinline__ double chunk_square(const ClipChunk& c) {
  const T* g = static_cast<const T*>(c.g);
  double sum = 0.0;
  int done = 0;
  if (c.kind & kClipWide) {
    const int head = c.kind >> 8, packs = (c.count - head) / 8;
    if (static_cast<int>(threadIdx.x) < head) {
      const double x = to_f32(g[threadIdx.x]);
      sum += x * x;
    }
    for (int i = threadIdx.x; i < packs; i += kClipAhead * kClipThreads) {
      Pack<T, 8> p[kClipAhead];
#pragma unroll
      for (int u = 0; u < kClipAhead; ++u)
        if (i + u * kClipThreads < packs) p[u] = load_pack<T, 8>(g + head + (i + u * kClipThreads) * 8);
#pragma unroll
      for (int u = 0; u < kClipAhead; ++u) {
        if (i + u * kClipThreads < packs) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const double x = to_f32(p[u].e[e]);
            sum += x * x;
          }
        }
      }
    }
    done = head + packs * 8;
  }
#pragma unroll 4
  for (int i = done + threadIdx.x; i < c.count; i += kClipThreads) {
    const double x = to_f32(g[i]);
    sum += x * x;
  }
  return sum;
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

__global__ void __launch_bounds__(kClipThreads) gradient_square_kernel(const ClipChunk* chunks, int count, double* partial) {
  __shared__ double share[kClipThreads / 32];
  grid_dependency_wait();
  double sum = 0.0;
  for (int c = blockIdx.x; c < count; c += gridDim.x) {
    const ClipChunk chunk = chunks[c];
    sum += (chunk.kind & kClipF32) ? chunk_square<float>(chunk) : chunk_square<__nv_bfloat16>(chunk);
  }
  sum = block_sum(sum, share);
  if (threadIdx.x == 0) partial[blockIdx.x] = sum;
  grid_launch_dependents();
}

template <typename TI, typename TO>
__device__ __forceinline__ void chunk_scale(const ClipChunk& c, float first, float by) {
  const TI* g = static_cast<const TI*>(c.g);
  TO* out = static_cast<TO*>(c.out);
  int done = 0;
  if (c.kind & kClipWide) {
    const int head = c.kind >> 8, packs = (c.count - head) / 8;
    if (static_cast<int>(threadIdx.x) < head) out[threadIdx.x] = from_f32<TO>(to_f32(g[threadIdx.x]) * first * by);
    for (int i = threadIdx.x; i < packs; i += kClipAhead * kClipThreads) {
      Pack<TI, 8> p[kClipAhead];
#pragma unroll
      for (int u = 0; u < kClipAhead; ++u)
        if (i + u * kClipThreads < packs) p[u] = load_pack<TI, 8>(g + head + (i + u * kClipThreads) * 8);
#pragma unroll
      for (int u = 0; u < kClipAhead; ++u) {
        if (i + u * kClipThreads < packs) {
          float x[8];
          unpack(p[u], x);
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = x[e] * first * by;
          store_f32<TO, 8>(out + head + (i + u * kClipThreads) * 8, x);
        }
      }
    }
    done = head + packs * 8;
  }
#pragma unroll 4
  for (int i = done + threadIdx.x; i < c.count; i += kClipThreads) out[i] = from_f32<TO>(to_f32(g[i]) * first * by);
}

// blocks: of the kernel before.
__global__ void __launch_bounds__(kClipThreads) gradient_scale_kernel(const ClipChunk* chunks, int count, const double* partial, int blocks,
                                                                      float max_norm, float* out_norm) {
  __shared__ double share[kClipThreads / 32];
  grid_dependency_wait();
  double sum = 0.0;
  for (int i = threadIdx.x; i < blocks; i += kClipThreads) sum += partial[i];
  const double norm = sqrt(block_sum(sum, share));
  if (blockIdx.x == 0 && threadIdx.x == 0) out_norm[0] = static_cast<float>(norm);
  // A norm that is not finite scales nothing: the gradients stay as they are.
  const double ratio = norm > max_norm && norm <= 1.7976931348623157e308 ? max_norm / norm : 1.0;
  // A ratio near the end of fp32's range is multiplied in two steps, the first a power of two.
  const float first = ratio < 0x1p-100 ? 0x1p-64f : 1.f, by = static_cast<float>(ratio / first);
  for (int c = count - 1 - static_cast<int>(blockIdx.x); c >= 0; c -= gridDim.x) {
    const ClipChunk chunk = chunks[c];
    if (chunk.out == nullptr || (chunk.out == chunk.g && ratio == 1.0)) continue;
    if (chunk.kind & kClipF32) {
      if (chunk.kind & kClipOutF32) chunk_scale<float, float>(chunk, first, by);
      else chunk_scale<float, __nv_bfloat16>(chunk, first, by);
    } else {
      if (chunk.kind & kClipOutF32) chunk_scale<__nv_bfloat16, float>(chunk, first, by);
      else chunk_scale<__nv_bfloat16, __nv_bfloat16>(chunk, first, by);
    }
  }
  grid_launch_dependents();
}

}  // namespace mtpc
