// Adjacent elements of fp32 or bf16 rows, as the streaming kernels around the head read and write them.
#pragma once
#include <cuda_bf16.h>
#include <stdint.h>

#include "mtpc_ptx.cuh"

namespace mtpc {

// V adjacent elements, at most 32 bytes, moved as one access (the address is a multiple of their size).
template <typename T, int V>
struct alignas(sizeof(T) * V) Pack {
  T e[V];
};
template <typename T, int V>
__device__ __forceinline__ Pack<T, V> load_pack(const T* p) {
  static_assert(sizeof(T) * V <= 32, "a load moves 32 bytes at most");
  if constexpr (sizeof(T) * V == 32) {
    Pack<T, V> x;
    uint32_t* r = reinterpret_cast<uint32_t*>(x.e);
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "l"(p));
    return x;
  } else {
    return *reinterpret_cast<const Pack<T, V>*>(p);
  }
}
template <typename T, int V>
__device__ __forceinline__ void store_pack(T* p, const Pack<T, V>& x) {
  if constexpr (sizeof(T) * V == 32) st_global_v8_b32(p, reinterpret_cast<const uint32_t*>(x.e));
  else *reinterpret_cast<Pack<T, V>*>(p) = x;
}
__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T>
__device__ __forceinline__ T from_f32(float x);
template <>
__device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

template <typename T, int V>
__device__ __forceinline__ void unpack(const Pack<T, V>& p, float (&x)[V]) {
#pragma unroll
  for (int i = 0; i < V; ++i) x[i] = to_f32(p.e[i]);
}
template <typename T, int V>
__device__ __forceinline__ void store_f32(T* p, const float (&x)[V]) {
  Pack<T, V> o;
#pragma unroll
  for (int i = 0; i < V; ++i) o.e[i] = from_f32<T>(x[i]);
  store_pack<T, V>(p, o);
}

// 16 bytes from global to shared memory without registers; they are there once the thread has waited for the group they were committed in.
__device__ __forceinline__ void copy_async16(uint32_t dst_smem, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst_smem), "l"(src) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// The sum over the threads of a row: a warp, or (blockDim.x > 32) the whole block, every thread with the same result, added up in the same order.
// red: 32 floats in shared memory; a buffer may be used again after the next barrier.
__device__ __forceinline__ float row_sum(float x, float* red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  if (blockDim.x == 32) return x;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  if (lane == 0) red[warp] = x;
  __syncthreads();
  x = lane < warps ? red[lane] : 0.f;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}
// Two sums at once, for blocks that take many rows: within a warp they take the shuffles of one and another (half of the lanes carry each), the warps'
// sums are read as vectors. red: 32 floats each, zero from the row's number of warps on.
__device__ __forceinline__ void row_sum(float (&x)[2], float (*red)[32]) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  const bool upper = lane & 16;
  float mine = (upper ? x[1] : x[0]) + __shfl_xor_sync(0xffffffffu, upper ? x[0] : x[1], 16);
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
  if (blockDim.x == 32) {
    x[0] = __shfl_sync(0xffffffffu, mine, 0);
    x[1] = __shfl_sync(0xffffffffu, mine, 16);
    return;
  }
  if ((lane & 15) == 0) red[lane >> 4][warp] = mine;
  __syncthreads();
  x[0] = x[1] = 0.f;
  for (int w = 0; w < warps; w += 4) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float4 y = *reinterpret_cast<const float4*>(&red[i][w]);
      x[i] += (y.x + y.y) + (y.z + y.w);
    }
  }
}

// Before the first such sums on a block's buffers (`count` floats): the words of warps that are not there.
__device__ __forceinline__ void clear_row_sums(float* red, int count) {
  if (blockDim.x == 32) return;
  for (int i = threadIdx.x; i < count; i += blockDim.x) red[i] = 0.f;
  __syncthreads();
}

// V adjacent weights (fp32 or bf16; none: ones).
template <int V>
__device__ __forceinline__ void load_weight(const void* weight, bool f32, int col, float (&w)[V]) {
  if (weight == nullptr) {
#pragma unroll
    for (int i = 0; i < V; ++i) w[i] = 1.f;
  } else if (f32) {
    unpack(load_pack<float, V>(static_cast<const float*>(weight) + col), w);
  } else {
    unpack(load_pack<__nv_bfloat16, V>(static_cast<const __nv_bfloat16*>(weight) + col), w);
  }
}

}  // namespace mtpc
