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
// Two sums at once, of a block of at most sixteen warps: half of the lanes carry each. red: 32 floats, zero from the number of warps on (and from 16 and it on).
__device__ __forceinline__ void row_sums(float (&x)[2], float* red) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const bool upper = lane & 16;
  float mine = (upper ? x[1] : x[0]) + __shfl_xor_sync(0xffffffffu, upper ? x[0] : x[1], 16);
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
  if (blockDim.x > 32) {
    if ((lane & 15) == 0) red[lane + warp] = mine;
    __syncthreads();
    mine = red[lane];
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
  }
  x[0] = __shfl_sync(0xffffffffu, mine, 0);
  x[1] = __shfl_sync(0xffffffffu, mine, 16);
}

// Two fp32 values as one operand: the packed multiply-adds do both in one instruction.
__device__ __forceinline__ uint64_t pack2(float lo, float hi) {
  uint64_t d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(lo), "f"(hi));
  return d;
}
__device__ __forceinline__ float2 unpack2(uint64_t x) {
  float2 d;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(d.x), "=f"(d.y) : "l"(x));
  return d;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}

// V adjacent elements as they were read, by a load that stays where it is written (of a Pack's bf16 elements a conditional load is taken apart at once, so
// that each waits for its own data); and as fp32, one by one or in pairs.
template <typename T, int V>
struct Raw {
  static constexpr int kBytes = sizeof(T) * V;
  uint32_t r[kBytes < 4 ? 1 : kBytes / 4];
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (kBytes == 32)
      asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                   : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                   : "l"(p));
    else if constexpr (kBytes == 16)
      asm volatile("ld.global.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "l"(p));
    else if constexpr (kBytes == 8)
      asm volatile("ld.global.v2.b32 {%0, %1}, [%2];" : "=r"(r[0]), "=r"(r[1]) : "l"(p));
    else if constexpr (kBytes == 4)
      asm volatile("ld.global.b32 %0, [%1];" : "=r"(r[0]) : "l"(p));
    else
      asm volatile("ld.global.u16 %0, [%1];" : "=r"(r[0]) : "l"(p));
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (uint32_t& x : r) x = 0;
  }
  __device__ __forceinline__ float value(int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(r[i]);
    else return __uint_as_float(i & 1 ? r[i / 2] & 0xffff0000u : r[i / 2] << 16);
  }
  __device__ __forceinline__ uint64_t pair(int i) const { return pack2(value(2 * i), value(2 * i + 1)); }
};
template <typename T>
__device__ __forceinline__ void store_pairs(T* p, const uint64_t (&x)[4]) {
  float y[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 v = unpack2(x[i]);
    y[2 * i] = v.x, y[2 * i + 1] = v.y;
  }
  store_f32<T, 8>(p, y);
}

// A row of d elements whose first vector of eight elements does not start it: `head` elements, `packs` vectors, `rest` elements. The elements beside the
// vectors, at most fourteen, go one to a thread (beside: its column, -1: none). Rows at a pitch that is no multiple of eight start at
// different places; those of several matrices do so alike if their addresses and pitches are alike modulo eight elements (`shift`, `pitch`).
struct SplitRow {
  int head, packs, rest;
  __device__ __forceinline__ SplitRow(int shift, int pitch, int row, int d) {
    head = min((8 - ((shift + (row & 7) * pitch) & 7)) & 7, d);
    packs = (d - head) / 8;
    rest = d - head - packs * 8;
  }
  __device__ __forceinline__ int beside(int tid) const { return tid < head ? tid : tid < head + rest ? packs * 8 + tid : -1; }
};

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

// One weight, and eight that lie anywhere.
__device__ __forceinline__ float load_weight1(const void* weight, bool f32, int col) {
  if (weight == nullptr) return 1.f;
  return f32 ? static_cast<const float*>(weight)[col] : to_f32(static_cast<const __nv_bfloat16*>(weight)[col]);
}
__device__ __forceinline__ void load_weight8(const void* weight, bool f32, int col, float (&w)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = load_weight1(weight, f32, col + i);
}

}  // namespace mtpc
