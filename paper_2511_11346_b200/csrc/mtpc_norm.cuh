// Residual addition and root-mean-square norm of the rows that the head reads as hidden states, and their gradients.
//   s = x + residual,  rstd = (mean(s^2) + eps)^(-1/2),  out = s rstd weight
//   d s = rstd (weight d_out - s rstd^2 mean(weight d_out s)) + d_stream,   d weight = sum over the rows of d_out s rstd
// (d s is the gradient of x and of residual alike.) Everything between the loads and the one rounding of each output is fp32.
//
// Both are streams: a row is read once, into registers, and everything is formed from there. A row is a warp's up to 64 vectors of eight
// elements, beyond that a block's with one vector a thread, so that a single row (one sequence being decoded) is spread over as
// many warps as it can be.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <stdint.h>

#include "mtpc_ptx.cuh"
#include "mtpc_rows.cuh"

namespace mtpc {

constexpr int kNormMaxWidth = 32768;     // columns: 1024 threads of 32
constexpr int kNormMinGroup = 32;        // columns that share a scale: 32, 64 or 128 (or the row)
constexpr float kE4m3Max = 448.f;
// Rows whose squares overflow fp32 are formed once more from s times this. What 2^-100 takes below the range is 2^-20 of
// the row's largest value at most.
constexpr float kNormRescue = 0x1p-100f;

struct NormArgs {
  const void *x, *residual, *weight;      // residual, weight: may be NULL
  void *sum, *out;                        // may be NULL
  uint8_t* codes;                         // e4m3, may be NULL
  float* scales;                          // [T, groups]
  long long x_stride, residual_stride, sum_stride, out_stride, codes_stride;
  int T, d, group, groups;                // group: columns that share a scale (0: the row)
  int group_shift;                        // its logarithm
  bool weight_f32;
  float eps, inv_d;
};

// Largest magnitude as the bits of an fp32: compared as integers a NaN is larger than everything, so it is not lost.
__device__ __forceinline__ unsigned magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// What a code of 1 stands for where the largest magnitude is `bits`.
__device__ __forceinline__ float code_scale(unsigned bits) {
  const float s = __uint_as_float(bits) * (1.f / kE4m3Max);
  return s == 0.f ? 1.f : s;
}
// x / scale as x * first * second (a reciprocal beside eight products, where eight divisions took longer than the row's bytes). Scales whose
// reciprocal fp32 cannot hold go in two steps, the first a power of two.
__device__ __forceinline__ float2 code_factors(float scale) {
  const float first = scale < 0x1p-100f ? 0x1p64f : 1.f;
  return make_float2(first, __fdividef(1.f, scale * first));          // (scale * first is between 2^-100 and 2^120)
}

template <typename IO, int V, int NV, int THREADS, int CTAS>
__global__ void __launch_bounds__(THREADS, CTAS) residual_rmsnorm_kernel(const __grid_constant__ NormArgs a) {
  __shared__ float red[2][32];
  __shared__ unsigned group_max[V == 1 ? kNormMaxWidth / kNormMinGroup : 1];
  const int row = blockIdx.x * blockDim.y + threadIdx.y;
  const int tid = threadIdx.x, lane = tid & 31;
  if (V == 1 && a.codes != nullptr) {            // (rows of single elements are a block's: blockDim.y = 1)
    for (int g = tid; g < a.groups && a.group != 0; g += blockDim.x) group_max[g] = 0;
    __syncthreads();
  }
  grid_dependency_wait();
  grid_launch_dependents();
  if (row >= a.T) return;                                    // a whole warp, or no thread
  const IO* x = static_cast<const IO*>(a.x) + row * a.x_stride;
  const IO* residual = static_cast<const IO*>(a.residual) + (a.residual ? row * a.residual_stride : 0);
  IO* sum = static_cast<IO*>(a.sum) + (a.sum ? row * a.sum_stride : 0);

  float s[NV][V];
  {
    Pack<IO, V> px[NV], pr[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int col = (tid + j * blockDim.x) * V;
      if (col < a.d) {
        px[j] = load_pack<IO, V>(x + col);
        if (a.residual) pr[j] = load_pack<IO, V>(residual + col);
      }
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int col = (tid + j * blockDim.x) * V;
#pragma unroll
      for (int i = 0; i < V; ++i) s[j][i] = 0.f;
      if (col < a.d) {
        unpack(px[j], s[j]);
        if (a.residual) {
          float r[V];
          unpack(pr[j], r);
#pragma unroll
          for (int i = 0; i < V; ++i) s[j][i] += r[i];
        }
        if (a.sum) store_f32<IO, V>(sum + col, s[j]);
      }
    }
  }
  float square = 0.f;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
#pragma unroll
    for (int i = 0; i < V; ++i) square += s[j][i] * s[j][i];
  }
  square = row_sum(square, red[0]);
  float rstd = rsqrtf(square * a.inv_d + a.eps);
  if (__float_as_uint(square) == 0x7f800000u) {              // the same in every thread of the row
    square = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        s[j][i] *= kNormRescue;
        square += s[j][i] * s[j][i];
      }
    }
    square = row_sum(square, red[1]);
    rstd = rsqrtf(square * a.inv_d);
  }
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int col = (tid + j * blockDim.x) * V;
    if (col < a.d) {
      float w[V];
      load_weight<V>(a.weight, a.weight_f32, col, w);
#pragma unroll
      for (int i = 0; i < V; ++i) s[j][i] = s[j][i] * rstd * w[i];
      if (a.out) store_f32<IO, V>(static_cast<IO*>(a.out) + row * a.out_stride + col, s[j]);
    }
  }
  if (a.codes == nullptr) return;

  // The scale of every vector's group, then its codes.
  unsigned largest[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    largest[j] = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) largest[j] = max(largest[j], magnitude(s[j][i]));        // (columns past the row's end are zeros)
  }
  uint8_t* codes = a.codes + row * a.codes_stride;
  float* scales = a.scales + static_cast<long long>(row) * a.groups;
  if (a.group == 0) {
    unsigned m = 0;
#pragma unroll
    for (int j = 0; j < NV; ++j) m = max(m, largest[j]);
    m = __reduce_max_sync(0xffffffffu, m);
    if (blockDim.x > 32) {
      unsigned* share = reinterpret_cast<unsigned*>(red[1]);
      __syncthreads();                                       // red[1] may still be read (rows whose squares overflowed)
      if (lane == 0) share[tid >> 5] = m;
      __syncthreads();
      m = __reduce_max_sync(0xffffffffu, lane < static_cast<int>(blockDim.x >> 5) ? share[lane] : 0u);
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) largest[j] = m;
    if (tid == 0) scales[0] = code_scale(m);
  } else if (V > 1) {
    const int lanes = a.group / V;                           // 4 to 16 lanes hold a group
#pragma unroll
    for (int j = 0; j < NV; ++j) {
#pragma unroll
      for (int o = 1; o < 16; o <<= 1)
        if (o < lanes) largest[j] = max(largest[j], __shfl_xor_sync(0xffffffffu, largest[j], o));
      const int col = (tid + j * blockDim.x) * V;
      if (col < a.d && (lane & (lanes - 1)) == 0) scales[col >> a.group_shift] = code_scale(largest[j]);
    }
  } else {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const unsigned m = __reduce_max_sync(0xffffffffu, largest[j]);       // 32 columns of one group
      const int col = tid + j * blockDim.x;
      if (lane == 0 && col < a.d) atomicMax(&group_max[col >> a.group_shift], m);
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int col = tid + j * blockDim.x;
      if (col < a.d) {
        largest[j] = group_max[col >> a.group_shift];
        if ((col & (a.group - 1)) == 0) scales[col >> a.group_shift] = code_scale(largest[j]);
      }
    }
  }
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int col = (tid + j * blockDim.x) * V;
    if (col >= a.d) continue;
    const float2 by = code_factors(code_scale(largest[j]));
    if constexpr (V > 1) {
      Pack<uint16_t, V / 2> o;
#pragma unroll
      for (int i = 0; i < V; i += 2)
        o.e[i / 2] = __nv_cvt_float2_to_fp8x2(make_float2(s[j][i] * by.x * by.y, s[j][i + 1] * by.x * by.y), __NV_SATFINITE, __NV_E4M3);
      store_pack<uint16_t, V / 2>(reinterpret_cast<uint16_t*>(codes + col), o);
    } else {
      codes[col] = __nv_cvt_float_to_fp8(s[j][0] * by.x * by.y, __NV_SATFINITE, __NV_E4M3);
    }
  }
}

struct NormGradArgs {
  const void *sum, *weight, *d_out, *d_stream;      // weight, d_stream: may be NULL
  void* d_x;
  float* partial;                                   // [gridDim.x, d]: the blocks' parts of d weight (NULL: not wanted)
  long long sum_stride, d_out_stride, d_stream_stride, d_x_stride;
  int T, d;
  bool weight_f32;
  float eps, inv_d;
};

// A thread's eight elements of a row in its own places of shared memory, in pieces of 16 bytes `pitch` apart, a piece's neighbours the other threads'.
template <typename T>
struct RingRow {
  static constexpr int kPieces = sizeof(T) * 8 / 16;
  static __device__ __forceinline__ void fetch(uint32_t at, const T* src, uint32_t pitch) {
#pragma unroll
    for (int i = 0; i < kPieces; ++i) copy_async16(at + i * pitch, reinterpret_cast<const uint8_t*>(src) + i * 16);
  }
  static __device__ __forceinline__ void read(uint32_t at, uint32_t pitch, float (&x)[8]) {
    Pack<T, 8> p;
    uint32_t* r = reinterpret_cast<uint32_t*>(p.e);
#pragma unroll
    for (int i = 0; i < kPieces; ++i)
      asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                   : "=r"(r[4 * i]), "=r"(r[4 * i + 1]), "=r"(r[4 * i + 2]), "=r"(r[4 * i + 3])
                   : "r"(at + i * pitch));
    unpack(p, x);
  }
};
// Bytes of a thread's part of a row.
template <typename IO, typename DY, typename DX>
__host__ __device__ constexpr int norm_grad_thread_bytes() { return 8 * (sizeof(IO) + sizeof(DY) + sizeof(DX)); }

// Every block has every gridDim.x-th row and keeps its part of d weight in registers. STAGES > 0: rows come through shared memory, the next
// STAGES - 1 on their way while one is worked on, every thread copying and reading its own elements (no barrier of their own). With one row at a
// time in registers two blocks of 512 threads an SM waited for memory half of the time (8192 rows of 4096, bf16, d_out fp32: 88 us); with eight
// elements a thread and the row read from the ring twice, shared memory and shuffles were the bound (74 us). Otherwise (wider rows, and rows that no
// vectors fit) a row is read twice, the second time from L1 or L2.
template <typename IO, typename DY, typename DX, int V, int NV, int STAGES, int THREADS, int CTAS>
__global__ void __launch_bounds__(THREADS, CTAS) rmsnorm_grad_kernel(const __grid_constant__ NormGradArgs a) {
  constexpr bool kRing = STAGES > 0;
  static_assert(!kRing || V == 8, "a piece of the ring is 16 bytes of eight elements");
  constexpr int kHeld = kRing ? NV : 1;                      // vectors of s, d_out and the weight that a thread holds at a time
  // (a ring of two vectors a thread is for rows that fill the first ones: its block is THREADS wide, and addresses are offsets known to the compiler)
  constexpr bool kFixed = kRing && NV > 1;
  const uint32_t threads = kFixed ? THREADS : blockDim.x;
  extern __shared__ __align__(16) uint8_t ring[];
  __shared__ __align__(16) float red[3][2][32];
  const int tid = threadIdx.x;
  const uint32_t pitch = threads * 16, vector_bytes = norm_grad_thread_bytes<IO, DY, DX>() * threads, stage_bytes = NV * vector_bytes;
  const uint32_t place = smem_u32(ring) + tid * 16, dy_at = RingRow<IO>::kPieces * pitch, stream_at = dy_at + RingRow<DY>::kPieces * pitch;
  bool inside[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) inside[j] = (kFixed && j + 1 < NV) || (tid + j * threads) * V < a.d;
  clear_row_sums(&red[0][0][0], 3 * 2 * 32);
  grid_dependency_wait();
  int next_row = blockIdx.x;                                 // the next to be fetched, and where the thread's first vector of it is
  const IO* next_s = static_cast<const IO*>(a.sum) + next_row * a.sum_stride + tid * V;
  const DY* next_dy = static_cast<const DY*>(a.d_out) + next_row * a.d_out_stride + tid * V;
  const DX* next_stream = static_cast<const DX*>(a.d_stream) + next_row * a.d_stream_stride + tid * V;
  auto fetch = [&](int stage) {
    if (next_row < a.T) {
      const uint32_t at = place + stage * stage_bytes;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        if (inside[j]) {
          RingRow<IO>::fetch(at + j * vector_bytes, next_s + j * threads * V, pitch);
          RingRow<DY>::fetch(at + j * vector_bytes + dy_at, next_dy + j * threads * V, pitch);
          if (a.d_stream) RingRow<DX>::fetch(at + j * vector_bytes + stream_at, next_stream + j * threads * V, pitch);
        }
      }
      next_row += gridDim.x;
      next_s += gridDim.x * a.sum_stride;
      next_dy += gridDim.x * a.d_out_stride;
      next_stream += gridDim.x * a.d_stream_stride;
    }
    copy_commit();
  };
  if constexpr (kRing) {
#pragma unroll
    for (int q = 0; q < STAGES - 1; ++q) fetch(q);
  }
  float s[kHeld][V], dy[kHeld][V], w[kHeld][V], dw[NV][V];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    if constexpr (kRing) {
#pragma unroll
      for (int i = 0; i < V; ++i) w[j][i] = 0.f;
      if (inside[j]) load_weight<V>(a.weight, a.weight_f32, (tid + j * threads) * V, w[j]);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) dw[j][i] = 0.f;
  }
  int turn = 0, stage = 0;
  DX* out_row = static_cast<DX*>(a.d_x) + blockIdx.x * a.d_x_stride;
  for (int row = blockIdx.x; row < a.T; row += gridDim.x, turn ^= 1, out_row += gridDim.x * a.d_x_stride) {
    const IO* s_row = static_cast<const IO*>(a.sum) + row * a.sum_stride;
    const DY* dy_row = static_cast<const DY*>(a.d_out) + row * a.d_out_stride;
    const uint32_t at = place + stage * stage_bytes;
    if constexpr (kRing) {
      // (the stage that is fetched into was read by this thread alone, a turn ago)
      fetch(stage == 0 ? STAGES - 1 : stage - 1);
      copy_wait<STAGES - 1>();
      stage = stage + 1 == STAGES ? 0 : stage + 1;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
#pragma unroll
        for (int i = 0; i < V; ++i) s[j][i] = dy[j][i] = 0.f;
        if (inside[j]) {
          RingRow<IO>::read(at + j * vector_bytes, pitch, s[j]);
          RingRow<DY>::read(at + j * vector_bytes + dy_at, pitch, dy[j]);
        }
      }
    }
    // vector j of s times `by`, d_out and the weight into the one place held (those of the ring are there); false past the row's end
    auto read = [&](int j, float by) {
      const int col = (tid + j * threads) * V;
      if (!inside[j]) return false;
      unpack(load_pack<IO, V>(s_row + col), s[0]);
      unpack(load_pack<DY, V>(dy_row + col), dy[0]);
      load_weight<V>(a.weight, a.weight_f32, col, w[0]);
#pragma unroll
      for (int i = 0; i < V; ++i) s[0][i] *= by;
      return true;
    };
    auto add_up = [&](float by, float (&sums)[2], float (*share)[32]) {      // s^2 and weight d_out s
      sums[0] = sums[1] = 0.f;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int h = kRing ? j : 0;
        if (!kRing && !read(j, by)) continue;
#pragma unroll
        for (int i = 0; i < V; ++i) {
          sums[0] += s[h][i] * s[h][i];
          sums[1] += dy[h][i] * w[h][i] * s[h][i];
        }
      }
      row_sum(sums, share);
    };
    float sums[2], by = 1.f;
    add_up(by, sums, red[turn]);
    float rstd = rsqrtf(sums[0] * a.inv_d + a.eps);
    if (__float_as_uint(sums[0]) == 0x7f800000u) {
      by = kNormRescue;
#pragma unroll
      for (int j = 0; j < kHeld; ++j) {
#pragma unroll
        for (int i = 0; i < V; ++i) s[j][i] *= by;
      }
      __syncthreads();                                       // red[2] may still be read for an earlier row
      add_up(by, sums, red[2]);
      rstd = rsqrtf(sums[0] * a.inv_d);
    }
    // with unit = s rstd: d s = step (weight d_out) - back unit + d_stream
    const float step = rstd * by, back = step * (sums[1] * rstd * a.inv_d);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int col = (tid + j * threads) * V, h = kRing ? j : 0;
      float dx[V];
      if (kRing ? !inside[j] : !read(j, by)) continue;
#pragma unroll
      for (int i = 0; i < V; ++i) dx[i] = 0.f;
      if (a.d_stream) {
        if constexpr (kRing) RingRow<DX>::read(at + j * vector_bytes + stream_at, pitch, dx);
        else unpack(load_pack<DX, V>(static_cast<const DX*>(a.d_stream) + row * a.d_stream_stride + col), dx);
      }
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float unit = s[h][i] * rstd;
        dx[i] = (dx[i] - back * unit) + step * (dy[h][i] * w[h][i]);
        dw[j][i] += dy[h][i] * unit;
      }
      store_f32<DX, V>(out_row + col, dx);
    }
  }
  if (a.partial) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      if (inside[j]) store_f32<float, V>(a.partial + static_cast<size_t>(blockIdx.x) * a.d + (tid + j * threads) * V, dw[j]);
    }
  }
  if constexpr (kRing) copy_wait<0>();
  grid_launch_dependents();
}

// d weight from the blocks' parts: 32 columns a block, warp y adds up parts y, y + 32, ..., then the warps' sums in their order.
__global__ void __launch_bounds__(1024) norm_weight_grad_kernel(const float* partial, int parts, int d, float* d_weight) {
  __shared__ float share[32][33];
  const int col = blockIdx.x * 32 + threadIdx.x;
  grid_dependency_wait();
  float sum = 0.f;
  if (col < d) {
#pragma unroll 16
    for (int p = threadIdx.y; p < parts; p += 32) sum += partial[static_cast<size_t>(p) * d + col];
  }
  share[threadIdx.y][threadIdx.x] = sum;
  __syncthreads();
  sum = share[threadIdx.x][threadIdx.y];                     // warp y: the 32 parts of column y
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  const int mine = blockIdx.x * 32 + threadIdx.y;
  if (threadIdx.x == 0 && mine < d) d_weight[mine] = sum;
  grid_launch_dependents();
}

}  // namespace mtpc
