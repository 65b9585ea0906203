// Residual addition and root-mean-square norm of the rows that the head reads as hidden states, and their gradients.
//   s = x + residual,  rstd = (mean(s^2) + eps)^(-1/2),  out = s rstd weight
//   d s = rstd (weight d_out - s rstd^2 mean(weight d_out s)) + d_stream,   d weight = sum over the rows of d_out s rstd
// (d s is the gradient of x and of residual alike.) Everything between the loads and the one rounding of each output is fp32.
//
// Both are streams: a row is read once, into registers, and everything is formed from there. Forward, a row is a warp's up to 64 vectors of eight elements (one or
// two a lane), beyond that a block's with two vectors a thread, from 8192 columns on four. Gradient: a warp's up to 32 vectors, beyond that a block's with one
// or two vectors a thread, by what a row ahead leaves of the registers. Rows that no vectors fit go element by element; the gradient
// reads those, and rows of more than 8192 columns, twice, the second time from L1 or L2.
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
// Rows whose squares (or their mean with eps) overflow fp32 are formed once more from s times this: 32768 squares of it times fp32's largest value still
// fit. What it takes below the range leaves an output off by 2^-134 of its weight at most, half the smallest step times rstd: the roots of such
// rows' means are above 2^56.
constexpr float kNormRescue = 0x1p-72f;
// Rows whose mean with eps is below this, whose squares lose digits below the range, from s times 2^60.
constexpr float kNormLowMean = 0x1p-96f, kNormRaise = 0x1p60f;
__device__ __forceinline__ bool norm_far(float mean) { return mean == INFINITY || mean < kNormLowMean; }
__device__ __forceinline__ float norm_factor(float mean) { return mean < kNormLowMean ? kNormRaise : kNormRescue; }

struct NormArgs {
  const void *x, *residual, *weight;      // residual, weight: may be NULL
  void *sum, *out;                        // may be NULL
  uint8_t* codes;                         // e4m3, may be NULL
  float* scales;                          // [T, groups]
  long long x_stride, residual_stride, sum_stride, out_stride, codes_stride;
  int T, d, group, groups;                // group: columns that share a scale (0: the row)
  int group_shift;                        // its logarithm
  int shift, pitch;                       // of split rows (SplitRow)
  bool weight_f32;
  float eps, width, inv_width;            // d and 1 / d
};

// A row's sum divided by its width: the product with the reciprocal and one step of Newton's iteration, rounded once (the remainder is exact in a fused
// multiply-add; a division in its place costs registers that the gradients do not have). The product alone has the reciprocal's rounding in every row alike.
template <typename Args>
__device__ __forceinline__ float row_mean(const Args& a, float sum) {
  const float q = sum * a.inv_width;
  return fabsf(sum) < INFINITY ? fmaf(fmaf(-q, a.width, sum), a.inv_width, q) : q;
}
// Largest magnitude as the bits of an fp32: compared as integers a NaN is larger than everything, so it is not lost.
__device__ __forceinline__ unsigned magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }
// The larger magnitude of two values (of either sign), NaN if one is.
__device__ __forceinline__ float larger(float x, float y) {
  float d;
  asm("max.NaN.xorsign.abs.f32 %0, %1, %2;" : "=f"(d) : "f"(x), "f"(y));
  return d;
}

// 1 / x to 23 digits, for x well within the range.
__device__ __forceinline__ float reciprocal_near(float x) {
  float d;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(d) : "f"(x));
  return d;
}
// How the elements of a group become codes whose largest magnitude is `bits`: scale, what a code of 1 stands for, is the quotient by 448 rounded once (the
// product with the reciprocal and one step of Newton's iteration, whose remainder is exact in a fused multiply-add), and x / scale is x first hi + x first lo,
// where hi + lo is the reciprocal to twice the digits by the same step: rounded once, to the nearest fp32 but for 2^-46 of it. (The products with reciprocals of
// 24 digits move codes that lie near the middle of two; eight divisions beside a vector's loads take longer than the row's bytes.)
// Magnitudes far from one take the division for the scale, below whose digits a remainder may fall, and go to the middle of the range first, by
// a power of two, where no digit of lo is lost. A scale that is not finite has hi = 0: what is finite gives 0.
struct CodeFactors {
  float scale, first, hi, lo;
};
__device__ __forceinline__ CodeFactors code_factors(unsigned bits) {
  const float x = __uint_as_float(bits);
  CodeFactors f;
  if (bits - 0x26800000u < 0x61000000u - 0x26800000u) {      // 2^-50 to 2^67
    const float q = x * (1.f / kE4m3Max);
    f.scale = fmaf(fmaf(q, -kE4m3Max, x), 1.f / kE4m3Max, q);
    f.first = 1.f;
    f.hi = reciprocal_near(f.scale);
    f.lo = fmaf(-f.hi, f.scale, 1.f) * f.hi;
  } else {
    f.scale = x / kE4m3Max;
    if (f.scale == 0.f) f.scale = 1.f;
    f.first = f.scale < 0x1p-59f ? 0x1p64f : f.scale > 0x1p58f ? 0x1p-64f : 1.f;
    const float s = f.scale * f.first;                       // (between 2^-85 and 2^60, or not finite)
    f.hi = s < 0x1p100f ? reciprocal_near(s) : isnan(s) ? s : 0.f;
    f.lo = s < 0x1p100f ? fmaf(-f.hi, s, 1.f) * f.hi : 0.f;
  }
  return f;
}
__device__ __forceinline__ float code_quotient(float x, const CodeFactors& f) {
  x *= f.first;
  return fmaf(x, f.hi, x * f.lo);
}
__device__ __forceinline__ uint64_t code_quotients(uint64_t x, const CodeFactors& f) {
  if (f.first != 1.f) x = mul2(x, pack2(f.first, f.first));
  return fma2(x, pack2(f.hi, f.hi), mul2(x, pack2(f.lo, f.lo)));
}

// The largest magnitude of the row's columns, every thread with the same.
__device__ __forceinline__ unsigned row_max(unsigned m, unsigned* share) {
  m = __reduce_max_sync(0xffffffffu, m);
  if (blockDim.x > 32) {
    const int lane = threadIdx.x & 31;
    __syncthreads();                                         // `share` may still be read
    if (lane == 0) share[threadIdx.x >> 5] = m;
    __syncthreads();
    m = __reduce_max_sync(0xffffffffu, lane < static_cast<int>(blockDim.x >> 5) ? share[lane] : 0u);
  }
  return m;
}

// NV vectors of eight elements a thread. Beside its bytes a row costs what an SM issues for it, so the arithmetic goes by packed pairs: with 8-bit
// output, 2005 rows of 4096, element by element 16.6 to 24 us. SPLIT: rows that start off their vectors (no groups of columns with scales of their own).
template <typename IO, int NV, int THREADS, int CTAS, bool SPLIT>
__global__ void __launch_bounds__(THREADS, CTAS) residual_rmsnorm_kernel(const __grid_constant__ NormArgs a) {
  __shared__ float red[2][32];
  const int row = blockIdx.x * blockDim.y + threadIdx.y;
  const int tid = threadIdx.x, lane = tid & 31, threads = blockDim.x;
  grid_dependency_wait();
  grid_launch_dependents();
  if (row >= a.T) return;                                    // a whole warp, or no thread
  const SplitRow split(SPLIT ? a.shift : 0, SPLIT ? a.pitch : 0, row, a.d);
  const int begin = (SPLIT ? split.head : 0) + tid * 8, beside = SPLIT ? split.beside(tid) : -1;       // the thread's first column, and a single one
  bool inside[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) inside[j] = SPLIT ? tid + j * threads < split.packs : begin + j * threads * 8 < a.d;
  uint64_t s[NV][4];
  float single = 0.f;
  {
    Raw<IO, 8> x[NV], r[NV];
    const IO* x_row = static_cast<const IO*>(a.x) + row * a.x_stride;
    const IO* r_row = static_cast<const IO*>(a.residual) + row * a.residual_stride;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      x[j].clear();
      if (inside[j]) {
        x[j].load(x_row + begin + j * threads * 8);
        if (a.residual) r[j].load(r_row + begin + j * threads * 8);
      }
    }
    if (SPLIT && beside >= 0) {
      single = a.residual ? to_f32(x_row[beside]) + to_f32(r_row[beside]) : to_f32(x_row[beside]);
      if (a.sum) static_cast<IO*>(a.sum)[row * a.sum_stride + beside] = from_f32<IO>(single);
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
#pragma unroll
      for (int i = 0; i < 4; ++i) s[j][i] = x[j].pair(i);
      if (inside[j]) {
        if (a.residual) {
#pragma unroll
          for (int i = 0; i < 4; ++i) s[j][i] = add2(s[j][i], r[j].pair(i));
        }
        if (a.sum) store_pairs<IO>(static_cast<IO*>(a.sum) + row * a.sum_stride + begin + j * threads * 8, s[j]);
      }
    }
  }
  auto squares = [&]() {
    uint64_t sum = 0;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
#pragma unroll
      for (int i = 0; i < 4; ++i) sum = fma2(s[j][i], s[j][i], sum);
    }
    const float2 x = unpack2(sum);
    return SPLIT ? x.x + x.y + single * single : x.x + x.y;
  };
  float square = row_sum(squares(), red[0]);
  const float mean = row_mean(a, square) + a.eps;
  float rstd = rsqrtf(mean);
  if (norm_far(mean)) {                                      // the same in every thread of the row
    const float by = norm_factor(mean);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
#pragma unroll
      for (int i = 0; i < 4; ++i) s[j][i] = mul2(s[j][i], pack2(by, by));
    }
    single *= by;
    square = row_sum(squares(), red[1]);
    rstd = rsqrtf(row_mean(a, square) + a.eps * by * by);
  }
  const uint64_t rstd2 = pack2(rstd, rstd);
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int col = begin + j * threads * 8;
    if (inside[j]) {
      float w[8];
      if constexpr (SPLIT) load_weight8(a.weight, a.weight_f32, col, w);
      else load_weight<8>(a.weight, a.weight_f32, col, w);
#pragma unroll
      for (int i = 0; i < 4; ++i) s[j][i] = mul2(mul2(s[j][i], rstd2), pack2(w[2 * i], w[2 * i + 1]));
      if (a.out) store_pairs<IO>(static_cast<IO*>(a.out) + row * a.out_stride + col, s[j]);
    }
  }
  if (SPLIT && beside >= 0) {
    single = single * rstd * load_weight1(a.weight, a.weight_f32, beside);
    if (a.out) static_cast<IO*>(a.out)[row * a.out_stride + beside] = from_f32<IO>(single);
  }
  if (a.codes == nullptr) return;

  // The scale of every vector's group, then its codes. (Columns past the row's end are zeros.)
  unsigned largest[NV];
  CodeFactors by[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 x = unpack2(s[j][i]);
      m = larger(larger(m, x.x), x.y);
    }
    largest[j] = magnitude(m);
  }
  float* scales = a.scales + static_cast<long long>(row) * a.groups;
  if (a.group == 0) {
    unsigned m = SPLIT ? max(largest[0], magnitude(single)) : largest[0];
#pragma unroll
    for (int j = 1; j < NV; ++j) m = max(m, largest[j]);
    m = row_max(m, reinterpret_cast<unsigned*>(red[1]));
    by[0] = code_factors(m);
#pragma unroll
    for (int j = 1; j < NV; ++j) by[j] = by[0];
    if (tid == 0) scales[0] = by[0].scale;
  } else {
    const int lanes = a.group / 8;                           // 4 to 16 lanes hold a group
#pragma unroll
    for (int j = 0; j < NV; ++j) {
#pragma unroll
      for (int o = 1; o < 16; o <<= 1)
        if (o < lanes) largest[j] = max(largest[j], __shfl_xor_sync(0xffffffffu, largest[j], o));
      const int col = begin + j * threads * 8;
      by[j] = code_factors(largest[j]);
      if (inside[j] && (lane & (lanes - 1)) == 0) scales[col >> a.group_shift] = by[j].scale;
    }
  }
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int col = begin + j * threads * 8;
    if (!inside[j]) continue;
    Pack<uint16_t, 4> o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o.e[i] = __nv_cvt_float2_to_fp8x2(unpack2(code_quotients(s[j][i], by[j])), __NV_SATFINITE, __NV_E4M3);
    store_pack<uint16_t, 4>(reinterpret_cast<uint16_t*>(a.codes + row * a.codes_stride + col), o);
  }
  if (SPLIT && beside >= 0) {
    a.codes[row * a.codes_stride + beside] =
        __nv_cvt_float_to_fp8(code_quotient(single, by[0]), __NV_SATFINITE, __NV_E4M3);
  }
}

// The same of rows that no vectors fit: a block per row, NV single elements a thread, 32 adjacent ones to a warp.
template <typename IO, int NV>
__global__ void __launch_bounds__(1024) residual_rmsnorm_plain_kernel(const __grid_constant__ NormArgs a) {
  __shared__ float red[2][32];
  __shared__ unsigned group_max[kNormMaxWidth / kNormMinGroup];
  const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 31;
  if (a.codes != nullptr && a.group != 0) {
    for (int g = tid; g < a.groups; g += blockDim.x) group_max[g] = 0;
    __syncthreads();
  }
  grid_dependency_wait();
  grid_launch_dependents();
  const IO* x = static_cast<const IO*>(a.x) + row * a.x_stride;
  const IO* residual = static_cast<const IO*>(a.residual) + row * a.residual_stride;
  float s[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int col = tid + j * blockDim.x;
    s[j] = 0.f;
    if (col < a.d) s[j] = a.residual ? to_f32(x[col]) + to_f32(residual[col]) : to_f32(x[col]);
  }
  float square = 0.f;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int col = tid + j * blockDim.x;
    if (a.sum && col < a.d) static_cast<IO*>(a.sum)[row * a.sum_stride + col] = from_f32<IO>(s[j]);
    square += s[j] * s[j];
  }
  square = row_sum(square, red[0]);
  const float mean = row_mean(a, square) + a.eps;
  float rstd = rsqrtf(mean);
  if (norm_far(mean)) {                                      // the same in every thread of the row
    const float by = norm_factor(mean);
    square = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      s[j] *= by;
      square += s[j] * s[j];
    }
    square = row_sum(square, red[1]);
    rstd = rsqrtf(row_mean(a, square) + a.eps * by * by);
  }
  unsigned m = 0;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int col = tid + j * blockDim.x;
    if (col < a.d) {
      float w[1];
      load_weight<1>(a.weight, a.weight_f32, col, w);
      s[j] = s[j] * rstd * w[0];
      if (a.out) static_cast<IO*>(a.out)[row * a.out_stride + col] = from_f32<IO>(s[j]);
    }
    m = max(m, magnitude(s[j]));                             // (columns past the row's end are zeros)
    if (a.codes && a.group != 0) {
      const unsigned here = __reduce_max_sync(0xffffffffu, magnitude(s[j]));       // 32 columns of one group
      if (lane == 0 && col < a.d) atomicMax(&group_max[col >> a.group_shift], here);
    }
  }
  if (a.codes == nullptr) return;
  float* scales = a.scales + static_cast<long long>(row) * a.groups;
  CodeFactors by;
  if (a.group == 0) {
    m = row_max(m, reinterpret_cast<unsigned*>(red[1]));
    by = code_factors(m);
    if (tid == 0) scales[0] = by.scale;
  } else {
    __syncthreads();
  }
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int col = tid + j * blockDim.x;
    if (col >= a.d) continue;
    if (a.group != 0) {
      by = code_factors(group_max[col >> a.group_shift]);
      if ((col & (a.group - 1)) == 0) scales[col >> a.group_shift] = by.scale;
    }
    a.codes[row * a.codes_stride + col] = __nv_cvt_float_to_fp8(code_quotient(s[j], by), __NV_SATFINITE, __NV_E4M3);
  }
}

struct NormGradArgs {
  const void *sum, *weight, *d_out, *d_stream;      // weight, d_stream: may be NULL
  void* d_x;
  float* partial;                                   // [gridDim.x, d]: the blocks' parts of d weight (NULL: not wanted)
  long long sum_stride, d_out_stride, d_stream_stride, d_x_stride;
  int T, d;
  int shift, pitch;                                 // of split rows (SplitRow)
  bool weight_f32;
  float eps, width, inv_width;                      // d and 1 / d
};

// Every block has every gridDim.x-th row (of ROWS > 1 threadIdx.y each, rows of a warp: 16384 rows of 64 11 instead of 15 us) and keeps its part of
// d weight in registers, NV vectors of eight elements a thread; its vectors of the next row are on their way to registers. What bounds it is what the
// SM issues for a row beside its bytes, so the arithmetic goes by packed pairs: 8192 rows of 4096 (bf16, d_out fp32) one by one 88 to 104 us, with rows
// fetched by cp.async through shared memory, where issuing the copies took 1000 of 3500 cycles a row, 65 to 78. SPLIT: rows that start off their
// vectors, at the same columns in all rows of a block.
template <typename IO, typename DY, typename DX, int NV, int THREADS, int CTAS, bool SPLIT, int ROWS>
__global__ void __launch_bounds__(THREADS, CTAS) rmsnorm_grad_kernel(const __grid_constant__ NormGradArgs a) {
  __shared__ float red[3][32];
  const int tid = threadIdx.x, threads = blockDim.x;
  const int first_row = ROWS > 1 ? blockIdx.x * ROWS + threadIdx.y : blockIdx.x, row_step = gridDim.x * ROWS;
  const SplitRow split(SPLIT ? a.shift : 0, SPLIT ? a.pitch : 0, first_row, a.d);          // (row_step: a multiple of eight, or one row a block)
  const int begin = (SPLIT ? split.head : 0) + tid * 8, beside = SPLIT ? split.beside(tid) : -1;       // the thread's first column, and a single one
  bool inside[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) inside[j] = SPLIT ? tid + j * threads < split.packs : begin + j * threads * 8 < a.d;
  for (int i = tid; i < 96; i += threads) red[i >> 5][i & 31] = 0.f;
  __syncthreads();
  grid_dependency_wait();
  struct Row {
    Raw<IO, 8> s[NV];
    Raw<DY, 8> dy[NV];
    Raw<DX, 8> stream[NV];
    Raw<IO, 1> s1;                                           // the single column's
    Raw<DY, 1> dy1;
    Raw<DX, 1> stream1;
  } ahead;
  const IO* next_s = static_cast<const IO*>(a.sum) + first_row * a.sum_stride;          // the row to be fetched next
  const DY* next_dy = static_cast<const DY*>(a.d_out) + first_row * a.d_out_stride;
  const DX* next_stream = static_cast<const DX*>(a.d_stream) + first_row * a.d_stream_stride;
  int next = first_row;
  auto fetch = [&](Row& x) {
    if (next < a.T) {
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        if (inside[j]) {
          x.s[j].load(next_s + begin + j * threads * 8);
          x.dy[j].load(next_dy + begin + j * threads * 8);
          if (a.d_stream) x.stream[j].load(next_stream + begin + j * threads * 8);
        }
      }
      if (SPLIT && beside >= 0) {
        x.s1.load(next_s + beside);
        x.dy1.load(next_dy + beside);
        if (a.d_stream) x.stream1.load(next_stream + beside);
      }
      next += row_step;
      next_s += row_step * a.sum_stride;
      next_dy += row_step * a.d_out_stride;
      next_stream += row_step * a.d_stream_stride;
    }
  };
#pragma unroll
  for (int j = 0; j < NV; ++j) {               // (what lies past the row's end stays zero, and so does d_stream if there is none)
    ahead.s[j].clear();
    ahead.dy[j].clear();
    ahead.stream[j].clear();
  }
  ahead.s1.clear();
  ahead.dy1.clear();
  ahead.stream1.clear();
  fetch(ahead);
  uint64_t w[NV][4], dw[NV][4];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    float x[8] = {};
    if (inside[j]) {
      if constexpr (SPLIT) load_weight8(a.weight, a.weight_f32, begin + j * threads * 8, x);
      else load_weight<8>(a.weight, a.weight_f32, begin + j * threads * 8, x);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w[j][i] = pack2(x[2 * i], x[2 * i + 1]);
      dw[j][i] = 0;
    }
  }
  const float w1 = SPLIT && beside >= 0 ? load_weight1(a.weight, a.weight_f32, beside) : 0.f;
  float dw1 = 0.f;
  int turn = 0;
  DX* out = static_cast<DX*>(a.d_x) + first_row * a.d_x_stride;
  for (int row = first_row; row < a.T; row += row_step) {
    uint64_t s[NV][4], dy[NV][4];
    Raw<DX, 8> stream[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[j][i] = ahead.s[j].pair(i);
        dy[j][i] = ahead.dy[j].pair(i);
      }
      stream[j] = ahead.stream[j];
    }
    float s1 = ahead.s1.value(0);
    const float dy1 = ahead.dy1.value(0), stream1 = ahead.stream1.value(0);
    fetch(ahead);
    auto add_up = [&](float (&sums)[2], float* share) {        // s^2 and weight d_out s
      uint64_t squares = 0, products = 0;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          squares = fma2(s[j][i], s[j][i], squares);
          products = fma2(mul2(dy[j][i], w[j][i]), s[j][i], products);
        }
      }
      const float2 x = unpack2(squares), y = unpack2(products);
      sums[0] = SPLIT ? x.x + x.y + s1 * s1 : x.x + x.y;
      sums[1] = SPLIT ? y.x + y.y + dy1 * w1 * s1 : y.x + y.y;
      row_sums(sums, share);
    };
    float sums[2], by = 1.f;
    add_up(sums, red[turn]);
    const float mean = row_mean(a, sums[0]) + a.eps;
    float rstd = rsqrtf(mean);
    if (norm_far(mean)) {
      by = norm_factor(mean);
#pragma unroll
      for (int j = 0; j < NV; ++j) {
#pragma unroll
        for (int i = 0; i < 4; ++i) s[j][i] = mul2(s[j][i], pack2(by, by));
      }
      s1 *= by;
      if constexpr (ROWS == 1) __syncthreads();              // red[2] may still be read for an earlier row
      add_up(sums, red[2]);
      rstd = rsqrtf(row_mean(a, sums[0]) + a.eps * by * by);
    }
    // with unit = s rstd: d s = step (weight d_out) - back unit + d_stream
    const float step = rstd * by, back = -step * (row_mean(a, sums[1]) * rstd);
    const uint64_t rstd2 = pack2(rstd, rstd), step2 = pack2(step, step), back2 = pack2(back, back);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      uint64_t dx[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint64_t unit = mul2(s[j][i], rstd2);
        dx[i] = fma2(step2, mul2(dy[j][i], w[j][i]), fma2(back2, unit, stream[j].pair(i)));
        dw[j][i] = fma2(dy[j][i], unit, dw[j][i]);
      }
      if (inside[j]) store_pairs<DX>(out + begin + j * threads * 8, dx);
    }
    if (SPLIT && beside >= 0) {
      const float unit = s1 * rstd;
      out[beside] = from_f32<DX>((stream1 + back * unit) + step * (dy1 * w1));
      dw1 += dy1 * unit;
    }
    out += row_step * a.d_x_stride;
    turn ^= 1;
  }
  if (a.partial) {
    float* part = a.partial + static_cast<size_t>(blockIdx.x) * a.d;
    __shared__ alignas(16) float share[ROWS > 1 ? ROWS : 1][ROWS > 1 ? 32 * 8 * NV : 1];
    float* mine = ROWS > 1 ? share[threadIdx.y] : part;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      if (!inside[j]) continue;
      if constexpr (SPLIT) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 x = unpack2(dw[j][i]);
          mine[begin + j * threads * 8 + 2 * i] = x.x;
          mine[begin + j * threads * 8 + 2 * i + 1] = x.y;
        }
      } else if constexpr (ROWS > 1) {
#pragma unroll
        for (int i = 0; i < 4; ++i) *reinterpret_cast<uint64_t*>(mine + begin + j * threads * 8 + 2 * i) = dw[j][i];
      } else {
        store_pairs<float>(part + begin + j * threads * 8, dw[j]);
      }
    }
    if (SPLIT && beside >= 0) mine[beside] = dw1;
    if constexpr (ROWS > 1) {
      __syncthreads();
      for (int col = threadIdx.y * 32 + tid; col < a.d; col += 32 * ROWS) {
        float sum = 0.f;
#pragma unroll
        for (int r = 0; r < ROWS; ++r) sum += share[r][col];
        part[col] = sum;
      }
    }
  }
  grid_launch_dependents();
}

// The same of rows that no vectors fit, or that are wider than the registers of a block: element after element of a thread, read twice, the second time
// from L1 or L2.
template <typename IO, typename DY, typename DX, int V, int NV>
__global__ void __launch_bounds__(1024) rmsnorm_grad_plain_kernel(const __grid_constant__ NormGradArgs a) {
  __shared__ float red[2][32];
  const int tid = threadIdx.x;
  grid_dependency_wait();
  float dw[NV][V];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
#pragma unroll
    for (int i = 0; i < V; ++i) dw[j][i] = 0.f;
  }
  for (int row = blockIdx.x; row < a.T; row += gridDim.x) {
    const IO* s_row = static_cast<const IO*>(a.sum) + row * a.sum_stride;
    const DY* dy_row = static_cast<const DY*>(a.d_out) + row * a.d_out_stride;
    float s[V], dy[V], w[V];
    auto read = [&](int j, float by) {                       // vector j of s times `by`, d_out and the weight; false past the row's end
      const int col = (tid + j * blockDim.x) * V;
      if (col >= a.d) return false;
      unpack(load_pack<IO, V>(s_row + col), s);
      unpack(load_pack<DY, V>(dy_row + col), dy);
      load_weight<V>(a.weight, a.weight_f32, col, w);
#pragma unroll
      for (int i = 0; i < V; ++i) s[i] *= by;
      return true;
    };
    auto add_up = [&](float by, float (&sums)[2]) {           // s^2 and weight d_out s
      sums[0] = sums[1] = 0.f;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        if (!read(j, by)) continue;
#pragma unroll
        for (int i = 0; i < V; ++i) {
          sums[0] += s[i] * s[i];
          sums[1] += dy[i] * w[i] * s[i];
        }
      }
      __syncthreads();                                       // the last sums have been read
      sums[0] = row_sum(sums[0], red[0]);
      sums[1] = row_sum(sums[1], red[1]);
    };
    float sums[2], by = 1.f;
    add_up(by, sums);
    const float mean = row_mean(a, sums[0]) + a.eps;
    float rstd = rsqrtf(mean);
    if (norm_far(mean)) {
      by = norm_factor(mean);
      add_up(by, sums);
      rstd = rsqrtf(row_mean(a, sums[0]) + a.eps * by * by);
    }
    const float step = rstd * by, back = step * (row_mean(a, sums[1]) * rstd);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int col = (tid + j * blockDim.x) * V;
      float dx[V];
      if (!read(j, by)) continue;
#pragma unroll
      for (int i = 0; i < V; ++i) dx[i] = 0.f;
      if (a.d_stream) unpack(load_pack<DX, V>(static_cast<const DX*>(a.d_stream) + row * a.d_stream_stride + col), dx);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float unit = s[i] * rstd;
        dx[i] = (dx[i] - back * unit) + step * (dy[i] * w[i]);
        dw[j][i] += dy[i] * unit;
      }
      store_f32<DX, V>(static_cast<DX*>(a.d_x) + row * a.d_x_stride + col, dx);
    }
  }
  if (a.partial) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int col = (tid + j * blockDim.x) * V;
      if (col < a.d) store_f32<float, V>(a.partial + static_cast<size_t>(blockIdx.x) * a.d + col, dw[j]);
    }
  }
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
