// Dropout: out = residual + (x / (1 - p) where the draw of an element is at least `cut`, else 0), p = cut / 65536.
//
// Draws are the eight 16-bit parts of Philox4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3; 2011) of the counter
// (element / 8, step) under a 64-bit key, element = row * d + column whatever the strides. The mask is so a function of seed, step and place:
// it is nowhere stored, and the gradient's call draws it again. Sixteen bits an element: ten rounds are about 80 instructions, for eight elements
// a third of the time that their bytes take, for four (32 bits each) two thirds, which would leave no room beside bf16 rows; the scale is that of the p in steps
// of 2^-16, so the mean is kept exactly.
//
// Bound by HBM: 8192 x 4096 bf16 with a residual 33 to 36 us, the bytes alone 31; small calls by their launch.
#pragma once
#include <stdint.h>

#include "mtpc_rows.cuh"

namespace mtpc {

struct DropoutArgs {
  const void *x, *residual;             // residual: NULL, or of out's type
  void* out;
  const int64_t* rng;                   // [2]: seed, step
  int64_t x_stride, residual_stride, out_stride;
  int64_t offset;
  int64_t count;                        // T * d
  int d;                                // <= 0: rows adjacent in all matrices, one run of `count` elements
  uint32_t cut;
  float scale;
};

// Eight draws, two to a word.
__device__ __forceinline__ uint4 philox_block(uint64_t block, uint64_t step, uint64_t seed) {
  uint32_t c0 = static_cast<uint32_t>(block), c1 = static_cast<uint32_t>(block >> 32);
  uint32_t c2 = static_cast<uint32_t>(step), c3 = static_cast<uint32_t>(step >> 32);
  uint32_t k0 = static_cast<uint32_t>(seed), k1 = static_cast<uint32_t>(seed >> 32);
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t a = static_cast<uint64_t>(c0) * 0xD2511F53u, b = static_cast<uint64_t>(c2) * 0xCD9E8D57u;
    c0 = static_cast<uint32_t>(b >> 32) ^ c1 ^ k0;
    c2 = static_cast<uint32_t>(a >> 32) ^ c3 ^ k1;
    c1 = static_cast<uint32_t>(b);
    c3 = static_cast<uint32_t>(a);
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return make_uint4(c0, c1, c2, c3);
}
__device__ __forceinline__ uint32_t draw_of(const uint4& w, int i) {
  const uint32_t word = i < 4 ? (i < 2 ? w.x : w.y) : (i < 6 ? w.z : w.w);
  return i & 1 ? word >> 16 : word & 0xffffu;
}

// Blocks of eight elements that lie within rows: d a multiple of eight, or adjacent rows (a.d <= 0) but for the last, short block. N blocks a thread, all
// loads ahead of the draws.
template <typename TI, typename TO, bool RESIDUAL, int N>
__global__ void __launch_bounds__(256) dropout_kernel(const DropoutArgs a) {
  grid_launch_dependents();
  grid_dependency_wait();
  const uint64_t seed = static_cast<uint64_t>(a.rng[0]), step = static_cast<uint64_t>(a.rng[1]) + static_cast<uint64_t>(a.offset);
  const int64_t blocks = a.count / 8, first = static_cast<int64_t>(blockIdx.x) * (256 * N) + threadIdx.x;
  const TI* x = static_cast<const TI*>(a.x);
  const TO* residual = static_cast<const TO*>(a.residual);
  TO* out = static_cast<TO*>(a.out);
  Raw<TI, 8> xv[N];
  Raw<TO, 8> rv[N];
  int64_t to[N];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int64_t b = first + n * 256;
    if (b >= blocks) continue;
    int64_t from = b * 8, res = b * 8;
    to[n] = b * 8;
    if (a.d > 0) {
      const int64_t row = b / (a.d / 8);
      const int64_t col = b * 8 - row * a.d;
      from = row * a.x_stride + col;
      res = row * a.residual_stride + col;
      to[n] = row * a.out_stride + col;
    }
    xv[n].load(x + from);
    if constexpr (RESIDUAL) rv[n].load(residual + res);
  }
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int64_t b = first + n * 256;
    if (b > blocks) continue;
    const uint4 w = philox_block(static_cast<uint64_t>(b), step, seed);
    if (b == blocks) {                               // what is behind the last whole block
      for (int i = 0; i < static_cast<int>(a.count - blocks * 8); ++i) {
        float y = draw_of(w, i) >= a.cut ? to_f32(x[blocks * 8 + i]) * a.scale : 0.f;
        if constexpr (RESIDUAL) y += to_f32(residual[blocks * 8 + i]);
        out[blocks * 8 + i] = from_f32<TO>(y);
      }
      continue;
    }
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      y[i] = draw_of(w, i) >= a.cut ? xv[n].value(i) * a.scale : 0.f;
      if constexpr (RESIDUAL) y[i] += rv[n].value(i);
    }
    store_f32<TO, 8>(out + to[n], y);
  }
}

// Any rows: a thread has the eight elements of a block one by one, wherever their rows end.
template <typename TI, typename TO, bool RESIDUAL>
__global__ void __launch_bounds__(256) dropout_plain_kernel(const DropoutArgs a) {
  grid_launch_dependents();
  grid_dependency_wait();
  const uint64_t seed = static_cast<uint64_t>(a.rng[0]), step = static_cast<uint64_t>(a.rng[1]) + static_cast<uint64_t>(a.offset);
  const int64_t b = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, begin = b * 8;
  if (begin >= a.count) return;
  const uint4 w = philox_block(static_cast<uint64_t>(b), step, seed);
  int64_t row = begin / a.d;
  int col = static_cast<int>(begin - row * a.d);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (begin + i >= a.count) return;
    float y = draw_of(w, i) >= a.cut ? to_f32(static_cast<const TI*>(a.x)[row * a.x_stride + col]) * a.scale : 0.f;
    if constexpr (RESIDUAL) y += to_f32(static_cast<const TO*>(a.residual)[row * a.residual_stride + col]);
    static_cast<TO*>(a.out)[row * a.out_stride + col] = from_f32<TO>(y);
    if (++col == a.d) col = 0, ++row;
  }
}

}  // namespace mtpc
