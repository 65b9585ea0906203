// A projection with low-rank adaptors of many requests beside it, and its gradients:
//   out[t] = W x[t] + A[i] low[t],   low[t] = scale[i] B[i] x'[t],   i = which[t] (negative: no adaptor)
//   d_x[t] = W^T g[t] + B[i]^T v[t], v[t] = scale[i] A[i]^T g[t],    dA[i] = sum of g low^T, dB[i] = sum of v x'^T over the rows of i
// x, W, A, B, g bf16; low, v, dA, dB fp32; out, d_x bf16.
//
// adaptor_low_kernel    low or v of many rows: K in chunks of 512 at most, each its own accumulator, added up in fp32. The tensor cores round every accumulation towards
//                       zero, so that one accumulator over K = 4096 is 4e-6 off, chunks 4e-7. The result is split into bf16 terms: two (16 bits) for the
//                       product with A or B whose result is rounded to bf16, three (24 bits) for the fp32 gradients. (4096 rows of 4096 x 4096, k = 16: against the exact result
//                       rounded once, two terms alone move 8e-5 of the result, as roundings to the other side; the whole kernel 1.3e-4, and without adaptors 1.5e-4, the cut
//                       accumulations', as a library's product does. The rounding to bf16 itself is 1.7e-3.)
// adapted_gemm_kernel   the shared product; the adaptors of a tile's rows follow as K blocks of their own.
// low_rows_kernel, adapted_rows_kernel   the same of few rows (decoding), where W is read once by the whole device.
// adaptor_grad_kernel, adaptor_grad_join_kernel   dA and dB.
//
// Rows keep their order. A tile of 128 (256) rows has a K block for every adaptor that occurs in it, whose MMAs leave the accumulator rows of others alone
// (the instruction's lane mask): no row's result holds another adaptor's weights, also not as zero times them, so that what one request's
// weights hold (infinities, NaN) reaches no other. Rows of a request that follow each other, as in prompts and training batches, give one to three
// such blocks a tile; in the worst case, 128 adaptors in every tile, they are as many K blocks more.
#pragma once
#include <cuda_bf16.h>
#include <math_constants.h>
#include <stdint.h>

#include "mtpc_pipeline.cuh"
#include "mtpc_rows.cuh"

namespace mtpc {

constexpr uint32_t kStatusBadAdaptor = 32u;
constexpr int kMaxRank = 64;
constexpr int kPieceRank = 32;                     // rank columns of one K block: their high terms, then their low ones
constexpr int kChunkBlocks = 8;                    // K blocks of one accumulator at most where fp32 is returned

// ---- instructions
// 3-D tiled loads: x innermost (a multiple of 16 bytes), then row, then matrix.
__device__ __forceinline__ void tma_load_3d(uint32_t lead, uint32_t dst_smem, const CUtensorMap* tm, uint32_t bar, int32_t x, int32_t y, int32_t z) {
  asm volatile(
      "{\n"
      ".reg .pred e;\n"
      "setp.ne.b32 e, %6, 0;\n"
      "@e cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];\n"
      "}\n" ::"r"(dst_smem),
      "l"(reinterpret_cast<uint64_t>(tm)), "r"(bar), "r"(x), "r"(y), "r"(z), "r"(lead)
      : "memory");
}
__device__ __forceinline__ void tma_load_3d_pair(uint32_t lead, uint32_t dst_smem, const CUtensorMap* tm, uint32_t cluster_bar, int32_t x, int32_t y,
                                                 int32_t z) {
  asm volatile(
      "{\n"
      ".reg .pred e;\n"
      "setp.ne.b32 e, %6, 0;\n"
      "@e cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];\n"
      "}\n" ::"r"(dst_smem),
      "l"(reinterpret_cast<uint64_t>(tm)), "r"(cluster_bar), "r"(x), "r"(y), "r"(z), "r"(lead)
      : "memory");
}
// The MMA that leaves accumulator rows alone: bit l of off[w] is TMEM lane 32 w + l (pairs: words 4 to 7 are the peer's lanes).
__device__ __forceinline__ void umma_bf16_rows(uint32_t lead, uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate,
                                               const uint32_t (&off)[4]) {
  asm volatile(
      "{\n"
      ".reg .pred p, e;\n"
      "setp.ne.b32 p, %4, 0;\n"
      "setp.ne.b32 e, %5, 0;\n"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, {%6, %7, %8, %9}, p;\n"
      "}\n" ::"r"(d_tmem),
      "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(lead), "r"(off[0]), "r"(off[1]), "r"(off[2]), "r"(off[3])
      : "memory");
}
__device__ __forceinline__ void umma_bf16_rows(uint32_t lead, uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate,
                                               const uint32_t (&off)[8]) {
  asm volatile(
      "{\n"
      ".reg .pred p, e;\n"
      "setp.ne.b32 p, %4, 0;\n"
      "setp.ne.b32 e, %5, 0;\n"
      "@e tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, {%6, %7, %8, %9, %10, %11, %12, %13}, p;\n"
      "}\n" ::"r"(d_tmem),
      "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate), "r"(lead), "r"(off[0]), "r"(off[1]), "r"(off[2]), "r"(off[3]), "r"(off[4]), "r"(off[5]),
      "r"(off[6]), "r"(off[7])
      : "memory");
}
__device__ __forceinline__ float ld_cluster_f32(uint32_t addr) {
  float x;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(x) : "r"(addr) : "memory");
  return x;
}

__device__ __forceinline__ float4 ld_cluster_v4(uint32_t addr) {
  float4 x;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w) : "r"(addr) : "memory");
  return x;
}

// ---- which adaptors a tile's rows have
// Row t's adaptor; -1: none, or one that does not exist (its rows are refused by whoever writes results).
__device__ __forceinline__ int adaptor_of(const int* which, int S, int t, int T) {
  if (t >= T) return -1;
  const int i = which == nullptr ? 0 : which[t];
  return i < S ? i : -1;
}
__device__ __forceinline__ bool adaptor_refused(const int* which, int S, int t) { return which != nullptr && which[t] >= S; }

// The adaptors of 32 * WORDS rows one after the other, in the order of their first rows; every warp that walks over them sees the same.
template <int WORDS>
struct TileAdaptors {
  int mine[WORDS];                      // of row 32 w + lane
  uint32_t left[WORDS];
  __device__ __forceinline__ void load(const int* which, int S, int row0, int T, int lane) {
#pragma unroll
    for (int w = 0; w < WORDS; ++w) mine[w] = adaptor_of(which, S, row0 + 32 * w + lane, T);
#pragma unroll
    for (int w = 0; w < WORDS; ++w) left[w] = __ballot_sync(0xffffffffu, mine[w] >= 0);
  }
  __device__ __forceinline__ bool none() const {
    uint32_t any = 0;
#pragma unroll
    for (int w = 0; w < WORDS; ++w) any |= left[w];
    return any == 0;
  }
  // The next adaptor and, in `off`, the rows that are not its own; false: there is none left.
  __device__ __forceinline__ bool next(int& adaptor, uint32_t (&off)[WORDS]) {
    int from = -1;
#pragma unroll
    for (int w = WORDS - 1; w >= 0; --w)
      if (left[w] != 0) from = w;
    if (from < 0) return false;
    int value = 0;
    uint32_t bits = 0;
#pragma unroll
    for (int w = 0; w < WORDS; ++w)
      if (w == from) value = mine[w], bits = left[w];
    adaptor = __shfl_sync(0xffffffffu, value, __ffs(bits) - 1);
#pragma unroll
    for (int w = 0; w < WORDS; ++w) {
      const uint32_t rows = __ballot_sync(0xffffffffu, mine[w] == adaptor);
      off[w] = ~rows;
      left[w] &= ~rows;
    }
    return true;
  }
};

// ---- low (or v) of many rows
// A cluster has a tile of 128 rows; its CTAs share the chunks of K, add theirs up in registers and meet in shared memory, where each finishes its share of the rows:
// sum, scale, low, its terms. For the gradients it splits given values into terms as well, and blocks behind the tiles' say which 64 rows have an adaptor's.
// Bound by the rows' bytes where there are many (8192 x 4096, k = 16: 15.4 us, 10 of them HBM's), by its chain of latencies where there are few (512 rows 6.3).
struct LowParams {
  CUtensorMap tm_a;                     // rows [T, K]          box 64 x 128
  CUtensorMap tm_f;                     // factors: B [S, k, K] box 64 x k16 (K-major), or A [S, K, k] box factor_columns(k16) x 64 (MN-major)
  const int* which;
  const float* scale;                   // [S] or NULL: ones
  float* low;                           // [T, k] or NULL
  __nv_bfloat16* two;                   // [T][pieces][64] or NULL
  __nv_bfloat16* three;                 // [T][3][k16] or NULL
  const float* given;                   // [T, k]
  __nv_bfloat16* given_three;           // [T][3][k16]
  uint32_t *present, *whole;            // bit b % 32 of [(b / 32) S + i]: block b has rows of i, and no others
  unsigned* status;                     // or NULL
  uint64_t wait_limit_ns;
  int T, S, k, k16, pieces;             // k16: the rank, rounded up to 16
  int kblocks, chunk_blocks, chunks, tiles, split, stages, stage_bytes;              // split: CTAs of a cluster; chunks 0: no sums are wanted
  int group;                            // adaptors whose factors share a stage with a tile of the rows, 64 columns in all: one pass over the rows gives the products with all of them,
                                        // and every row takes those of its own
  int present_blocks;
};
constexpr int kLowThreads = 192;
constexpr int kLowSlots = 4, kLowSlotCols = kMaxRank, kLowTmemCols = kLowSlots * kLowSlotCols;
// MN-major factors lie in shared memory as 64 rows (of K) of 16, 32 or 64 columns, swizzled over the 32, 64 or 128 bytes that a row has: a quarter of what boxes of 64
// columns would move for a rank of 16. Eight rows are 8 row-lengths apart, sixteen (an MMA's K) twice that.
__host__ __device__ constexpr int factor_columns(int k16) { return k16 <= 32 ? k16 : 64; }
__device__ __forceinline__ uint64_t umma_smem_desc_factor(uint32_t smem_addr, int columns) {
  const uint64_t layout = columns == 16 ? 6 : columns == 32 ? 4 : 2;
  uint64_t d = 0;
  d |= static_cast<uint64_t>((smem_addr & 0x3FFFFu) >> 4);
  d |= static_cast<uint64_t>((columns * kBlockK * 2) >> 4) << 16;      // the next adaptor's box continues the columns
  d |= static_cast<uint64_t>(columns) << 32;                           // eight rows of 2 columns bytes, in units of 16
  d |= static_cast<uint64_t>(1) << 46;
  d |= layout << 61;
  return d;
}
// x as a sum of bf16 values: the nearest, and the nearest to what is left (twice, where a third is wanted). A value that is not finite keeps its first.
__device__ __forceinline__ void split_terms(float x, __nv_bfloat16& hi, __nv_bfloat16& mid, __nv_bfloat16& lo) {
  hi = __float2bfloat16_rn(x);
  const float r = isfinite(x) ? x - __bfloat162float(hi) : 0.f;
  mid = __float2bfloat16_rn(r);
  lo = __float2bfloat16_rn(r - __bfloat162float(mid));
}
// Four values of row t from rank j0 on (those past the rank are zeros) as terms.
__device__ __forceinline__ void store_terms(const LowParams& p, int t, int j0, const float (&x)[4], __nv_bfloat16* two, __nv_bfloat16* three) {
  __align__(8) __nv_bfloat16 h[4], m[4], l[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) split_terms(j0 + q < p.k ? x[q] : 0.f, h[q], m[q], l[q]);
  const uint2 hv = *reinterpret_cast<const uint2*>(h), mv = *reinterpret_cast<const uint2*>(m), lv = *reinterpret_cast<const uint2*>(l);
  if (two != nullptr) {
    __nv_bfloat16* dst = two + (static_cast<size_t>(t) * p.pieces + j0 / kPieceRank) * 64 + j0 % kPieceRank;
    *reinterpret_cast<uint2*>(dst) = hv;
    *reinterpret_cast<uint2*>(dst + kPieceRank) = mv;
  }
  if (three != nullptr) {
    __nv_bfloat16* dst = three + static_cast<size_t>(t) * 3 * p.k16 + j0;
    *reinterpret_cast<uint2*>(dst) = hv;
    *reinterpret_cast<uint2*>(dst + p.k16) = mv;
    *reinterpret_cast<uint2*>(dst + 2 * p.k16) = lv;
  }
}
// The terms of given values of rows [t0, t1), by the 128 threads of the epilogue.
__device__ __forceinline__ void given_terms(const LowParams& p, int t0, int t1, int thread) {
  const int quads = p.k16 / 4, all = (min(t1, p.T) - t0) * quads;
#pragma unroll 4
  for (int at = thread; at < all; at += 128) {
    const int t = t0 + at / quads, j0 = at % quads * 4;
    const bool any = adaptor_of(p.which, p.S, t, p.T) >= 0;
    float x[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) x[q] = any && j0 + q < p.k ? p.given[static_cast<size_t>(t) * p.k + j0 + q] : 0.f;
    store_terms(p, t, j0, x, nullptr, p.given_three);
  }
}
__device__ __forceinline__ void present_rows(const LowParams& p, int group, uint32_t* words) {       // words: S + 1
  uint32_t* mixed = words + p.S;
  for (int i = threadIdx.x; i <= p.S; i += kLowThreads) words[i] = 0;
  __syncthreads();
  for (int r = threadIdx.x; r < 32 * 64; r += kLowThreads) {
    const long long t = static_cast<long long>(group) * (32 * 64) + r;
    if (t >= p.T) continue;
    const int i = adaptor_of(p.which, p.S, static_cast<int>(t), p.T), head = adaptor_of(p.which, p.S, static_cast<int>(t) - r % 64, p.T);
    if (i >= 0) atomicOr(&words[i], 1u << (r / 64));
    if (i != head) atomicOr(mixed, 1u << (r / 64));
    // Where sums are wanted, whoever finishes them reports it. (In given_terms, the same line made the compiler's code of the tiles slower: 1024 rows 28.9 -> 35.0 us.)
    if (p.chunks == 0 && p.status != nullptr && adaptor_refused(p.which, p.S, static_cast<int>(t))) atomicOr(p.status, kStatusBadAdaptor);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < p.S; i += kLowThreads) {
    p.present[static_cast<size_t>(group) * p.S + i] = words[i];
    p.whole[static_cast<size_t>(group) * p.S + i] = words[i] & ~*mixed;
  }
}

template <bool F_MN>
__global__ void __launch_bounds__(kLowThreads, 2) adaptor_low_kernel(const __grid_constant__ LowParams p) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw_addr = smem_u32(smem_raw);
  const uint32_t tiles_addr = (raw_addr + 1023u) & ~1023u;
  if (static_cast<int>(blockIdx.x) >= p.tiles * p.split) {           // (whole clusters of such blocks)
    grid_dependency_wait();
    grid_launch_dependents();
    const int block = blockIdx.x - p.tiles * p.split;
    if (block < p.present_blocks) present_rows(p, block, reinterpret_cast<uint32_t*>(smem_raw));
    return;
  }
  GemmControl* ctl = reinterpret_cast<GemmControl*>(smem_raw + (tiles_addr - raw_addr) + static_cast<size_t>(p.stages) * p.stage_bytes);
  const int warp = static_cast<int>(warp_uniform(threadIdx.x >> 5));
  const int lane = threadIdx.x & 31;
  const int tile = blockIdx.x / p.split, rank = blockIdx.x - tile * p.split, row0 = tile * kBlockM;
  if (threadIdx.x == 0) {
    for (int s = 0; s < p.stages; ++s) {
      mbar_init(smem_u32(&ctl->full[s]), 1);
      mbar_init(smem_u32(&ctl->empty[s]), 1);
    }
    for (int s = 0; s < kLowSlots; ++s) {
      mbar_init(smem_u32(&ctl->tfull[s]), 1);
      mbar_init(smem_u32(&ctl->tempty[s]), 4);
    }
    mbar_init(smem_u32(&ctl->drain), 1);
    ctl->abort = 0;
    ctl->wait_limit_ns = p.wait_limit_ns;
    fence_mbar_init();
    if (p.chunks > 0) {
      tma_prefetch_desc(&p.tm_a);
      tma_prefetch_desc(&p.tm_f);
    }
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(&ctl->tmem_base), kLowTmemCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = warp_uniform(ctl->tmem_base);
  grid_dependency_wait();
  grid_launch_dependents();             // (a gate: what is behind may read all but what is written here)
  const uint32_t full0 = smem_u32(&ctl->full[0]), empty0 = smem_u32(&ctl->empty[0]);
  // sums [128][k16] of this CTA, over the stages once these have been multiplied; rows four floats apart from their neighbours' banks
  float* sums = reinterpret_cast<float*>(smem_raw + (tiles_addr - raw_addr));
  const int pitch = p.k16 + 4;
  TileAdaptors<4> ta;
  ta.load(p.which, p.S, row0, p.T, lane);
  const bool none = ta.none();
  int adaptor = 0;
  uint32_t off[4];
  const int group = p.group;
  const uint32_t f_bytes = static_cast<uint32_t>(F_MN ? factor_columns(p.k16) : p.k16) * (kBlockK * 2);

  if (warp >= 2 && p.given != nullptr) given_terms(p, row0 + rank * (kBlockM / p.split), row0 + (rank + 1) * (kBlockM / p.split), threadIdx.x - 64);
  if (none || p.chunks == 0) {
  } else if (warp == 0) {
    const uint32_t lead = elect_one();
    uint32_t stage = 0, phase = 0, issued = 0;
    bool ok = true;
    for (int c = rank; c < p.chunks && ok; c += p.split) {
      const int kb0 = c * p.chunk_blocks, kb1 = min(p.kblocks, kb0 + p.chunk_blocks);
      TileAdaptors<4> each = ta;
      while (ok) {
        int of[4], n = 0;
        while (n < group && each.next(adaptor, off)) {
#pragma unroll
          for (int q = 0; q < 4; ++q)
            if (q == n) of[q] = adaptor;
          ++n;
        }
        if (n == 0) break;
        for (int kb = kb0; kb < kb1; ++kb) {
          if (!bounded_wait_all(empty0 + 8 * stage, phase ^ 1u, ctl, p)) { ok = false; break; }
          const uint32_t full = full0 + 8 * stage, a_dst = tiles_addr + stage * p.stage_bytes;
          mbar_arrive_expect_tx(lead, full, kABytes + n * f_bytes);
          tma_load_2d(lead, a_dst, &p.tm_a, full, kb * kBlockK, row0);
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            if (q >= n) break;
            if (F_MN) tma_load_3d(lead, a_dst + kABytes + q * f_bytes, &p.tm_f, full, 0, kb * kBlockK, of[q]);
            else tma_load_3d(lead, a_dst + kABytes + q * f_bytes, &p.tm_f, full, kb * kBlockK, 0, of[q]);
          }
          ++issued;
          if (++stage == static_cast<uint32_t>(p.stages)) { stage = 0; phase ^= 1u; }
        }
      }
    }
    for (uint32_t s = 0; s < static_cast<uint32_t>(p.stages) && s < issued; ++s) drain_wait(full0 + 8 * s, ((issued - 1 - s) / p.stages) & 1u);
    __syncwarp();
  } else if (warp == 1) {
    const uint32_t lead = elect_one();
    uint32_t stage = 0, phase = 0, use = 0;
    bool ok = rank >= p.chunks || first_wait(full0, ctl, p);
    const uint32_t f_step = F_MN ? 2u * factor_columns(p.k16) : 2u;
    const uint64_t a_desc0 = umma_smem_desc_sw128(tiles_addr);
    const uint64_t f_desc0 = F_MN ? umma_smem_desc_factor(tiles_addr + kABytes, factor_columns(p.k16)) : umma_smem_desc_sw128(tiles_addr + kABytes);
    for (int c = rank; c < p.chunks && ok; c += p.split) {
      const int kb0 = c * p.chunk_blocks, kb1 = min(p.kblocks, kb0 + p.chunk_blocks);
      TileAdaptors<4> each = ta;
      while (ok) {
        int n = 0;
        while (n < group && each.next(adaptor, off)) ++n;
        if (n == 0) break;
        const uint32_t slot = use % kLowSlots, idesc = umma_idesc_bf16(kBlockM, n * p.k16, false, F_MN);
        if (!bounded_wait_all(smem_u32(&ctl->tempty[slot]), ((use / kLowSlots) & 1u) ^ 1u, ctl, p)) { ok = false; break; }
        ++use;
        tc_fence_after();
        const uint32_t d_tmem = tmem_base + slot * kLowSlotCols;
        for (int kb = kb0; kb < kb1; ++kb) {
          if (!bounded_wait_all(full0 + 8 * stage, phase, ctl, p)) { ok = false; break; }
          tc_fence_after();
          const uint64_t a_desc = a_desc0 + stage * (p.stage_bytes >> 4), f_desc = f_desc0 + stage * (p.stage_bytes >> 4);
#pragma unroll
          for (int kk = 0; kk < kBlockK / 16; ++kk) umma_bf16(lead, d_tmem, a_desc + 2 * kk, f_desc + f_step * kk, idesc, (kb != kb0 || kk != 0) ? 1u : 0u);
          umma_commit(lead, empty0 + 8 * stage);
          if (++stage == static_cast<uint32_t>(p.stages)) { stage = 0; phase ^= 1u; }
        }
        if (ok) umma_commit(lead, smem_u32(&ctl->tfull[slot]));
      }
    }
    __syncwarp();
  } else {
    const int quarter = warp & 3;
    const uint32_t lane_base = tmem_base + (static_cast<uint32_t>(quarter * 32) << 16);
    float acc[kMaxRank];
#pragma unroll
    for (int j = 0; j < kMaxRank; ++j) acc[j] = 0.f;
    uint32_t use = 0;
    bool ok = true;
    for (int c = rank; c < p.chunks && ok; c += p.split) {
      TileAdaptors<4> each = ta;
      while (true) {
        int n = 0, place = -1;                                       // which of the group's adaptors this thread's row has
        while (n < group && each.next(adaptor, off)) {
          uint32_t others = 0;
#pragma unroll
          for (int w = 0; w < 4; ++w)
            if (w == quarter) others = off[w];
          if (!(others >> lane & 1)) place = n;
          ++n;
        }
        if (n == 0) break;
        const uint32_t slot = use % kLowSlots;
        if (!bounded_wait_warp(smem_u32(&ctl->tfull[slot]), (use / kLowSlots) & 1u, ctl, p.status, lane)) { ok = false; break; }
        ++use;
        tc_fence_after();
        for (int q = 0; q < n; ++q) {
#pragma unroll
          for (int b = 0; b < kMaxRank / 16; ++b) {
            if (b * 16 >= p.k16) break;
            float x[16];
            tmem_ld16(lane_base + slot * kLowSlotCols + q * p.k16 + b * 16, x);
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[b * 16 + e] += place == q ? x[e] : 0.f;
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&ctl->tempty[slot]));
      }
    }
    float4* dst = reinterpret_cast<float4*>(sums + (quarter * 32 + lane) * pitch);
#pragma unroll
    for (int j = 0; j < kMaxRank / 4; ++j) {
      if (4 * j >= p.k16) break;
      dst[j] = make_float4(acc[4 * j], acc[4 * j + 1], acc[4 * j + 2], acc[4 * j + 3]);
    }
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();                                                // the other CTAs' sums
  const int quads = p.k16 / 4, rows = kBlockM / p.split;
  for (int at = threadIdx.x; at < (p.chunks > 0 ? rows * quads : 0); at += kLowThreads) {
    const int r = at / quads, j0 = (at - r * quads) * 4, row = rank * rows + r, t = row0 + row;
    if (t >= p.T) break;
    const int i = adaptor_of(p.which, p.S, t, p.T);
    float x[4] = {0.f, 0.f, 0.f, 0.f};
    if (i >= 0) {
      float4 y[8];
      const uint32_t own = smem_u32(sums + row * pitch + j0);
#pragma unroll
      for (int c = 0; c < 8; ++c)
        if (c < p.split) y[c] = ld_cluster_v4(cluster_map_shared(own, c));
#pragma unroll
      for (int c = 0; c < 8; ++c)
        if (c < p.split) x[0] += y[c].x, x[1] += y[c].y, x[2] += y[c].z, x[3] += y[c].w;
      const float s = p.scale == nullptr ? 1.f : p.scale[i];
#pragma unroll
      for (int q = 0; q < 4; ++q) x[q] *= s;
    }
    const bool refused = adaptor_refused(p.which, p.S, t);
    if (refused && p.status != nullptr && j0 == 0) atomicOr(p.status, kStatusBadAdaptor);
    if (p.low != nullptr) {
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (j0 + q < p.k) p.low[static_cast<size_t>(t) * p.k + j0 + q] = refused ? CUDART_NAN_F : x[q];
    }
    store_terms(p, t, j0, x, p.two, p.three);
  }
  __syncthreads();
  if (warp == 1) drain_after_abort<1>(ctl, true);
  __syncthreads();
  cluster_sync_all();                                                // nobody reads this CTA's sums any more
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, kLowTmemCols);
  }
}

// ---- the shared product and the adaptors' part
// Bound by the tensor pipe: 8192 x 4096 x 4096, k = 16, eight adaptors 172 us with the pipe 88 % busy; 2005 rows in one round of 64 pairs 26 us (at the peak rate 20).
struct AdaptedParams {
  CUtensorMap tm_a;                     // rows [T, K]              box 64 x 128
  CUtensorMap tm_b;                     // W [N, K] box 64 x (TN / CTAS), or [K, N] box 64 x 64 (MN-major)
  CUtensorMap tm_u;                     // two terms of low [T, 64 pieces]  box 64 x 128
  CUtensorMap tm_f;                     // A [S, N, k] box 64 x (TN / CTAS), or B [S, k, N] box 64 x 64
  const int* which;
  __nv_bfloat16* out;
  int64_t out_stride;
  unsigned* status;
  uint64_t wait_limit_ns;
  int T, S, N, k, pieces;               // pieces 0: no adaptors
  int kblocks;                          // 0: the adaptors' part alone
  int m_units, n_tiles, stages, stage_bytes;
  int store;                            // bytes that rows of out allow a store: 32, 16 or 2
};
constexpr int kAdaptedThreads = 320;

// Thirty-two columns of 32 rows from `col` on, a row a lane (`rows` of them exist), x in fp32. Rows that allow no vectors are written a row at a time, its columns
// side by side, by way of `stage` (2005 x 2003: each lane its own row, two bytes at a time, the kernel took 51 us, so 11).
constexpr int kStorePitch = 17;                   // words of a staged row: 32 columns and one over, so that lanes meet no bank twice
constexpr int kStoreBytes = 8 * 32 * kStorePitch * 4;
__device__ __forceinline__ void store_rows32(const AdaptedParams& p, __nv_bfloat16* first, int lane, int rows, int col, const uint32_t (&x)[32], uint32_t* stage) {
  uint32_t y[16];
#pragma unroll
  for (int q = 0; q < 16; ++q) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(__uint_as_float(x[2 * q]), __uint_as_float(x[2 * q + 1]));
    y[q] = *reinterpret_cast<const uint32_t*>(&v);
  }
  if (p.store >= 16) {
    if (lane >= rows) return;
    __nv_bfloat16* dst = first + lane * p.out_stride + col;
    if (col + 32 <= p.N && p.store == 32) {
      st_global_v8_b32(dst, y);
      st_global_v8_b32(dst + 16, y + 8);
      return;
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if (col + 8 * q + 8 <= p.N) {
        *reinterpret_cast<uint4*>(dst + 8 * q) = make_uint4(y[4 * q], y[4 * q + 1], y[4 * q + 2], y[4 * q + 3]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (col + 8 * q + e < p.N) dst[8 * q + e] = __ushort_as_bfloat16(static_cast<unsigned short>(y[4 * q + e / 2] >> (16 * (e & 1))));
      }
    }
    return;
  }
#pragma unroll
  for (int q = 0; q < 16; ++q) stage[lane * kStorePitch + q] = y[q];
  __syncwarp();
  if (col + lane < p.N) {
    __nv_bfloat16* dst = first + col + lane;
#pragma unroll 8
    for (int r = 0; r < rows; ++r)
      dst[r * p.out_stride] = __ushort_as_bfloat16(static_cast<unsigned short>(stage[r * kStorePitch + lane / 2] >> (16 * (lane & 1))));
  }
  __syncwarp();
}

template <bool B_MN, int TN, int CTAS>
__global__ void __launch_bounds__(kAdaptedThreads, 1) adapted_gemm_kernel(const __grid_constant__ AdaptedParams p) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw_addr = smem_u32(smem_raw);
  const uint32_t tiles_addr = (raw_addr + 1023u) & ~1023u;
  GemmControl* ctl = reinterpret_cast<GemmControl*>(smem_raw + (tiles_addr - raw_addr) + static_cast<size_t>(p.stages) * p.stage_bytes);
  const int warp = static_cast<int>(warp_uniform(threadIdx.x >> 5));
  const int lane = threadIdx.x & 31;
  const int items = p.m_units * p.n_tiles;
  const uint32_t cta_rank = CTAS == 2 ? warp_uniform(cluster_cta_rank()) : 0u;      // 0 = the pair's leader
  const int first_item = CTAS == 2 ? static_cast<int>(blockIdx.x >> 1) : static_cast<int>(blockIdx.x);
  const int item_step = CTAS == 2 ? static_cast<int>(gridDim.x >> 1) : static_cast<int>(gridDim.x);
  constexpr uint32_t kSlots = 2;
  constexpr int kBCols = TN / CTAS;
  constexpr uint32_t kBBytes = kBCols * kBlockK * 2;
  constexpr int kWords = 4 * CTAS;
  if (threadIdx.x == 0) {
    for (int s = 0; s < p.stages; ++s) {
      mbar_init(smem_u32(&ctl->full[s]), 1);
      mbar_init(smem_u32(&ctl->empty[s]), 1);
    }
    for (uint32_t s = 0; s < kSlots; ++s) {
      mbar_init(smem_u32(&ctl->tfull[s]), 1);
      mbar_init(smem_u32(&ctl->tempty[s]), 8 * CTAS);
    }
    mbar_init(smem_u32(&ctl->drain), 1);
    ctl->abort = 0;
    ctl->wait_limit_ns = p.wait_limit_ns;
    fence_mbar_init();
    if (p.kblocks > 0) {
      tma_prefetch_desc(&p.tm_a);
      tma_prefetch_desc(&p.tm_b);
    }
    if (p.pieces > 0) {
      tma_prefetch_desc(&p.tm_u);
      tma_prefetch_desc(&p.tm_f);
    }
  }
  if (warp == 1) {
    if (CTAS == 2) {
      tmem_alloc_pair(smem_u32(&ctl->tmem_base), kTmemCols);
      tmem_relinquish_pair();
    } else {
      tmem_alloc(smem_u32(&ctl->tmem_base), kTmemCols);
      tmem_relinquish();
    }
  }
  tc_fence_before();
  __syncthreads();
  if (CTAS == 2) cluster_sync_all();   // the peer's barriers are initialised before anything arrives on them
  tc_fence_after();
  const uint32_t tmem_base = warp_uniform(ctl->tmem_base);
  // Ahead of this kernel is adaptor_low_kernel, a gate (or this kernel itself, of d_x): rows and W are there, the terms of low are waited for where they are read. It is a
  // gate again: what is behind it starts when the epilogue warps have waited.
  TileAdaptors<kWords> ta;
  int adaptor = 0;
  uint32_t off[kWords];

  if (warp == 0) {
    const uint32_t lead = elect_one(), expects = cta_rank == 0 ? lead : 0u;
    uint32_t stage = 0, phase = 0, issued = 0;
    bool ok = true;
    const uint32_t own_full = smem_u32(&ctl->full[0]), empty0 = smem_u32(&ctl->empty[0]);
    const uint32_t full0 = CTAS == 2 ? warp_uniform(cluster_map_shared(own_full, 0)) : own_full;   // the leader's barriers
    uint32_t full = 0, a_dst = 0;
    bool waited = false;
    auto begin = [&]() {
      ok = bounded_wait_all(empty0 + 8 * stage, phase ^ 1u, ctl, p);
      if (!ok) return false;
      full = full0 + 8 * stage;
      a_dst = tiles_addr + stage * p.stage_bytes;
      mbar_arrive_expect_tx(expects, own_full + 8 * stage, CTAS * (kABytes + kBBytes));      // of both CTAs' copies when paired
      ++issued;
      if (++stage == static_cast<uint32_t>(p.stages)) { stage = 0; phase ^= 1u; }
      return true;
    };
    auto load2 = [&](uint32_t dst, const CUtensorMap* tm, int x, int y) {
      if (CTAS == 2) tma_load_2d_pair(lead, dst, tm, full, x, y);
      else tma_load_2d(lead, dst, tm, full, x, y);
    };
    auto load3 = [&](uint32_t dst, const CUtensorMap* tm, int x, int y, int z) {
      if (CTAS == 2) tma_load_3d_pair(lead, dst, tm, full, x, y, z);
      else tma_load_3d(lead, dst, tm, full, x, y, z);
    };
    for (int item = first_item; item < items && ok; item += item_step) {
      const int mt = item / p.n_tiles, nt = item - mt * p.n_tiles;
      const int am = (mt * CTAS + static_cast<int>(cta_rank)) * kBlockM, bn = nt * TN + static_cast<int>(cta_rank) * kBCols;
      for (int k = 0; k < p.kblocks * kBlockK; k += kBlockK) {
        if (!begin()) break;
        load2(a_dst, &p.tm_a, k, am);
        if (B_MN) {
#pragma unroll
          for (int q = 0; q < kBCols / 64; ++q) load2(a_dst + kABytes + q * kMnBoxBytes, &p.tm_b, bn + q * 64, k);
        } else {
          load2(a_dst + kABytes, &p.tm_b, k, bn);
        }
      }
      if (p.pieces == 0) continue;
      ta.load(p.which, p.S, mt * CTAS * kBlockM, p.T, lane);
      if (!waited) grid_dependency_wait();
      waited = true;
      while (ok && ta.next(adaptor, off)) {
        for (int q = 0; q < p.pieces; ++q) {
          if (!begin()) break;
          load2(a_dst, &p.tm_u, q * 64, am);
          if (B_MN) {
#pragma unroll
            for (int c = 0; c < kBCols / 64; ++c) load3(a_dst + kABytes + c * kMnBoxBytes, &p.tm_f, bn + c * 64, q * kPieceRank, adaptor);
          } else {
            load3(a_dst + kABytes, &p.tm_f, q * kPieceRank, bn, adaptor);
          }
        }
      }
    }
    // no copy may still be in flight when the CTA goes away (they have all landed unless some warp gave up)
    if (CTAS == 1 || cta_rank == 0) {
      for (uint32_t s = 0; s < static_cast<uint32_t>(p.stages) && s < issued; ++s)
        drain_wait(own_full + 8 * s, ((issued - 1 - s) / p.stages) & 1u);
    }
    __syncwarp();
  } else if (warp == 1) {
    if (cta_rank == 0) {
      const uint32_t lead = elect_one();
      uint32_t stage = 0, phase = 0, use = 0;
      bool ok = first_item >= items || p.kblocks == 0 || first_wait(smem_u32(&ctl->full[0]), ctl, p);
      const uint32_t idesc = umma_idesc_bf16(kBlockM * CTAS, TN, false, B_MN);
      constexpr uint32_t kStepB = B_MN ? 128u : 2u;
      const uint64_t a_desc0 = umma_smem_desc_sw128(tiles_addr);
      const uint64_t b_desc0 = B_MN ? umma_smem_desc_mn_sw128(tiles_addr + kABytes, kMnBoxBytes) : umma_smem_desc_sw128(tiles_addr + kABytes);
      const uint32_t stage_step = p.stage_bytes >> 4, full0 = smem_u32(&ctl->full[0]), empty0 = smem_u32(&ctl->empty[0]);
      auto commit = [&](uint32_t bar) {                        // pairs: in both CTAs
        if (CTAS == 2) umma_commit_pair(lead, bar);
        else umma_commit(lead, bar);
      };
      uint64_t a_desc = 0, b_desc = 0;
      auto begin = [&]() {
        ok = bounded_wait_all(full0 + 8 * stage, phase, ctl, p);
        if (!ok) return false;
        tc_fence_after();
        a_desc = a_desc0 + stage * stage_step;
        b_desc = b_desc0 + stage * stage_step;
        return true;
      };
      auto end = [&]() {
        commit(empty0 + 8 * stage);
        if (++stage == static_cast<uint32_t>(p.stages)) { stage = 0; phase ^= 1u; }
      };
      for (int item = first_item; item < items && ok; item += item_step, ++use) {
        const int mt = item / p.n_tiles;
        const uint32_t slot = use % kSlots;
        if (!bounded_wait_all(smem_u32(&ctl->tempty[slot]), ((use / kSlots) & 1u) ^ 1u, ctl, p)) { ok = false; break; }
        tc_fence_after();
        const uint32_t d_tmem = tmem_base + slot * TN;
        for (int kb = 0; kb < p.kblocks; ++kb) {
          if (!begin()) break;
#pragma unroll
          for (int kk = 0; kk < kBlockK / 16; ++kk) {
            if (CTAS == 2) umma_bf16_pair(lead, d_tmem, a_desc + 2 * kk, b_desc + kStepB * kk, idesc, (kb | kk) != 0 ? 1u : 0u);
            else umma_bf16(lead, d_tmem, a_desc + 2 * kk, b_desc + kStepB * kk, idesc, (kb | kk) != 0 ? 1u : 0u);
          }
          end();
        }
        if (p.pieces > 0) {
          ta.load(p.which, p.S, mt * CTAS * kBlockM, p.T, lane);
          while (ok && ta.next(adaptor, off)) {
            for (int q = 0; q < p.pieces; ++q) {
              if (!begin()) break;
              const int steps = p.k - q * kPieceRank > 16 ? 2 : 1;
              for (int j = 0; j < steps; ++j) {
                const uint32_t acc = p.kblocks > 0 || q > 0 || j > 0 ? 1u : 0u;
                umma_bf16_rows(lead, d_tmem, a_desc + 2 * j, b_desc + kStepB * j, idesc, acc, off);          // the high terms,
                umma_bf16_rows(lead, d_tmem, a_desc + 4 + 2 * j, b_desc + kStepB * j, idesc, 1u, off);       // 64 bytes on, the low ones
              }
              end();
            }
          }
        }
        if (!ok) break;
        commit(smem_u32(&ctl->tfull[slot]));
      }
    }
    __syncwarp();
  } else {
    const int quarter = warp & 3, sub = (warp - 2) >> 2;
    const uint32_t lane_base = tmem_base + (static_cast<uint32_t>(quarter * 32) << 16);
    uint32_t* stage = reinterpret_cast<uint32_t*>(ctl + 1) + (warp - 2) * (32 * kStorePitch);        // (there with p.store == 2 only)
    uint32_t use = 0;
    grid_dependency_wait();
    grid_launch_dependents();
    for (int item = first_item; item < items; item += item_step, ++use) {
      const int mt = item / p.n_tiles, nt = item - mt * p.n_tiles;
      const uint32_t slot = use % kSlots;
      const int row = (mt * CTAS + static_cast<int>(cta_rank)) * kBlockM + quarter * 32 + lane;
      const bool inside = row < p.T;
      const bool refused = p.pieces > 0 && inside && adaptor_refused(p.which, p.S, row);
      const bool empty = p.kblocks == 0 && adaptor_of(p.which, p.S, row, p.T) < 0;
      if (!bounded_wait_warp(smem_u32(&ctl->tfull[slot]), (use / kSlots) & 1u, ctl, p.status, lane)) break;
      tc_fence_after();
      const uint32_t tcol = lane_base + slot * TN;
      __nv_bfloat16* out = p.out + (row - lane) * p.out_stride;
      const int batches = (min(TN, p.N - nt * TN) + 31) / 32;
      for (int b = sub; b < batches; b += 2) {
        uint32_t x[32];
        tmem_ld32_issue(tcol + b * 32, x);
        tmem_ld_wait32(x);
        if (refused || empty) {
#pragma unroll
          for (int q = 0; q < 32; ++q) x[q] = refused ? 0x7fffffffu : 0u;
        }
        store_rows32(p, out, lane, min(32, p.T - (row - lane)), nt * TN + b * 32, x, stage);
        __syncwarp();
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        if (CTAS == 2) mbar_arrive_cluster(cluster_map_shared(smem_u32(&ctl->tempty[slot]), 0));
        else mbar_arrive(smem_u32(&ctl->tempty[slot]));
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 1) drain_after_abort<CTAS>(ctl, cta_rank == 0);
  if (CTAS == 2) {        // a CTA of a pair may leave only when its partner no longer needs it
    __syncthreads();
    cluster_sync_all();
  }
  if (warp == 1) {
    tc_fence_after();
    if (CTAS == 2) tmem_dealloc_pair(tmem_base, kTmemCols);
    else tmem_dealloc(tmem_base, kTmemCols);
  }
}

// ---- few rows
// low of few rows: a block has four of a row's rank values, its warps a quarter of d each. Bound by latency: 64 rows, d = 4096, k = 16, 32 adaptors 5 us, of which 1.4 are
// the dot products.
struct LowRowsParams {
  const __nv_bfloat16 *x, *B;
  int64_t x_stride;
  const int* which;
  const float* scale;
  float* low;                           // [T, k]
  unsigned* status;                     // or NULL
  int T, d, k, S, wide;                 // wide: vectors of eight elements
};
__global__ void __launch_bounds__(128) low_rows_kernel(const LowRowsParams p) {
  __shared__ float4 red[4];
  grid_dependency_wait();
  grid_launch_dependents();             // (a gate: what is behind may read all but low before it waits)
  const int t = blockIdx.x, j0 = blockIdx.y * 4, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int i = adaptor_of(p.which, p.S, t, p.T);
  float s[4] = {0.f, 0.f, 0.f, 0.f};
  if (i >= 0) {
    const __nv_bfloat16* x = p.x + t * p.x_stride;
    const __nv_bfloat16* f = p.B + (static_cast<size_t>(i) * p.k + j0) * p.d;
    const int js = min(4, p.k - j0);
    if (p.wide) {
#pragma unroll 4
      for (int c = threadIdx.x * 8; c < p.d; c += 1024) {
        Raw<__nv_bfloat16, 8> xv, fv[4];
        xv.load(x + c);
#pragma unroll
        for (int q = 0; q < 4; ++q) fv[q].load(f + static_cast<size_t>(min(q, js - 1)) * p.d + c);
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
          for (int e = 0; e < 8; ++e) s[q] = fmaf(xv.value(e), fv[q].value(e), s[q]);
      }
    } else {
      for (int c = threadIdx.x; c < p.d; c += 128) {
        const float xv = to_f32(x[c]);
#pragma unroll
        for (int q = 0; q < 4; ++q) s[q] = fmaf(xv, to_f32(f[static_cast<size_t>(min(q, js - 1)) * p.d + c]), s[q]);
      }
    }
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) s[q] += __shfl_xor_sync(0xffffffffu, s[q], o);
  }
  if (lane == 0) red[warp] = make_float4(s[0], s[1], s[2], s[3]);
  __syncthreads();
  if (threadIdx.x < 4 && j0 + threadIdx.x < p.k) {
    const float* r = reinterpret_cast<const float*>(red) + threadIdx.x;
    const bool refused = adaptor_refused(p.which, p.S, t);
    const float y = i < 0 ? 0.f : ((r[0] + r[4]) + (r[8] + r[12])) * (p.scale == nullptr ? 1.f : p.scale[i]);
    p.low[static_cast<size_t>(t) * p.k + j0 + threadIdx.x] = refused ? CUDART_NAN_F : y;
    if (refused && threadIdx.x == 0 && j0 == 0 && p.status != nullptr) atomicOr(p.status, kStatusBadAdaptor);
  }
}

// out of few rows: W's rows are the MMA's M (128 of them a cluster), the tokens its N. The CTAs of a cluster share K; each has every SPLIT-th token, forms its adaptors'
// part, adds it to its own sums, and adds the cluster's sums of its tokens up, which meet in shared memory.
// A few rank values in all (T k <= kOwnLow): every cluster forms low itself, each CTA over its share of K, one launch less; W, which is all but a few of the bytes, is asked
// into L2 while the kernels ahead still run.
struct RowsParams {
  CUtensorMap tm_w;                     // W [N, K]   box 64 x 128
  CUtensorMap tm_x;                     // x [T, K]   box 64 x tokens
  const __nv_bfloat16* A;               // [S, N, k]
  const float* low;                     // [T, k] (low_rows_kernel's)
  const int* which;
  __nv_bfloat16* out;
  int64_t out_stride;
  unsigned* status;
  uint64_t wait_limit_ns;
  int T, S, N, k, tokens;               // tokens: T rounded up to 16
  int kblocks, stages, stage_bytes;
  int wide;                             // rows of A are vectors of eight elements
  int store4;                           // rows of out allow stores of four elements
  // where low is formed here
  LowRowsParams own;                    // low: NULL or where it is wanted
};
constexpr int kOwnLow = 32;
struct RowsShared {
  float part[kOwnLow], low[kOwnLow];
};
constexpr int kRowsThreads = 320;
// The adaptors' part of column n of ROWS rows t, t + step, t + 2 step, ... (those that exist): begin() asks for A, finish() needs low, whose rows are low_step apart in
// shared memory.
template <int ROWS>
struct RowsAdaptors {
  int i[ROWS];
  Raw<__nv_bfloat16, 8> a[ROWS][2];     // sixteen of A's row, where rows are vectors
  __device__ __forceinline__ const __nv_bfloat16* row(const RowsParams& p, int q, int n) const { return p.A + (static_cast<size_t>(i[q]) * p.N + n) * p.k; }
  __device__ __forceinline__ void load(const RowsParams& p, int n, int j) {
#pragma unroll
    for (int q = 0; q < ROWS; ++q) {
      if (i[q] < 0) continue;
      a[q][0].load(row(p, q, n) + j);
      if (p.k > j + 8) a[q][1].load(row(p, q, n) + j + 8);
    }
  }
  __device__ __forceinline__ void begin(const RowsParams& p, int step, int t, int n) {
#pragma unroll
    for (int q = 0; q < ROWS; ++q) i[q] = n < p.N ? adaptor_of(p.which, p.S, t + q * step, p.T) : -1;
    if (p.wide) load(p, n, 0);
    if (!p.wide || p.k > 16) {
#pragma unroll
      for (int q = 0; q < ROWS; ++q)
        if (i[q] >= 0) prefetch_l2(row(p, q, n) + p.k - 1);
    }
  }
  __device__ __forceinline__ void finish(const RowsParams& p, const float* low_row, int low_step, int n, float* y) {
#pragma unroll
    for (int q = 0; q < ROWS; ++q) y[q] = 0.f;
    if (p.wide) {
      for (int j = 0; j < p.k; j += 16) {
        if (j > 0) load(p, n, j);
#pragma unroll
        for (int q = 0; q < ROWS; ++q) {
          if (i[q] < 0) continue;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (j + 8 * h >= p.k) break;
            const float4* low = reinterpret_cast<const float4*>(low_row + q * low_step + j + 8 * h);
            const float4 l0 = low[0], l1 = low[1];
            const float l[8] = {l0.x, l0.y, l0.z, l0.w, l1.x, l1.y, l1.z, l1.w};
#pragma unroll
            for (int e = 0; e < 8; ++e) y[q] = fmaf(a[q][h].value(e), l[e], y[q]);
          }
        }
      }
    } else {
#pragma unroll
      for (int q = 0; q < ROWS; ++q) {
        if (i[q] < 0) continue;
        const __nv_bfloat16* at = row(p, q, n);
        for (int j = 0; j < p.k; ++j) y[q] = fmaf(to_f32(at[j]), low_row[q * low_step + j], y[q]);
      }
    }
  }
};
// This CTA's share [c0, c1) of K of the T k dot products, four at a time a warp.
__device__ __forceinline__ void own_low_parts(const LowRowsParams& p, int c0, int c1, int warp, int lane, float* part) {
  for (int base = warp * 4; base < p.T * p.k; base += 32) {
    const __nv_bfloat16 *x[4], *f[4];
    float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int id = min(base + q, p.T * p.k - 1), t = id / p.k, i = max(adaptor_of(p.which, p.S, t, p.T), 0);       // (what a row without adaptor gives is not used)
      x[q] = p.x + t * p.x_stride;
      f[q] = p.B + (static_cast<size_t>(i) * p.k + (id - t * p.k)) * p.d;
    }
    if (p.wide) {
#pragma unroll 2
      for (int c = c0 + lane * 8; c < c1; c += 256) {
        Raw<__nv_bfloat16, 8> xv[4], fv[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          xv[q].load(x[q] + c);
          fv[q].load(f[q] + c);
        }
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
          for (int e = 0; e < 8; ++e) s[q] = fmaf(xv[q].value(e), fv[q].value(e), s[q]);
      }
    } else {
      for (int c = c0 + lane; c < c1; c += 32)
#pragma unroll
        for (int q = 0; q < 4; ++q) s[q] = fmaf(to_f32(x[q][c]), to_f32(f[q][c]), s[q]);
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) s[q] += __shfl_xor_sync(0xffffffffu, s[q], o);
      if (lane == 0 && base + q < p.T * p.k) part[base + q] = s[q];
    }
  }
}
__device__ __forceinline__ void rows_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }      // warps 2 to 9

// AHEAD: rows of a thread whose adaptors' part is formed while W is on its way (all loads in flight together: eight rows a thread, 4096 x 4096, 64 rows 15.1 -> 14.3 us against
// twice four; one or two, 1024 x 1024, 16 rows 5.5 -> 5.9).
template <int SPLIT, bool OWN_LOW, int AHEAD>
__global__ void __launch_bounds__(kRowsThreads, 2) adapted_rows_kernel(const __grid_constant__ RowsParams p) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw_addr = smem_u32(smem_raw);
  const uint32_t tiles_addr = (raw_addr + 1023u) & ~1023u;
  GemmControl* ctl = reinterpret_cast<GemmControl*>(smem_raw + (tiles_addr - raw_addr) + static_cast<size_t>(p.stages) * p.stage_bytes);
  RowsShared* shared = reinterpret_cast<RowsShared*>((reinterpret_cast<uintptr_t>(ctl + 1) + 15) & ~static_cast<uintptr_t>(15));
  float* lows = reinterpret_cast<float*>(shared + 1);                // of this CTA's tokens [T / SPLIT][k] (without OWN_LOW)
  const int warp = static_cast<int>(warp_uniform(threadIdx.x >> 5));
  const int lane = threadIdx.x & 31;
  const int rank = static_cast<int>(blockIdx.x % SPLIT), tile = blockIdx.x / SPLIT;
  const int kb0 = rank * p.kblocks / SPLIT, kb1 = (rank + 1) * p.kblocks / SPLIT;
  const uint32_t tmem_cols = p.tokens <= 32 ? 32u : p.tokens <= 64 ? 64u : 128u;
  if (threadIdx.x == 0) {
    for (int s = 0; s < p.stages; ++s) {
      mbar_init(smem_u32(&ctl->full[s]), 1);
      mbar_init(smem_u32(&ctl->empty[s]), 1);
    }
    mbar_init(smem_u32(&ctl->tfull[0]), 1);
    mbar_init(smem_u32(&ctl->drain), 1);
    ctl->abort = 0;
    ctl->wait_limit_ns = p.wait_limit_ns;
    fence_mbar_init();
    tma_prefetch_desc(&p.tm_w);
    tma_prefetch_desc(&p.tm_x);
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(&ctl->tmem_base), tmem_cols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = warp_uniform(ctl->tmem_base);
  const uint32_t full0 = smem_u32(&ctl->full[0]), empty0 = smem_u32(&ctl->empty[0]);
  float part[AHEAD];                    // the adaptors' part of this CTA's rows
  // sums [tokens][128] fp32, over the stages once these have been multiplied
  float* sums = reinterpret_cast<float*>(smem_raw + (tiles_addr - raw_addr));

  if (warp == 0) {
    const uint32_t lead = elect_one();
    // low_rows_kernel ahead is a gate: x and W are there. Without it W is asked into L2 while the kernel ahead still runs.
    if (OWN_LOW) {
      for (int kb = kb0; kb < kb1; ++kb) tma_prefetch_2d(lead, &p.tm_w, kb * kBlockK, tile * kBlockM);
      grid_dependency_wait();
    }
    const uint32_t bytes = kABytes + static_cast<uint32_t>(p.tokens) * (kBlockK * 2);
    uint32_t stage = 0, phase = 0, issued = 0;
    for (int kb = kb0; kb < kb1; ++kb) {
      if (!bounded_wait_all(empty0 + 8 * stage, phase ^ 1u, ctl, p)) break;
      const uint32_t full = full0 + 8 * stage, dst = tiles_addr + stage * p.stage_bytes;
      mbar_arrive_expect_tx(lead, full, bytes);
      tma_load_2d(lead, dst, &p.tm_w, full, kb * kBlockK, tile * kBlockM);
      tma_load_2d(lead, dst + kABytes, &p.tm_x, full, kb * kBlockK, 0);
      ++issued;
      if (++stage == static_cast<uint32_t>(p.stages)) { stage = 0; phase ^= 1u; }
    }
    for (uint32_t s = 0; s < static_cast<uint32_t>(p.stages) && s < issued; ++s) drain_wait(full0 + 8 * s, ((issued - 1 - s) / p.stages) & 1u);
    __syncwarp();
  } else if (warp == 1) {
    const uint32_t lead = elect_one();
    const uint32_t idesc = umma_idesc_bf16(kBlockM, p.tokens);
    const uint64_t a_desc0 = umma_smem_desc_sw128(tiles_addr), b_desc0 = umma_smem_desc_sw128(tiles_addr + kABytes);
    uint32_t stage = 0, phase = 0;
    bool ok = first_wait(full0, ctl, p);
    for (int kb = kb0; kb < kb1 && ok; ++kb) {
      if (!bounded_wait_all(full0 + 8 * stage, phase, ctl, p)) { ok = false; break; }
      tc_fence_after();
      const uint64_t a_desc = a_desc0 + stage * (p.stage_bytes >> 4), b_desc = b_desc0 + stage * (p.stage_bytes >> 4);
#pragma unroll
      for (int kk = 0; kk < kBlockK / 16; ++kk) umma_bf16(lead, tmem_base, a_desc + 2 * kk, b_desc + 2 * kk, idesc, (kb != kb0 || kk != 0) ? 1u : 0u);
      umma_commit(lead, empty0 + 8 * stage);
      if (++stage == static_cast<uint32_t>(p.stages)) { stage = 0; phase ^= 1u; }
    }
    if (ok) umma_commit(lead, smem_u32(&ctl->tfull[0]));
    __syncwarp();
  } else {
    const int quarter = warp & 3, sub = (warp - 2) >> 2, n = tile * kBlockM + quarter * 32 + lane;
    const uint32_t lane_base = tmem_base + (static_cast<uint32_t>(quarter * 32) << 16);
    const int first = rank + SPLIT * sub;
    if (OWN_LOW) {
      grid_dependency_wait();
      grid_launch_dependents();
      for (int t = first; t < p.T; t += 2 * SPLIT) {
        const int i = adaptor_of(p.which, p.S, t, p.T);
        if (i >= 0 && n < p.N) prefetch_l2(p.A + (static_cast<size_t>(i) * p.N + n) * p.k);
      }
      own_low_parts(p.own, kb0 * kBlockK, min(kb1 * kBlockK, p.own.d), warp - 2, lane, shared->part);
    } else {
      RowsAdaptors<AHEAD> ra;
      ra.begin(p, 2 * SPLIT, first, n);
      for (int t = first + AHEAD * 2 * SPLIT; t < p.T; t += 2 * SPLIT) {
        const int i = adaptor_of(p.which, p.S, t, p.T);
        if (i >= 0 && n < p.N) prefetch_l2(p.A + (static_cast<size_t>(i) * p.N + n) * p.k);
      }
      grid_dependency_wait();
      grid_launch_dependents();
      const int values = (p.T - rank + SPLIT - 1) / SPLIT * p.k;
      for (int e = threadIdx.x - 64; e < values; e += 256) {
        const int j = e / p.k;
        lows[e] = p.low[static_cast<size_t>(rank + SPLIT * j) * p.k + (e - j * p.k)];
      }
      rows_sync();
      ra.finish(p, lows + sub * p.k, 2 * p.k, n, part);
    }
    if (bounded_wait_warp(smem_u32(&ctl->tfull[0]), 0, ctl, p.status, lane)) {
      tc_fence_after();
      for (int b = sub; b < p.tokens / 16; b += 2) {
        float x[16];
        tmem_ld16(lane_base + b * 16, x);
#pragma unroll
        for (int q = 0; q < 16; ++q) sums[(b * 16 + q) * kBlockM + quarter * 32 + lane] = x[q];
      }
    }
    tc_fence_before();
    if (!OWN_LOW) {
      rows_sync();                                                   // this CTA's sums are there: its tokens' parts are added to them
      float* mine = sums + quarter * 32 + lane;
#pragma unroll
      for (int q = 0; q < AHEAD; ++q)
        if (first + q * 2 * SPLIT < p.T) mine[(first + q * 2 * SPLIT) * kBlockM] += part[q];
      for (int q = AHEAD; first + q * 2 * SPLIT < p.T; q += AHEAD) {
        RowsAdaptors<AHEAD> ra;
        ra.begin(p, 2 * SPLIT, first + q * 2 * SPLIT, n);
        ra.finish(p, lows + (sub + 2 * q) * p.k, 2 * p.k, n, part);
#pragma unroll
        for (int e = 0; e < AHEAD; ++e)
          if (first + (q + e) * 2 * SPLIT < p.T) mine[(first + (q + e) * 2 * SPLIT) * kBlockM] += part[e];
      }
    }
  }
  __syncthreads();
  cluster_sync_all();                                                // the other CTAs' sums
  if (OWN_LOW && warp >= 2) {
    const int m = (warp & 3) * 32 + lane, n = tile * kBlockM + m, first = rank + SPLIT * ((warp - 2) >> 2);
    const uint32_t own = smem_u32(sums) + 4u * m;
    const int id = threadIdx.x - 64;
    if (id < p.T * p.k) {
      float v[SPLIT], all = 0.f;
#pragma unroll
      for (int r = 0; r < SPLIT; ++r) v[r] = ld_cluster_f32(cluster_map_shared(smem_u32(shared->part + id), r));
#pragma unroll
      for (int r = 0; r < SPLIT; ++r) all += v[r];
      const int t = id / p.k, i = adaptor_of(p.which, p.S, t, p.T);
      const bool refused = adaptor_refused(p.which, p.S, t);
      all = i < 0 ? 0.f : all * (p.own.scale == nullptr ? 1.f : p.own.scale[i]);
      shared->low[id] = all;
      if (blockIdx.x == 0) {
        if (p.own.low != nullptr) p.own.low[id] = refused ? CUDART_NAN_F : all;
        if (refused && p.own.status != nullptr) atomicOr(p.own.status, kStatusBadAdaptor);
      }
    }
    rows_sync();
    for (int t = first; t < p.T; t += 8 * SPLIT) {
      float y[4], sum[4][SPLIT];
      RowsAdaptors<4> ra;
      ra.begin(p, 2 * SPLIT, t, n);
#pragma unroll
      for (int q = 0; q < 4; ++q)                                    // four rows: all loads in flight together
#pragma unroll
        for (int r = 0; r < SPLIT; ++r)
          sum[q][r] = t + q * 2 * SPLIT < p.T ? ld_cluster_f32(cluster_map_shared(own + 4u * kBlockM * (t + q * 2 * SPLIT), r)) : 0.f;
      ra.finish(p, shared->low + t * p.k, 2 * SPLIT * p.k, n, y);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int at = t + q * 2 * SPLIT;
        if (at >= p.T || n >= p.N) continue;
        float all = y[q];
#pragma unroll
        for (int r = 0; r < SPLIT; ++r) all += sum[q][r];
        p.out[at * p.out_stride + n] = __float2bfloat16_rn(adaptor_refused(p.which, p.S, at) ? CUDART_NAN_F : all);
      }
    }
  } else if (warp >= 2) {
    // a warp to a token, four columns to a lane
#pragma unroll 2
    for (int t = rank + SPLIT * (warp - 2); t < p.T; t += SPLIT * 8) {
      const uint32_t own = smem_u32(sums + t * kBlockM + 4 * lane);
      float4 v[SPLIT];
#pragma unroll
      for (int r = 0; r < SPLIT; ++r) v[r] = ld_cluster_v4(cluster_map_shared(own, r));
      float x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int r = 0; r < SPLIT; ++r) x[0] += v[r].x, x[1] += v[r].y, x[2] += v[r].z, x[3] += v[r].w;
      const bool refused = adaptor_refused(p.which, p.S, t);
      __align__(8) __nv_bfloat16 y[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) y[q] = __float2bfloat16_rn(refused ? CUDART_NAN_F : x[q]);
      const int n = tile * kBlockM + 4 * lane;
      __nv_bfloat16* dst = p.out + t * p.out_stride + n;
      if (p.store4 && n + 4 <= p.N) {
        *reinterpret_cast<uint2*>(dst) = *reinterpret_cast<const uint2*>(y);
      } else {
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (n + q < p.N) dst[q] = y[q];
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) drain_after_abort<1>(ctl, true);
  __syncthreads();
  cluster_sync_all();                                                // nobody reads this CTA's sums any more
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, tmem_cols);
  }
}

// ---- gradients of the adaptors
// dA (product 0: rows g, terms of low) and dB (product 1: rows x', terms of v): 128 columns of the rows are the MMA's M, the 3 k16 terms its N, rows its K. An item is
// one tile of columns of one adaptor over one of `splits` runs of row blocks; every eight blocks the accumulators are added to fp32 registers. Bound by the rows' bytes:
// 8192 rows, 4096 + 4096 columns, k = 16: 26 us for 136 MB.
struct GradParams {
  CUtensorMap tm_rows[2];                        // [T, cols]    box 64 x 64
  CUtensorMap tm_terms[2];                       // [T, 3 k16]   box 64 x 64
  const int* which;
  const uint32_t *present, *whole;               // LowParams
  float* out[2];                                 // dA [S, m, k], dB [S, k, d]; either may be NULL
  float* part;                                   // [splits][S][columns of both, whole tiles][k16], splits > 1
  unsigned* status;
  uint64_t wait_limit_ns;
  int T, S, k, cols[2], tiles[2];                // tiles of an absent product: 0
  int blocks, splits, stages, stage_bytes;
  int after_low, wide_a;                         // wide_a: rows of dA are vectors of eight
};
constexpr int kGradThreads = 192;
constexpr int kGradWords = 1024;
// CTAs of an SM: two where both have stages enough (256 rows, k = 16, eight adaptors: all gradients 23.1 -> 21.2 us; 2005 rows, k = 64: 52 with one, 64 with two).
__host__ __device__ constexpr int grad_ctas(int k16) { return k16 <= 32 ? 2 : 1; }

struct GradItem {
  int product, tile, adaptor, split;
};
__device__ __forceinline__ GradItem grad_item(const GradParams& p, int item) {
  const int tiles = p.tiles[0] + p.tiles[1];
  GradItem g;
  int rest = item / tiles;
  g.tile = item - rest * tiles;
  g.product = g.tile >= p.tiles[0] ? 1 : 0;
  if (g.product) g.tile -= p.tiles[0];
  g.adaptor = rest / p.splits;
  g.split = rest - g.adaptor * p.splits;
  return g;
}
// The row blocks of an item that have rows of its adaptor, in order; a warp walks over them as a whole.
struct BlockWalk {
  const uint32_t *present, *whole;      // in shared memory, where they are few
  int block, end;
  uint32_t word, alone;
  __device__ __forceinline__ BlockWalk(const uint32_t* present_, const uint32_t* whole_) : present(present_), whole(whole_) {}
  __device__ __forceinline__ void look(const GradParams& p, const GradItem& g, int b) {
    const size_t at = static_cast<size_t>(b >> 5) * p.S + g.adaptor;
    word = present[at];
    alone = whole[at];
  }
  __device__ __forceinline__ void start(const GradParams& p, const GradItem& g) {
    block = static_cast<int>(static_cast<long long>(g.split) * p.blocks / p.splits) - 1;
    end = static_cast<int>(static_cast<long long>(g.split + 1) * p.blocks / p.splits);
    word = alone = 0;
    if (block + 1 < end) look(p, g, block + 1);
  }
  __device__ __forceinline__ bool next(const GradParams& p, const GradItem& g) {
    while (true) {
      if (++block >= end) return false;
      if ((block & 31) == 0) look(p, g, block);
      const uint32_t ahead = word >> (block & 31);
      if (ahead != 0) {
        block += __ffs(ahead) - 1;
        return block < end;
      }
      block |= 31;
    }
  }
  // Whether all rows of the block are the adaptor's.
  __device__ __forceinline__ bool all() const { return alone >> (block & 31) & 1; }
};

template <int K16>
__global__ void __launch_bounds__(kGradThreads, grad_ctas(K16)) adaptor_grad_kernel(const __grid_constant__ GradParams p) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw_addr = smem_u32(smem_raw);
  const uint32_t tiles_addr = (raw_addr + 1023u) & ~1023u;
  GemmControl* ctl = reinterpret_cast<GemmControl*>(smem_raw + (tiles_addr - raw_addr) + static_cast<size_t>(p.stages) * p.stage_bytes);
  const int warp = static_cast<int>(warp_uniform(threadIdx.x >> 5));
  const int lane = threadIdx.x & 31;
  const int items = (p.tiles[0] + p.tiles[1]) * p.S * p.splits;
  constexpr int kTermBoxes = (3 * K16 + 63) / 64;
  constexpr uint32_t kSlots = 2, kSlotCols = K16 == 16 ? 64 : K16 == 32 ? 128 : 256, kCols = kSlots * kSlotCols;
  if (threadIdx.x == 0) {
    for (int s = 0; s < p.stages; ++s) {
      mbar_init(smem_u32(&ctl->full[s]), 1);
      mbar_init(smem_u32(&ctl->empty[s]), 1);
    }
    for (uint32_t s = 0; s < kSlots; ++s) {
      mbar_init(smem_u32(&ctl->tfull[s]), 1);
      mbar_init(smem_u32(&ctl->tempty[s]), 4);
    }
    mbar_init(smem_u32(&ctl->drain), 1);
    ctl->abort = 0;
    ctl->wait_limit_ns = p.wait_limit_ns;
    fence_mbar_init();
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(&ctl->tmem_base), kCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = warp_uniform(ctl->tmem_base);
  // The kernel ahead is the product, a gate: what adaptor_low_kernel wrote is there, and nothing here needs the product. Or (after_low) that kernel itself.
  if (p.after_low) grid_dependency_wait();
  grid_launch_dependents();
  const uint32_t *present = p.present, *whole_blocks = p.whole;
  const int words = ((p.blocks + 31) >> 5) * p.S;
  if (words <= kGradWords) {            // every role looks them up for every item
    uint32_t* near = reinterpret_cast<uint32_t*>(ctl + 1);
    for (int i = threadIdx.x; i < words; i += kGradThreads) {
      near[i] = p.present[i];
      near[kGradWords + i] = p.whole[i];
    }
    __syncthreads();
    present = near;
    whole_blocks = near + kGradWords;
  }
  const uint32_t full0 = smem_u32(&ctl->full[0]), empty0 = smem_u32(&ctl->empty[0]);

  if (warp == 0) {
    const uint32_t lead = elect_one();
    uint32_t stage = 0, phase = 0, issued = 0;
    bool ok = true;
    for (int item = blockIdx.x; item < items && ok; item += gridDim.x) {
      const GradItem g = grad_item(p, item);
      const CUtensorMap *rows = &p.tm_rows[g.product], *terms = &p.tm_terms[g.product];
      BlockWalk walk(present, whole_blocks);
      walk.start(p, g);
      while (walk.next(p, g)) {
        const int t0 = walk.block * 64;
        if (!bounded_wait_all(empty0 + 8 * stage, phase ^ 1u, ctl, p)) { ok = false; break; }
        const uint32_t full = full0 + 8 * stage, dst = tiles_addr + stage * p.stage_bytes;
        mbar_arrive_expect_tx(lead, full, kABytes + kTermBoxes * kMnBoxBytes);
#pragma unroll
        for (int q = 0; q < 2; ++q) tma_load_2d(lead, dst + q * kMnBoxBytes, rows, full, g.tile * kBlockM + q * 64, t0);
#pragma unroll
        for (int q = 0; q < kTermBoxes; ++q) tma_load_2d(lead, dst + kABytes + q * kMnBoxBytes, terms, full, q * 64, t0);
        ++issued;
        if (++stage == static_cast<uint32_t>(p.stages)) { stage = 0; phase ^= 1u; }
      }
    }
    for (uint32_t s = 0; s < static_cast<uint32_t>(p.stages) && s < issued; ++s) drain_wait(full0 + 8 * s, ((issued - 1 - s) / p.stages) & 1u);
    __syncwarp();
  } else if (warp == 1) {
    const uint32_t lead = elect_one();
    const uint32_t idesc = umma_idesc_bf16(kBlockM, 3 * K16, true, true);
    const uint64_t a_desc0 = umma_smem_desc_mn_sw128(tiles_addr, kMnBoxBytes), b_desc0 = umma_smem_desc_mn_sw128(tiles_addr + kABytes, kMnBoxBytes);
    const uint32_t stage_step = p.stage_bytes >> 4;
    uint32_t stage = 0, phase = 0, use = 0;
    bool ok = true;
    for (int item = blockIdx.x; item < items && ok; item += gridDim.x) {
      const GradItem g = grad_item(p, item);
      BlockWalk walk(present, whole_blocks);
      walk.start(p, g);
      int n = 0;                                                     // blocks in the open accumulator
      uint32_t slot = 0;
      while (walk.next(p, g)) {
        if (n == 0) {
          slot = use % kSlots;
          if (!bounded_wait_all(smem_u32(&ctl->tempty[slot]), ((use / kSlots) & 1u) ^ 1u, ctl, p)) { ok = false; break; }
          if (use == 0 && !first_wait(full0, ctl, p)) { ok = false; break; }
          ++use;
        }
        const bool whole = walk.all();
        bool foreign[2] = {false, false};                            // rows lane and lane + 32 of the block
        if (!whole) {
#pragma unroll
          for (int q = 0; q < 2; ++q) foreign[q] = adaptor_of(p.which, p.S, walk.block * 64 + 32 * q + lane, p.T) != g.adaptor;
        }
        if (!bounded_wait_all(full0 + 8 * stage, phase, ctl, p)) { ok = false; break; }
        if (!whole) {
          // rows of other adaptors, which may hold anything, become zeros in both operands where they landed: a row is 128 bytes of every box
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            if (!foreign[q]) continue;
            const uint32_t row = tiles_addr + stage * p.stage_bytes + (32 * q + lane) * 128;
#pragma unroll
            for (int c = 0; c < 8; ++c)                              // neighbours start at other banks
#pragma unroll
              for (int box = 0; box < 2 + kTermBoxes; ++box) st_shared_v4(row + box * kMnBoxBytes + ((c + lane) & 7) * 16, 0, 0, 0, 0);
          }
          fence_proxy_async_shared();
          __syncwarp();
        }
        tc_fence_after();
        const uint64_t a_desc = a_desc0 + stage * stage_step, b_desc = b_desc0 + stage * stage_step;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
          umma_bf16(lead, tmem_base + slot * kSlotCols, a_desc + 128 * kk, b_desc + 128 * kk, idesc, (n | kk) != 0 ? 1u : 0u);
        umma_commit(lead, empty0 + 8 * stage);
        if (++stage == static_cast<uint32_t>(p.stages)) { stage = 0; phase ^= 1u; }
        if (++n == kChunkBlocks) {
          umma_commit(lead, smem_u32(&ctl->tfull[slot]));
          n = 0;
        }
      }
      if (ok && n > 0) umma_commit(lead, smem_u32(&ctl->tfull[slot]));
    }
    __syncwarp();
  } else {
    const int quarter = warp & 3;
    const uint32_t lane_base = tmem_base + (static_cast<uint32_t>(quarter * 32) << 16);
    uint32_t use = 0;
    bool ok = true;
    for (int item = blockIdx.x; item < items && ok; item += gridDim.x) {
      const GradItem g = grad_item(p, item);
      BlockWalk walk(present, whole_blocks);
      walk.start(p, g);
      float acc[K16];
#pragma unroll
      for (int j = 0; j < K16; ++j) acc[j] = 0.f;
      int n = 0;
      bool more = walk.next(p, g);
      while (more) {
        more = walk.next(p, g);
        if (++n < kChunkBlocks && more) continue;
        n = 0;
        const uint32_t slot = use % kSlots;
        if (!bounded_wait_warp(smem_u32(&ctl->tfull[slot]), (use / kSlots) & 1u, ctl, p.status, lane)) { ok = false; break; }
        ++use;
        tc_fence_after();
#pragma unroll
        for (int b = 0; b < K16 / 16; ++b) {
          float hi[16], mid[16], lo[16];
          tmem_ld16(lane_base + slot * kSlotCols + b * 16, hi);
          tmem_ld16(lane_base + slot * kSlotCols + K16 + b * 16, mid);
          tmem_ld16(lane_base + slot * kSlotCols + 2 * K16 + b * 16, lo);
#pragma unroll
          for (int q = 0; q < 16; ++q) acc[b * 16 + q] += hi[q] + (mid[q] + lo[q]);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&ctl->tempty[slot]));
      }
      if (!ok) break;
      const int col = g.tile * kBlockM + quarter * 32 + lane, cols = p.cols[g.product];
      if (p.splits > 1) {
        const size_t all = static_cast<size_t>(p.tiles[0] + p.tiles[1]) * kBlockM;
        float* dst = p.part + ((static_cast<size_t>(g.split) * p.S + g.adaptor) * all + (g.product ? p.tiles[0] * kBlockM : 0) + col) * K16;
#pragma unroll
        for (int j = 0; j < K16; j += 8) st_global_v8(dst + j, acc + j);
      } else if (col < cols && g.product == 0 && p.wide_a) {
        float* dst = p.out[0] + (static_cast<size_t>(g.adaptor) * cols + col) * p.k;
#pragma unroll
        for (int j = 0; j < K16; j += 8)
          if (j < p.k) st_global_v8(dst + j, acc + j);
      } else if (col < cols) {
#pragma unroll
        for (int j = 0; j < K16; ++j) {
          if (j >= p.k) break;
          if (g.product) p.out[1][(static_cast<size_t>(g.adaptor) * p.k + j) * cols + col] = acc[j];
          else p.out[0][(static_cast<size_t>(g.adaptor) * cols + col) * p.k + j] = acc[j];
        }
      }
    }
  }
  grid_dependency_wait();               // so that the end of this grid is that of all before it
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    drain_after_abort<1>(ctl, true);
    tc_fence_after();
    tmem_dealloc(tmem_base, kCols);
  }
}

// Adds the splits' parts up, in order: a thread has one column's rank values four at a time. (Four runs of 64 tiles of 128 columns, k = 16: 6 us, a launch's latency.)
__global__ void __launch_bounds__(256) adaptor_grad_join_kernel(const __grid_constant__ GradParams p, int k16) {
  grid_dependency_wait();
  grid_launch_dependents();
  const size_t all = static_cast<size_t>(p.tiles[0] + p.tiles[1]) * kBlockM;
  const int quads = k16 / 4;
  // columns fastest across a warp's eight, so that both layouts are written in runs
  const size_t at = static_cast<size_t>(blockIdx.x) * 256 + threadIdx.x;
  const size_t total = static_cast<size_t>(p.S) * all * quads;
  if (at >= total) return;
  const int j0 = static_cast<int>(at % quads) * 4;
  const size_t row = at / quads;
  const int i = static_cast<int>(row / all);
  int col = static_cast<int>(row - static_cast<size_t>(i) * all);
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
  for (int q = 0; q < p.splits; ++q) {
    const float4 x = *reinterpret_cast<const float4*>(p.part + (static_cast<size_t>(q) * p.S * all + row) * k16 + j0);
    s.x += x.x, s.y += x.y, s.z += x.z, s.w += x.w;
  }
  const float y[4] = {s.x, s.y, s.z, s.w};
  const int product = col >= p.tiles[0] * kBlockM ? 1 : 0;
  if (product) col -= p.tiles[0] * kBlockM;
  if (col >= p.cols[product]) return;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (j0 + e >= p.k) break;
    if (product) p.out[1][(static_cast<size_t>(i) * p.k + j0 + e) * p.cols[1] + col] = y[e];
    else p.out[0][(static_cast<size_t>(i) * p.cols[0] + col) * p.k + j0 + e] = y[e];
  }
}

// ---- rows that the tensor maps cannot address (an address or pitch that is no multiple of 16 bytes), copied to ones that they can (2005 and 2003 rows of 1001: 7 us)
struct CopyRows {
  const __nv_bfloat16* src;
  __nv_bfloat16* dst;
  int64_t stride, rows;
  int cols, pitch;                      // pitch: cols rounded up to eight
};
struct CopyParams {
  CopyRows m[4];
  int64_t begin[5];                     // in vectors of eight elements
};
__global__ void __launch_bounds__(256) copy_rows_kernel(const CopyParams p) {
  grid_dependency_wait();
  grid_launch_dependents();
  const int64_t at = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (at >= p.begin[4]) return;
  int q = 0;
#pragma unroll
  for (int i = 1; i < 4; ++i)
    if (at >= p.begin[i]) q = i;
  const CopyRows& m = p.m[q];
  const int64_t v = at - p.begin[q];
  const int per = m.pitch / 8;
  const int64_t row = v / per;
  const int col = static_cast<int>(v - row * per) * 8;
  const __nv_bfloat16* src = m.src + row * m.stride + col;
  __align__(16) __nv_bfloat16 x[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = col + e < m.cols ? src[e] : __float2bfloat16_rn(0.f);
  *reinterpret_cast<uint4*>(m.dst + row * m.pitch + col) = *reinterpret_cast<const uint4*>(x);
}

}  // namespace mtpc
