// Losses of log-likelihoods in packed sequences, and their gradients.
//
// Policy: per valid position t of sequence s, ratio r = exp(logp - old), advantage a of the sequence:
//   value = -min(r a, clip(r, 1 - low, 1 + high) a) + beta (e^q - 1 - q),   q = ref - logp
//   slope = -(r a, or 0 where the clipped one is smaller) + beta (1 - e^q)
// weighted by 1 / (all valid positions), or by 1 / (S * the sequence's valid positions).
// Preference: sequences 2p and 2p + 1, h = beta (sum of logp - ref over the one's valid positions - over the other's),
//   loss = mean of -(1 - s) log sigmoid(h) - s log sigmoid(-h),   slope = +- beta (s - sigmoid(-h)) / pairs.
//
// Differences of log-likelihoods lose nothing: the policy loss takes them as two fp32 terms, the nearest value and what it leaves, and e^(d + rest) as e^d (1 + rest); the sums of pairs
// take them in fp64. Whether a ratio is clipped is decided on both terms, against the logarithms of the ends in two terms as well, since a position beside an end would else
// change sides by a rounding. What a position comes to (ratios, products, slopes) is fp32; sums are fp64, in an order that sizes fix.
//
// Work is dealt in items: a warp has one of P equal slices of one sequence, so that no position has to look for its sequence. P is the same for all sequences, 4736 / S at most
// (the warps that the device holds), so lengths that differ leave warps idle: 1.6 million positions in 256 sequences alike 15 us (masked, policy), with all but 255 x 128 of them
// in one sequence, which 18 warps then have, 760. Weights need the counts of valid positions first, so the call goes over the data twice (the mask alone
// for the counts, every warp over that of its own sequence where that is all it needs; logp and ref for the sums of pairs). Few positions: all phases in one launch of one cluster, with its barrier between
// them (a chain of four kernels of 2 us each otherwise); many: a launch for each phase. Bound by launches and their chains of loads: 1.6 million masked positions 16.0 us (policy; with differences and
// sums of four in fp32 alone 14.5) and 12.0 (preference), of which the bytes are 4 and 3; a few hundred positions 8, mostly the host's.
#pragma once
#include <math_constants.h>
#include <stdint.h>

#include "mtpc_ptx.cuh"

namespace mtpc {

constexpr uint32_t kStatusBadOffset = 16u;
constexpr int kObjectiveThreads = 512, kObjectiveWarps = kObjectiveThreads / 32;
constexpr int kObjectiveCtas = 8;                  // of the cluster that does a small call alone
constexpr int kSmallItems = 1024;                  // that such a call has at most
constexpr int kMostBlocks = 148 * 2;               // of a launch for one phase: what the device holds at once

struct ObjectiveArgs {
  const float *logp, *old, *ref, *advantage;       // ref: NULL without the KL term; advantage [S], or [T] with an advantage for every position (policy)
  const uint8_t* mask;                             // [T] or NULL
  const int* offsets;                              // [S + 1]
  int T, S, parts;                                 // parts: slices of a sequence
  int by_sequence;
  int own_count;                                   // every warp counts the valid positions of its sequence itself
  float log_low[2], log_high[2];                   // logarithms of the ends, in two terms
  float low, high;                                 // the ends: 1 - clip_low, 1 + clip_high
  double beta, smoothing;
  float *loss, *stats, *d_logp, *h;                // stats [3] or NULL; h [S / 2] or NULL
  uint32_t* status;
  // workspace
  int* count;                                      // [S * parts] valid positions of every slice
  long long* block_count;                          // [kMostBlocks] of all slices of a block
  double* sum;                                     // [kMostBlocks][3] of all slices of a block (policy), or [S * parts] (preference)
  double* term;                                    // [S / 2] a pair's loss
  float* slope;                                    // [S / 2]
};

// Where sequence s lies; offsets that decrease or leave [0, T] are brought into it and refused at the end.
struct Span {
  int begin, end;
  bool refused;
};
__device__ __forceinline__ Span span_of(const ObjectiveArgs& a, int s) {
  const int lo = a.offsets[s], hi = a.offsets[s + 1];
  Span x;
  x.refused = lo < 0 || hi < lo || hi > a.T;
  x.begin = min(max(lo, 0), a.T);
  x.end = max(x.begin, min(max(hi, 0), a.T));
  return x;
}
// The sequences that a warp takes, in order: none begins before the end of the one ahead, whatever the offsets say. (Refused ones may name all positions for every
// sequence, S T of them together; so a warp has T at most.)
struct Taken {
  int s, from, end;                                // the last sequence, where it may begin, where it ends
  __device__ __forceinline__ Taken() : s(-1), from(0), end(0) {}
  __device__ __forceinline__ Span span(const ObjectiveArgs& a, int next) {
    Span x = span_of(a, next);
    if (next != s) from = max(from, end), s = next;
    x.begin = max(x.begin, from);
    x.end = max(x.end, x.begin);
    end = x.end;
    return x;
  }
};
// Item `item`: slice `item % parts` of sequence `item / parts`, cut at multiples of four positions (equal steps: a 64-bit division for either end was a third of a warp's
// instructions).
struct Slice {
  int s, begin, end;
  Span of;                                         // its sequence
};
__device__ __forceinline__ Slice slice_of(const ObjectiveArgs& a, int item, Taken& taken) {
  Slice c;
  c.s = item / a.parts;
  const int part = item - c.s * a.parts;
  const Span x = c.of = taken.span(a, c.s);
  const int base = x.begin & ~3, step = ((x.end - base + a.parts - 1) / a.parts + 3) & ~3;       // (parts * step: below 2^30 + 8 * 4736)
  c.begin = min(x.end, max(x.begin, base + part * step));
  c.end = min(x.end, base + (part + 1) * step);
  c.end = max(c.begin, c.end);
  return c;
}

template <typename F>
__device__ __forceinline__ F warp_total(F x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}

// body(first position, four flags) for every group of four positions that a warp's lanes have of [begin, end): the flags say which are inside and valid.
template <bool WIDE, typename Body>
__device__ __forceinline__ void over_slice(const ObjectiveArgs& a, const Slice& c, int lane, Body body) {
  for (int q = (c.begin >> 2) + lane; q * 4ll < c.end; q += 32) {
    const int t = q * 4;
    uint32_t valid = 0;
    const bool inside = t >= c.begin && t + 4 <= c.end;
    if (WIDE && inside && a.mask != nullptr) {
      const uint32_t m = *reinterpret_cast<const uint32_t*>(a.mask + t);
#pragma unroll
      for (int i = 0; i < 4; ++i) valid |= ((m >> (8 * i)) & 0xffu) ? 1u << i : 0u;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (t + i >= c.begin && t + i < c.end && (a.mask == nullptr || a.mask[t + i] != 0)) valid |= 1u << i;
    }
    body(t, valid, inside);
  }
}
template <bool WIDE>
__device__ __forceinline__ void load4(const float* p, int t, bool inside, uint32_t valid, float (&x)[4]) {
  if (WIDE && inside) {
    const float4 v = *reinterpret_cast<const float4*>(p + t);
    x[0] = v.x, x[1] = v.y, x[2] = v.z, x[3] = v.w;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = valid >> i & 1 ? p[t + i] : 0.f;
  }
}
template <bool WIDE>
__device__ __forceinline__ void store4(float* p, const Slice& c, int t, bool inside, const float (&x)[4]) {
  if (WIDE && inside) {
    *reinterpret_cast<float4*>(p + t) = make_float4(x[0], x[1], x[2], x[3]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (t + i >= c.begin && t + i < c.end) p[t + i] = x[i];
  }
}

// ---- phases, each over items first, first + step, ... of a warp
// N sums over the warps of a block, each warp's in its lane 0; thread 0 gets them. red: N * kObjectiveWarps values.
template <int N, typename F>
__device__ __forceinline__ void block_sum(F (&x)[N], F* red) {
  __syncthreads();
  if ((threadIdx.x & 31) == 0) {
#pragma unroll
    for (int k = 0; k < N; ++k) red[k * kObjectiveWarps + (threadIdx.x >> 5)] = x[k];
  }
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int k = 0; k < N; ++k) {
      x[k] = 0;
#pragma unroll
      for (int i = 0; i < kObjectiveWarps; ++i) x[k] += red[k * kObjectiveWarps + i];
    }
  }
}
// Bytes that are not zero of mask[begin, end): this one's of `lanes` threads.
__device__ __forceinline__ int count_mask(const uint8_t* mask, int begin, int end, int lane, int lanes) {
  int n = 0;
  auto word = [](uint32_t w) { return __popc((w | ((w & 0x7f7f7f7fu) + 0x7f7f7f7fu)) & 0x80808080u); };
  const uint8_t *from = mask + begin, *to = mask + end;
  const uint8_t* first = reinterpret_cast<const uint8_t*>((reinterpret_cast<uintptr_t>(from) + 15) & ~static_cast<uintptr_t>(15));
  const uint8_t* last = reinterpret_cast<const uint8_t*>(reinterpret_cast<uintptr_t>(to) & ~static_cast<uintptr_t>(15));
  if (first >= last) {
    for (const uint8_t* b = from + lane; b < to; b += lanes) n += *b != 0;
  } else {
    if (from + lane < first) n += from[lane] != 0;
#pragma unroll 4
    for (const uint8_t* b = first + 16 * lane; b < last; b += 16 * lanes) {
      const uint4 v = *reinterpret_cast<const uint4*>(b);
      n += word(v.x) + word(v.y) + word(v.z) + word(v.w);
    }
    if (last + lane < to) n += last[lane] != 0;
  }
  return n;
}
template <bool WIDE>
__device__ __forceinline__ void count_phase(const ObjectiveArgs& a, int block, int blocks, int lane, long long* red) {
  const int first = block * kObjectiveWarps + (threadIdx.x >> 5), step = blocks * kObjectiveWarps;
  long long all[1] = {0};
  Taken taken;
  for (int item = first; item < a.S * a.parts; item += step) {
    const Slice c = slice_of(a, item, taken);
    int n = 0;
    over_slice<WIDE>(a, c, lane, [&](int, uint32_t valid, bool) { n += __popc(valid); });
    n = warp_total(n);
    if (lane == 0) a.count[item] = n;
    all[0] += n;
  }
  block_sum(all, red);
  if (threadIdx.x == 0) a.block_count[block] = all[0];
}

// x - y in two terms: the nearest fp32 value, and what it leaves (exactly).
__device__ __forceinline__ float difference_rest(float x, float y, float d) {
  const float back = __fadd_rn(d, y);
  return __fsub_rn(__fsub_rn(x, back), __fsub_rn(y, __fsub_rn(back, d)));
}
// Whether an exponential of the difference takes the rest into account: up to where fp32 ends, so that no infinity is multiplied by it.
__device__ __forceinline__ bool rest_counts(float d) { return fabsf(d) < 88.f; }
// e^q - 1 - q, and e^q - 1, of four: near zero by the series, whose next term is below 2^-28 of the first; the function less q is off by q's rounding.
__device__ __forceinline__ void exp_beyond(const float (&q)[4], float (&beyond)[4], float (&m1)[4]) {
  bool far = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float s = 1.f / 362880.f;
    s = fmaf(s, q[i], 1.f / 40320.f);
    s = fmaf(s, q[i], 1.f / 5040.f);
    s = fmaf(s, q[i], 1.f / 720.f);
    s = fmaf(s, q[i], 1.f / 120.f);
    s = fmaf(s, q[i], 1.f / 24.f);
    s = fmaf(s, q[i], 1.f / 6.f);
    s = fmaf(s, q[i], 0.5f);
    beyond[i] = q[i] * q[i] * s;
    m1[i] = q[i] + beyond[i];
    far |= fabsf(q[i]) >= 0.5f;
  }
  if (far) {
#pragma unroll 1
    for (int i = 0; i < 4; ++i) {
      const float x = i < 2 ? (i == 0 ? q[0] : q[1]) : (i == 2 ? q[2] : q[3]);
      if (fabsf(x) < 0.5f) continue;
      const float y = expm1f(x);
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (k == i) m1[k] = y, beyond[k] = y < CUDART_INF_F ? y - x : y;       // (of infinity: itself)
    }
  }
}
// What an advantage's sign says about clipping: the end that counts (its logarithm in two terms) and the value beyond it.
struct ClipOf {
  float adv, sign, end, end_rest, held;
};
__device__ __forceinline__ ClipOf clip_of(const ObjectiveArgs& a, float adv) {
  const bool up = adv > 0.f;
  return ClipOf{adv, up ? 1.f : adv < 0.f ? -1.f : 0.f, up ? a.log_high[0] : a.log_low[0], up ? a.log_high[1] : a.log_low[1], (up ? a.high : a.low) * adv};
}
// (logp - old) - the end's logarithm, where roundings would decide: both in two terms.
__device__ __forceinline__ float beyond_end(float d, float rest, const ClipOf& side) { return __fadd_rn(__fsub_rn(d, side.end), __fsub_rn(rest, side.end_rest)); }

// A slice's values on their way into L2 while its weight is formed, a line of 32 to a lane.
__device__ __forceinline__ void prefetch_slice(const ObjectiveArgs& a, const Slice& c, int lane) {
  for (int t = (c.begin & ~31) + 32 * lane; t < c.end; t += 32 * 32) {
    const int at = max(t, c.begin);
    prefetch_l2(a.logp + at);
    prefetch_l2(a.old + at);
    if (a.ref != nullptr) prefetch_l2(a.ref + at);
  }
}
// total: all valid positions. EACH: an advantage for every position.
template <bool WIDE, bool EACH>
__device__ __forceinline__ void policy_phase(const ObjectiveArgs& a, int block, int blocks, int lane, long long total, double* red) {
  const int items = a.S * a.parts;
  double all[3] = {0.0, 0.0, 0.0};
  Taken taken;
  for (int base = block * kObjectiveWarps; base < items; base += blocks * kObjectiveWarps) {
    const int item = base + (threadIdx.x >> 5);
    const Slice c = slice_of(a, min(item, items - 1), taken);
    int own = 0;
    const bool together = a.own_count && a.parts >= kObjectiveWarps / 2;       // the block's warps share two or three sequences: counted by all of them
    if (together) {
      __shared__ int counted[4];
      if (threadIdx.x < 4) counted[threadIdx.x] = 0;
      if (item < items) prefetch_slice(a, c, lane);
      __syncthreads();
      const int s0 = base / a.parts, s1 = (min(base + kObjectiveWarps, items) - 1) / a.parts;
      for (int s = s0; s <= s1; ++s) {
        const Span x = span_of(a, s);
        const int n = warp_total(count_mask(a.mask, x.begin, x.end, threadIdx.x, kObjectiveThreads));
        if (lane == 0 && n) atomicAdd(&counted[s - s0], n);
      }
      __syncthreads();
      if (item < items) own = counted[c.s - s0];
      __syncthreads();
    }
    if (item >= items) continue;
    long long n = total;
    if (a.by_sequence) {
      int here = c.of.end - c.of.begin;
      if (together) {
        here = own;
      } else if (a.own_count) {
        prefetch_slice(a, c, lane);
        here = warp_total(count_mask(a.mask, c.of.begin, c.of.end, lane, 32));
      } else if (a.mask != nullptr) {
        here = 0;
        for (int q = lane; q < a.parts; q += 32) here += a.count[c.s * a.parts + q];
        here = warp_total(here);
      }
      n = static_cast<long long>(here) * a.S;
    }
    const double weight = n > 0 ? 1.0 / static_cast<double>(n) : 0.0;
    const float w = static_cast<float>(weight), beta = static_cast<float>(a.beta);
    const ClipOf one = clip_of(a, EACH ? 0.f : a.advantage[c.s]);
    double value = 0.0, kl = 0.0;
    int clipped = 0;
    over_slice<WIDE>(a, c, lane, [&](int t, uint32_t valid, bool inside) {
      float lp[4], old[4], ref[4], adv[4], g[4];
      load4<WIDE>(a.logp, t, inside, valid, lp);
      load4<WIDE>(a.old, t, inside, valid, old);
      if (a.ref != nullptr) load4<WIDE>(a.ref, t, inside, valid, ref);
      if (EACH) load4<WIDE>(a.advantage, t, inside, valid, adv);
      float diff[4], rest[4], over[4], beyond[4] = {0.f, 0.f, 0.f, 0.f}, m1[4] = {0.f, 0.f, 0.f, 0.f};
      bool near = false;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const ClipOf side = EACH ? clip_of(a, adv[i]) : one;
        diff[i] = __fsub_rn(lp[i], old[i]);
        rest[i] = difference_rest(lp[i], old[i], diff[i]);
        over[i] = diff[i] - side.end;
        near |= fabsf(over[i]) < fmaf(fabsf(diff[i]), 1e-6f, 1e-6f);                  // (both roundings are below 2^-23 of diff and end)
      }
      if (near) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (fabsf(over[i]) < fmaf(fabsf(diff[i]), 1e-6f, 1e-6f)) over[i] = beyond_end(diff[i], rest[i], EACH ? clip_of(a, adv[i]) : one);
      }
      if (a.ref != nullptr) {
        const float q[4] = {__fsub_rn(ref[0], lp[0]), __fsub_rn(ref[1], lp[1]), __fsub_rn(ref[2], lp[2]), __fsub_rn(ref[3], lp[3])};
        exp_beyond(q, beyond, m1);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float more = difference_rest(ref[i], lp[i], q[i]);
          if (!rest_counts(q[i])) continue;
          beyond[i] = fmaf(more, m1[i], beyond[i]);
          m1[i] = fmaf(more, 1.f + m1[i], m1[i]);
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const ClipOf side = EACH ? clip_of(a, adv[i]) : one;
        const bool out = side.sign * over[i] > 0.f, counts = valid >> i & 1;
        const float ratio = expf(diff[i]);
        float gain = (rest_counts(diff[i]) ? fmaf(ratio, rest[i], ratio) : ratio) * side.adv;
        if (out) gain = side.held;
        if (side.adv == 0.f) gain = 0.f;
        float slope = out ? 0.f : -gain;
        if (a.ref != nullptr) slope = fmaf(-beta, m1[i], slope);
        g[i] = counts ? w * slope : 0.f;
        value -= static_cast<double>(counts ? gain : 0.f);
        kl += static_cast<double>(counts ? beyond[i] : 0.f);
        clipped += counts && out ? 1 : 0;
      }
      store4<WIDE>(a.d_logp, c, t, inside, g);
    });
    value = warp_total(value);
    kl = warp_total(kl);
    clipped = warp_total(clipped);
    all[0] += value * weight;
    all[1] += kl * weight;
    all[2] += clipped * weight;
  }
  block_sum(all, red);
  if (threadIdx.x == 0) {
#pragma unroll
    for (int i = 0; i < 3; ++i) a.sum[3 * block + i] = all[i];
  }
}

// N sums of n values each that the threads of a block have in turn, in an order that n fixes; every thread gets them. red: N * kObjectiveWarps values.
template <int N, typename F, typename Get>
__device__ __forceinline__ void block_totals(int n, F (&x)[N], F* red, Get get) {
#pragma unroll
  for (int k = 0; k < N; ++k) x[k] = 0;
#pragma unroll 4
  for (int i = threadIdx.x; i < n; i += kObjectiveThreads) get(i, x);
#pragma unroll
  for (int k = 0; k < N; ++k) x[k] = warp_total(x[k]);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) {
#pragma unroll
    for (int k = 0; k < N; ++k) red[k * kObjectiveWarps + (threadIdx.x >> 5)] = x[k];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < N; ++k) {
    x[k] = 0;
#pragma unroll
    for (int i = 0; i < kObjectiveWarps; ++i) x[k] += red[k * kObjectiveWarps + i];
  }
}
// All valid positions (whole numbers: any order gives the same).
__device__ __forceinline__ long long all_valid(const ObjectiveArgs& a, int blocks, long long* red) {
  long long n[1];
  if (a.mask != nullptr) {
    block_totals<1>(blocks, n, red, [&](int i, long long (&x)[1]) { x[0] += a.block_count[i]; });
  } else {
    block_totals<1>(a.S, n, red, [&](int s, long long (&x)[1]) {
      const Span c = span_of(a, s);
      x[0] += c.end - c.begin;
    });
  }
  return n[0];
}
// Whether offsets were refused: the loss has no value then.
__device__ __forceinline__ bool any_refused(const ObjectiveArgs& a, long long* red) {
  long long n[1];
  block_totals<1>(a.S, n, red, [&](int s, long long (&x)[1]) { x[0] += span_of(a, s).refused ? 1 : 0; });
  if (n[0] > 0 && threadIdx.x == 0 && a.status != nullptr) atomicOr(a.status, kStatusBadOffset);
  return n[0] > 0;
}
__device__ __forceinline__ void policy_final(const ObjectiveArgs& a, int blocks, double* red) {
  const bool refused = any_refused(a, reinterpret_cast<long long*>(red));
  double s[3];
  block_totals<3>(blocks, s, red, [&](int block, double (&x)[3]) {
#pragma unroll
    for (int i = 0; i < 3; ++i) x[i] += a.sum[3 * block + i];
  });
  if (threadIdx.x == 0) {
    a.loss[0] = refused ? CUDART_NAN_F : static_cast<float>(s[0] + a.beta * s[1]);
    if (a.stats != nullptr)
      for (int i = 0; i < 3; ++i) a.stats[i] = refused ? CUDART_NAN_F : static_cast<float>(s[i]);
  }
}

template <bool WIDE>
__device__ __forceinline__ void ratio_phase(const ObjectiveArgs& a, int first, int step, int lane) {
  Taken taken;
  for (int item = first; item < a.S * a.parts; item += step) {
    const Slice c = slice_of(a, item, taken);
    double sum = 0.0;
    over_slice<WIDE>(a, c, lane, [&](int t, uint32_t valid, bool inside) {
      float lp[4], ref[4];
      load4<WIDE>(a.logp, t, inside, valid, lp);
      load4<WIDE>(a.ref, t, inside, valid, ref);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (valid >> i & 1) sum += static_cast<double>(lp[i]) - static_cast<double>(ref[i]);
    });
    sum = warp_total(sum);
    if (lane == 0) a.sum[item] = sum;
  }
}
// A factor of zero takes its term away, also where that has no bound (a window without probability).
__device__ __forceinline__ double of_share(double share, double x) { return share > 0.0 ? share * x : 0.0; }
// h of pair p, by a warp: the difference of its sequences' sums.
__device__ __forceinline__ double pair_h(const ObjectiveArgs& a, int p, int lane) {
  double h = 0.0;
  for (int q = lane; q < 2 * a.parts; q += 32) {
    const double x = a.sum[static_cast<size_t>(2 * p) * a.parts + q];
    h += q < a.parts ? x : -x;
  }
  return of_share(a.beta, warp_total(h));
}
// The pair's loss and the slope of its first sequence. e = exp(-|h|): log sigmoid(h) = min(h, 0) - log(1 + e).
__device__ __forceinline__ double pair_loss(const ObjectiveArgs& a, double h) {
  return log1p(exp(-fabs(h))) + of_share(1.0 - a.smoothing, fmax(-h, 0.0)) + of_share(a.smoothing, fmax(h, 0.0));
}
__device__ __forceinline__ float pair_slope(const ObjectiveArgs& a, double h) {
  const double e = exp(-fabs(h)), low = e / (1.0 + e), of_other = h > 0.0 ? low : 1.0 - low;      // sigmoid(-h)
  return static_cast<float>(a.beta * (a.smoothing - of_other) / (a.S / 2));
}
// Pairs first, first + step, ... of a warp: h, slope and loss.
__device__ __forceinline__ void pairs_phase(const ObjectiveArgs& a, int first, int step, int lane) {
  for (int p = first; p < a.S / 2; p += step) {
    const double h = pair_h(a, p, lane);
    if (lane == 0) {
      a.term[p] = pair_loss(a, h);
      a.slope[p] = pair_slope(a, h);
      if (a.h != nullptr) a.h[p] = static_cast<float>(h);
    }
  }
}
// All pairs by one block: their sums a warp to a pair, four at once, then a thread to each pair's loss (one after the other by its warp, 128 pairs took 10 us).
__device__ __forceinline__ void all_pairs(const ObjectiveArgs& a) {
  const int pairs = a.S / 2, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int base = warp * 4; base < pairs; base += 4 * kObjectiveWarps) {
    double h[4] = {0.0, 0.0, 0.0, 0.0};
    for (int q = lane; q < 2 * a.parts; q += 32) {
      const double sign = q < a.parts ? 1.0 : -1.0;
#pragma unroll
      for (int i = 0; i < 4; ++i) h[i] += sign * a.sum[static_cast<size_t>(2 * min(base + i, pairs - 1)) * a.parts + q];
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
      for (int i = 0; i < 4; ++i) h[i] += __shfl_xor_sync(0xffffffffu, h[i], o);
    if (lane < 4 && base + lane < pairs) a.term[base + lane] = of_share(a.beta, lane == 0 ? h[0] : lane == 1 ? h[1] : lane == 2 ? h[2] : h[3]);
  }
  __syncthreads();
  for (int p = threadIdx.x; p < pairs; p += kObjectiveThreads) {
    const double h = a.term[p];
    a.term[p] = pair_loss(a, h);
    if (a.h != nullptr) a.h[p] = static_cast<float>(h);
  }
  __syncthreads();
}
__device__ __forceinline__ void preference_final(const ObjectiveArgs& a, double* red) {
  const bool refused = any_refused(a, reinterpret_cast<long long*>(red));
  double s[1];
  block_totals<1>(a.S / 2, s, red, [&](int p, double (&x)[1]) { x[0] += a.term[p]; });
  if (threadIdx.x == 0) a.loss[0] = refused ? CUDART_NAN_F : static_cast<float>(s[0] / (a.S / 2));
}
// own: every warp forms its pair's slope itself.
template <bool WIDE>
__device__ __forceinline__ void spread_phase(const ObjectiveArgs& a, int first, int step, int lane, bool own) {
  Taken taken;
  for (int item = first; item < a.S * a.parts; item += step) {
    const Slice c = slice_of(a, item, taken);
    float slope = own ? pair_slope(a, pair_h(a, c.s >> 1, lane)) : a.slope[c.s >> 1];
    if (c.s & 1) slope = -slope;
    over_slice<WIDE>(a, c, lane, [&](int t, uint32_t valid, bool inside) {
      float g[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) g[i] = valid >> i & 1 ? slope : 0.f;
      store4<WIDE>(a.d_logp, c, t, inside, g);
    });
  }
}

// ---- one cluster does the whole call; what its CTAs hand each other lies in the first one's shared memory
struct ObjectiveShared {
  double sum[kSmallItems], term[kSmallItems / 2];
  long long block_count[kObjectiveCtas];
  int count[kSmallItems];
  float slope[kSmallItems / 2];
};
__device__ __forceinline__ void use_first_cta(ObjectiveArgs& a, ObjectiveShared* own) {
  uint64_t at;
  asm("mapa.u64 %0, %1, 0;" : "=l"(at) : "l"(reinterpret_cast<uint64_t>(own)));
  ObjectiveShared* first = reinterpret_cast<ObjectiveShared*>(at);
  a.sum = first->sum;
  a.term = first->term;
  a.block_count = first->block_count;
  a.count = first->count;
  a.slope = first->slope;
}
template <bool WIDE, bool EACH>
__global__ void __launch_bounds__(kObjectiveThreads) policy_cluster_kernel(ObjectiveArgs a) {
  __shared__ double red[3 * kObjectiveWarps];
  __shared__ ObjectiveShared shared;
  use_first_cta(a, &shared);
  const int rank = static_cast<int>(cluster_cta_rank()), lane = threadIdx.x & 31;
  grid_launch_dependents();
  cluster_sync_all();                              // the first CTA is there
  grid_dependency_wait();
  if (a.mask != nullptr && !a.own_count) {
    count_phase<WIDE>(a, rank, kObjectiveCtas, lane, reinterpret_cast<long long*>(red));
    cluster_sync_all();
  }
  const long long total = a.by_sequence ? 0 : all_valid(a, kObjectiveCtas, reinterpret_cast<long long*>(red));
  policy_phase<WIDE, EACH>(a, rank, kObjectiveCtas, lane, total, red);
  cluster_sync_all();
  if (rank == 0) policy_final(a, kObjectiveCtas, red);
}
template <bool WIDE>
__global__ void __launch_bounds__(kObjectiveThreads) preference_cluster_kernel(ObjectiveArgs a) {
  __shared__ double red[kObjectiveWarps];
  __shared__ ObjectiveShared shared;
  use_first_cta(a, &shared);
  const int rank = static_cast<int>(cluster_cta_rank()), lane = threadIdx.x & 31;
  const int first = rank * kObjectiveWarps + (threadIdx.x >> 5), step = kObjectiveCtas * kObjectiveWarps;
  grid_launch_dependents();
  cluster_sync_all();
  grid_dependency_wait();
  ratio_phase<WIDE>(a, first, step, lane);
  cluster_sync_all();
  pairs_phase(a, first, step, lane);
  cluster_sync_all();
  spread_phase<WIDE>(a, first, step, lane, false);
  if (rank == 0) preference_final(a, red);
  cluster_sync_all();                              // nobody reads the first CTA's any more
}

// ---- a launch for each phase
template <bool WIDE>
__global__ void __launch_bounds__(kObjectiveThreads) count_kernel(const ObjectiveArgs a) {
  __shared__ long long red[kObjectiveWarps];
  grid_launch_dependents();
  grid_dependency_wait();
  count_phase<WIDE>(a, blockIdx.x, gridDim.x, threadIdx.x & 31, red);
}
template <bool WIDE, bool EACH>
__global__ void __launch_bounds__(kObjectiveThreads, 2) policy_kernel(const ObjectiveArgs a) {
  __shared__ double red[3 * kObjectiveWarps];
  grid_launch_dependents();
  grid_dependency_wait();
  const long long total = a.by_sequence ? 0 : all_valid(a, gridDim.x, reinterpret_cast<long long*>(red));
  policy_phase<WIDE, EACH>(a, blockIdx.x, gridDim.x, threadIdx.x & 31, total, red);
}
__global__ void __launch_bounds__(kObjectiveThreads) policy_final_kernel(const ObjectiveArgs a, int blocks) {
  __shared__ double red[3 * kObjectiveWarps];
  grid_launch_dependents();
  grid_dependency_wait();
  policy_final(a, blocks, red);
}
template <bool WIDE>
__global__ void __launch_bounds__(kObjectiveThreads) ratio_kernel(const ObjectiveArgs a) {
  grid_launch_dependents();
  grid_dependency_wait();
  ratio_phase<WIDE>(a, blockIdx.x * kObjectiveWarps + (threadIdx.x >> 5), gridDim.x * kObjectiveWarps, threadIdx.x & 31);
}
__global__ void __launch_bounds__(kObjectiveThreads) pairs_kernel(const ObjectiveArgs a) {
  grid_launch_dependents();
  grid_dependency_wait();
  pairs_phase(a, blockIdx.x * kObjectiveWarps + (threadIdx.x >> 5), gridDim.x * kObjectiveWarps, threadIdx.x & 31);
}
// The last block adds up the loss. own: without pairs_kernel ahead, every warp forms what it needs of the sums, the last block all pairs'.
template <bool WIDE>
__global__ void __launch_bounds__(kObjectiveThreads) spread_kernel(const ObjectiveArgs a, bool own) {
  __shared__ double red[kObjectiveWarps];
  grid_launch_dependents();
  grid_dependency_wait();
  if (blockIdx.x + 1 == gridDim.x) {
    if (own) all_pairs(a);
    preference_final(a, red);
  } else {
    spread_phase<WIDE>(a, blockIdx.x * kObjectiveWarps + (threadIdx.x >> 5), (gridDim.x - 1) * kObjectiveWarps, threadIdx.x & 31, own);
  }
}

}  // namespace mtpc
