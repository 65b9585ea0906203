// Host side of the calls that fit a model to tasks beside its head (include/mtpc.h): dropout and the losses of log-likelihoods.
// Argument checks, carving of the caller's workspace, choice of the build, launches.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <algorithm>
#include <initializer_list>

#include "../../include/mtpc.h"
#include "mtpc_dropout.cuh"
#include "mtpc_host.cuh"
#include "mtpc_launch.cuh"
#include "mtpc_objective.cuh"

namespace {

using namespace mtpc;

// ---------------------------------------------------------------- dropout
template <typename TI, typename TO, bool RESIDUAL>
void launch_dropout(const DropoutArgs& a, bool vectors, cudaStream_t st) {
  const int64_t blocks = (a.count + 7) / 8;
  // Two blocks of draws a thread where there are enough for every SM.
  if (!vectors) launch_kernel(dropout_plain_kernel<TI, TO, RESIDUAL>, ceil_div(blocks, 256), 256, 0, st, true, a);
  else if (blocks >= static_cast<int64_t>(kSms) * 2048) launch_kernel(dropout_kernel<TI, TO, RESIDUAL, 2>, ceil_div(blocks, 512), 256, 0, st, true, a);
  else launch_kernel(dropout_kernel<TI, TO, RESIDUAL, 1>, ceil_div(blocks, 256), 256, 0, st, true, a);
}
template <typename TI, typename TO>
void launch_dropout(const DropoutArgs& a, bool vectors, cudaStream_t st) {
  if (a.residual) launch_dropout<TI, TO, true>(a, vectors, st);
  else launch_dropout<TI, TO, false>(a, vectors, st);
}

// ---------------------------------------------------------------- losses
constexpr int kMaxSequences = 1 << 20;
constexpr int kSmallPositions = 1 << 16;
constexpr int kOwnParts = 64, kOwnPairs = 1024;
constexpr int kOwnCount = 1 << 14;      // mean length up to which a sequence's positions are counted by each of its warps: 32 vectors of 16 bytes a lane
struct ObjectivePlan {
  int parts;
  bool small;                           // one cluster does it, without a workspace
  size_t off_count, off_blocks, off_sum, off_term, off_slope, total;
};
// Slices for every warp that the device holds at once, of 128 positions (a vector of a lane) at least; of a small call for those of its cluster.
void plan_objective(int T, int S, ObjectivePlan* p) {
  const int most = T <= kSmallPositions ? kSmallItems : kMostBlocks * kObjectiveWarps;
  p->parts = std::max(1, std::min(ceil_div(T, static_cast<long long>(S) * 128), most / S));
  const size_t items = static_cast<size_t>(S) * p->parts;
  p->small = T <= kSmallPositions && items <= kSmallItems;
  p->total = 0;
  if (p->small) return;
  size_t off = 0;
  auto take = [&](size_t bytes) { size_t o = off; off += align_up(bytes); return o; };
  p->off_count = take(items * 4);
  p->off_blocks = take(kMostBlocks * 8);
  p->off_sum = take(std::max<size_t>(items, 3 * kMostBlocks) * 8);
  p->off_term = take(static_cast<size_t>(S / 2 + 1) * 8);
  p->off_slope = take(static_cast<size_t>(S / 2 + 1) * 4);
  p->total = off;
}
int check_sequences(int T, int S) {
  if (T < 0 || S < 1) return MTPC_ERR_SHAPE;
  if (T > kMaxRows || S > kMaxSequences) return MTPC_ERR_UNSUPPORTED;
  return MTPC_OK;
}
void two_terms(double x, float* y) {
  y[0] = static_cast<float>(x);
  y[1] = isinf(y[0]) ? 0.f : static_cast<float>(x - y[0]);
}
bool a_share(float x) { return x >= 0.f && x <= 1.f; }      // (no NaN)
void carve(const ObjectivePlan& p, void* workspace, ObjectiveArgs* a) {
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  a->parts = p.parts;
  if (p.small) return;
  a->count = reinterpret_cast<int*>(ws + p.off_count);
  a->block_count = reinterpret_cast<long long*>(ws + p.off_blocks);
  a->sum = reinterpret_cast<double*>(ws + p.off_sum);
  a->term = reinterpret_cast<double*>(ws + p.off_term);
  a->slope = reinterpret_cast<float*>(ws + p.off_slope);
}
int item_blocks(const ObjectiveArgs& a) { return std::min(ceil_div(static_cast<long long>(a.S) * a.parts, kObjectiveWarps), kMostBlocks); }
template <bool WIDE, bool EACH>
void launch_policy(const ObjectiveArgs& a, bool small, cudaStream_t st) {
  if (small) {
    launch_clusters(policy_cluster_kernel<WIDE, EACH>, kObjectiveCtas, kObjectiveCtas, kObjectiveThreads, 0, st, true, a);
    return;
  }
  if (a.mask && !a.own_count) launch_kernel(count_kernel<WIDE>, item_blocks(a), kObjectiveThreads, 0, st, true, a);
  launch_kernel(policy_kernel<WIDE, EACH>, item_blocks(a), kObjectiveThreads, 0, st, true, a);
  launch_kernel(policy_final_kernel, 1, kObjectiveThreads, 0, st, true, a, item_blocks(a));
}
template <bool WIDE>
void launch_preference(const ObjectiveArgs& a, bool small, cudaStream_t st) {
  if (small) {
    launch_clusters(preference_cluster_kernel<WIDE>, kObjectiveCtas, kObjectiveCtas, kObjectiveThreads, 0, st, true, a);
    return;
  }
  launch_kernel(ratio_kernel<WIDE>, item_blocks(a), kObjectiveThreads, 0, st, true, a);
  // Where a pair's sums are few, whoever needs its slope forms it, and the last block has all of them for the loss in little time: one launch less.
  const bool own = a.parts <= kOwnParts && a.S <= kOwnPairs;
  if (!own) launch_kernel(pairs_kernel, std::min(ceil_div(a.S / 2, kObjectiveWarps), kSms * 4), kObjectiveThreads, 0, st, true, a);
  launch_kernel(spread_kernel<WIDE>, item_blocks(a) + 1, kObjectiveThreads, 0, st, true, a, own);
}

}  // namespace

extern "C" {

int mtpc_dropout(const void* x, int64_t x_stride, int32_t x_dtype, const void* residual, int64_t residual_stride, int32_t T, int32_t d,
                 float p, const int64_t* rng, int64_t offset, void* out, int64_t out_stride, int32_t out_dtype, void* stream) {
  if (T < 0 || T > kMaxRows || d < 1 || d > kMaxRows || !known(x_dtype) || !known(out_dtype) || !(p >= 0.f && p < 1.f)) return MTPC_ERR_SHAPE;
  if (static_cast<int64_t>(T) * d > (static_cast<int64_t>(1) << 40)) return MTPC_ERR_UNSUPPORTED;
  if (T == 0) return MTPC_OK;
  if (!x || !rng || !out) return MTPC_ERR_NULL;
  if (!input_rows(x, x_stride, T) || !input_rows(residual, residual_stride, T) || !output_rows(out, out_stride, T, d)) return MTPC_ERR_SHAPE;
  const size_t ei = element(x_dtype), eo = element(out_dtype);
  if (!aligned(x, ei) || !aligned(residual, eo) || !aligned(out, eo) || !aligned(rng, 8)) return MTPC_ERR_SHAPE;
  const int rc = check_device();
  if (rc != MTPC_OK) return rc;
  DropoutArgs a;
  memset(&a, 0, sizeof(a));
  a.x = x;
  a.residual = residual;
  a.out = out;
  a.rng = rng;
  a.x_stride = x_stride;
  a.residual_stride = residual_stride;
  a.out_stride = out_stride;
  a.offset = offset;
  a.count = static_cast<int64_t>(T) * d;
  a.cut = static_cast<uint32_t>(std::min(65535.f, floorf(p * 65536.f + 0.5f)));
  a.scale = 65536.f / static_cast<float>(65536u - a.cut);
  const bool one_run = T == 1 || (x_stride == d && out_stride == d && (!residual || residual_stride == d));
  a.d = one_run ? 0 : d;
  const bool vectors = (one_run || d % 8 == 0) && rows_allow(x, one_run ? 0 : x_stride, ei, 8, T) &&
                       rows_allow(residual, one_run ? 0 : residual_stride, eo, 8, T) && rows_allow(out, one_run ? 0 : out_stride, eo, 8, T);
  if (!vectors) a.d = d;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (x_dtype == MTPC_F32) {
    if (out_dtype == MTPC_F32) launch_dropout<float, float>(a, vectors, st);
    else launch_dropout<float, __nv_bfloat16>(a, vectors, st);
  } else {
    if (out_dtype == MTPC_F32) launch_dropout<__nv_bfloat16, float>(a, vectors, st);
    else launch_dropout<__nv_bfloat16, __nv_bfloat16>(a, vectors, st);
  }
  return check_launch();
}

int mtpc_objective_workspace_bytes(int32_t T, int32_t S, size_t* out_bytes) {
  if (!out_bytes) return MTPC_ERR_NULL;
  const int rc = check_sequences(T, S);
  if (rc != MTPC_OK) return rc;
  ObjectivePlan p;
  plan_objective(T, S, &p);
  *out_bytes = p.total;
  return MTPC_OK;
}

int mtpc_policy_loss(const float* logp, const float* old_logp, const float* ref_logp, const float* advantage, int32_t advantage_by_position,
                     const uint8_t* mask, const int32_t* offsets, int32_t T, int32_t S, float clip_low, float clip_high, float beta,
                     int32_t by_sequence, float* out_loss, float* out_stats, float* d_logp, void* workspace, size_t workspace_bytes,
                     uint32_t* out_status, void* stream) {
  int rc = check_sequences(T, S);
  if (rc != MTPC_OK) return rc;
  if (!(clip_low >= 0.f && clip_low < INFINITY) || !(clip_high >= 0.f && clip_high < INFINITY) || !(beta >= 0.f && beta < INFINITY)) return MTPC_ERR_SHAPE;
  if (!offsets || !out_loss || (!advantage && (T > 0 || !advantage_by_position)) || (T > 0 && (!logp || !old_logp || !d_logp))) return MTPC_ERR_NULL;
  if (beta > 0.f && T > 0 && !ref_logp) return MTPC_ERR_NULL;
  for (const void* q : {static_cast<const void*>(logp), static_cast<const void*>(old_logp), static_cast<const void*>(ref_logp),
                        static_cast<const void*>(advantage), static_cast<const void*>(offsets), static_cast<const void*>(out_loss),
                        static_cast<const void*>(out_stats), static_cast<const void*>(d_logp), static_cast<const void*>(out_status)})
    if (!aligned(q, 4)) return MTPC_ERR_SHAPE;
  ObjectivePlan p;
  plan_objective(T, S, &p);
  if (p.total > 0 && !workspace) return MTPC_ERR_NULL;
  if (workspace_bytes < p.total || !aligned(workspace, kAlign)) return MTPC_ERR_WORKSPACE;
  if ((rc = check_device()) != MTPC_OK) return rc;
  ObjectiveArgs a;
  memset(&a, 0, sizeof(a));
  a.logp = logp;
  a.old = old_logp;
  a.ref = beta > 0.f ? ref_logp : nullptr;
  a.advantage = advantage;
  a.mask = mask;
  a.offsets = offsets;
  a.T = T;
  a.S = S;
  a.by_sequence = by_sequence != 0;
  a.own_count = a.by_sequence && mask && T / S <= kOwnCount;
  a.low = static_cast<float>(1.0 - static_cast<double>(clip_low));
  a.high = static_cast<float>(1.0 + static_cast<double>(clip_high));
  two_terms(clip_low < 1.f ? log1p(-static_cast<double>(clip_low)) : -INFINITY, a.log_low);
  two_terms(log1p(static_cast<double>(clip_high)), a.log_high);
  a.beta = beta;
  a.loss = out_loss;
  a.stats = out_stats;
  a.d_logp = d_logp;
  a.status = out_status;
  carve(p, workspace, &a);
  const bool each = advantage_by_position != 0;
  const bool wide = aligned(logp, 16) && aligned(old_logp, 16) && aligned(a.ref, 16) && aligned(d_logp, 16) && aligned(mask, 4) &&
                    (!each || aligned(advantage, 16));
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (each) wide ? launch_policy<true, true>(a, p.small, st) : launch_policy<false, true>(a, p.small, st);
  else wide ? launch_policy<true, false>(a, p.small, st) : launch_policy<false, false>(a, p.small, st);
  return check_launch();
}

int mtpc_preference_loss(const float* logp, const float* ref_logp, const uint8_t* mask, const int32_t* offsets, int32_t T, int32_t S, float beta,
                         float smoothing, float* out_loss, float* out_h, float* d_logp, void* workspace, size_t workspace_bytes,
                         uint32_t* out_status, void* stream) {
  int rc = check_sequences(T, S);
  if (rc != MTPC_OK) return rc;
  if (S % 2 != 0 || !(beta >= 0.f && beta < INFINITY) || !a_share(smoothing)) return MTPC_ERR_SHAPE;
  if (!offsets || !out_loss || (T > 0 && (!logp || !ref_logp || !d_logp))) return MTPC_ERR_NULL;
  for (const void* q : {static_cast<const void*>(logp), static_cast<const void*>(ref_logp), static_cast<const void*>(offsets),
                        static_cast<const void*>(out_loss), static_cast<const void*>(out_h), static_cast<const void*>(d_logp),
                        static_cast<const void*>(out_status)})
    if (!aligned(q, 4)) return MTPC_ERR_SHAPE;
  ObjectivePlan p;
  plan_objective(T, S, &p);
  if (p.total > 0 && !workspace) return MTPC_ERR_NULL;
  if (workspace_bytes < p.total || !aligned(workspace, kAlign)) return MTPC_ERR_WORKSPACE;
  if ((rc = check_device()) != MTPC_OK) return rc;
  ObjectiveArgs a;
  memset(&a, 0, sizeof(a));
  a.logp = logp;
  a.ref = ref_logp;
  a.mask = mask;
  a.offsets = offsets;
  a.T = T;
  a.S = S;
  a.beta = beta;
  a.smoothing = smoothing;
  a.loss = out_loss;
  a.h = out_h;
  a.d_logp = d_logp;
  a.status = out_status;
  carve(p, workspace, &a);
  const bool wide = aligned(logp, 16) && aligned(ref_logp, 16) && aligned(d_logp, 16) && aligned(mask, 4);
  if (wide) launch_preference<true>(a, p.small, static_cast<cudaStream_t>(stream));
  else launch_preference<false>(a, p.small, static_cast<cudaStream_t>(stream));
  return check_launch();
}

}  // extern "C"
