// What the tensor-core kernels' roles share: tile sizes, the barriers of a CTA, and waits that end.
#pragma once
#include <stdint.h>

#include "mtpc_ptx.cuh"

namespace mtpc {

constexpr int kBlockM = 128;         // positions per tile (= TMEM lanes)
constexpr int kBlockK = 64;          // bf16 elements per 128-byte swizzled row
constexpr int kMaxStages = 16;
constexpr int kMaxSlots = 8;
constexpr int kTmemCols = 512;
constexpr int kGemmThreads = 192;
constexpr uint64_t kWaitLimitNs = 1000ull * 1000ull * 1000ull;   // 1 s per barrier wait (the default, and always the limit of the drain waits)
constexpr uint64_t kAwakeNs = 100ull * 1000ull;                  // limits below this: see first_wait
constexpr uint64_t kAbortSettleNs = 200ull * 1000ull;            // 0.2 ms: far longer than any copy or MMA in flight takes
constexpr int kABytes = kBlockM * kBlockK * 2;                   // 16 KB
constexpr uint32_t kStatusBadTarget = 1u, kStatusBadUniform = 2u, kStatusTimeout = 4u;
constexpr uint32_t kMnBoxBytes = 64 * kBlockK * 2;   // one 64 x 64 bf16 box: 8 KB

struct GemmControl {
  uint64_t full[kMaxStages];
  uint64_t empty[kMaxStages];
  uint64_t tfull[kMaxSlots];
  uint64_t tempty[kMaxSlots];
  uint64_t drain;
  uint64_t wait_limit_ns;
  uint32_t tmem_base;
  volatile int abort;
};

__device__ __forceinline__ bool bounded_wait(uint32_t bar, uint32_t parity, GemmControl* ctl, unsigned* status) {
  if (mbar_try_wait(bar, parity)) return true;
  const uint64_t t0 = global_timer_ns();
  uint32_t it = 0;
  while (true) {
    if (mbar_try_wait(bar, parity)) return true;
    if ((++it & 15u) == 0) {
      if (ctl->abort) return false;
      if (global_timer_ns() - t0 > ctl->wait_limit_ns) {
        ctl->abort = 1;
        if (status != nullptr) atomicOr(status, kStatusTimeout);
        return false;
      }
    }
  }
}
// Lane 0 waits, the whole warp learns the outcome (keeps the warp converged for the .sync.aligned TMEM loads).
__device__ __forceinline__ bool bounded_wait_warp(uint32_t bar, uint32_t parity, GemmControl* ctl, unsigned* status,
                                                  int lane) {
  int ok = 1;
  if (lane == 0) ok = bounded_wait(bar, parity, ctl, status) ? 1 : 0;
  return __shfl_sync(0xffffffffu, ok, 0) != 0;
}

// The whole warp waits and learns the outcome, known to be the same in every lane. It sleeps in try_wait until the barrier's phase is over or for
// as long as the hardware lets it (a suspend-time hint of 50 ns does not shorten that), and then looks whether another role has given up. P: the
// kernel's parameters.
template <typename P>
__device__ __forceinline__ bool bounded_wait_all(uint32_t bar, uint32_t parity, GemmControl* ctl, const P& p) {
  constexpr unsigned all = 0xffffffffu;
  if (__all_sync(all, mbar_try_wait(bar, parity))) return true;
  const uint64_t t0 = global_timer_ns();
  while (true) {
    if (__any_sync(all, ctl->abort)) return false;
    if (__all_sync(all, mbar_try_wait(bar, parity))) return true;
    if (__any_sync(all, global_timer_ns() - t0 > p.wait_limit_ns)) {
      ctl->abort = 1;
      if (elect_one() && p.status != nullptr) atomicOr(p.status, kStatusTimeout);
      return false;
    }
  }
}
// A sleep outlasts limits of microseconds, and a choice between sleeping and not at every wait costs GEMMs 1.5 % (5 x 401 positions of a training call
// 990 -> 1005 us). So with a limit that short the MMA issuer keeps awake for its first copies, and what it decides reaches the other roles by the
// abort flag.
template <typename P>
__device__ __forceinline__ bool first_wait(uint32_t bar, GemmControl* ctl, const P& p) {
  constexpr unsigned all = 0xffffffffu;
  if (p.wait_limit_ns >= kAwakeNs) return true;
  const uint64_t t0 = global_timer_ns();
  while (!__all_sync(all, mbar_test_wait(bar, 0))) {
    if (__any_sync(all, global_timer_ns() - t0 > p.wait_limit_ns)) {
      ctl->abort = 1;
      if (elect_one() && p.status != nullptr) atomicOr(p.status, kStatusTimeout);
      return false;
    }
  }
  return true;
}
// A wait that decides nothing: for what may still be in flight when a CTA goes away.
__device__ __forceinline__ void drain_wait(uint32_t bar, uint32_t parity) {
  const uint64_t t0 = global_timer_ns();
  while (!mbar_try_wait(bar, parity) && global_timer_ns() - t0 < kWaitLimitNs) {}
}

// Warp 1 of a CTA whose roles have all ended and met: if a wait gave up in any of them, its MMAs may still be in flight, also where it had issued
// all it had to. They are waited for before tensor memory is freed and the CTA goes away. Pairs: the leader's (`issuer`), and then as long
// as any copy of either CTA takes, since the peer's are counted on the leader's barriers and cannot be awaited.
template <int CTAS>
__device__ __forceinline__ void drain_after_abort(GemmControl* ctl, bool issuer) {
  if (!__any_sync(0xffffffffu, ctl->abort)) return;
  if (issuer) {
    const uint32_t lead = elect_one();                          // the lane that issued them
    if (CTAS == 2) umma_commit_pair(lead, smem_u32(&ctl->drain));
    else umma_commit(lead, smem_u32(&ctl->drain));
    drain_wait(smem_u32(&ctl->drain), 0);
  }
  if (CTAS == 2) {
    const uint64_t t0 = global_timer_ns();
    while (global_timer_ns() - t0 < kAbortSettleNs) {}
  }
  __syncwarp();
}

}  // namespace mtpc
