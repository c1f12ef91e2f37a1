// Bounded waits: no wait inside a kernel lasts longer than kWaitLimitNs.
#pragma once

#include "ozk_common.cuh"
#include "ozk_ptx.cuh"

namespace ozk {

constexpr uint64_t kWaitLimitNs = 2000000000ull;

// Bounded wait on an mbarrier phase.  Returns false after the time limit or when another role
// of this CTA has already given up.
__device__ __forceinline__ bool wait_bounded(uint32_t bar, uint32_t parity, volatile int* abort, StatusBlock* status, int where) {
  if (ptx::mbar_try_wait(bar, parity)) return true;
  const uint64_t t0 = ptx::global_timer_ns();
  for (uint32_t it = 1;; ++it) {
    if (ptx::mbar_try_wait(bar, parity)) return true;
    if ((it & 63u) == 0u) {
      if (*abort) return false;
      if (ptx::global_timer_ns() - t0 > kWaitLimitNs) {
        *abort = 1;
        atomicMin(&status->code, (int)OZK_ERR_DEVICE_TIMEOUT);
        atomicExch(&status->where, where);
        return false;
      }
    }
  }
}
// The same for all lanes of a converged warp, with one answer for all.
__device__ __forceinline__ bool wait_warp(uint32_t bar, uint32_t parity, volatile int* abort, StatusBlock* status, int where) {
  return __all_sync(0xFFFFFFFFu, wait_bounded(bar, parity, abort, status, where));
}

}  // namespace ozk
