// Bounded waits on shared-memory mbarriers: a wait that is not served within its limit raises the (sticky) status
// word of the caller's workspace to SDVG_ERR_TIMEOUT and returns false, so that the kernel can leave its roles and exit.
#pragma once

#include <stdint.h>

#include "sdvg.h"
#include "sm100_ptx.cuh"

namespace sm100 {

// Every wait on an mbarrier ends at an absolute deadline taken at kernel start.
struct Deadline {
  uint64_t t_ns;                       // globaltimer value after which waits give up
  unsigned int* status;                // global status word
};

// Slow path of the bounded wait: poll until the phase completes or the deadline passes.  Kept out
// of line of the first attempt so that the timer read never sits on the fast path.  Waiting threads
// that poll less often (a suspend-time hint on the try_wait, the timer read once per 256 polls) or that
// never suspend (test_wait) were measured 2-5% slower: how soon a waiter notices counts for more than the
// issue slots its polling takes.
__device__ __forceinline__ bool wait_bar_slow(uint32_t bar_addr, uint32_t parity, uint64_t deadline_ns,
                                           unsigned int* status) {
  uint32_t ok;
  asm volatile(
      "{\n\t"
      ".reg .pred p, q;\n\t"
      ".reg .u64 t;\n\t"
      "SDVG_WAIT:\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "@p bra SDVG_DONE;\n\t"
      "mov.u64 t, %%globaltimer;\n\t"
      "setp.lt.u64 q, t, %3;\n\t"
      "@q bra SDVG_WAIT;\n\t"
      "SDVG_DONE:\n\t"
      "selp.u32 %0, 1, 0, p;\n\t"
      "}"
      : "=r"(ok)
      : "r"(bar_addr), "r"(parity), "l"(deadline_ns)
      : "memory");
  if (!ok) atomicMax(status, (unsigned)SDVG_ERR_TIMEOUT);      // sticky: only a reset clears it
  return ok != 0;
}

// Bounded mbarrier wait.  One try_wait (which itself suspends the thread for a hardware-chosen
// time) settles almost every wait; only if it fails does the thread enter the timed poll loop.
// Returns false (and records SDVG_ERR_TIMEOUT) once the deadline has passed.
__device__ __forceinline__ bool wait_bar(uint64_t* bar, uint32_t parity, const Deadline& d) {
  if (mbar_try_wait(bar, parity)) return true;
  return wait_bar_slow(smem_u32(bar), parity, d.t_ns, d.status);
}

// The same wait made by all 32 lanes of a warp, with a warp-uniform result.
__device__ __forceinline__ bool wait_warp(uint64_t* bar, uint32_t parity, const Deadline& d) {
  return __all_sync(0xffffffffu, wait_bar(bar, parity, d));
}

// A wait whose limit runs from the wait itself: for kernels whose run time grows with the problem without bound.
__device__ __forceinline__ bool wait_for(uint64_t* bar, uint32_t parity, unsigned int* status, uint64_t limit_ns) {
  if (mbar_try_wait(bar, parity)) return true;
  return wait_bar_slow(smem_u32(bar), parity, globaltimer_ns() + limit_ns, status);
}

}  // namespace sm100
