// Which workgroup of a launch ends last (gfx950, wave64).
#pragma once

#include "device_common.hpp"

namespace vtrace {

// Workgroups that finish together would queue for one counter (about 10 ns each: 1024 of them
// 10 us), so each of 32 counters, a 128-byte line apiece, takes a share of them, and the
// workgroup that is the last of its counter draws the ticket.  All return to zero.
constexpr int kCounters = 32, kCounterWords = 32;
static_assert(kCounters * kCounterWords * sizeof(unsigned) == kWsCounterBytes, "their place in a workspace");

// True in every thread of the workgroup that is the last of the grid to get here; what the
// thread 0 of each workgroup stored before (with device-scope atomic stores) is then there to
// be read (with device-scope atomic loads).  Ordering as in finish_ticket.
__device__ __forceinline__ bool last_workgroup(unsigned* ticket, unsigned* counters) {
  __shared__ int s_last;
  if (threadIdx.x == 0) {
    __atomic_signal_fence(__ATOMIC_SEQ_CST);  // keep the compiler from moving the stores past the wait
    __builtin_amdgcn_s_waitcnt(kWaitVmcnt0);  // the stores have completed
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    const unsigned mine = blockIdx.x % kCounters;
    const unsigned sharers = (gridDim.x - mine + kCounters - 1) / kCounters;
    unsigned* const counter = counters + mine * kCounterWords;
    bool last = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == sharers - 1;
    if (last) {
      __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      const unsigned used = gridDim.x < kCounters ? gridDim.x : kCounters;
      last = __hip_atomic_fetch_add(ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == used - 1;
      if (last) __hip_atomic_store(ticket, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    s_last = last;
  }
  __syncthreads();
  return s_last != 0;
}

}  // namespace vtrace
