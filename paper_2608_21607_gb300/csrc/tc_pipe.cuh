// What the tensor-core kernels' pipelines share: bounded mbarrier waits and the
// driver's tensor-map encoder.
#pragma once

#include <cudaTypedefs.h>

#include <mutex>

#include "nmd_internal.cuh"
#include "tc_ptx.cuh"

namespace nmd {
namespace tc {

constexpr uint64_t kTimeoutNs = 2000000000ull;

__device__ __forceinline__ void record(int* status, int code, int detail) {
  if (atomicCAS(status, 0, code) == 0) status[1] = detail;
}

// Bounded wait on an mbarrier phase.  Returns false if the kernel is aborting.
// The polls suspend in hardware until the phase completes (or 20 us pass), so
// waiting warps do not take issue slots from the MMA and copy threads.
static __device__ __noinline__ bool wait_bar_slow(uint32_t bar, uint32_t parity, volatile int* abort_flag, int* status,
                                           int where, uint64_t limit_ns = kTimeoutNs) {
  const uint64_t t0 = globaltimer_ns();
  for (;;) {
    if (mbar_try_wait(bar, parity)) return true;
    if (*abort_flag) return false;
    if (globaltimer_ns() - t0 > limit_ns) {
      *abort_flag = 1;
      record(status, NMD_ERR_TIMEOUT, where);
      return false;
    }
  }
}
__device__ __forceinline__ bool wait_bar(uint32_t bar, uint32_t parity, volatile int* abort_flag, int* status,
                                         int where) {
  if (mbar_try_wait(bar, parity)) return true;
  return wait_bar_slow(bar, parity, abort_flag, status, where);
}

// Wait for a converged warp: every lane tests the phase; if it has not
// completed, lane 0 polls and the outcome is broadcast.
__device__ __forceinline__ bool conv_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, int* status,
                                          int where) {
  if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
  int ok = 0;
  if ((threadIdx.x & 31) == 0) ok = wait_bar_slow(bar, parity, abort_flag, status, where);
  ok = __shfl_sync(0xffffffffu, ok, 0);
  return ok != 0;
}

// Warp-uniform wait: lane 0 polls, the outcome is broadcast to the warp.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, int* status,
                                          int where) {
  int ok = 0;
  if ((threadIdx.x & 31) == 0) ok = wait_bar(bar, parity, abort_flag, status, where);
  ok = __shfl_sync(0xffffffffu, ok, 0);
  __syncwarp();
  return ok != 0;
}

inline PFN_cuTensorMapEncodeTiled_v12000 encode_fn() {
  static PFN_cuTensorMapEncodeTiled_v12000 fn = nullptr;
  static std::once_flag once;
  std::call_once(once, [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) ==
            cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
      fn = (PFN_cuTensorMapEncodeTiled_v12000)p;
  });
  return fn;
}

}  // namespace tc
}  // namespace nmd
