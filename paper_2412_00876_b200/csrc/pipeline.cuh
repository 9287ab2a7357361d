// mbarrier and bulk-copy wrappers (inline PTX) shared by the pipelined kernels.
// Every wait is bounded: after kSpinLimit polls the caller's abort flag is raised and the
// wait returns false, so a broken pipeline ends with an error status instead of a hang.
#pragma once

#include <stdint.h>

namespace dl {

constexpr int kSpinLimit = 1 << 22;
constexpr int kSpinLimitBusy = 1 << 21;     // polls of the sleepless wait (each try_wait may itself suspend)

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void fence_mbar_init() {
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
}
__device__ __forceinline__ void mbar_expect_tx(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool mbar_try_wait(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
// One poll that never suspends the thread (for a role that watches several barriers in turn).
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
// Bounded wait.  Returns false (and raises *abort) when the bound is hit or another warp aborted.
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, volatile int* abort, int limit = kSpinLimit) {
  if (mbar_try_wait(bar, parity)) return !*abort;            // fast path: the phase is already complete
  for (int i = 0; i < limit; ++i) {
    if (*abort) return false;
    if (mbar_try_wait(bar, parity)) return true;
    if (i > 32) __nanosleep(40);
  }
  *abort = 1;
  return false;
}
// The same bound without the sleep between polls, for hand-offs inside a pipeline whose stages are a
// few hundred cycles long (try_wait itself suspends the thread for a hardware-chosen time).
__device__ __forceinline__ bool mbar_wait_spin(uint32_t bar, uint32_t parity, volatile int* abort) {
  if (mbar_test(bar, parity)) return true;                  // fast path: one non-suspending poll
  for (int i = 0; i < kSpinLimitBusy; ++i) {
    if (mbar_try_wait(bar, parity)) return true;
    if ((i & 63) == 63 && *abort) return false;
  }
  *abort = 1;
  return false;
}
// One answer for a whole warp whose lanes have waited each for itself: true if none of them gave up.  Lanes may leave a loop
// of votes, shuffles or matrix instructions on nothing else: a wait that runs out may do so for some of them only.
__device__ __forceinline__ bool warp_agreed(bool ok) { return __all_sync(0xffffffffu, ok); }
// 1-D bulk copy global -> shared; both addresses 16-byte aligned, bytes a multiple of 16.
__device__ __forceinline__ void bulk_g2s(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}

// 1-D bulk copy shared -> global, tracked by the issuing thread's bulk groups; both addresses 16-byte
// aligned, bytes a multiple of 16.
__device__ __forceinline__ void bulk_s2g(void* dst, uint32_t src, uint32_t bytes) {
  asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst), "r"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bulk_group_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
// until every bulk group of this thread has read its shared-memory source
__device__ __forceinline__ void bulk_group_wait_read_all() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }

}  // namespace dl
