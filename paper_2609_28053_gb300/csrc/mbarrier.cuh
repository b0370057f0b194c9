// mbarrier.cuh -- shared-memory mbarriers with bounded waits, for the kernels
// that load asynchronously, and the barrier of a cluster.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace eqb {

namespace {

constexpr uint32_t kSpinLimit = 1u << 20;  // polls of at most ~1 us: about a second

__device__ __forceinline__ uint32_t smem_u32(const void* p) {
  return static_cast<uint32_t>(__cvta_generic_to_shared(p));
}

__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_expect_tx(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes)
               : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool mbar_try_wait(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity), "r"(1000u)
      : "memory");
  return ok != 0;
}
// Bounded wait for the phase of parity `parity`; false if it timed out or
// another role aborted.
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
  for (uint32_t i = 0; i < kSpinLimit; ++i) {
    if (mbar_try_wait(bar, parity)) return true;
    if ((i & 63u) == 63u && *abort_flag) return false;
  }
  *abort_flag = 1;
  return false;
}

// After a wait ran out: tile loads may still be on their way into shared
// memory, which is not this block's any more once it has returned.  Waits for
// the last min(S, issued) of the `issued` loads of a ring of S stages (load i
// completes the phase of parity (i / S) & 1 of barrier(i % S)), within one
// limit for all of them.
template <class Barrier>
__device__ __forceinline__ void drain_loads(int issued, int S, Barrier barrier) {
  uint32_t left = kSpinLimit;
  for (int i = issued > S ? issued - S : 0; i < issued; ++i)
    while (left > 0u && !mbar_try_wait(barrier(i % S), static_cast<uint32_t>(i / S) & 1u)) --left;
}

// An untiled copy into shared memory, counted by a barrier: addresses and size
// are multiples of 16 bytes.
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src),
               "r"(bytes), "r"(bar)
               : "memory");
}

// This block's place in its cluster, and the cluster's barrier.
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

}  // namespace

}  // namespace eqb
