// Inline PTX of the policy update's kernels, beside what they share with the forward's
// (dora_ptx.cuh): a header of their own, so that the forward's sources, and what is
// keyed by them, stay as they are when these change.
//
// Like the training side's other kernels these do not trigger their dependents: a
// kernel that follows starts when they end.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "dora_ptx.cuh"

namespace dora {

// mbar_wait on a barrier that other CTAs of the cluster arrive on: what they wrote
// here before (release at cluster scope) is visible after it.
__device__ __forceinline__ bool mbar_try_wait_cluster(uint64_t* bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(smem_u32(bar)), "r"(parity)
      : "memory");
  return ok != 0;
}
__device__ __forceinline__ bool mbar_wait_cluster(uint64_t* bar, uint32_t parity,
                                                  volatile int* abort) {
  if (mbar_try_wait_cluster(bar, parity)) return true;
  const uint64_t t0 = globaltimer_ns();
  uint32_t spins = 0;
  while (true) {
    if (mbar_try_wait_cluster(bar, parity)) return true;
    if ((++spins & 63u) == 0u) {
      if (*abort) return false;
      if (globaltimer_ns() - t0 > kWaitLimitNs) {
        *abort = 1;
        return false;
      }
    }
  }
}

// One more CTA is done: its number, from 0.  What the thread wrote before is visible to
// the one that gets the last number, and to what follows a barrier of its CTA.
__device__ __forceinline__ unsigned take_ticket(unsigned* ticket) {
  unsigned n;
  asm volatile("atom.acq_rel.gpu.global.add.u32 %0, [%1], 1;" : "=r"(n) : "l"(ticket) : "memory");
  return n;
}

// A word into CTA `cta` of the cluster.
__device__ __forceinline__ void store_remote(int v, int* to, uint32_t cta) {
  asm volatile(
      "{\n\t.reg .b32 ra;\n\t"
      "mapa.shared::cluster.u32 ra, %0, %1;\n\t"
      "st.shared::cluster.u32 [ra], %2;\n\t}" ::"r"(smem_u32(to)),
      "r"(cta), "r"(v)
      : "memory");
}

__device__ __forceinline__ uint64_t f2_mul(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}

}  // namespace dora
