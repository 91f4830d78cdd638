// layer_device.cuh -- device helpers of the kernels around the verification attention:
// a decoder layer's, trees of drafts', a bounded cache's.  (sf_device.cuh is part of the
// attention's and the LM head's sources, by which their captures are known.)
#pragma once

#include "sf_device.cuh"

namespace sf {

// tmem_ld_32x32b_x16 without the wait: v must not be touched before tmem_ld_wait_x16(v).
__device__ __forceinline__ void tmem_ld_async_x16(uint32_t taddr, uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
        "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
      : "r"(taddr)
      : "memory");
}

// Waits for this thread's tcgen05.ld; v are registers that the last one brings (they
// pass through the statement, so that nothing uses them in front of it).
__device__ __forceinline__ void tmem_ld_wait_x16(uint32_t (&v)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]),
                 "+r"(v[8]), "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15])
               :
               : "memory");
}

// Two fp32 values in one 64-bit register: one instruction for both.
__device__ __forceinline__ unsigned long long f32x2(float x, float y) {
  unsigned long long v;
  asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(x), "f"(y));
  return v;
}
__device__ __forceinline__ void f32x2_split(unsigned long long v, float &x, float &y) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(v));
}
__device__ __forceinline__ unsigned long long f32x2_fma(unsigned long long a, unsigned long long b, unsigned long long c) {
  unsigned long long d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ unsigned long long f32x2_add(unsigned long long a, unsigned long long b) {
  unsigned long long d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}

// Lets the next kernel on the stream start once all stores of the grid can be read by
// it, also by bulk copies that it issues before it waits for this one.  All threads of
// the block call it, behind their stores.  (A block stays until its stores have arrived:
// the append of 35k rows 104 -> 110 us.)
__device__ __forceinline__ void launch_dependents_after_stores() {
  asm volatile("fence.proxy.async.global;" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();
    grid_launch_dependents();
  }
}

}  // namespace sf
