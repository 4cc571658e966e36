// Small device helpers shared by the kernels of libslidedp: BF16 packing and streaming accesses.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace slidedp {

// ---- small helpers -----------------------------------------------------------------

__device__ __forceinline__ float bf16_lo(uint32_t x) { return __uint_as_float(x << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t x) { return __uint_as_float(x & 0xFFFF0000u); }

// FP32 -> BF16 bits, round to nearest even, NaN stays NaN.
__device__ __forceinline__ uint32_t f32_to_bf16_bits(float x) {
  uint16_t r;
  asm("cvt.rn.bf16.f32 %0, %1;" : "=h"(r) : "f"(x));
  return (uint32_t)r;
}

// The same for two values: lo in the lower half.
__device__ __forceinline__ uint32_t f32x2_to_bf16x2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// The address of a shared-memory object in the form that the shared-memory instructions take.
__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

// Two FP32 values per instruction.
__device__ __forceinline__ uint64_t pair(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void split(uint64_t v, float* lo, float* hi) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(*lo), "=f"(*hi) : "l"(v));
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// Streaming (read-once / write-once) 128-bit accesses: keep them out of L1 and mark them
// evict-first in L2, since nothing on this path is ever re-read.
__device__ __forceinline__ uint4 ld_stream(const void* p) {
  return __ldcs(reinterpret_cast<const uint4*>(p));
}
__device__ __forceinline__ void st_stream(void* p, uint4 v) {
  __stcs(reinterpret_cast<uint4*>(p), v);
}

// Programmatic dependent launch: a kernel launched with the programmatic-stream-serialization
// attribute may be scheduled while the kernel before it in the stream is still finishing; this
// wait holds it until that kernel has completed and its writes are visible. Launched the plain
// way the instruction does nothing. Every kernel that can be launched that way executes it
// before its first global-memory access.
__device__ __forceinline__ void wait_for_previous_kernel() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
}
// Lets a kernel launched that way start as soon as every block of this one has come here or ended.
__device__ __forceinline__ void allow_next_kernel() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
// For kernels that have nothing to do before their first access to memory.
__device__ __forceinline__ void start_after_previous_kernel() {
  allow_next_kernel();
  wait_for_previous_kernel();
}

}  // namespace slidedp
