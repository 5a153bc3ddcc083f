// Two fp32 values in one register pair, and the instructions that work on both at once (each rounded as its own); asynchronous
// copies of a thread's own 4, 8 or 16 bytes into shared memory.
#pragma once

#include "common.cuh"

namespace ist {
namespace {

// A product and a sum of pairs may be fused by the assembler, their rounding modifiers notwithstanding (seen in results).  Where
// the product's own rounding counts, the sum is taken with add_rounded.
typedef unsigned long long pair;        // two fp32 values
__device__ __forceinline__ pair make_pair2(float a, float b) {
  pair p;
  asm("mov.b64 %0, {%1, %2};" : "=l"(p) : "f"(a), "f"(b));
  return p;
}
__device__ __forceinline__ float first_of(pair p) { return __uint_as_float((uint32_t)p); }
__device__ __forceinline__ float second_of(pair p) { return __uint_as_float((uint32_t)(p >> 32)); }
__device__ __forceinline__ pair both(float a) { return make_pair2(a, a); }
__device__ __forceinline__ pair add(pair a, pair b) {
  pair d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ pair add_rounded(pair a, pair b) {
  return make_pair2(__fadd_rn(first_of(a), first_of(b)), __fadd_rn(second_of(a), second_of(b)));
}
__device__ __forceinline__ pair mul(pair a, pair b) {
  pair d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ pair fma(pair a, pair b, pair c) {
  pair d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}

__device__ __forceinline__ uint32_t shared_address(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
template <int BYTES>
__device__ __forceinline__ void copy_async(uint32_t to, const void* from) {
  if (BYTES == 16)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(to), "l"(from), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

}  // namespace
}  // namespace ist
