// Operand types, the softmax's small steps, counted waits and LDS fragment reads of the packed attention kernels.
#ifndef PF_PACKED_STEPS_H
#define PF_PACKED_STEPS_H

#include <utility>
#include "pf_internal.h"

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;   // 16-byte register quad
typedef __attribute__((ext_vector_type(2))) unsigned int u32x2;

template <int N>
struct IntC { static constexpr int value = N; };
template <int B, class F, int... I>
__device__ __forceinline__ void static_for_impl(F &&f, std::integer_sequence<int, I...>) {
  (f(IntC<B + I>()), ...);
}
template <int B, int E, class F>
__device__ __forceinline__ void static_for(F &&f) {
  static_for_impl<B>(f, std::make_integer_sequence<int, E - B>());
}

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// A row's weights are formed against the reference maximum that it has; only where a lane's sum of one tile's weights (no weight exceeds
// it) passes this bound is the tile's maximum looked up, the reference moved and the weights formed again.  fp32 and bf16 share the 8-bit
// exponent, so both hold such weights without loss of relative precision.  An unordered comparison: a NaN takes the same way once.
constexpr float PACKED_MAX_TILE_SUM = 256.0f;
__device__ __forceinline__ bool tile_sum_too_large(float sum) {
  return __builtin_amdgcn_fcmpf(sum, PACKED_MAX_TILE_SUM, 10 /* ugt */) != 0;
}

// max / sum with the lane that holds the other half of the same query row (lane ^ 32)
__device__ __forceinline__ float partner_max(float x) {
  const int xi = __float_as_int(x);
  auto r = __builtin_amdgcn_permlane32_swap(xi, xi, false, false);
  return fmaxf(__int_as_float(r[0]), __int_as_float(r[1]));
}
__device__ __forceinline__ float partner_sum(float x) {
  const int xi = __float_as_int(x);
  auto r = __builtin_amdgcn_permlane32_swap(xi, xi, false, false);
  return __int_as_float(r[0]) + __int_as_float(r[1]);
}

template <int N>
__device__ __forceinline__ void wait_vm() {                       // at most N vector-memory operations outstanding
  static_assert(N < 64, "vmcnt field");
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | ((N >> 4) << 14));
  __builtin_amdgcn_sched_barrier(0);
}
template <int N>
__device__ __forceinline__ void wait_lds() {                      // at most N LDS operations outstanding
  static_assert(N < 16, "lgkmcnt field");
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_waitcnt(0xC07F | (N << 8));
  __builtin_amdgcn_sched_barrier(0);
}

// Fragment reads by hand: the compiler would wait for all outstanding copies before an LDS read it knows about
template <int OFF = 0>
__device__ __forceinline__ void read_k(u32x4 &f, unsigned a) {
  asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(f) : "v"(a), "n"(OFF));
}
template <int OFF>
__device__ __forceinline__ void read_vt(u32x2 &f, unsigned a) {   // transposed: the lanes' rows become their columns
  asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(f) : "v"(a), "n"(OFF));
}

#endif  // PF_PACKED_STEPS_H
