// Building blocks of the bf16 attention kernels: vector types, weights packed for
// the matrix cores, exchanges between the two halves of a wave, and the
// dispatch order.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#define LDS_AS __attribute__((address_space(3)))

namespace fademem {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Two weights rounded to bf16 and packed as one B-operand word of P.V.
__device__ __forceinline__ uint32_t round_pair(float p0, float p1) {
  bf16x2 pk;
  pk[0] = (__bf16)p0;
  pk[1] = (__bf16)p1;
  return __builtin_bit_cast(uint32_t, pk);
}

__device__ __forceinline__ float pair_max(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __builtin_elementwise_maximum(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float pair_sum(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// A pointer the whole wave holds, moved to scalar registers.
__device__ __forceinline__ const char* uniform_ptr(const char* p) {
  const uint64_t u = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane(uint32_t(u));
  const uint32_t hi = __builtin_amdgcn_readfirstlane(uint32_t(u >> 32));
  return reinterpret_cast<const char*>((uint64_t(hi) << 32) | lo);
}

// XCD-aware group index: blocks are dealt to the 8 XCDs round-robin, so
// block b runs on XCD b % 8; give each XCD a contiguous run of groups.
__device__ __forceinline__ int xcd_group(int bid, int groups) {
  const int per = groups / 8, rem = groups % 8;
  const int xcd = bid % 8, local = bid / 8;
  return (xcd < rem) ? xcd * (per + 1) + local : rem * (per + 1) + (xcd - rem) * per + local;
}

}  // namespace
}  // namespace fademem
