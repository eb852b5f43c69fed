// What the attention kernels over the paged cache share.
#pragma once

#include "hifa4_device.h"
#include "hifa4_packed.h"
#include "hifa4_paged.h"

namespace hifa4 {

typedef float f4v_t __attribute__((ext_vector_type(4)));
typedef half_t h8v_t __attribute__((ext_vector_type(8)));

__device__ __forceinline__ int pages_of(const PagedCache& c, int b) {
  return b < c.batch ? (paged_len(c, b) + kPage - 1) / kPage : 0;
}
// q s to fp16, the exact product rounded once: the fp32 product made odd where
// it is not exact, so that the second rounding is the only one.
__device__ __forceinline__ half_t round_product(half_t q, float s) {
  const float p = (float)q * s, e = fmaf((float)q, s, -p);
  uint32_t b = __float_as_uint(p);
  if ((__float_as_uint(e) ^ b) & 0x80000000u) b -= e != 0.0f;      // |p| is above the product: one step toward zero
  return (half_t)__uint_as_float(e != 0.0f ? b | 1u : b);
}

// x and y lane values of (own, partner) exchanges
__device__ __forceinline__ float max_across_rows(float v) {      // over the four lanes of a column
  const Pair32 p = pair32(__float_as_uint(v));
  v = fmaxf(__uint_as_float(p.x), __uint_as_float(p.y));
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_across_rows(float v) {
  v = add_with_partner(v);
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// A scalar address that the compiler takes as given: sums with a lane's 32-bit
// offset stay in that form instead of becoming 64-bit vector additions.
typedef const __attribute__((address_space(1))) uint8_t* global_ptr;
__device__ __forceinline__ global_ptr scalar_address(const uint8_t* p) {
  global_ptr g = (global_ptr)p;
  asm("" : "+s"(g));
  return g;
}
template <typename T>
__device__ __forceinline__ T load_at(global_ptr p, uint32_t offset) {
  return *(const __attribute__((address_space(1))) T*)(p + offset);
}
// Nothing is scheduled across: a page's loads stay between the last use of the
// registers that they fill and the next page's, K's before V's, so that they
// need no registers of their own and a wait for K's does not wait for V's.
__device__ __forceinline__ void keep_order() { __builtin_amdgcn_sched_barrier(0); }

// The pages of a run, as their records: 64 table entries at a time, one a lane.
struct Pages {
  int mine, base;
};
__device__ __forceinline__ void load_pages(Pages& p, const PagedCache& c, int b, int from, int last, int lane) {
  p.base = from;
  p.mine = from + lane <= last ? c.table[(size_t)b * c.max_pages + from + lane] : -1;
}

template <int N, int kStep>
__device__ __forceinline__ void load_operands(h8v_t (&x)[N], const uint8_t* p, uint32_t lane) {
  constexpr int kSome = 4096 / kStep;
#pragma unroll
  for (int i = 0; i < N; i += kSome) {
    const global_ptr at = scalar_address(p + kStep * i);
#pragma unroll
    for (int u = 0; u < kSome; ++u) x[i + u] = load_at<h8v_t>(at, 16 * lane + kStep * u);
  }
}

}  // namespace hifa4
