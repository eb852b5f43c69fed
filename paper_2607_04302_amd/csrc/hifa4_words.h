// Packed-fp16 pieces of the quantizers that hold a group as eight words of
// eight values, one or more words a lane: the canonical Q^, K^ and V^ kernels
// and the paged cache's append.
#pragma once

#include "hifa4_packed.h"

namespace hifa4 {

typedef unsigned short u16x2_t __attribute__((ext_vector_type(2)));

__device__ __forceinline__ u16x2_t as_u16(h2_t x) { return __builtin_bit_cast(u16x2_t, x); }

// Level-2 and level-3 decisions of both halves of a pair of 4-block maxima a4
// whose 8-block maxima are a8, against the half- and quarter-range floors
// (per half): n = 2 - (E2 + E3) and the complement of E2, as 0..2 and 0..1 in
// 16-bit halves (non-negative fp16 values order like their bit patterns).
__device__ __forceinline__ void block_levels(h2_t a4, h2_t a8, h2_t th_h, h2_t th_q, u16x2_t& n, u16x2_t& not_e2) {
  const u16x2_t one = {1, 1};
  const u16x2_t big4 = __builtin_elementwise_min(__builtin_elementwise_sub_sat(as_u16(a4), as_u16(th_h)), one);
  not_e2 = __builtin_elementwise_min(__builtin_elementwise_sub_sat(as_u16(a8), as_u16(th_h)), one);
  const u16x2_t quarter = __builtin_elementwise_min(__builtin_elementwise_sub_sat(as_u16(a4), as_u16(th_q)), one);
  n = big4 + __builtin_elementwise_max(not_e2, quarter);
}

// fp16(a*R + C) per half (R fp32 per half, C fp16 per half): the code u sits in
// the low mantissa bits, since C = 1.5 * 2^(10-sh) has the grid 2^-sh as its
// last place.  Returns u in 0..7 per half.
__device__ __forceinline__ uint32_t codes2(h2_t a, float r0, float r1, u16x2_t n) {
  const u16x2_t c = n * (unsigned short)0x400 + (unsigned short)(kGrid10 & 0xFFFFu);
  h2_t y;
  asm("v_fma_mixlo_f16 %0, %1, %2, %4 op_sel:[0,0,0] op_sel_hi:[1,0,1]\n\t"
      "v_fma_mixhi_f16 %0, %1, %3, %4 op_sel:[1,0,1] op_sel_hi:[1,0,1]"
      : "=&v"(y)
      : "v"(a), "v"(r0), "v"(r1), "v"(__builtin_bit_cast(uint32_t, c)));
  return __builtin_bit_cast(uint32_t, y) & 0x00070007u;
}

// Sign-magnitude nibbles of both halves: u | sign << 3, a zero code without a
// sign (u + 7 carries into bit 3 exactly where u > 0).
__device__ __forceinline__ uint32_t nibbles2(uint32_t u, h2_t x) {
  const uint32_t s = (__builtin_bit_cast(uint32_t, x) >> 12) & 0x00080008u;
  return u | ((u + 0x00070007u) & s);
}

// fp16(k/s) for a pair of fp16 values from r0, r1 = RN32(1/s) of each: with the
// reciprocal taken two units in the last place (ulps) down and up, the fp32
// products bracket the exact quotient (two ulps exceed the reciprocal's half
// ulp and the product's rounding together), so where both ends round to the
// same fp16 the quotient does too.  `open`: the lanes in which they differ
// (about one value in 2000).
__device__ __forceinline__ h2_t divide2(h2_t k, float r0, float r1, unsigned long long& open) {
  const float d0 = __uint_as_float(__float_as_uint(r0) - 2u), u0 = __uint_as_float(__float_as_uint(r0) + 2u);
  const float d1 = __uint_as_float(__float_as_uint(r1) - 2u), u1 = __uint_as_float(__float_as_uint(r1) + 2u);
  float a, b, c, d;
  asm("v_fma_mix_f32 %0, %4, %5, 0 op_sel:[0,0,0] op_sel_hi:[1,0,0]\n\t"
      "v_fma_mix_f32 %1, %4, %6, 0 op_sel:[1,0,0] op_sel_hi:[1,0,0]\n\t"
      "v_fma_mix_f32 %2, %4, %7, 0 op_sel:[0,0,0] op_sel_hi:[1,0,0]\n\t"
      "v_fma_mix_f32 %3, %4, %8, 0 op_sel:[1,0,0] op_sel_hi:[1,0,0]"
      : "=&v"(a), "=&v"(b), "=&v"(c), "=&v"(d)
      : "v"(k), "v"(d0), "v"(d1), "v"(u0), "v"(u1));
  const h2_t lo = pack2_f16(a, b), hi = pack2_f16(c, d);
  open = __builtin_amdgcn_ballot_w64(__builtin_bit_cast(uint32_t, lo) != __builtin_bit_cast(uint32_t, hi));
  return lo;
}

// fp16(k/s) of N pairs: s and rs are the scales and their reciprocals.  A pair
// that is open in any lane takes the exact division.
template <int N, typename S, typename R>
__device__ __forceinline__ void divide_pairs(h2_t (&x)[N], const S& s, const R& rs) {
  h2_t y[N];
  unsigned long long open[N], any = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    y[i] = divide2(x[i], rs[2 * i], rs[2 * i + 1], open[i]);
    any |= open[i];
  }
  if (__builtin_expect(any != 0, 0)) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (open[i]) y[i] = h2_t{div_rn16((float)x[i][0], s[2 * i]), div_rn16((float)x[i][1], s[2 * i + 1])};
  }
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = y[i];
}

// Reductions over aligned sets of eight lanes (quad permutes, then the mirror
// of eight, which pairs the two quads).
template <typename F>
__device__ __forceinline__ uint32_t reduce8(uint32_t v, F f) {
  v = f(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, true));    // quad_perm [1,0,3,2]
  v = f(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xF, 0xF, true));    // quad_perm [2,3,0,1]
  return f(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x141, 0xF, 0xF, true));  // row_half_mirror
}

}  // namespace hifa4
