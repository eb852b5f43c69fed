// Rotary positions: the pair (x, y) of frequency w at position p becomes
//   (x cos pw - y sin pw, x sin pw + y cos pw) times a magnitude;
// the pairs are the channels (i, i + r/2) or (2i, 2i + 1) of the first r.
//
// Angles are counted in turns, as whole numbers of 2^-64: p times the frequency's
// turns, taken modulo one turn, is an integer product whose carry is dropped: exact at
// every position, for the frequency as it stands in the table.  That one comes out of fp64
// (2^-52 of itself, about), so that the angle is off by up to 2^-21 rad near position
// 2^31, and by less before (an angle in fp32 is off by 2^-24 of itself: by 0.06 rad at a
// million).  What is left of the angle after its quarter turns lies within pi/4, where the series of sine and cosine are cut behind the
// 9th and 10th power (errors below 2^-28).  The rotated values are rounded once, to
// fp16.
//
// Bound by the bytes: 20011 tokens of 24 heads of 256 channels (492 MB) in 96 us, 5.12
// TB/s, what a large copy reaches; 8192 tokens of 40 heads of 128 (168 MB) in 27 us, out
// of the last-level cache in part; 32 tokens 3.7 us, a chain of two loads.
#include "hifa4_rope.h"

#include <algorithm>

namespace hifa4 {

typedef half_t h8v_t __attribute__((ext_vector_type(8)));
typedef half_t h4v_t __attribute__((ext_vector_type(4)));

// (cos, sin) of 2 pi times the fraction t 2^-64.
__device__ __forceinline__ float2 unit_of(uint64_t t) {
  const uint32_t quarter = (uint32_t)((t + (1ull << 61)) >> 62);
  const int rest = (int)(uint32_t)((t - ((uint64_t)quarter << 62)) >> 32);       // within 2^29, units of 2^-32
  const float x = (float)rest * 0x1.921fb6p-30f, z = x * x;                     // 2 pi 2^-32
  float s = fmaf(z, 2.7557319e-6f, -1.9841270e-4f);
  s = fmaf(s, z, 8.3333333e-3f);
  s = fmaf(s, z, -1.6666667e-1f);
  s = fmaf(s * z, x, x);
  float c = fmaf(z, -2.7557319e-7f, 2.4801587e-5f);
  c = fmaf(c, z, -1.3888889e-3f);
  c = fmaf(c, z, 4.1666667e-2f);
  c = fmaf(c, z, -0.5f);
  c = fmaf(c, z, 1.0f);
  const float a = quarter & 1 ? s : c, b = quarter & 1 ? c : s;
  return make_float2((quarter + 1) & 2 ? -a : a, quarter & 2 ? -b : b);
}

// A lane keeps its place in the head (2 V channels: V and their partners, or V pairs,
// or 2 V that are only copied) and its V angles, and goes through the heads of one token.
template <int V, bool kInterleaved>
__global__ void __launch_bounds__(256) k_rope(RopeArgs a, int units, int slices) {
  typedef half_t vec_t __attribute__((ext_vector_type(V)));
  const long item = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int token = (int)(item / slices), slice = (int)(item % slices), lane = threadIdx.x & 63;
  if (token >= a.tokens) return;
  const int pos = a.pos[token];
  if (pos < 0) return;
  const int u = lane % units, per = 64 / units, heads = a.q.heads + a.k.heads;
  const bool rotates = u < a.rot / (2 * V);
  const int at0 = kInterleaved || !rotates ? 2 * V * u : V * u, at1 = kInterleaved || !rotates ? at0 + V : at0 + a.rot / 2;
  float2 w[V];
  if (rotates) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      w[i] = unit_of((uint64_t)pos * a.turns[V * u + i]);
      w[i].x *= a.magnitude;
      w[i].y *= a.transposed ? -a.magnitude : a.magnitude;
    }
  }
  const auto head_rows = [&](int h, const half_t*& x, half_t*& y) {
    const bool is_q = h < a.q.heads;
    const RopeRows& r = is_q ? a.q : a.k;
    const int head = is_q ? h : h - a.q.heads;
    x = r.x + token * r.x_stride + (long)head * a.D;
    y = r.y + token * r.y_stride + (long)head * a.D;
  };
  // kHeads of the lane's heads at a time, all fetched before the first is used (a call over
  // the 20011 tokens 95.5 us, one at a time 99.2; over the 8192 30.8 and 30.7)
  constexpr int kHeads = 4;
  const int step = slices * per;
  for (int h0 = slice * per + lane / units; h0 < heads; h0 += kHeads * step) {
    vec_t x0[kHeads], x1[kHeads];
    half_t* y[kHeads];
#pragma unroll
    for (int u = 0; u < kHeads; ++u) {
      const half_t* x;
      head_rows(min(h0 + u * step, heads - 1), x, y[u]);
      if (h0 + u * step < heads) {
        x0[u] = *reinterpret_cast<const vec_t*>(x + at0);
        x1[u] = *reinterpret_cast<const vec_t*>(x + at1);
      }
    }
#pragma unroll
    for (int u = 0; u < kHeads; ++u) {
      if (h0 + u * step >= heads) break;
      vec_t y0 = x0[u], y1 = x1[u];
      if (rotates) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
          if (kInterleaved) {
            const vec_t& in = i < V / 2 ? x0[u] : x1[u];
            const float p = (float)in[2 * i % V], q = (float)in[2 * i % V + 1];
            vec_t& out = i < V / 2 ? y0 : y1;
            out[2 * i % V] = (half_t)(p * w[i].x - q * w[i].y);
            out[2 * i % V + 1] = (half_t)(p * w[i].y + q * w[i].x);
          } else {
            const float p = (float)x0[u][i], q = (float)x1[u][i];
            y0[i] = (half_t)(p * w[i].x - q * w[i].y);
            y1[i] = (half_t)(p * w[i].y + q * w[i].x);
          }
        }
      }
      *reinterpret_cast<vec_t*>(y[u] + at0) = y0;
      *reinterpret_cast<vec_t*>(y[u] + at1) = y1;
    }
  }
}

template <int V>
static void launch(const RopeArgs& a, hipStream_t st) {
  const int units = a.D / (2 * V), per = 64 / units, heads = a.q.heads + a.k.heads;
  // a token's heads are shared out among waves while those of the tokens alone (each with
  // its angles) are fewer than the chip holds at 16 a CU
  const int most = (heads + per - 1) / per;
  const int slices = std::max(1, std::min(most, 4096 / std::max(1, a.tokens)));
  const long items = (long)a.tokens * slices;
  const dim3 grid((unsigned)((items + 3) / 4));
  if (a.interleaved)
    k_rope<V, true><<<grid, 256, 0, st>>>(a, units, slices);
  else
    k_rope<V, false><<<grid, 256, 0, st>>>(a, units, slices);
}

hipError_t launch_rope(const RopeArgs& a, hipStream_t st) {
  // (16-byte loads; 8-byte ones where half of rot_dim is no multiple of 8 channels)
  if (a.rot % 16 == 0)
    launch<8>(a, st);
  else
    launch<4>(a, st);
  return hipGetLastError();
}

}  // namespace hifa4
