// Rotary positions (hifa4_rope.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace hifa4 {

typedef _Float16 half_t;

struct RopeRows {
  const half_t* x;
  half_t* y;
  long x_stride, y_stride;      // elements from token to token
  int heads;
};
struct RopeArgs {
  RopeRows q, k;
  const int* pos;
  const uint64_t* turns;        // [rot / 2], turns per position in units of 2^-64
  int tokens, D, rot;
  bool interleaved, transposed;
  float magnitude;
};

hipError_t launch_rope(const RopeArgs& a, hipStream_t st);

}  // namespace hifa4
