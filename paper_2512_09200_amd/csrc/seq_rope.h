// Rotary angle of a position, shared by the batch kernels and the
// single-event step.
#pragma once
#include "seq.h"

namespace lat {

// cos and sin of 2 pi * position * turns.  The product and its reduction to
// [-1/2, 1/2] are in 64 bits: in 32 the angle of position 3e7 would be off by
// whole radians.  What is left goes through sinpi / cospi in 32 bits (2 ulp).
__device__ inline float2 rope_cs(int pos, double turns) {
  const double t = (double)pos * turns;
  const float r = (float)(t - rint(t));
  float2 v;
  sincospif(2.f * r, &v.y, &v.x);
  return v;
}

}  // namespace lat
