// OCP e4m3 codes: the hardware conversions, shared by the FP8 linear layers,
// the norm's 8-bit output and the 8-bit ring caches.
#pragma once
#include "common.h"

namespace lat {

constexpr float E4M3_MAX = 448.f;

// Four fp32 values (already scaled) -> four e4m3 codes in one word, byte e
// = value e: round to nearest even, saturating at +-448.
__device__ inline uint32_t e4m3x4(float a, float b, float c, float d) {
  auto cl = [](float v) { return __builtin_amdgcn_fmed3f(v, -E4M3_MAX, E4M3_MAX); };
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(cl(a), cl(b), 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(cl(c), cl(d), w, true);
  return (uint32_t)w;
}

}  // namespace lat
