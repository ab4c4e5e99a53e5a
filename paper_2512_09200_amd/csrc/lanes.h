// Joins over a wave's lanes in registers.
#pragma once
#include "common.h"

#include <type_traits>

namespace lat {

// f over the lane's LANES (2, 4, .. 64) neighbours.  Every level joins two equal
// shares, so all lanes get the same bits.
template <int LANES, typename V, typename F>
__device__ inline V lanes_join(V x, F f) {
  auto dpp = [&](auto ctrl) __attribute__((always_inline)) {
    const int o = __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(ctrl)::value, 0xf, 0xf, true);
    x = f(x, __builtin_bit_cast(V, o));
  };
  dpp(std::integral_constant<int, 0xB1>());        // lane ^ 1
  if constexpr (LANES >= 4) dpp(std::integral_constant<int, 0x4E>());      // lane ^ 2
  if constexpr (LANES >= 8) dpp(std::integral_constant<int, 0x141>());     // mirrored in 8
  if constexpr (LANES >= 16) dpp(std::integral_constant<int, 0x140>());    // mirrored in 16
  if constexpr (LANES >= 32) {
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    x = f(__builtin_bit_cast(V, (uint32_t)r[0]), __builtin_bit_cast(V, (uint32_t)r[1]));
  }
  if constexpr (LANES >= 64) {
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    x = f(__builtin_bit_cast(V, (uint32_t)r[0]), __builtin_bit_cast(V, (uint32_t)r[1]));
  }
  return x;
}
struct Add { template <typename V> __device__ inline V operator()(V a, V b) const { return a + b; } };
struct Max { template <typename V> __device__ inline V operator()(V a, V b) const { return a > b ? a : b; } };
template <> __device__ inline float Max::operator()(float a, float b) const { return fmaxf(a, b); }

}  // namespace lat
