// Sums over neighbouring lanes without LDS.
#pragma once
#include <hip/hip_runtime.h>

#include <type_traits>

namespace marl {

// Sum over L lanes next to each other, in all of them
template <int L>
__device__ __forceinline__ float sum_lanes(float v) {
  auto add = [&](auto control) { v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(control)::value, 0xf, 0xf, true)); };
  if constexpr (L >= 2) add(std::integral_constant<int, 0xB1>());   // the neighbour
  if constexpr (L >= 4) add(std::integral_constant<int, 0x4E>());   // the other pair
  if constexpr (L >= 8) add(std::integral_constant<int, 0x141>());  // mirrored in eight
  if constexpr (L >= 16) add(std::integral_constant<int, 0x140>()); // mirrored in sixteen
  if constexpr (L >= 32) v += __shfl_xor(v, 16);
  if constexpr (L >= 64) v += __shfl_xor(v, 32);
  return v;
}

}  // namespace marl
