#pragma once
#include "common.h"

namespace marl {

// Division of n < 2^31 by a number fixed at launch: a product and a shift.  (magic d = 2^shift + e with 0 < e <= 2^(shift - 31), so n magic / 2^shift
// is less than n / d + 1 / d.)
struct Divisor {
  uint32_t d = 1, magic = 0;
  int shift = 0;
  __device__ __forceinline__ uint32_t operator()(uint32_t n) const { return __umulhi(2 * n, magic) >> (shift - 31); }
};
inline Divisor divisor(uint32_t d) {
  Divisor r;
  r.d = d;
  int lg = 0;
  while ((1u << lg) < d) ++lg;
  r.shift = 31 + lg;
  r.magic = (uint32_t)(((uint64_t)1 << r.shift) / d + 1);
  return r;
}

}  // namespace marl
