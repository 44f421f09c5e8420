// Division by a number that the host knows (attn_bias.h, rotary.hip, cross_attention.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace spa {

// x / d for 0 <= x < 2^31 by one high product: with 2^s >= d > 2^(s-1), M = floor(2^(31+s) / d) + 1 < 2^32 is at most 2^s / d too
// large in units of its last place, which times x is below 2^(31+s) / d: the quotient is exact.  (d = 1: M = 0.)
struct Divisor {
  uint32_t d, M, shift;
};
inline Divisor divisor(uint32_t d) {
  uint32_t s = 0;
  while ((1ull << s) < d) ++s;
  return d == 1 ? Divisor{1, 0, 0} : Divisor{d, (uint32_t)((1ull << (31 + s)) / d + 1), s - 1};
}
__device__ __forceinline__ uint32_t quotient(uint32_t x, const Divisor& d) { return d.M == 0 ? x : __umulhi(x, d.M) >> d.shift; }

}  // namespace spa
