// What a split takes of the rows or keys that several workgroups share (cross_attention.h); no device code, so that a host program can ask
// it.
#pragma once

#include <hip/hip_runtime.h>

namespace spa {

struct Share {
  int from, n, live;             // first row, rows (<= 0: none), splits that have any
};
// A split's share of n rows in steps of STEP: all of them but the last have as many.  Nothing here passes 2^31 for n below it (a
// split behind the last has no first row).
template <int STEP>
__host__ __device__ inline Share share_of(int n, int splits, int split) {
  if (splits == 1) return {0, n, 1};
  if (n <= 0) return {0, 0, 1};
  const int steps = (n - 1) / STEP + 1, each = ((steps - 1) / splits + 1) * STEP, live = (n - 1) / each + 1;
  if (split >= live) return {0, 0, live};
  const int from = split * each, left = n - from;
  return {from, left < each ? left : each, live};
}

}  // namespace spa
