// Places, steps and tiles of the fp32 products (f32_tiles.h); no device code, so that a host program can ask them.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>

namespace spa {

// Numbers of rows, columns and contraction elements reach 2^31 - 1: what is past the end of the last tile or step has no place in an int.
// Element first + i of n, or the last one (0 <= first < n, i a place in a tile or step).
__host__ __device__ inline int f32_at(int first, int i, int n) {
  const unsigned at = (unsigned)first + (unsigned)i, last = (unsigned)n - 1u;
  return (int)(at < last ? at : last);
}
__host__ __device__ inline bool f32_inside(int first, int i, int n) { return i < n - first; }
__host__ __device__ inline int f32_steps(int n, int step) { return n > 0 ? (n - 1) / step + 1 : 0; }
// The larger tiles where there are enough of them for most units.  us, 32 | 64: 1000 x 2800 -> 1000 (256 tiles of 64) backward 109 | 87, 3000 x 5760 -> 320 (235) 193 | 160,
// weights of 1600 x 400 (175) 182 | 190.
inline bool f32_wide(long rows, long cols) { return ((rows + 63) / 64) * ((cols + 63) / 64) >= 192; }
inline long f32_tiles(long rows, long cols, int edge) { return ((rows + edge - 1) / edge) * ((cols + edge - 1) / edge); }

}  // namespace spa
