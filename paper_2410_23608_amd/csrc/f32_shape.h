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
// The larger tiles where there are enough of them for most units.  us, 32 | 64: 1000 x 2800 -> 1000 (256 tiles of 64) backward 109 | 87,
// 3000 x 5760 -> 320 (235) 193 | 160, weights of 1600 x 400 (175) 182 | 190.
inline bool f32_wide(long rows, long cols) { return ((rows + 63) / 64) * ((cols + 63) / 64) >= 192; }
inline long f32_tiles(long rows, long cols, int edge) { return ((rows + edge - 1) / edge) * ((cols + edge - 1) / edge); }

// A thread an element instead of tiles, where the contraction is short: the same chain, the same bits.  A step of the tiles holds 32 or 64
// contraction elements of 32 or 64 rows and columns, whatever of them there are, and a workgroup has two rounds of loads before its first
// product. us, a thread an element | tiles: forward 1000000 x 1 -> 1 4.1 | 97, 300000 x 4 -> 4 6.0 | 34, 300000 x 16 -> 1 14 | 36, x 8 ->
// 16 73 | 36, x 4 -> 64 82 | 43, 20000 x 16 -> 4 3.4 | 7.0, x 1 -> 512 20.3 | 23.6, x 4 -> 512 47 | 24, 1000 x 8 -> 64 3.0 | 3.7, x 32 -> 4
// 4.1 | 3.8; input side, 300000 rows, 8 elements of 16 columns 22 | 46, of 64 83 | 50, 32 of 4 46 | 51; weights 64 x 64, 1 row 2.2 | 4.9, 8
// 3.5 | 4.9, 16 5.2 | 5.0, 1000 x 1000, 2 5.6 | 6.1, 4 7.4 | 6.1.  The times below are lines through these, in us.
enum class F32Side { kForward, kInput, kWeight };
inline bool f32_by_element(F32Side side, long rows, long cols, long kc) {
  const double n = (double)rows * (double)cols, k = (double)kc, tiles64 = (double)f32_tiles(rows, cols, 64);
  double elements, start = f32_wide(rows, cols) ? 5.0 : 3.5;
  if (side == F32Side::kWeight) {
    start = 4.8;
    elements = 1.9 + 0.2 * k + 1e-6 * n * (1.8 + 0.72 * k);
  } else {
    // (forward neighbouring lanes read along rows of W: up to 16 bytes, or few rows, cost less)
    const double each = side == F32Side::kInput ? 1.3 + 0.3 * k : kc <= 4 ? 0.7 + 1.1 * k : (cols < 8 ? 1.1 : 1.85) * k;
    elements = 2.0 + 0.07 * k + 1e-6 * std::max(n * each, 2.5 * (double)rows * k);
  }
  return elements <= start + 0.012 * k + (side == F32Side::kInput ? 0.008 : 0.006) * tiles64 + 0.45e-6 * n;
}

}  // namespace spa
