// Paths of a token tree, by a warp.
#pragma once
#include "common.cuh"

namespace laser {

// The rows on the path from the root to row `lane` (mask[0]) and to row lane + 32 (mask[1]), themselves included: bit j = row j.  parents: of the
// nr (at most 64) rows of one tree; entry 0 is not read, and a parent that is not an earlier row ends its path.  Each of the six passes
// joins the paths of twice as many steps.
__device__ __forceinline__ void tree_paths(const int32_t* parents, int nr, int lane, unsigned long long (&mask)[2]) {
  int up[2];
#pragma unroll
  for (int y = 0; y < 2; ++y) {
    const int i = lane + 32 * y;
    up[y] = i > 0 && i < nr ? parents[i] : -1;
    if (up[y] >= i) up[y] = -1;
    mask[y] = 1ull << i;
  }
#pragma unroll 1
  for (int hop = 1; hop < 64; hop <<= 1) {
    unsigned long long more[2];
    int next[2];
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const int from = max(up[y], 0);
      const unsigned long long m0 = __shfl_sync(0xffffffffu, mask[0], from & 31), m1 = __shfl_sync(0xffffffffu, mask[1], from & 31);
      const int u0 = __shfl_sync(0xffffffffu, up[0], from & 31), u1 = __shfl_sync(0xffffffffu, up[1], from & 31);
      more[y] = up[y] < 0 ? 0ull : from < 32 ? m0 : m1;
      next[y] = up[y] < 0 ? -1 : from < 32 ? u0 : u1;
    }
#pragma unroll
    for (int y = 0; y < 2; ++y) { mask[y] |= more[y]; up[y] = next[y]; }
  }
}
// Of what tree_paths gave the warp: the path of any row.
__device__ __forceinline__ unsigned long long tree_path_of(const unsigned long long (&mask)[2], int row) {
  const unsigned long long a = __shfl_sync(0xffffffffu, mask[0], row & 31), b = __shfl_sync(0xffffffffu, mask[1], row & 31);
  return row < 32 ? a : b;
}

}  // namespace laser
