// Kernels that move whole rows, a wave or a few a row: their launch and loops.
#pragma once

#include <type_traits>

#include "serving.h"

namespace bo {

constexpr int kRowWg = 256;
constexpr int kRowWaves = kRowWg / 64;

// The wave's number in the grid, and how many there are: units of work are
// taken in a loop, since a grid of one wave a unit may pass a launch's limit.
__device__ __forceinline__ int64_t first_unit() {
  return static_cast<int64_t>(blockIdx.x) * kRowWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
}
__device__ __forceinline__ int64_t units() { return static_cast<int64_t>(gridDim.x) * kRowWaves; }

inline unsigned row_blocks(int64_t units) {
  const int64_t b = (units + kRowWaves - 1) / kRowWaves;
  return static_cast<unsigned>(b < (1 << 22) ? b : 1 << 22);
}

// log2 of the waves that share a row of H elements: one, unless rows are too few
// to fill the device.
inline int row_split(int type, int64_t rows, int64_t H) {
  const int64_t vecs = 64 * (16 / static_cast<int64_t>(type_bytes(type)));
  int s = 0;
  while (s < 10 && (rows << s) < 8192 && (vecs << s) < H) ++s;
  return s;
}

template <typename F>
void by_type(int type, F&& f) {
  if (type == BO_TYPE_F32) f(std::integral_constant<int, BO_TYPE_F32>());
  else if (type == BO_TYPE_BF16) f(std::integral_constant<int, BO_TYPE_BF16>());
  else f(std::integral_constant<int, BO_TYPE_F16>());
}

}  // namespace bo
