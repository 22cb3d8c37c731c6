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

// A row's i-th vector: where H ends inside it, it is moved back to end with the row
// (its first `skip` elements stand in the vector before as well). A row shorter
// than a vector has one, of H elements.
template <int TYPE>
struct RowVec {
  static constexpr int kVec = Vec<TYPE>::kVec;
  using T = typename Elem<TYPE>::T;
  int64_t h;
  int skip, n;
  __device__ __forceinline__ RowVec(int64_t i, int64_t H)
      : h(H >= kVec ? min(i * kVec, H - kVec) : 0), skip(static_cast<int>(i * kVec - h)),
        n(H >= kVec ? kVec : static_cast<int>(H)) {}
  template <bool STREAM = false>
  __device__ __forceinline__ void load(Vec<TYPE>& v, const T* row) const {
    if (n == kVec) v.template load<STREAM>(row + h);
    else v.load_part(row, n);
  }
  template <bool STREAM = false>
  __device__ __forceinline__ void store(const Vec<TYPE>& v, T* row) const {
    if (n == kVec) v.template store<STREAM>(row + h);
    else v.store_part(row, n);
  }
};
__device__ __forceinline__ int64_t vectors(int64_t H, int vec) { return (H + vec - 1) / vec; }

template <int TYPE>
__device__ __forceinline__ Vec<TYPE> zero_vec() {
  Vec<TYPE> v;
  v.q[0] = v.q[1] = v.q[2] = v.q[3] = 0;
  return v;
}

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
