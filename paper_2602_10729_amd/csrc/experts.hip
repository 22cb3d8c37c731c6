// Tokens into rows grouped by expert, the experts' outputs back under the
// router's weights, and the gradients.
//
//   grouped[position[t,k]] = x[t]                   (a row that no pair fills: 0)
//   y[t] = sum_k w[t,k] rows[position[t,k]]         (fp32, k rising, rounded once)
//   grad_rows[position[t,k]] = w[t,k] grad[t],  grad_w[t,k] = grad[t] . rows[position[t,k]]
//
// The gradient of the first is the second without weights. All of it is moving
// rows of H elements, and memory bounds it: 262144 rows of 2048 bf16 (1.07 GB) from
// or to 32768 tokens take 244 us (gather), 226 (combine) and 487 (gradient), 5.0 TB/s.
// The experts' rows are read past the caches, being read once. Rows that are
// written pass them by above kStreamBytes, where the next product would find few of
// them there (1184 against 1251 us for the four passes of a training step).
// Gathering row by row of the output instead reads tokens `top` times: 300 us; a
// wave a pair beside its token's others: 335.
#include "rows.h"

namespace bo {
namespace {

// Sum over the wave, in every lane; the order is fixed.
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int off = 32; off; off >>= 1) v += __shfl_xor(v, off);
  return v;
}

// The lanes whose pair of the token has a row, and each one's row in its lane.
struct Pairs {
  int at;
  unsigned long long there;
  __device__ __forceinline__ Pairs(const int32_t* __restrict__ position, int64_t t, int top, int64_t R) {
    const int lane = threadIdx.x & 63;
    at = lane < top ? position[t * top + lane] : -1;
    there = __ballot(at >= 0 && at < R);
  }
  // the lowest of those left, and its row
  __device__ __forceinline__ int next(int64_t& row) {
    const int k = __ffsll(there) - 1;
    there &= there - 1;
    row = __builtin_amdgcn_readlane(at, k);
    return k;
  }
};

// 2^split waves a token, vector after vector of its row: read once and written to
// each of its places. The same waves clear row p for the token's pairs p where no
// pair fills that row (order[p] < 0): p runs over all rows.
template <int TYPE, bool STREAM>
__global__ __launch_bounds__(kRowWg) void k_expert_gather(
    const typename Elem<TYPE>::T* __restrict__ x, int64_t T, int64_t H, int64_t stride, int top,
    const int32_t* __restrict__ order, int64_t R, const int32_t* __restrict__ position,
    typename Elem<TYPE>::T* __restrict__ out, int64_t out_stride, int split) {
  const int lane = threadIdx.x & 63;
  const int64_t vecs = vectors(H, Vec<TYPE>::kVec);
  for (int64_t unit = first_unit(); unit < T << split; unit += units()) {
    const int64_t t = unit >> split;
    const Pairs all(position, t, top, R);
    const int64_t p = t * top + lane;
    const unsigned long long clear = __ballot(lane < top && p < R && order[p] < 0);
    for (int64_t i = (unit & ((1 << split) - 1)) * 64 + lane; i < vecs; i += static_cast<int64_t>(64) << split) {
      const RowVec<TYPE> r(i, H);
      Vec<TYPE> v;
      r.load(v, x + t * stride);
      Pairs pairs = all;
      while (pairs.there) {
        int64_t at;
        pairs.next(at);
        r.template store<STREAM>(v, out + at * out_stride);
      }
      for (unsigned long long c = clear; c; c &= c - 1)
        r.template store<STREAM>(zero_vec<TYPE>(), out + (t * top + __ffsll(c) - 1) * out_stride);
    }
  }
}

// 2^split waves a token; the rows of up to eight pairs are on their way at once.
template <int TYPE>
__global__ __launch_bounds__(kRowWg) void k_expert_combine(
    const typename Elem<TYPE>::T* __restrict__ rows, int64_t R, int64_t H, int64_t stride,
    const int32_t* __restrict__ position, int64_t T, int top, const float* __restrict__ weights,
    typename Elem<TYPE>::T* __restrict__ out, int64_t out_stride, int split) {
  constexpr int kVec = Vec<TYPE>::kVec;
  const int lane = threadIdx.x & 63;
  const int64_t vecs = vectors(H, kVec);
  for (int64_t unit = first_unit(); unit < T << split; unit += units()) {
    const int64_t t = unit >> split;
    const Pairs all(position, t, top, R);
    const int w = __float_as_int(weights && lane < top ? weights[t * top + lane] : 1.0f);
    for (int64_t i = (unit & ((1 << split) - 1)) * 64 + lane; i < vecs; i += static_cast<int64_t>(64) << split) {
      const RowVec<TYPE> r(i, H);
      float sum[kVec];
#pragma unroll
      for (int e = 0; e < kVec; ++e) sum[e] = 0.0f;
      Pairs pairs = all;
      const auto take = [&](auto count) {
        constexpr int N = decltype(count)::value;
        Vec<TYPE> v[N];
        float f[N];
#pragma unroll
        for (int c = 0; c < N; ++c) {
          int64_t at;
          f[c] = __int_as_float(__builtin_amdgcn_readlane(w, pairs.next(at)));
          r.template load<true>(v[c], rows + at * stride);
        }
#pragma unroll
        for (int c = 0; c < N; ++c)
#pragma unroll
          for (int e = 0; e < kVec; ++e) sum[e] = fmaf(f[c], v[c].get(e), sum[e]);
      };
      int left = __popcll(pairs.there);
      for (; left >= 8; left -= 8) take(std::integral_constant<int, 8>());
      if (left & 4) take(std::integral_constant<int, 4>());
      if (left & 2) take(std::integral_constant<int, 2>());
      if (left & 1) take(std::integral_constant<int, 1>());
      Vec<TYPE> o;
      o.set_all(sum);
      r.store(o, out + t * out_stride);
    }
  }
}

// A workgroup a token, whose waves take its pairs in turn: the token's row of grad
// comes from the caches for all but one of them.
template <int TYPE, bool STREAM>
__global__ __launch_bounds__(512) void k_expert_combine_grad(
    const typename Elem<TYPE>::T* __restrict__ grad, int64_t T, int64_t H, int64_t grad_stride,
    const typename Elem<TYPE>::T* __restrict__ rows, int64_t R, int64_t stride, int top,
    const int32_t* __restrict__ order, const int32_t* __restrict__ position,
    const float* __restrict__ weights, typename Elem<TYPE>::T* __restrict__ grad_rows,
    int64_t grad_rows_stride, float* __restrict__ grad_weights) {
  constexpr int kVec = Vec<TYPE>::kVec;
  const int lane = threadIdx.x & 63, waves = blockDim.x >> 6;
  const int64_t vecs = vectors(H, kVec);
  for (int64_t t = blockIdx.x; t < T; t += gridDim.x) {
    for (int k = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); k < top; k += waves) {
      const int64_t p = t * top + k;
      const int32_t at = position[p];
      const bool there = at >= 0 && at < R;
      const bool clear = grad_rows && p < R && order[p] < 0;
      const float w = weights ? weights[p] : 1.0f;
      float dot = 0.0f;
      if (there)
#pragma unroll 2
        for (int64_t i = lane; i < vecs; i += 64) {
          const RowVec<TYPE> r(i, H);
          Vec<TYPE> g;
          r.load(g, grad + t * grad_stride);
          if (grad_weights) {
            Vec<TYPE> z;
            r.template load<true>(z, rows + at * stride);
#pragma unroll
            for (int e = 0; e < kVec; ++e)
              if (e >= r.skip && e < r.n) dot = fmaf(g.get(e), z.get(e), dot);
          }
          if (grad_rows) {
            float d[kVec];
#pragma unroll
            for (int e = 0; e < kVec; ++e) d[e] = w * g.get(e);
            Vec<TYPE> o;
            o.set_all(d);
            r.template store<STREAM>(o, grad_rows + at * grad_rows_stride);
          }
        }
      if (clear)
        for (int64_t i = lane; i < vecs; i += 64)
          RowVec<TYPE>(i, H).template store<STREAM>(zero_vec<TYPE>(), grad_rows + p * grad_rows_stride);
      if (grad_weights) {
        dot = wave_sum(dot);
        if (lane == 0) grad_weights[p] = dot;
      }
    }
  }
}

template <typename F>
void by_stream(bool stream, F&& f) {
  if (stream) f(std::true_type());
  else f(std::false_type());
}
constexpr int64_t kStreamBytes = (int64_t)160 << 20;
bool streams(const ExpertArgs& a) {
  return a.R * a.H * static_cast<int64_t>(type_bytes(a.type)) > kStreamBytes;
}

}  // namespace

hipError_t launch_expert_gather(const ExpertArgs& a, hipStream_t st) {
  const int split = row_split(a.type, a.T, a.H);
  by_type(a.type, [&](auto ty) {
    by_stream(streams(a), [&](auto past) {
      using E = typename Elem<decltype(ty)::value>::T;
      k_expert_gather<decltype(ty)::value, decltype(past)::value><<<row_blocks(a.T << split), kRowWg, 0, st>>>(
          static_cast<const E*>(a.tokens), a.T, a.H, a.stride, a.top, a.order, a.R, a.position,
          static_cast<E*>(a.out), a.out_stride, split);
    });
  });
  return hipGetLastError();
}

hipError_t launch_expert_combine(const ExpertArgs& a, hipStream_t st) {
  const int split = row_split(a.type, a.T, a.H);
  by_type(a.type, [&](auto ty) {
    using E = typename Elem<decltype(ty)::value>::T;
    k_expert_combine<decltype(ty)::value><<<row_blocks(a.T << split), kRowWg, 0, st>>>(
        static_cast<const E*>(a.rows), a.R, a.H, a.rows_stride, a.position, a.T, a.top, a.weights,
        static_cast<E*>(a.out), a.out_stride, split);
  });
  return hipGetLastError();
}

hipError_t launch_expert_combine_grad(const ExpertArgs& a, hipStream_t st) {
  const unsigned waves = a.top > 4 ? 8 : a.top > 2 ? 4 : a.top;
  const unsigned grid = static_cast<unsigned>(a.T < (1 << 22) ? a.T : 1 << 22);
  by_type(a.type, [&](auto ty) {
    by_stream(streams(a), [&](auto past) {
      using E = typename Elem<decltype(ty)::value>::T;
      k_expert_combine_grad<decltype(ty)::value, decltype(past)::value><<<grid, 64 * waves, 0, st>>>(
          static_cast<const E*>(a.tokens), a.T, a.H, a.stride, static_cast<const E*>(a.rows), a.R,
          a.rows_stride, a.top, a.order, a.position, a.weights, static_cast<E*>(a.out), a.out_stride,
          a.grad_weights);
    });
  });
  return hipGetLastError();
}

}  // namespace bo
