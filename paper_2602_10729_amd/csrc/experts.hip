// Tokens into rows grouped by expert, the experts' outputs back under the
// router's weights, and the gradients.
//
//   grouped[position[t,k]] = x[t]                   (a row that no pair fills: 0)
//   y[t] = sum_k w[t,k] rows[position[t,k]]         (fp32, k rising, rounded once)
//   grad_rows[position[t,k]] = w[t,k] grad[t],  grad_w[t,k] = grad[t] . rows[position[t,k]]
//
// The gradient of the first is the second without weights. All of it is moving
// rows of H elements: what bounds it is memory.
#include "rows.h"

namespace bo {
namespace {

// Sum over the wave, in every lane; the order is fixed.
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int off = 32; off; off >>= 1) v += __shfl_xor(v, off);
  return v;
}

// 2^split waves a token, vector after vector of its row: read once and written to
// each of its places. The same waves clear row p for the token's pairs p where no
// pair fills that row (order[p] < 0): p runs over all rows.
template <int TYPE>
__global__ __launch_bounds__(kRowWg) void k_expert_gather(
    const typename Elem<TYPE>::T* __restrict__ x, int64_t T, int64_t H, int64_t stride, int top,
    const int32_t* __restrict__ order, int64_t R, const int32_t* __restrict__ position,
    typename Elem<TYPE>::T* __restrict__ out, int64_t out_stride, int split) {
  constexpr int kVec = Vec<TYPE>::kVec;
  const int lane = threadIdx.x & 63;
  Vec<TYPE> zero;
  zero.q[0] = zero.q[1] = zero.q[2] = zero.q[3] = 0;
  for (int64_t unit = first_unit(); unit < T << split; unit += units()) {
    const int64_t t = unit >> split;
    for (int64_t h = ((unit & ((1 << split) - 1)) * 64 + lane) * kVec; h < H; h += (64 * kVec) << split) {
      const int n = static_cast<int>(min<int64_t>(kVec, H - h));
      Vec<TYPE> v;
      if (n == kVec) v.load(x + t * stride + h);
      else v.load_part(x + t * stride + h, n);
      for (int k = 0; k < top; ++k) {
        const int64_t p = t * top + k;
        const int32_t at = position[p];
        if (at >= 0 && at < R) {
          if (n == kVec) v.store(out + at * out_stride + h);
          else v.store_part(out + at * out_stride + h, n);
        }
        if (p < R && order[p] < 0) {
          if (n == kVec) zero.store(out + p * out_stride + h);
          else zero.store_part(out + p * out_stride + h, n);
        }
      }
    }
  }
}

// 2^split waves a token.
template <int TYPE>
__global__ __launch_bounds__(kRowWg) void k_expert_combine(
    const typename Elem<TYPE>::T* __restrict__ rows, int64_t R, int64_t H, int64_t stride,
    const int32_t* __restrict__ position, int64_t T, int top, const float* __restrict__ weights,
    typename Elem<TYPE>::T* __restrict__ out, int64_t out_stride, int split) {
  constexpr int kVec = Vec<TYPE>::kVec;
  const int lane = threadIdx.x & 63;
  for (int64_t unit = first_unit(); unit < T << split; unit += units()) {
    const int64_t t = unit >> split;
    for (int64_t h = ((unit & ((1 << split) - 1)) * 64 + lane) * kVec; h < H; h += (64 * kVec) << split) {
      const int n = static_cast<int>(min<int64_t>(kVec, H - h));
      float sum[kVec];
#pragma unroll
      for (int e = 0; e < kVec; ++e) sum[e] = 0.0f;
      for (int k = 0; k < top; ++k) {
        const int32_t at = position[t * top + k];
        if (at < 0 || at >= R) continue;
        const float w = weights ? weights[t * top + k] : 1.0f;
        Vec<TYPE> v;
        if (n == kVec) v.load(rows + at * stride + h);
        else v.load_part(rows + at * stride + h, n);
#pragma unroll
        for (int e = 0; e < kVec; ++e) sum[e] = fmaf(w, v.get(e), sum[e]);
      }
      Vec<TYPE> o;
      o.set_all(sum);
      if (n == kVec) o.store(out + t * out_stride + h);
      else o.store_part(out + t * out_stride + h, n);
    }
  }
}

// A wave a pair.
template <int TYPE>
__global__ __launch_bounds__(kRowWg) void k_expert_combine_grad(
    const typename Elem<TYPE>::T* __restrict__ grad, int64_t T, int64_t H, int64_t grad_stride,
    const typename Elem<TYPE>::T* __restrict__ rows, int64_t R, int64_t stride, int top,
    const int32_t* __restrict__ order, const int32_t* __restrict__ position,
    const float* __restrict__ weights, typename Elem<TYPE>::T* __restrict__ grad_rows,
    int64_t grad_rows_stride, float* __restrict__ grad_weights) {
  constexpr int kVec = Vec<TYPE>::kVec;
  const int lane = threadIdx.x & 63;
  Vec<TYPE> zero;
  zero.q[0] = zero.q[1] = zero.q[2] = zero.q[3] = 0;
  for (int64_t p = first_unit(); p < T * top; p += units()) {
    const int64_t t = p / top;
    const int32_t at = position[p];
    const bool there = at >= 0 && at < R;
    const bool clear = grad_rows && p < R && order[p] < 0;
    const float w = weights ? weights[p] : 1.0f;
    float dot = 0.0f;
    for (int64_t h = static_cast<int64_t>(lane) * kVec; h < H; h += 64 * kVec) {
      const int n = static_cast<int>(min<int64_t>(kVec, H - h));
      if (there) {
        Vec<TYPE> g;
        if (n == kVec) g.load(grad + t * grad_stride + h);
        else g.load_part(grad + t * grad_stride + h, n);
        if (grad_weights) {
          Vec<TYPE> z;
          if (n == kVec) z.load(rows + at * stride + h);
          else z.load_part(rows + at * stride + h, n);
#pragma unroll
          for (int e = 0; e < kVec; ++e)
            if (e < n) dot = fmaf(g.get(e), z.get(e), dot);
        }
        if (grad_rows) {
          float d[kVec];
#pragma unroll
          for (int e = 0; e < kVec; ++e) d[e] = w * g.get(e);
          Vec<TYPE> o;
          o.set_all(d);
          if (n == kVec) o.store(grad_rows + at * grad_rows_stride + h);
          else o.store_part(grad_rows + at * grad_rows_stride + h, n);
        }
      }
      if (clear) {
        if (n == kVec) zero.store(grad_rows + p * grad_rows_stride + h);
        else zero.store_part(grad_rows + p * grad_rows_stride + h, n);
      }
    }
    if (grad_weights) {
      dot = wave_sum(dot);
      if (lane == 0) grad_weights[p] = dot;
    }
  }
}

}  // namespace

hipError_t launch_expert_gather(const ExpertArgs& a, hipStream_t st) {
  const int split = row_split(a.type, a.T, a.H);
  by_type(a.type, [&](auto ty) {
    using E = typename Elem<decltype(ty)::value>::T;
    k_expert_gather<decltype(ty)::value><<<row_blocks(a.T << split), kRowWg, 0, st>>>(
        static_cast<const E*>(a.tokens), a.T, a.H, a.stride, a.top, a.order, a.R, a.position,
        static_cast<E*>(a.out), a.out_stride, split);
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
  by_type(a.type, [&](auto ty) {
    using E = typename Elem<decltype(ty)::value>::T;
    k_expert_combine_grad<decltype(ty)::value><<<row_blocks(a.T * a.top), kRowWg, 0, st>>>(
        static_cast<const E*>(a.tokens), a.T, a.H, a.stride, static_cast<const E*>(a.rows), a.R,
        a.rows_stride, a.top, a.order, a.position, a.weights, static_cast<E*>(a.out), a.out_stride,
        a.grad_weights);
  });
  return hipGetLastError();
}

}  // namespace bo
