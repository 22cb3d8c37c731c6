// Routing to experts: scores, the choice of groups and experts, weights, and
// the gradient of the router's logits.
//
// One wave per row; lane l holds experts l, l + 64, ..; each choice is a
// reduction of (value, lowest index) over the wave.
#include "serving.h"

namespace bo {
namespace {

constexpr int kWg = 256;
constexpr float kNegInf = -__builtin_huge_valf();
constexpr int kPerLane = BO_MAX_EXPERTS / 64;

__device__ __forceinline__ float wave_max(float v) {
  for (int off = 32; off > 0; off >>= 1) v = fmaxf(v, __shfl_xor(v, off));
  return v;
}
__device__ __forceinline__ float wave_sum(float v) {
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off);
  return v;
}
__device__ __forceinline__ unsigned long long wave_best(unsigned long long k) {
  for (int off = 32; off > 0; off >>= 1) {
    const unsigned long long o = __shfl_xor(k, off);
    k = o > k ? o : k;
  }
  return k;
}
__device__ __forceinline__ float sigmoid(float l) { return 1.0f / (1.0f + expf(-l)); }

template <int TYPE>
__global__ __launch_bounds__(kWg) void k_route(RouteArgs a) {
  using El = Elem<TYPE>;
  __shared__ float value[kWg / 64][BO_MAX_EXPERTS];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float* val = value[wave];
  const int64_t rows = (int64_t)gridDim.x * (kWg / 64);
  const int per = a.E / a.groups;
  for (int64_t row0 = (int64_t)blockIdx.x * (kWg / 64); row0 < a.T; row0 += rows) {
    const int64_t row = row0 + wave;
    const bool live = row < a.T;
    const typename El::T* x = static_cast<const typename El::T*>(a.logits) + (live ? row : 0) * a.stride;
    // the softmax statistics (a NaN stays in the sum)
    float m = kNegInf, sum = 1.0f;
    if (a.score == BO_SCORE_SOFTMAX) {
      for (int j = lane; j < a.E; j += 64) m = fmaxf(m, El::load(x[j]));
      m = wave_max(m);
      const float mr = m == kNegInf ? 0.0f : m;
      sum = 0.0f;
      for (int j = lane; j < a.E; j += 64) sum += expf(El::load(x[j]) - mr);
      sum = wave_sum(sum);
    }
    const auto score = [&](float l) {
      return a.score == BO_SCORE_SOFTMAX ? expf(l - (m == kNegInf ? 0.0f : m)) / sum : sigmoid(l);
    };
    __syncthreads();
    for (int j = lane; j < a.E; j += 64) {
      const float l = El::load(x[j]), s = score(l), b = a.bias ? a.bias[j] : 0.0f;
      float v = s + b;
      if (!(l > kNegInf) || !(b > kNegInf) || !(v > kNegInf)) v = kNegInf;
      val[j] = v;
    }
    __syncthreads();
    // groups: each of the top_groups best in turn leaves its mark
    unsigned long long kept[BO_MAX_EXPERTS / 64] = {};
    if (a.groups > 1) {
      unsigned long long gk[kPerLane];
      for (int i = 0; i < kPerLane; ++i) {
        gk[i] = 0;
        const int g = lane + 64 * i;
        if (g < a.groups) {
          float b1 = kNegInf, b2 = kNegInf;
          for (int e = 0; e < per; ++e) {
            const float v = val[g * per + e];
            b2 = fmaxf(b2, fminf(b1, v));
            b1 = fmaxf(b1, v);
          }
          gk[i] = pack_key(a.group_best == 2 ? b1 + b2 : b1, g);
        }
      }
      for (int n = 0; n < a.top_groups; ++n) {
        unsigned long long best = 0;
        for (int i = 0; i < kPerLane; ++i) best = gk[i] > best ? gk[i] : best;
        best = wave_best(best);
        const unsigned g = 0xFFFFFFFFu - static_cast<unsigned>(best);
        for (int i = 0; i < kPerLane; ++i) {
          if (gk[i] == best) gk[i] = 0;
          if (static_cast<int>(g >> 6) == i) kept[i] |= 1ull << (g & 63);
        }
      }
    }
    unsigned long long key[kPerLane];
    for (int i = 0; i < kPerLane; ++i) {
      const int j = lane + 64 * i;
      key[i] = 0;
      if (j < a.E && val[j] > kNegInf) {
        const float v = a.bias ? val[j] : El::load(x[j]);
        const int g = j / per;
        bool in = a.groups == 1;
        for (int q = 0; q < kPerLane; ++q)
          if ((g >> 6) == q) in = in || ((kept[q] >> (g & 63)) & 1);
        if (in) key[i] = pack_key(v, j);
      }
    }
    int mine = -1;
    for (int n = 0; n < a.top; ++n) {
      unsigned long long best = 0;
      for (int i = 0; i < kPerLane; ++i) best = key[i] > best ? key[i] : best;
      best = wave_best(best);
      for (int i = 0; i < kPerLane; ++i)
        if (key[i] == best) key[i] = 0;
      if (lane == n && best) mine = static_cast<int>(0xFFFFFFFFu - static_cast<unsigned>(best));
    }
    // weights: lane n holds choice n; relative to the largest chosen logit
    // where they are renormalised
    const float l = mine >= 0 ? El::load(x[mine]) : kNegInf;
    float w = 0.0f;
    if (a.renorm) {
      float top = wave_max(l);
      if (a.score == BO_SCORE_SIGMOID) top = fminf(top, 0.0f);
      if (mine >= 0) w = a.score == BO_SCORE_SOFTMAX ? expf(l - top)
                         : l > 0.0f ? sigmoid(l) : expf(l - top) / (1.0f + expf(l));
      const float total = wave_sum(w);
      if (mine >= 0) w = w / total;
    } else if (mine >= 0) {
      w = score(l);
    }
    if (live && lane < a.top) {
      a.ids[row * a.top + lane] = mine;
      a.weights[row * a.top + lane] = a.scale * w;
    }
  }
}

template <int TYPE>
__global__ __launch_bounds__(kWg) void k_route_grad(RouteGradArgs a) {
  using El = Elem<TYPE>;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t rows = (int64_t)gridDim.x * (kWg / 64);
  for (int64_t row = (int64_t)blockIdx.x * (kWg / 64) + wave; row < a.T; row += rows) {
    const typename El::T* x = static_cast<const typename El::T*>(a.logits) + row * a.stride;
    typename El::T* out = static_cast<typename El::T*>(a.out) + row * a.out_stride;
    int id = lane < a.top ? a.ids[row * a.top + lane] : -1;
    if (id >= a.E) id = -1;
    const bool on = id >= 0;
    const float g = on ? a.g[row * a.top + lane] : 0.0f;
    const float l = on ? El::load(x[id]) : kNegInf;
    const bool any = __ballot(on) != 0;
    float m = kNegInf, sum = 1.0f, s = 0.0f, w = 0.0f, inner = 0.0f, d = 0.0f;
    if (any && a.renorm) {
      float top = wave_max(l);
      if (a.score == BO_SCORE_SIGMOID) top = fminf(top, 0.0f);
      if (on) w = a.score == BO_SCORE_SOFTMAX ? expf(l - top)
                  : l > 0.0f ? sigmoid(l) : expf(l - top) / (1.0f + expf(l));
      const float total = wave_sum(w);
      if (on) w = w / total;
      const float mean = wave_sum(w * g);
      d = on ? a.scale * w * (g - mean) : 0.0f;
      if (on && a.score == BO_SCORE_SIGMOID) d *= sigmoid(-l);
    } else if (any && a.score == BO_SCORE_SIGMOID) {
      d = on ? a.scale * g * sigmoid(l) * sigmoid(-l) : 0.0f;
    } else if (any) {
      for (int j = lane; j < a.E; j += 64) m = fmaxf(m, El::load(x[j]));
      m = wave_max(m);
      sum = 0.0f;
      for (int j = lane; j < a.E; j += 64) sum += expf(El::load(x[j]) - m);
      sum = wave_sum(sum);
      s = on ? expf(l - m) / sum : 0.0f;
      inner = wave_sum(s * g);
      d = a.scale * s * g;
    }
    const bool dense = any && !a.renorm && a.score == BO_SCORE_SOFTMAX;
    for (int j0 = 0; j0 < a.E; j0 += 64) {
      const int j = j0 + lane;
      float v = 0.0f;
      if (dense && j < a.E) v = -a.scale * inner * (expf(El::load(x[j]) - m) / sum);
      for (int n = 0; n < a.top; ++n) {
        const int at = __shfl(id, n);
        const float dn = __shfl(d, n);
        if (at == j) v += dn;
      }
      if (j < a.E) out[j] = El::store(v);
    }
  }
}

template <typename F32, typename BF16, typename F16>
void by_type(int type, F32 f, BF16 b, F16 h) {
  if (type == BO_TYPE_F32) f();
  else if (type == BO_TYPE_BF16) b();
  else h();
}

unsigned row_blocks(int64_t T) {
  const int64_t b = (T + kWg / 64 - 1) / (kWg / 64);
  return static_cast<unsigned>(b < (1 << 20) ? b : (1 << 20));
}

}  // namespace

hipError_t launch_route(const RouteArgs& a, hipStream_t st) {
  const dim3 grid(row_blocks(a.T));
  by_type(a.type, [&] { k_route<BO_TYPE_F32><<<grid, kWg, 0, st>>>(a); },
          [&] { k_route<BO_TYPE_BF16><<<grid, kWg, 0, st>>>(a); },
          [&] { k_route<BO_TYPE_F16><<<grid, kWg, 0, st>>>(a); });
  return hipGetLastError();
}

hipError_t launch_route_grad(const RouteGradArgs& a, hipStream_t st) {
  const dim3 grid(row_blocks(a.T));
  by_type(a.type, [&] { k_route_grad<BO_TYPE_F32><<<grid, kWg, 0, st>>>(a); },
          [&] { k_route_grad<BO_TYPE_BF16><<<grid, kWg, 0, st>>>(a); },
          [&] { k_route_grad<BO_TYPE_F16><<<grid, kWg, 0, st>>>(a); });
  return hipGetLastError();
}

}  // namespace bo
