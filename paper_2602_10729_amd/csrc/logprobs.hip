// Log probabilities of given tokens, entropy, ranks and alternatives, and the
// gradient of the logits.
//
// One workgroup per row: the maximum, then the sums relative to it, then one
// sweep per alternative for the largest (value, lowest index) below the last.
#include "serving.h"

namespace bo {
namespace {

constexpr int kWg = 256;
constexpr float kNegInf = -__builtin_huge_valf();
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;
// A finite stand-in for -inf where it is multiplied by a probability of 0.
constexpr float kLow = -1e30f;

// Orders (value, index): larger value first, lower index among equals; the
// unsigned order of the result is the wanted one. -0 and +0 are equal.
__device__ __forceinline__ unsigned long long pack_key(float v, unsigned j) {
  const unsigned u = __float_as_uint(v + 0.0f);
  const unsigned o = (u & 0x80000000u) ? ~u : (u | 0x80000000u);
  return (static_cast<unsigned long long>(o) << 32) | (0xFFFFFFFFu - j);
}
__device__ __forceinline__ float key_value(unsigned long long k) {
  const unsigned o = static_cast<unsigned>(k >> 32);
  return __uint_as_float((o & 0x80000000u) ? (o & 0x7FFFFFFFu) : ~o);
}

template <typename V, typename F>
__device__ V block_reduce(V v, V* lds, F f) {
  for (int off = 32; off > 0; off >>= 1) v = f(v, __shfl_xor(v, off));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  v = lds[0];
  for (int i = 1; i < kWg / 64; ++i) v = f(v, lds[i]);
  return v;
}

template <int TYPE>
__global__ __launch_bounds__(kWg) void k_logprobs(LogprobArgs a) {
  using El = Elem<TYPE>;
  __shared__ float fl[kWg / 64];
  __shared__ int il[kWg / 64];
  __shared__ unsigned long long ul[kWg / 64];
  const auto add = [](auto x, auto y) { return x + y; };
  const auto larger = [](auto x, auto y) { return x > y ? x : y; };
  for (int64_t row = blockIdx.x; row < a.T; row += gridDim.x) {
    const typename El::T* x = static_cast<const typename El::T*>(a.logits) + row * a.stride;
    const int64_t tok = a.tokens ? a.tokens[row] : -1;
    const bool has = tok >= 0 && tok < a.V;
    const float xt = has ? El::load(x[tok]) : 0.0f;
    float m = kNegInf;
    for (int64_t j = threadIdx.x; j < a.V; j += kWg) m = fmaxf(m, El::load(x[j]));
    m = block_reduce(m, fl, [](float p, float q) { return fmaxf(p, q); });
    const float mr = m == kNegInf ? 0.0f : m, c = a.it * kLog2e;
    float s = 0.0f, w = 0.0f;
    int ahead = 0;
    for (int64_t j = threadIdx.x; j < a.V; j += kWg) {
      const float v = El::load(x[j]), t = (v - mr) * c, e = exp2f(t);
      s += e;
      w += e * fmaxf(t, kLow);
      ahead += (v > xt || (v == xt && j < tok)) ? 1 : 0;
    }
    s = block_reduce(s, fl, add);
    w = block_reduce(w, fl, add);
    ahead = block_reduce(ahead, il, add);
    const float ls = logf(s);
    if (threadIdx.x == 0) {
      a.stats[2 * row] = m;
      a.stats[2 * row + 1] = ls;
      a.entropy[row] = m == kNegInf && s == 0.0f ? 0.0f : ls - w / s * kLn2;
      float lp = 0.0f;
      if (has) lp = xt == kNegInf && s == s ? kNegInf : (xt - m) * a.it - ls;
      if (tok >= a.V) lp = __builtin_nanf("");
      a.logprob[row] = lp;
      a.rank[row] = has && xt > kNegInf ? ahead + 1 : 0;
    }
    unsigned long long last = ~0ull;
    for (int i = 0; i < a.top; ++i) {
      unsigned long long best = 0ull;
      for (int64_t j = threadIdx.x; j < a.V; j += kWg) {
        const float v = El::load(x[j]);
        if (v > kNegInf) {
          const unsigned long long k = pack_key(v, static_cast<unsigned>(j));
          if (k < last && k > best) best = k;
        }
      }
      best = block_reduce(best, ul, larger);
      if (threadIdx.x == 0) {
        const float v = key_value(best);
        a.top_ids[row * a.top + i] = best ? static_cast<int>(0xFFFFFFFFu - static_cast<unsigned>(best)) : -1;
        a.top_logprobs[row * a.top + i] = best ? (v - m) * a.it - ls : kNegInf;
      }
      last = best;
    }
    __syncthreads();
  }
}

template <int TYPE>
__global__ __launch_bounds__(kWg) void k_logprobs_grad(LogprobGradArgs a) {
  using El = Elem<TYPE>;
  __shared__ float onehot[BO_MAX_ALTERNATIVES + 1];
  __shared__ int at[BO_MAX_ALTERNATIVES + 1];
  for (int64_t row = blockIdx.x; row < a.T; row += gridDim.x) {
    const typename El::T* x = static_cast<const typename El::T*>(a.logits) + row * a.stride;
    typename El::T* out = static_cast<typename El::T*>(a.out) + row * a.out_stride;
    const float m = a.stats[2 * row], ls = a.stats[2 * row + 1];
    const int64_t tok = a.tokens ? a.tokens[row] : -1;
    const bool has = tok >= 0 && tok < a.V;
    const float gl = has && a.g_logprob ? a.g_logprob[row] : 0.0f;
    const float gh = a.g_entropy ? a.g_entropy[row] : 0.0f;
    float sum = gl;
    for (int i = 0; i < a.top; ++i) {
      const int id = a.top_ids[row * a.top + i];
      if (id >= 0 && id < a.V) sum += a.g_top[row * a.top + i];
    }
    __syncthreads();
    for (int i = threadIdx.x; i <= a.top; i += kWg) {
      const int64_t id = i < a.top ? a.top_ids[row * a.top + i] : (has ? tok : -1);
      at[i] = id >= 0 && id < a.V ? static_cast<int>(id) : -1;
      onehot[i] = i < a.top ? a.g_top[row * a.top + i] : gl;
    }
    __syncthreads();
    const bool empty = m == kNegInf && ls == kNegInf;
    float base = -sum - gh * a.entropy[row];
    if (tok >= a.V) base = __builtin_nanf("");
    for (int64_t j = threadIdx.x; j < a.V; j += kWg) {
      float g = 0.0f;
      if (!empty) {
        const float u = (El::load(x[j]) - m) * a.it - ls;
        g = exp2f(u * kLog2e) * (base - gh * fmaxf(u, kLow));
        for (int i = 0; i <= a.top; ++i)
          if (at[i] == j) g += onehot[i];
        g *= a.it;
      }
      out[j] = El::store(g);
    }
  }
}

template <typename F32, typename BF16, typename F16>
void by_type(int type, F32 f, BF16 b, F16 h) {
  if (type == BO_TYPE_F32) f();
  else if (type == BO_TYPE_BF16) b();
  else h();
}

}  // namespace

int64_t logprob_workspace(int64_t, int64_t, int) { return 0; }

hipError_t launch_logprobs(const LogprobArgs& a, hipStream_t st) {
  const dim3 grid(static_cast<unsigned>(a.T < (1 << 20) ? a.T : (1 << 20)));
  by_type(a.type, [&] { k_logprobs<BO_TYPE_F32><<<grid, kWg, 0, st>>>(a); },
          [&] { k_logprobs<BO_TYPE_BF16><<<grid, kWg, 0, st>>>(a); },
          [&] { k_logprobs<BO_TYPE_F16><<<grid, kWg, 0, st>>>(a); });
  return hipGetLastError();
}

hipError_t launch_logprobs_grad(const LogprobGradArgs& a, hipStream_t st) {
  const dim3 grid(static_cast<unsigned>(a.T < (1 << 20) ? a.T : (1 << 20)));
  by_type(a.type, [&] { k_logprobs_grad<BO_TYPE_F32><<<grid, kWg, 0, st>>>(a); },
          [&] { k_logprobs_grad<BO_TYPE_BF16><<<grid, kWg, 0, st>>>(a); },
          [&] { k_logprobs_grad<BO_TYPE_F16><<<grid, kWg, 0, st>>>(a); });
  return hipGetLastError();
}

}  // namespace bo
