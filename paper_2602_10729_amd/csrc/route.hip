// Routing to experts: scores, the choice of groups and experts, weights, and
// the gradient of the router's logits.
//
// Choice: a row is held by `lpt` neighbouring lanes (a power of two up to 32),
// each with 32 consecutive experts at most, so a wave takes 64 / lpt rows. An
// expert is one 64-bit key, larger for a larger value and, among equals, for a
// lower index: the value's order-preserving code and the index are the
// mantissa of a double in [2^52, 2^53), so that keys compare and exchange with
// one v_max_f64 and one v_min_f64, which this chip runs at the fp32 rate. A
// lane sorts its experts by eights, keeping the K >= top best; lanes then
// exchange lists by halves (the larger of a_i and b_{K-1-i} are the K best of
// two falling lists, and form a bitonic sequence that log2 K steps sort).
//
// What bounds it: the instructions of the sort, not memory. 32768 x 256 in 8
// groups (19 MB, 4 us at a copy's rate) take 17.4 us; 65537 x 61 fp32 take 8.2
// and their gradient 11.0 (35 MB, 7 us); a decoding step's 16 x 64 take 3.7, a
// launch's latency and a wave's way through the code once.
#include <algorithm>
#include <type_traits>

#include "serving.h"

namespace bo {
namespace {

constexpr int kWg = 256;
constexpr float kNegInf = -__builtin_huge_valf();
constexpr float kLog2e = 1.44269504088896340736f;
constexpr int kSpan = 32;                    // experts a lane holds
// Four waves on every SIMD (32768 x 256 takes 17 us; with eight, in half the
// experts a lane, 22; 65537 x 61 takes 8.3, with two 10.1, with eight 9.8).
constexpr int64_t kLanesWanted = 4096 * 64;
constexpr unsigned kExpTwo52 = 0x43300000u;  // high word of 2^52

// ---- keys -----------------------------------------------------------------
// Exchanges go through LDS' swizzle, not DPP: a DPP read needs wait states
// after the write, which the compiler does not know of behind inline assembly.
template <int XOR>
__device__ __forceinline__ int swap_lanes(int v) {
  return __builtin_amdgcn_ds_swizzle(v, (XOR << 10) | 0x1F);
}
template <int XOR>
__device__ __forceinline__ float swap_lanes(float v) {
  return __int_as_float(swap_lanes<XOR>(__float_as_int(v)));
}
template <int XOR>
__device__ __forceinline__ double swap_lanes(double v) {
  return __hiloint2double(swap_lanes<XOR>(__double2hiint(v)), swap_lanes<XOR>(__double2loint(v)));
}
__device__ __forceinline__ double kmax(double a, double b) {
  double d;
  asm("v_max_f64 %0, %1, %2" : "=v"(d) : "v"(a), "v"(b));
  return d;
}
__device__ __forceinline__ double kmin(double a, double b) {
  double d;
  asm("v_min_f64 %0, %1, %2" : "=v"(d) : "v"(a), "v"(b));
  return d;
}
// the larger first
__device__ __forceinline__ void order(double& a, double& b) {
  const double hi = kmax(a, b), lo = kmin(a, b);
  a = hi;
  b = lo;
}
// A bitonic sequence into falling order.
template <int N>
__device__ __forceinline__ void bitonic(double* a) {
#pragma unroll
  for (int h = N / 2; h > 0; h >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i)
      if ((i & h) == 0) order(a[i], a[i + h]);
}
// Any sequence into falling order: halves, the second taken backwards.
template <int N>
__device__ __forceinline__ void sort(double* a) {
  if constexpr (N > 1) {
    sort<N / 2>(a);
    sort<N / 2>(a + N / 2);
#pragma unroll
    for (int i = 0; i < N / 2; ++i) order(a[i], a[N - 1 - i]);
    // both halves are bitonic, every key of the first above the second's
    bitonic<N / 2>(a);
    bitonic<N / 2>(a + N / 2);
  }
}
// a: the K best of a and of the falling list b[0..NB), NB <= K.
template <int K, int NB>
__device__ __forceinline__ void keep_best(double* a, const double* b) {
#pragma unroll
  for (int i = 0; i < NB; ++i) a[K - 1 - i] = kmax(a[K - 1 - i], b[i]);
  bitonic<K>(a);
}

// The value's key with the place among the lane's experts. v is no NaN; -inf is
// none.
__device__ __forceinline__ double make_key(float v, int place) {
  const unsigned o = code_of(v);
  return __hiloint2double(static_cast<int>(kExpTwo52 | (o >> 12)),
                          static_cast<int>((o << 20) | static_cast<unsigned>(31 - place)));
}

// (the code of -inf is 0x007FFFFF, the next one 0x00800000)
__device__ __forceinline__ bool is_choice(double key) {
  return static_cast<unsigned>(__double2hiint(key)) >= (kExpTwo52 | (0x00800000u >> 12));
}

// ---- reductions over a row's lanes ------------------------------------------
template <typename F>
__device__ __forceinline__ float row_reduce(float v, int lpt, F f) {
  if (lpt > 1) v = f(v, swap_lanes<1>(v));
  if (lpt > 2) v = f(v, swap_lanes<2>(v));
  if (lpt > 4) v = f(v, swap_lanes<4>(v));
  if (lpt > 8) v = f(v, swap_lanes<8>(v));
  if (lpt > 16) v = f(v, swap_lanes<16>(v));
  return v;
}
// Every lane of the row takes the K best of the row's lists (one copy of the
// code for all distances: the kernel runs its code once, so its fetch counts).
template <int K>
__device__ __forceinline__ void join_lists(double* a, int lane, int lpt) {
#pragma unroll 1
  for (int x = 1; x < lpt; x <<= 1) {
    const int from = (lane ^ x) << 2;
    double b[K];
#pragma unroll
    for (int i = 0; i < K; ++i)
      b[i] = __hiloint2double(__builtin_amdgcn_ds_bpermute(from, __double2hiint(a[i])),
                              __builtin_amdgcn_ds_bpermute(from, __double2loint(a[i])));
    keep_best<K, K>(a, b);
  }
}

// A lane's SPAN elements of a row of E from `first` on, -inf past the end.
// Every lane loads (a load that only some lanes make waits for the one before
// it): what would reach past the row starts earlier and is moved up.
template <int TYPE, int SPAN>
__device__ __forceinline__ void load_span(Vec<TYPE> (&q)[SPAN / Vec<TYPE>::kVec],
                                          const typename Elem<TYPE>::T* x, int first, int E) {
  constexpr int KV = Vec<TYPE>::kVec;
  if (E >= KV) {
#pragma unroll
    for (int p = 0; p < SPAN / KV; ++p) q[p].load(x + min(first + p * KV, E - KV));
#pragma unroll
    for (int p = 0; p < SPAN / KV; ++p) {
      const int past = first + p * KV - (E - KV);
      if (__any(past > 0)) q[p].drop(max(past, 0));
    }
  } else {
#pragma unroll
    for (int p = 0; p < SPAN / KV; ++p) q[p].fill_masked();
    if (first == 0) q[0].load_part(x, E);
  }
}

// Expert j's place in LDS: a gap after every 32 keeps lanes that walk groups of
// 32 off one another's bank.
__device__ __forceinline__ int at_of(int j) { return j + (j >> 5); }

// LDS words of a row of n places.
__host__ __device__ constexpr int row_words(int n) { return n + (n >> 5) + 1; }

// The larger two of a falling pair and of another.
__device__ __forceinline__ void top_two(float& b1, float& b2, float o1, float o2) {
  b2 = max2(b2 < o2 ? o2 : b2, b1 < o1 ? b1 : o1);
  b1 = max2(b1, o1);
}

// How the groups lie: none (or none dropped), each of whole eights, or anyhow.
enum { kNoGroups, kBlockGroups, kAnyGroups };

// 1 << shift lanes a row, NB eights of experts each. `div` is 65536 / eights per group, rounded up
// (kBlockGroups): eight / (eights per group) = eight * div >> 16 for up to 128.
template <int TYPE, int K, int GROUPS, int NB>
__global__ __launch_bounds__(kWg, K <= 8 && GROUPS != kAnyGroups ? 4 : 1) void k_route(RouteArgs a, int shift, int div) {
  using El = Elem<TYPE>;
  using V = Vec<TYPE>;
  constexpr int SPAN = 8 * NB;
  // per wave: choices and what they weigh, and before them the groups' work
  constexpr int kChoice = 2 * 64 * K;
  constexpr int kGroup = GROUPS == kNoGroups ? 0 : GROUPS == kBlockGroups ? 64 * NB * 4
                                                                         : 64 * (SPAN + 1) + 64 * SPAN / 2;
  __shared__ float lds[kWg / 64][kChoice > kGroup ? kChoice : kGroup];
  __shared__ alignas(16) float lds_bias[BO_MAX_EXPERTS + 8 * kSpan];
  const auto fmax2 = [](float p, float q) { return fmaxf(p, q); };
  const auto fadd2 = [](float p, float q) { return p + q; };
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lpt = 1 << shift, sub = lane & (lpt - 1), slot = lane >> shift, rows = 64 >> shift;
  const int first = sub * SPAN;
  const bool scored = GROUPS != kNoGroups || a.bias;      // else the logits are compared
  if (a.bias) {
    for (int j = threadIdx.x; j < SPAN * lpt; j += kWg) lds_bias[j] = j < a.E ? a.bias[j] : kNegInf;
    __syncthreads();
  }
  const int64_t step = (int64_t)gridDim.x * (kWg / 64) * rows;
  for (int64_t base = (int64_t)blockIdx.x * (kWg / 64) * rows; base < a.T; base += step) {
    const int64_t row = base + wave * rows + slot;
    const bool live = row < a.T;
    const typename El::T* x =
        static_cast<const typename El::T*>(a.logits) + (live ? row : 0) * a.stride;
    V q[SPAN / V::kVec];
    load_span<TYPE, SPAN>(q, x, first, a.E);
    const auto logit = [&](int i) { return q[i / V::kVec].get(i % V::kVec); };
    // softmax statistics; a row with a NaN or +inf has no choice
    float m = 0.0f, inv = 1.0f;
    bool bad = false;
    if (a.score == BO_SCORE_SOFTMAX) {
      m = kNegInf;
#pragma unroll
      for (int i = 0; i < SPAN; ++i) {
        m = max2(m, logit(i));
        bad = bad || __builtin_isnan(logit(i));
      }
      m = row_reduce(m, lpt, fmax2);
      bad = bad || m == __builtin_huge_valf();
      bad = (__ballot(bad) >> (slot << shift) & (~0ull >> (64 - lpt))) != 0;
      m = m == kNegInf ? 0.0f : m;
      if (scored || !a.renorm) {
        float t = 0.0f;
#pragma unroll
        for (int i = 0; i < SPAN; ++i) t += __builtin_amdgcn_exp2f((logit(i) - m) * kLog2e);
        inv = 1.0f / row_reduce(t, lpt, fadd2);
      }
    }
    const auto score = [&](float t) {
      if (a.score == BO_SCORE_SIGMOID)
        return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-t * kLog2e));
      return __builtin_amdgcn_exp2f((t - m) * kLog2e) * inv;
    };
    // what is compared, eight experts at a time; -inf where one cannot be chosen
    const auto values = [&](int at, int b, float (&v)[8]) {      // (block b, held at place `at`)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = logit(8 * at + e);
      if (scored) {
        if (a.score == BO_SCORE_SIGMOID) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            v[e] = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-v[e] * kLog2e));
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = __builtin_amdgcn_exp2f((v[e] - m) * kLog2e) * inv;
        }
        if (a.bias) {
          const float4* t = reinterpret_cast<const float4*>(lds_bias + first + 8 * b);
          const float4 lo = t[0], hi = t[1];
          v[0] += lo.x; v[1] += lo.y; v[2] += lo.z; v[3] += lo.w;
          v[4] += hi.x; v[5] += hi.y; v[6] += hi.z; v[7] += hi.w;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = logit(8 * at + e) > kNegInf ? v[e] : kNegInf;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = fmaxf(v[e], kNegInf);     // a NaN is no choice
    };
    float kept[GROUPS == kBlockGroups ? SPAN : 1];
    float* val = lds[wave] + slot * lpt * (SPAN + 1);
    // a group that top_groups or more come before is dropped
    const auto dropped = [&](const unsigned* grp, int g) {
      const unsigned mine = grp[g];
      int before = 0;
      for (int o = 0; o < a.groups; ++o) before += grp[o] > mine || (grp[o] == mine && o < g);
      return before >= a.top_groups;
    };
    if constexpr (GROUPS == kBlockGroups) {
      // the best two of each eight, then of each group
      float2* two = reinterpret_cast<float2*>(lds[wave]) + slot * lpt * NB;
      unsigned* grp = reinterpret_cast<unsigned*>(lds[wave] + 64 * NB * 2) + slot * lpt * NB;
      unsigned* drop = grp + 64 * NB;
      const int eights = a.E / a.groups / 8, at = first >> 3;
#pragma unroll
      for (int b = 0; b < NB; ++b) {
          float v[8];
          values(b, b, v);
          float b1 = kNegInf, b2 = kNegInf;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            kept[8 * b + e] = v[e];
            b2 = __builtin_amdgcn_fmed3f(b1, b2, v[e]);
            b1 = max2(b1, v[e]);
          }
          two[at + b] = make_float2(b1, b2);
        }
      __syncthreads();
      for (int g = sub; g < a.groups; g += lpt) {
        float2 best = two[g * eights];
        for (int e = 1; e < eights; ++e) top_two(best.x, best.y, two[g * eights + e].x, two[g * eights + e].y);
        grp[g] = code_of(a.group_best == 2 ? best.x + best.y : best.x);
      }
      __syncthreads();
      for (int g = sub; g < a.groups; g += lpt) drop[g] = dropped(grp, g);
      __syncthreads();
#pragma unroll
      for (int b = 0; b < NB; ++b) {
          const bool out = drop[min((at + b) * div >> 16, a.groups - 1)];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float v = !a.bias && kept[8 * b + e] > kNegInf ? logit(8 * b + e) : kept[8 * b + e];
            kept[8 * b + e] = out ? kNegInf : v;
          }
        }
      __syncthreads();                      // (the choices take this memory's place)
    }
    if constexpr (GROUPS == kAnyGroups) {
      const int per = a.E / a.groups;
      unsigned* grp = reinterpret_cast<unsigned*>(lds[wave] + 64 * (SPAN + 1)) + slot * lpt * (SPAN / 2);
#pragma unroll
      for (int b = 0; b < NB; ++b) {
          float v[8];
          values(b, b, v);
#pragma unroll
          for (int e = 0; e < 8; ++e) val[at_of(first + 8 * b) + e] = v[e];
        }
      __syncthreads();
      for (int g = sub; g < a.groups; g += lpt) {
        float b1 = kNegInf, b2 = kNegInf;
        for (int e = g * per; e < (g + 1) * per; ++e) top_two(b1, b2, val[at_of(e)], kNegInf);
        grp[g] = code_of(a.group_best == 2 ? b1 + b2 : b1);
      }
      __syncthreads();
      for (int g = sub; g < a.groups; g += lpt)
        if (dropped(grp, g))
          for (int e = g * per; e < (g + 1) * per; ++e) val[at_of(e)] = kNegInf;
      __syncthreads();
    }
    // the lane's best, eight experts at a time in one copy of the code: what comes
    // next moves to the front
    double best[K];
    constexpr int B = K < 8 ? K : 8;
#pragma unroll
    for (int i = 0; i < K; ++i) best[i] = 0.0;
#pragma unroll 1
    for (int b = 0; b < NB; ++b) {
      float v[8];
      if constexpr (GROUPS == kBlockGroups) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = kept[e];
#pragma unroll
        for (int i = 0; i < SPAN - 8; ++i) kept[i] = kept[i + 8];
      } else {
        if constexpr (GROUPS == kAnyGroups) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            v[e] = val[at_of(first + 8 * b) + e];
            if (!a.bias) v[e] = v[e] > kNegInf ? logit(e) : kNegInf;
          }
        } else {
          values(0, b, v);
        }
#pragma unroll
        for (int p = 0; p < (SPAN - 8) / V::kVec; ++p) q[p] = q[p + 8 / V::kVec];
      }
#pragma unroll
      for (int p = 0; p < 8 / B; ++p) {
        double key[B];
#pragma unroll
        for (int e = 0; e < B; ++e) key[e] = make_key(v[p * B + e], 8 * b + p * B + e);
        sort<B>(key);
        keep_best<K, B>(best, key);
      }
    }
    // the row's best: the lane joins the key
#pragma unroll
    for (int i = 0; i < K; ++i)
      best[i] = __hiloint2double(__double2hiint(best[i]),
                                 __double2loint(best[i]) | ((31 - sub) << 5));
    join_lists<K>(best, lane, lpt);
    if constexpr (GROUPS == kAnyGroups) __syncthreads();
    // weights: lane `sub` takes choices sub, sub + lpt, ..
    int* cid = reinterpret_cast<int*>(lds[wave]) + slot * K;
    float* cw = lds[wave] + 64 * K + slot * K;
    if (sub == 0) {
#pragma unroll
      for (int i = 0; i < K; ++i) {
        const int lo = __double2loint(best[i]);
        cid[i] = is_choice(best[i]) && !bad ? (31 - ((lo >> 5) & 31)) * SPAN + (31 - (lo & 31)) : -1;
      }
    }
    __syncthreads();
    float hi = kNegInf, total = 0.0f, norm = 1.0f;
    for (int n = sub; n < a.top; n += lpt) {
      const int id = cid[n];
      const float t = id >= 0 ? El::load(x[id]) : kNegInf;
      hi = fmaxf(hi, t);
      cw[n] = t;
    }
    if (a.renorm) {
      // relative to the largest chosen score, so that none underflows
      hi = row_reduce(hi, lpt, fmax2);
      if (a.score == BO_SCORE_SIGMOID) hi = fminf(hi, 0.0f);
    }
    for (int n = sub; n < a.top; n += lpt) {
      const float t = cw[n];
      float w;
      if (!a.renorm || (a.score == BO_SCORE_SIGMOID && t > 0.0f)) w = score(t);
      else w = __builtin_amdgcn_exp2f((t - hi) * kLog2e);
      if (a.renorm && a.score == BO_SCORE_SIGMOID && !(t > 0.0f))
        w *= __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(t * kLog2e));
      w = cid[n] >= 0 ? w : 0.0f;
      cw[n] = w;
      total += w;
    }
    if (a.renorm) {
      total = row_reduce(total, lpt, fadd2);
      norm = total > 0.0f ? 1.0f / total : 0.0f;
    }
    if (live)
      for (int n = sub; n < a.top; n += lpt) {
        a.ids[row * a.top + n] = cid[n];
        a.weights[row * a.top + n] = a.scale * (cw[n] * norm);
      }
    __syncthreads();
  }
}

// The same lanes hold a row: each choice's term goes to its expert's place in
// LDS, then every lane adds the dense part (softmax, not renormalised: -scale
// s_j sum_k s_k g_k) to its experts' and writes them. A lane takes choices sub,
// sub + lpt, .., C at most.
template <int TYPE, int C, int NB>
__global__ __launch_bounds__(kWg) void k_route_grad(RouteGradArgs a, int shift) {
  using El = Elem<TYPE>;
  using V = Vec<TYPE>;
  constexpr int SPAN = 8 * NB, kParts = SPAN / V::kVec;
  extern __shared__ float lds_term[];       // [waves][rows][row_words]
  const auto fmax2 = [](float p, float q) { return fmaxf(p, q); };
  const auto fadd2 = [](float p, float q) { return p + q; };
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lpt = 1 << shift, sub = lane & (lpt - 1), slot = lane >> shift, rows = 64 >> shift;
  const int first = sub * SPAN;
  const int64_t step = (int64_t)gridDim.x * (kWg / 64) * rows;
  const bool softmax = a.score == BO_SCORE_SOFTMAX, dense = softmax && !a.renorm;
  float* term = lds_term + (wave * rows + slot) * row_words(SPAN << shift);
  for (int64_t base = (int64_t)blockIdx.x * (kWg / 64) * rows; base < a.T; base += step) {
    const int64_t row = base + wave * rows + slot;
    const bool live = row < a.T;
    const int64_t r = live ? row : 0;
    const typename El::T* x = static_cast<const typename El::T*>(a.logits) + r * a.stride;
    // a lane's choices: expert, logit, the weight's gradient
    int id[C];
    float l[C], g[C];
#pragma unroll
    for (int t = 0; t < C; ++t) {
      const int n = min(t * lpt + sub, a.top - 1);
      id[t] = a.ids[r * a.top + n];
      g[t] = a.g[r * a.top + n];
      if (id[t] >= a.E || t * lpt + sub >= a.top) id[t] = -1;
    }
#pragma unroll
    for (int t = 0; t < C; ++t) l[t] = El::load(x[max(id[t], 0)]);
    V q[kParts];
    float m = 0.0f, inv = 1.0f;
    if (dense) {
      load_span<TYPE, SPAN>(q, x, first, a.E);
      m = kNegInf;
#pragma unroll
      for (int i = 0; i < SPAN; ++i) m = max2(m, q[i / V::kVec].get(i % V::kVec));
      m = row_reduce(m, lpt, fmax2);
      m = m == kNegInf ? 0.0f : m;
      float t = 0.0f;
#pragma unroll
      for (int i = 0; i < SPAN; ++i)
        t += __builtin_amdgcn_exp2f((q[i / V::kVec].get(i % V::kVec) - m) * kLog2e);
      inv = 1.0f / row_reduce(t, lpt, fadd2);
    }
#pragma unroll
    for (int i = 0; i < SPAN; ++i) term[at_of(first) + i] = 0.0f;
    const auto sigm = [](float t) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-t * kLog2e)); };
    float hi = kNegInf, any = 0.0f;
#pragma unroll
    for (int t = 0; t < C; ++t) {
      hi = id[t] >= 0 ? fmaxf(hi, l[t]) : hi;
      any = id[t] >= 0 ? 1.0f : any;
    }
    if (a.renorm) {
      hi = row_reduce(hi, lpt, fmax2);
      if (!softmax) hi = fminf(hi, 0.0f);
    }
    any = row_reduce(any, lpt, fmax2);
    // the weights before their common factor, as in the forward pass
    const auto weight = [&](float t) {
      if (dense) return __builtin_amdgcn_exp2f((t - m) * kLog2e) * inv;
      if (!a.renorm) return sigm(t);
      if (!softmax && t > 0.0f) return sigm(t);
      const float w = __builtin_amdgcn_exp2f((t - hi) * kLog2e);
      return softmax ? w : w * sigm(-t);
    };
    float total = 0.0f, wg = 0.0f, w[C];
#pragma unroll
    for (int t = 0; t < C; ++t) {
      w[t] = id[t] >= 0 ? weight(l[t]) : 0.0f;
      total += w[t];
      wg = id[t] >= 0 ? fmaf(w[t], g[t], wg) : wg;
    }
    if (a.renorm) total = row_reduce(total, lpt, fadd2);
    if (a.renorm || dense) wg = row_reduce(wg, lpt, fadd2);
    const float norm = a.renorm ? 1.0f / total : 1.0f, mean = a.renorm ? wg * norm : 0.0f;
    __syncthreads();
#pragma unroll
    for (int t = 0; t < C; ++t)
      if (id[t] >= 0) {
        const float d = a.scale * (w[t] * norm) * (g[t] - mean);
        term[at_of(id[t])] = softmax ? d : d * sigm(-l[t]);
      }
    __syncthreads();
    typename El::T* out = static_cast<typename El::T*>(a.out) + r * a.out_stride;
    const float back = dense && any > 0.0f ? -a.scale * wg * inv : 0.0f;
#pragma unroll
    for (int p = 0; p < kParts; ++p) {
      const int j = first + p * V::kVec;
      float v[V::kVec];
#pragma unroll
      for (int e = 0; e < V::kVec; ++e) v[e] = term[at_of(first) + p * V::kVec + e];
      if (dense) {
#pragma unroll
        for (int e = 0; e < V::kVec; ++e) {
          const float s = __builtin_amdgcn_exp2f((q[p].get(e) - m) * kLog2e);
          v[e] = back != 0.0f ? fmaf(back, s, v[e]) : v[e];
        }
      }
      q[p].set_all(v);
      if (live && j + V::kVec <= a.E) q[p].store(out + j);
      else if (live && j < a.E) q[p].store_part(out + j, a.E - j);
    }
    __syncthreads();
  }
}

// As few lanes a row as hold it; more, down to eight experts each, while that
// leaves the chip short of waves.
int lanes_shift(int64_t T, int E) {
  int shift = 0;
  while ((kSpan << shift) < E) ++shift;
  while ((8 << shift) < E && shift < 5 && (T << shift) < kLanesWanted) ++shift;
  return shift;
}
unsigned row_blocks(int64_t T, int shift) {
  const int64_t rows = (64 >> shift) * (kWg / 64);
  return static_cast<unsigned>(std::min<int64_t>((T + rows - 1) / rows, 1 << 20));
}

// The smallest of 1, 2, 4, 8, 16, 32 that is at least n, as a constant.
template <typename F>
void by_size(int n, F f) {
  if (n <= 1) f(std::integral_constant<int, 1>());
  else if (n <= 2) f(std::integral_constant<int, 2>());
  else if (n <= 4) f(std::integral_constant<int, 4>());
  else if (n <= 8) f(std::integral_constant<int, 8>());
  else if (n <= 16) f(std::integral_constant<int, 16>());
  else f(std::integral_constant<int, 32>());
}
// Eights of experts that a lane holds (1, 2 or 4).
int eights_of(int E, int shift) { return (((E + 7) >> 3) + (1 << shift) - 1) >> shift; }

template <int TYPE>
hipError_t launch_typed(const RouteArgs& a, hipStream_t st) {
  const int shift = lanes_shift(a.T, a.E);
  const unsigned grid = row_blocks(a.T, shift);
  const int per = a.E / a.groups, eights = per / 8, div = eights ? (65536 + eights - 1) / eights : 0;
  // (the best of the best groups of one expert are the best experts, top_groups >= top)
  const bool grouped = per > 1 && a.top_groups < a.groups;
  by_size(a.top, [&](auto k) {
    by_size(eights_of(a.E, shift), [&](auto nb) {
      // (one code for lists of one and two; groups of any size, and long lists,
      // are rare: they take the widest lanes)
      constexpr int K = decltype(k)::value < 2 ? 2 : decltype(k)::value;
      constexpr int NB = K > 8 || decltype(nb)::value > 4 ? 4 : decltype(nb)::value;
      if (!grouped) k_route<TYPE, K, kNoGroups, NB><<<grid, kWg, 0, st>>>(a, shift, 0);
      else if (per % 8 == 0) k_route<TYPE, K, kBlockGroups, NB><<<grid, kWg, 0, st>>>(a, shift, div);
      else k_route<TYPE, K, kAnyGroups, 4><<<grid, kWg, 0, st>>>(a, shift, 0);
    });
  });
  return hipGetLastError();
}

template <int TYPE>
hipError_t launch_typed(const RouteGradArgs& a, hipStream_t st) {
  const int shift = lanes_shift(a.T, a.E), lpt = 1 << shift;
  const unsigned grid = row_blocks(a.T, shift);
  by_size((a.top + lpt - 1) / lpt, [&](auto c) {
    by_size(eights_of(a.E, shift), [&](auto nb) {
      constexpr int C = decltype(c)::value;
      constexpr int NB = C > 8 || decltype(nb)::value > 4 ? 4 : decltype(nb)::value;
      const size_t lds = sizeof(float) * (kWg >> shift) * row_words((8 * NB) << shift);
      k_route_grad<TYPE, C, NB><<<grid, kWg, lds, st>>>(a, shift);
    });
  });
  return hipGetLastError();
}

}  // namespace

hipError_t launch_route(const RouteArgs& a, hipStream_t st) {
  if (a.type == BO_TYPE_F32) return launch_typed<BO_TYPE_F32>(a, st);
  if (a.type == BO_TYPE_BF16) return launch_typed<BO_TYPE_BF16>(a, st);
  return launch_typed<BO_TYPE_F16>(a, st);
}

hipError_t launch_route_grad(const RouteGradArgs& a, hipStream_t st) {
  if (a.type == BO_TYPE_F32) return launch_typed<BO_TYPE_F32>(a, st);
  if (a.type == BO_TYPE_BF16) return launch_typed<BO_TYPE_BF16>(a, st);
  return launch_typed<BO_TYPE_F16>(a, st);
}

}  // namespace bo
