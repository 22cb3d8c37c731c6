// Log probabilities of given tokens, entropy, ranks and alternatives, and the
// gradient of the logits.
//
// Forward, one pass over a row, in powers of two: with c = log2(e) /
// temperature, a lane keeps a reference r near its largest logit, R = c r
// rounded, s = sum 2^t and w = sum t 2^t with t = c l - R (one fma). Lanes are
// joined by moving their sums to the row's maximum M:
//   s' = s 2^d,  w' = (w + d s) 2^d,  d = R - R_M;
// what R_M lost in rounding, c M - R_M, goes back into the logarithm of the
// sum. A masked logit makes t 2^t NaN, and so does a reference so far from 0
// (|c r| >= 2^24) that R says nothing about the last bits of an exponent: a chunk
// that ends with w not finite is summed again with t = c (l - r) + (c r - R), the
// second term 0 for a far reference, t bounded from below in the product; the
// wave stays on that path.
// The largest logits are collected on the way: a workgroup knows a threshold
// that at least `top` logits of the row reach, appends what lies above it to a
// list in LDS, and now and then keeps the list's `top` best, whose last raises
// the threshold. A row's first chunk sets it from its lanes' maxima. What is
// appended falls off with the place in the row, about top / chunk number a
// chunk, so the search costs one comparison of a vector's maximum.
//
// What bounds it: the logits' way from memory, read once. 16897 x 128000 bf16
// take 729 us, 5.9 TB/s (a copy of 4 GiB moves 4.7, reads and writes together).
// A workgroup of 256 takes a row whole, four vectors of 16 bytes a lane in
// flight. Few rows are split over workgroups by units of 8192 logits and joined
// by a second launch: 64 x 128000 with 20 alternatives take 16 + 7 us, bound by
// latency and barriers. One row of 32000 takes 14 us, four chunks one after the
// other.
#include <algorithm>
#include <type_traits>

#include "serving.h"

namespace bo {
namespace {

constexpr int kWg = 256;
constexpr float kNegInf = -__builtin_huge_valf();
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;
// A finite stand-in for -inf where it is multiplied by a probability of 0.
constexpr float kLow = -1e30f;
constexpr int kVecs = 4;                 // vectors a thread holds at once (16 bytes each)
constexpr int kUnit = 8192;              // elements by which a row is shared out
constexpr int kCand = 768;               // room for appended candidates
constexpr int kMergeAt = 32;             // candidates that are worth a merge
// A lane's reference follows its maximum when that is this far above (in
// powers of two). A wave pays for the move when one of its lanes makes it: at 4
// most vectors did (logits a few units wide), which took as many instructions
// as the sums. The entropy loses 16 units of its last place at most.
constexpr float kSlack = 16.0f;

// The largest fp32 value below v (v finite or +inf).
__device__ __forceinline__ float below(float v) {
  const unsigned u = __float_as_uint(v + 0.0f);
  if (v == 0.0f) return __uint_as_float(0x80000001u);
  return __uint_as_float(v > 0.0f ? u - 1 : u + 1);
}

// Reductions over the wave by DPP: rows of 16 by shifts, then across rows; the
// last lane holds the result, which is given to all. The order is fixed.
template <int CTRL, int ROWS>
__device__ __forceinline__ float dpp(float none, float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(none), __float_as_int(v), CTRL, ROWS, 0xF, false));
}
template <typename F>
__device__ __forceinline__ float wave_reduce(float v, float none, F f) {
  v = f(v, dpp<0x111, 0xF>(none, v));
  v = f(v, dpp<0x112, 0xF>(none, v));
  v = f(v, dpp<0x114, 0xF>(none, v));
  v = f(v, dpp<0x118, 0xF>(none, v));
  v = f(v, dpp<0x142, 0xA>(none, v));
  v = f(v, dpp<0x143, 0xC>(none, v));
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}
__device__ __forceinline__ float wave_max(float v) {
  return wave_reduce(v, kNegInf, [](float p, float q) { return fmaxf(p, q); });
}
__device__ __forceinline__ float wave_sum(float v) {
  return wave_reduce(v, 0.0f, [](float p, float q) { return p + q; });
}

// A scaled reference, NaN from 2^24 on: there its rounding is more than a unit of
// an exponent (a mask of -1e10 would be off by 2^100), so a lane with such a
// reference has to take differences first, t = c (l - r); the NaN in its sums
// tells the wave. (Rounded by itself: contracted into what uses it, the lanes'
// references would no longer be the ones that their sums are relative to.)
constexpr float kNear = 16777216.0f;
__device__ __forceinline__ float scaled_ref(float r, float c) {
#pragma clang fp contract(off)
  const float R = r * c;
  return fabsf(R) < kNear ? R : __builtin_nanf("");
}
// What R = scaled_ref(r, c) lost in rounding: sums are relative to c r - lost.
__device__ __forceinline__ float lost_of(float r, float c, float R) {
  return R == R ? fmaf(r, c, -R) : 0.0f;
}
// c (a - b), of halves: a - b may leave fp32 where c (a - b) does not.
__device__ __forceinline__ float scaled_diff(float a, float b, float c) {
  return fmaf(a, 0.5f, -0.5f * b) * (2.0f * c);
}
// (s, w) relative to r, moved to M >= r: a lane without a finite logit has
// r = -inf and s = 0 (or NaN, which stays).
__device__ __forceinline__ void move_to(float M, float r, float c, float& s, float& w) {
#pragma clang fp contract(off)
  if (r == kNegInf) return;
  const float Rr = scaled_ref(r, c), RM = scaled_ref(M, c);
  float d = Rr - RM;
  // (bounded, so that s d stays finite where it is multiplied by 0)
  if (d != d) d = fmaxf(scaled_diff(r, M, c) + (lost_of(M, c, RM) - lost_of(r, c, Rr)), -1e4f);
  const float f = __builtin_amdgcn_exp2f(d);
  w = (w + s * d) * f;
  s *= f;
  if (M - M != 0.0f) s = w = __builtin_nanf("");
}

// Workgroups go to the chip's dies in turn. Rows in that order would give all
// rows of a batch that are alike by a period of 2, 4 or 8 (masked ones cost more)
// to the same dies; a die takes consecutive rows instead.
constexpr int kXcds = 8;
__device__ __forceinline__ int64_t xcd_order(int64_t b, int64_t each) {
  return (b % kXcds) * each + b / kXcds;
}

// Logits and gradients of more bytes than these pass the caches by (256 MB of
// last level, and the dies' L2). A smaller gradient stays for what reads it
// next: at 131 MB it and a product that reads it take 128 us, past the caches
// 144, and both passes 71 against 74; at 205 MB both passes take 147 against 125,
// at 524 MB 307 against 267 (4 of them lost again in the product).
// The forward pass leaves its last rows for the gradient, which starts there.
// Only where those are few does it load past the caches: both passes at 1.0 GB
// 544 us against 557, at 2.1 GB 1087 against 1081; alone at 4.3 GB 747 against 729.
constexpr int64_t kStreamGrad = (int64_t)160 << 20;
constexpr int64_t kStreamForward = (int64_t)1536 << 20;

struct Partial {      // of one row's share
  float M, s, w;
  int ahead;
};

// The row's outputs from its joined sums (one thread).
__device__ __forceinline__ float finish(const LogprobArgs& a, int64_t row, const Partial& p,
                                        int64_t tok, float xt) {
  const bool has = tok >= 0 && tok < a.V;
  const float c = a.c;
  const float lost = lost_of(p.M, c, scaled_ref(p.M, c));
  const float ls0 = logf(p.s), ls = ls0 - lost * kLn2;
  a.stats[2 * row] = p.M;
  a.stats[2 * row + 1] = ls;
  a.entropy[row] = p.M == kNegInf && p.s == 0.0f ? 0.0f : ls0 - p.w / p.s * kLn2;
  float lp = 0.0f;
  if (has) lp = xt == kNegInf && p.s == p.s ? kNegInf : scaled_diff(xt, p.M, a.it) - ls;
  if (tok >= a.V) lp = __builtin_nanf("");
  a.logprob[row] = lp;
  a.rank[row] = has && xt > kNegInf ? p.ahead + 1 : 0;
  return ls;
}
__device__ __forceinline__ void finish_top(const LogprobArgs& a, int64_t row, int i,
                                           unsigned long long key, float M, float ls) {
  a.top_ids[row * a.top + i] = key ? key_index(key) : -1;
  a.top_logprobs[row * a.top + i] = key ? scaled_diff(key_value(key), M, a.it) - ls : kNegInf;
}

struct alignas(16) TopLds {
  unsigned long long list[2][BO_MAX_ALTERNATIVES];
  unsigned long long cand[kCand + 2];
  unsigned lane_max[kWg];
  float wave_th[kWg / 64];
  int count[2];
};

// How many of keys[0..n) are larger; keys aligned to 16 bytes, room to read one
// past an odd end.
__device__ __forceinline__ int count_larger(const unsigned long long* keys, int n,
                                            unsigned long long key) {
  int rank = 0;
#pragma unroll 4
  for (int j = 0; j < n; j += 2) {
    const ulonglong2 two = *reinterpret_cast<const ulonglong2*>(keys + j);
    rank += two.x > key;
    rank += j + 1 < n && two.y > key;
  }
  return rank;
}

// Keeps the k best of list[cur][0..kcur) and cand[0..n): each key's rank is
// the number of larger ones. Ends with a barrier; returns how many are kept.
__device__ int merge(TopLds& L, int cur, int kcur, int n, int k) {
  __syncthreads();
  const int all = kcur + n;
  for (int i = threadIdx.x; i < all; i += kWg) {
    const unsigned long long key = i < kcur ? L.list[cur][i] : L.cand[i - kcur];
    const int rank = count_larger(L.list[cur], kcur, key) + count_larger(L.cand, n, key);
    if (rank < k) L.list[cur ^ 1][rank] = key;
  }
  __syncthreads();
  return all < k ? all : k;
}

// A vector's largest logit, NaN where it holds one: a maximum that drops NaN
// turns a signalling one into a quiet one first, and what it was compared with
// is dropped with it by the next.
template <int TYPE>
__device__ __forceinline__ float vec_max(const Vec<TYPE>& q) {
  if constexpr (Vec<TYPE>::kVec == 8) {
    const float low = max3_nan(q.get(0), q.get(1), q.get(2));
    return max3_nan(low, max3_nan(q.get(3), q.get(4), q.get(5)), max3_nan(q.get(6), q.get(7), low));
  } else {
    return max3_nan(max3_nan(q.get(0), q.get(1), q.get(2)), q.get(3), q.get(3));
  }
}
// The largest of a vector that holds NaN (-inf when it holds nothing else).
template <int TYPE>
__device__ __forceinline__ float vec_max_beside_nan(const Vec<TYPE>& q) {
  float m = kNegInf;
#pragma unroll
  for (int e = 0; e < Vec<TYPE>::kVec; ++e) m = q.get(e) > m ? q.get(e) : m;
  return m;
}

// One workgroup per (row, share of the row's units).
template <int TYPE, bool TOP, bool STREAM>
__global__ __launch_bounds__(kWg) void k_logprobs(LogprobArgs a, int splits, int cps) {
  using El = Elem<TYPE>;
  using V = Vec<TYPE>;
  constexpr int KV = V::kVec, U = kVecs;
  __shared__ float fl[3][kWg / 64];
  __shared__ int il[kWg / 64 + 1];
  __shared__ float row_ls;
  __shared__ TopLds L;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int V_ = static_cast<int>(a.V), nv = V_ / KV, rest = V_ % KV;
  const float c = a.c, slack = a.slack;
  const int64_t work = a.T * splits, each = (work + kXcds - 1) / kXcds;
  for (int64_t b = blockIdx.x; b < each * kXcds; b += gridDim.x) {
    const int64_t g = xcd_order(b, each);
    if (g >= work) continue;
    const int64_t row = splits == 1 ? g : g / splits;
    const int part = splits == 1 ? 0 : static_cast<int>(g - row * splits);
    const typename El::T* x = static_cast<const typename El::T*>(a.logits) + row * a.stride;
    const int v0 = min(nv, part * cps * (kUnit / KV)), v1 = min(nv, v0 + cps * (kUnit / KV));
    // a chunk: every lane loads, past the share its last vector again (a load
    // that only some lanes make waits for the one before)
    V q[U];
    const auto fetch = [&](int vb) {
      const typename El::T* xc = x + (int64_t)vb * KV;
#pragma unroll
      for (int u = 0; u < U; ++u)
        q[u].template load<STREAM>(xc + static_cast<unsigned>(min(u * kWg + tid, v1 - 1 - vb)) * KV);
    };
    if (v0 < v1) fetch(v0);
    const int64_t tok = a.tokens ? a.tokens[row] : -1;
    const bool has = tok >= 0 && tok < a.V;
    const float xt = has ? El::load(x[tok]) : 0.0f;
    // what a logit must exceed to stand before the token: behind it and ahead
    const float gt = has ? xt : __builtin_huge_valf(), ge = has ? below(xt) : gt;
    // the token's vector (nv past the whole ones: then every vector is ahead of it,
    // and the logits before it in the rest are counted there)
    const int tv = has ? static_cast<int>(tok) / KV : -1;

    // the lane's reference: itself, as it is subtracted (0 for none), scaled (NaN
    // when it is far from 0), and what a logit must exceed to move it
    float m = kNegInf, ref = kNegInf, rz = 0.0f, R = 0.0f, lim = kNegInf, s = 0.0f, w = 0.0f;
    const auto set_ref = [&](float r) {
      ref = rz = r;
      R = scaled_ref(r, c);
      lim = r + slack;
    };
    int ahead = 0, ahead_lane = 0;
    bool bounded = false;                      // the row has met a masked or far logit (per wave)
    float th = kNegInf;
    int cur = 0, kcur = 0, pending = 0, parity = 0;
    int seen[2] = {0, 0};
    if (TOP && tid < 2) L.count[tid] = 0;

    // what is left of the row past its whole vectors: an element to a lane
    const bool owns_rest = part == splits - 1 && tid < rest;
    const int64_t jr = (int64_t)nv * KV + tid;
    float lr = owns_rest ? El::load(x[jr]) : kNegInf;
    for (int vb = v0; vb < v1; vb += kWg * U) {
      if (vb + kWg * U > v1) {
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (vb + u * kWg + tid >= v1) q[u].fill_masked();
      }
      if (TOP && vb == v0) {
        // the wave's k-th largest lane maximum; its low bits give way to the
        // lane, which only lowers it
        float cm = kNegInf;
#pragma unroll
        for (int u = 0; u < U; ++u) cm = max2(cm, vec_max<TYPE>(q[u]));
        const unsigned key = (code_of(cm == cm ? cm : kNegInf) & ~63u) | (63 - lane);
        L.lane_max[tid] = key;
        __syncthreads();
        int rank = 0;
        const uint4* four = reinterpret_cast<const uint4*>(L.lane_max + (tid & ~63));
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const uint4 o = four[j];
          rank += (o.x > key) + (o.y > key) + (o.z > key) + (o.w > key);
        }
        const unsigned long long who = __ballot(rank == a.top - 1);
        const unsigned kth = __builtin_amdgcn_readlane(key, __builtin_ctzll(who)) & ~63u;
        if (lane == 0) L.wave_th[wave] = ordered_value(kth);
        __syncthreads();
        // (the cleared bits may have left a NaN below -inf's code)
        th = kNegInf;
        for (int i = 0; i < kWg / 64; ++i)
          if (L.wave_th[i] > th) th = L.wave_th[i];
        if (th > kNegInf) th = below(th);
      }
      const auto pass = [&](auto is_bounded, auto is_first) {
        constexpr bool BOUNDED = decltype(is_bounded)::value, FIRST = decltype(is_first)::value;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (vb + u * kWg + wave * 64 >= v1) break;
          float vm = vec_max<TYPE>(q[u]);
          if (!(vm <= lim)) {
            if (vm != vm) vm = vec_max_beside_nan<TYPE>(q[u]);
            if (vm > lim) {
              move_to(vm, ref, c, s, w);
              set_ref(vm);
            }
          }
          const int v = vb + u * kWg + tid;
          const float thr = v < tv ? ge : gt;
          const float off = BOUNDED ? lost_of(rz, c, R) : 0.0f, half = -0.5f * rz;
          // (a token among its row's likeliest: few vectors hold what precedes it)
          if (FIRST && __any(vm > thr)) {
#pragma unroll
            for (int e = 0; e < KV; ++e) ahead += __builtin_popcountll(__ballot(q[u].get(e) > thr));
          }
#pragma unroll
          for (int e = 0; e < KV; ++e) {
            const float l = q[u].get(e);
            const float t = BOUNDED ? fmaf(fmaf(l, 0.5f, half), 2.0f * c, off) : fmaf(l, c, -R);
            const float ex = __builtin_amdgcn_exp2f(t);
            s += ex;
            w = fmaf(ex, BOUNDED ? max2(t, kLow) : t, w);
          }
          if (!FIRST) continue;
          m = max2(m, vm);
          if (v == tv && v < v1) {                         // one lane of one chunk
            for (int64_t j = (int64_t)v * KV; j < tok; ++j) ahead_lane += El::load(x[j]) == xt;
          }
          if (TOP && __any(!(vm <= th))) {
#pragma unroll
            for (int e = 0; e < KV; ++e) {
              const float l = q[u].get(e);
              if (__any(l > th) && l > th) {
                const int at = pending + atomicAdd(&L.count[parity], 1) - seen[parity];
                if (at < kCand) L.cand[at] = pack_key(l, static_cast<unsigned>(v) * KV + e);
              }
            }
          }
        }
      };
      if (bounded) {
        pass(std::true_type(), std::true_type());
      } else {
        const float s0 = s, w0 = w, ref0 = ref;
        pass(std::false_type(), std::true_type());
        if (__any(!(fabsf(w) < __builtin_huge_valf()))) {
          bounded = true;
          s = s0;
          w = w0;
          if (ref0 > kNegInf) {
            set_ref(ref0);
          } else {
            ref = lim = kNegInf;
            rz = R = 0.0f;
          }
          pass(std::true_type(), std::false_type());
        }
      }
      if (vb + kWg * U < v1) fetch(vb + kWg * U);     // (on its way during the barrier)
      if (TOP) {
        __syncthreads();
        const int got = L.count[parity] - seen[parity];
        seen[parity] += got;
        parity ^= 1;
        if (pending + got > kCand) {
          // more than there is room for (a row that rises, or is all equal):
          // the chunk again, 256 candidates at a time (its whole vectors: what
          // the row has past them comes on its own, and a key twice would
          // leave a rank without one)
          kcur = merge(L, cur, kcur, pending, a.top);
          cur ^= 1;
          const int64_t j0 = (int64_t)vb * KV, j1 = min((int64_t)v1 * KV, j0 + kWg * U * KV);
          for (int64_t j = j0; j < j1; j += kWg) {
            const unsigned long long least = kcur == a.top ? L.list[cur][kcur - 1] : 0ull;
            if (j + tid < j1) {
              const float l = El::load(x[j + tid]);
              if (l > kNegInf) {
                const unsigned long long key = pack_key(l, static_cast<unsigned>(j + tid));
                if (key > least) L.cand[atomicAdd(&L.count[parity], 1) - seen[parity]] = key;
              }
            }
            __syncthreads();
            const int n = L.count[parity] - seen[parity];
            seen[parity] += n;
            parity ^= 1;
            if (n > 0) {
              kcur = merge(L, cur, kcur, n, a.top);
              cur ^= 1;
            }
          }
          pending = 0;
          th = kcur == a.top ? key_value(L.list[cur][kcur - 1]) : kNegInf;
        } else {
          pending += got;
          if (pending >= kMergeAt || (vb == v0 && pending > a.top)) {
            kcur = merge(L, cur, kcur, pending, a.top);
            cur ^= 1;
            pending = 0;
            th = kcur == a.top ? key_value(L.list[cur][kcur - 1]) : kNegInf;
          }
        }
      }
    }

    if (rest > 0 && part == splits - 1 && wave == 0) {
      if (lr > lim) {
        move_to(lr, ref, c, s, w);
        set_ref(lr);
      }
      m = lr > m ? lr : m;
      const float t = scaled_diff(lr, rz, c) + lost_of(rz, c, R);
      const float ex = __builtin_amdgcn_exp2f(t);
      s += ex;
      w = fmaf(ex, max2(t, kLow), w);
      ahead += __builtin_popcountll(__ballot(lr > (jr < tok ? ge : gt)));
    }
    if (TOP) {
      __syncthreads();                         // (a row without whole vectors: the counters)
      if (lr > th) {
        const int at = pending + atomicAdd(&L.count[parity], 1) - seen[parity];
        L.cand[at] = pack_key(lr, static_cast<unsigned>(jr));
      }
      __syncthreads();
      pending += L.count[parity] - seen[parity];
      if (pending > 0) {
        kcur = merge(L, cur, kcur, pending, a.top);
        cur ^= 1;
      }
    }

    // join the lanes
    float M = wave_max(m);
    if (lane == 0) fl[0][wave] = M;
    if (tid == 0) il[kWg / 64] = 0;
    __syncthreads();
    for (int i = 0; i < kWg / 64; ++i) M = fmaxf(M, fl[0][i]);
    move_to(M, ref, c, s, w);
    s = wave_sum(s);
    w = wave_sum(w);
    if (ahead_lane) il[kWg / 64] = ahead_lane;       // (the token's lane, or none)
    if (lane == 0) {
      fl[1][wave] = s;
      fl[2][wave] = w;
      il[wave] = ahead;
    }
    __syncthreads();
    if (tid == 0) {
      Partial p{M, fl[1][0], fl[2][0], il[0] + il[kWg / 64]};
      for (int i = 1; i < kWg / 64; ++i) {
        p.s += fl[1][i];
        p.w += fl[2][i];
        p.ahead += il[i];
      }
      if (splits == 1) row_ls = finish(a, row, p, tok, xt);
      else static_cast<Partial*>(a.ws)[g] = p;
    }
    __syncthreads();
    if (TOP && tid < a.top) {
      const unsigned long long key = tid < kcur ? L.list[cur][tid] : 0ull;
      if (splits == 1) {
        finish_top(a, row, tid, key, M, row_ls);
      } else {
        unsigned long long* keys = reinterpret_cast<unsigned long long*>(static_cast<Partial*>(a.ws) + work);
        keys[g * a.top + tid] = key;
      }
    }
    __syncthreads();
  }
}

constexpr int kMaxSplits = 64;
constexpr int kMaxJoinKeys = 1024;

// One workgroup per row joins its shares.
template <int TYPE>
__global__ __launch_bounds__(kWg) void k_logprobs_join(LogprobArgs a, int splits) {
  using El = Elem<TYPE>;
  __shared__ alignas(16) unsigned long long keys[kMaxJoinKeys + 2];
  __shared__ int count;
  __shared__ unsigned long long best[BO_MAX_ALTERNATIVES];
  __shared__ float row_M, row_ls;
  const int tid = threadIdx.x;
  const float c = a.c;
  for (int64_t row = blockIdx.x; row < a.T; row += gridDim.x) {
    const Partial* ps = static_cast<const Partial*>(a.ws) + row * splits;
    const unsigned long long* ks =
        reinterpret_cast<const unsigned long long*>(static_cast<const Partial*>(a.ws) + a.T * splits) +
        row * splits * a.top;
    // a bound that `top` keys reach: every share's p-th best
    const int n = splits * a.top, p = (a.top + splits - 1) / splits;
    for (int i = tid; i < a.top; i += kWg) best[i] = 0ull;
    if (tid == 0) count = 0;
    unsigned long long key[kMaxJoinKeys / kWg];
#pragma unroll
    for (int i = 0; i < kMaxJoinKeys / kWg; ++i) key[i] = i * kWg + tid < n ? ks[i * kWg + tid] : 0ull;
    const int lane = tid & 63;
    unsigned long long bound = a.top > 0 && lane < splits ? ks[lane * a.top + p - 1] : ~0ull;
    for (int off = 32; off > 0; off >>= 1) bound = min(bound, __shfl_xor(bound, off));
    if (tid < 64) {
      Partial p{kNegInf, 0.0f, 0.0f, 0};
      if (tid < splits) p = ps[tid];
      const float M = wave_max(p.M);
      move_to(M, p.M, c, p.s, p.w);
      p.s = wave_sum(p.s);
      p.w = wave_sum(p.w);
      for (int off = 32; off > 0; off >>= 1) p.ahead += __shfl_xor(p.ahead, off);
      p.M = M;
      if (tid == 0) {
        const typename El::T* x = static_cast<const typename El::T*>(a.logits) + row * a.stride;
        const int64_t tok = a.tokens ? a.tokens[row] : -1;
        const float xt = tok >= 0 && tok < a.V ? El::load(x[tok]) : 0.0f;
        row_ls = finish(a, row, p, tok, xt);
        row_M = M;
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kMaxJoinKeys / kWg; ++i)
      if (key[i] && key[i] >= bound) keys[atomicAdd(&count, 1)] = key[i];
    __syncthreads();
    for (int i = tid; i < count; i += kWg) {
      const int rank = count_larger(keys, count, keys[i]);
      if (rank < a.top) best[rank] = keys[i];
    }
    __syncthreads();
    if (tid < a.top) finish_top(a, row, tid, best[tid], row_M, row_ls);
    __syncthreads();
  }
}

// One workgroup per (row, share of the row's chunks): with t = c (l - m),
//   grad_j = p_j (A + B u_j),  u_j = t - log2 s,  p_j = 2^u_j
// streamed once, then the token's and the alternatives' terms put in place of
// what the stream wrote there.
// Bound by memory: after the forward pass over 8192 x 32000 bf16, 167 us for
// 524 MB read and as many written, 6.3 TB/s. Rows go in the reverse of the
// forward pass' order: what that read last is still in the last-level cache
// (both passes 314 -> 307 us).
template <int TYPE, bool STREAM>
__global__ __launch_bounds__(kWg) void k_logprobs_grad(LogprobGradArgs a, int splits, int cps) {
  using El = Elem<TYPE>;
  using V = Vec<TYPE>;
  constexpr int KV = V::kVec, U = kVecs;
  __shared__ float hot[BO_MAX_ALTERNATIVES + 1];
  __shared__ int at[BO_MAX_ALTERNATIVES + 1];
  const int tid = threadIdx.x;
  const int V_ = static_cast<int>(a.V), nv = V_ / KV, rest = V_ % KV;
  const float c = a.it * kLog2e;
  const int64_t work = a.T * splits, each = (work + kXcds - 1) / kXcds;
  for (int64_t b = blockIdx.x; b < each * kXcds; b += gridDim.x) {
    const int64_t g = xcd_order(each * kXcds - 1 - b, each);
    if (g >= work) continue;
    const int64_t row = splits == 1 ? g : g / splits;
    const int part = splits == 1 ? 0 : static_cast<int>(g - row * splits);
    const typename El::T* x = static_cast<const typename El::T*>(a.logits) + row * a.stride;
    typename El::T* out = static_cast<typename El::T*>(a.out) + row * a.out_stride;
    const int v0 = min(nv, part * cps * (kUnit / KV)), v1 = min(nv, v0 + cps * (kUnit / KV));
    const float m0 = a.stats[2 * row], ls0 = a.stats[2 * row + 1];
    const bool empty = m0 == kNegInf && ls0 == kNegInf;
    const float half = empty ? 0.0f : -0.5f * m0, ls2 = empty ? 0.0f : ls0 * kLog2e;
    const int64_t tok = a.tokens ? a.tokens[row] : -1;
    const bool has = tok >= 0 && tok < a.V;
    const float gl = has && a.g_logprob ? a.g_logprob[row] : 0.0f;
    const float gh = a.g_entropy ? a.g_entropy[row] : 0.0f;
    // this thread's one-hot term: alternative tid, or the token
    int id = -1;
    float own = 0.0f;
    if (tid < a.top) {
      id = a.top_ids[row * a.top + tid];
      if (id < 0 || id >= V_) id = -1;
      else own = a.g_top[row * a.top + tid];
    } else if (tid == a.top && has) {
      id = static_cast<int>(tok);
      own = gl;
    }
    if (tid <= a.top) {
      at[tid] = id;
      hot[tid] = own;
    }
    // (the row's last share has what is left past the whole vectors)
    const bool last = part == splits - 1;
    if (id < v0 * KV || id >= (last ? V_ : v1 * KV) || empty) id = -1;
    const int64_t jr = (int64_t)nv * KV + tid;
    const float lr = last && tid < rest ? El::load(x[jr]) : 0.0f;
    const float xi = id >= 0 ? El::load(x[id]) : 0.0f;     // before the row may be overwritten
    __syncthreads();
    float total = 0.0f, mine = 0.0f;
    for (int i = 0; i <= a.top; ++i) {
      total += hot[i];
      if (at[i] == id) mine += hot[i];
    }
    float A = a.it * (-total - gh * a.entropy[row]), B = -a.it * gh * kLn2;
    if (tok >= a.V) A = __builtin_nanf("");
    if (empty) A = B = 0.0f;
    // where p is 0: no product with what may be infinite, NaN only as A's
    const float none = A != A ? A : 0.0f;
    const auto grad = [&](float l) {
      const float u = fmaf(fmaf(l, 0.5f, half), 2.0f * c, -ls2);   // c (l - m) - log2 s
      const float p = __builtin_amdgcn_exp2f(u);
      return p == 0.0f ? none : p * fmaf(B, u, A);
    };
    for (int vb = v0; vb < v1; vb += kWg * U) {
      V q[U];
#pragma unroll
      for (int u = 0; u < U; ++u) q[u].template load<STREAM>(x + (int64_t)min(vb + u * kWg + tid, v1 - 1) * KV);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int v = vb + u * kWg + tid;
        if (v < v1) {
          float r[KV];
#pragma unroll
          for (int e = 0; e < KV; ++e) r[e] = grad(q[u].get(e));
          q[u].set_all(r);
          q[u].template store<STREAM>(out + (int64_t)v * KV);
        }
      }
    }
    if (last && tid < rest) out[jr] = El::store(grad(lr));
    __syncthreads();
    // (an id that is given twice has all its terms in each of its threads)
    if (id >= 0) out[id] = El::store(grad(xi) + a.it * mine);
    __syncthreads();
  }
}

// Shares of a row: enough workgroups for every compute unit when the rows are
// few, whole units each.
struct Split {
  int splits, cps;
};
Split split_of(int64_t T, int64_t V, int64_t most) {
  const int64_t units = (V + kUnit - 1) / kUnit;
  int64_t want = T >= 1024 ? 1 : 1024 / T;
  want = std::min({want, units, most});
  const int64_t cps = (units + want - 1) / want;
  return {static_cast<int>((units + cps - 1) / cps), static_cast<int>(cps)};
}
// Forward, up to four units stay whole: the join's launch and workspace cost the
// host 5 us a call (1 x 32000 with 5 alternatives: 16.9 us a call back to back
// against 21.7; alone 38.7 against 36.8).
Split forward_split(int64_t T, int64_t V, int top) {
  if (V <= 4 * kUnit) return split_of(T, V, 1);
  return split_of(T, V, top > 0 ? std::min(kMaxSplits, kMaxJoinKeys / top) : kMaxSplits);
}

template <int TYPE>
hipError_t launch(const LogprobArgs& a, hipStream_t st) {
  const Split sp = forward_split(a.T, a.V, a.top);
  const int64_t work = (a.T * sp.splits + kXcds - 1) / kXcds * kXcds;
  const dim3 grid(static_cast<unsigned>(std::min<int64_t>(work, 1 << 22)));
  if (a.T * a.V * static_cast<int64_t>(type_bytes(TYPE)) > kStreamForward) {
    if (a.top > 0) k_logprobs<TYPE, true, true><<<grid, kWg, 0, st>>>(a, sp.splits, sp.cps);
    else k_logprobs<TYPE, false, true><<<grid, kWg, 0, st>>>(a, sp.splits, sp.cps);
  } else {
    if (a.top > 0) k_logprobs<TYPE, true, false><<<grid, kWg, 0, st>>>(a, sp.splits, sp.cps);
    else k_logprobs<TYPE, false, false><<<grid, kWg, 0, st>>>(a, sp.splits, sp.cps);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || sp.splits == 1) return e;
  k_logprobs_join<TYPE><<<dim3(static_cast<unsigned>(a.T)), kWg, 0, st>>>(a, sp.splits);
  return hipGetLastError();
}

template <int TYPE>
hipError_t launch(const LogprobGradArgs& a, hipStream_t st) {
  const Split sp = split_of(a.T, a.V, kMaxSplits);
  const int64_t work = (a.T * sp.splits + kXcds - 1) / kXcds * kXcds;
  const dim3 grid(static_cast<unsigned>(std::min<int64_t>(work, 1 << 22)));
  if (a.T * a.V * static_cast<int64_t>(type_bytes(TYPE)) > kStreamGrad)
    k_logprobs_grad<TYPE, true><<<grid, kWg, 0, st>>>(a, sp.splits, sp.cps);
  else
    k_logprobs_grad<TYPE, false><<<grid, kWg, 0, st>>>(a, sp.splits, sp.cps);
  return hipGetLastError();
}

}  // namespace

int64_t logprob_workspace(int64_t T, int64_t V, int top) {
  const Split sp = forward_split(T, V, top);
  return sp.splits == 1 ? 0 : T * sp.splits * static_cast<int64_t>(sizeof(Partial) + 8 * top);
}

hipError_t launch_logprobs(const LogprobArgs& args, hipStream_t st) {
  LogprobArgs a = args;
  a.c = a.it * kLog2e;
  a.slack = kSlack / a.c;
  if (a.type == BO_TYPE_F32) return launch<BO_TYPE_F32>(a, st);
  if (a.type == BO_TYPE_BF16) return launch<BO_TYPE_BF16>(a, st);
  return launch<BO_TYPE_F16>(a, st);
}

hipError_t launch_logprobs_grad(const LogprobGradArgs& a, hipStream_t st) {
  if (a.type == BO_TYPE_F32) return launch<BO_TYPE_F32>(a, st);
  if (a.type == BO_TYPE_BF16) return launch<BO_TYPE_BF16>(a, st);
  return launch<BO_TYPE_F16>(a, st);
}

}  // namespace bo
