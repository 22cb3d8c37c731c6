// Tiled products of the log probabilities from hidden rows, with what each does
// to its tile: out[n][m] = sum_k A(m, k) B(n, k).
//
//   kLogprobs  A = weight, B = hidden, k over H: logits; a tile leaves each
//              token's maximum, sum of exponentials and sum of exponent times
//              exponential, and the given token's logit
//   kDerivs    the same product again; a tile becomes d (see bo.h), rounded
//   kSums      fp32 sums, added to what is there or not
//   kRows      rounded results
// The gradients are A = weight by k over the vocabulary and B = d (grad_hidden),
// and A = hidden, B = d, both by k over the tokens (grad_weight).
//
// m is the side that lies together in out, so that a lane, which holds four
// consecutive m of one n, stores them together, and so that a token's logits
// stay in one lane but for its partner: softmax needs no exchange but one.
//
// An operand lies with k together in its rows (K) or with its own index together
// (kAcross: rows are k). Tiles come by loads straight into LDS, 16 bytes a lane,
// range-checked by the buffer's size: rows and granules past the end are 0. A
// wave reads fragments of 16 bytes a lane: for K its lane's row; for kAcross four
// rows at a time through the transposing read (16-bit types) or element by
// element (fp32). LDS rows hold their granules XORed with the row's low bits, so
// that lanes which read together fall on different banks.
#pragma once

#include <type_traits>

#include "serving.h"

namespace bo {

enum Epilogue { kLogprobs, kDerivs, kSums, kRows };

// What the gradient needs of a token, and whether it takes part.
struct TokenCoef {
  float m, ls, g, gh, entropy;            // stats; gradients times nothing yet
  int32_t token;                          // or -1
  int32_t live, pad;
};

struct TileArgs {
  const void* a;
  const void* b;
  int64_t a_stride, b_stride;             // bytes
  int64_t M, N, K;
  int m_tiles, n_tiles, splits;           // splits of k
  int64_t split_k;                        // k-tiles of a split
  // kLogprobs
  const int64_t* tokens;
  float c;                                // log2(e) inverse temperature
  float* part;                            // [slots][3][N]
  float* given;                           // [N]
  // kDerivs
  const TokenCoef* coef;                  // (kRows, kSums: of out's rows, or nullptr)
  const float* largest;                   // [64], for the scale of f16
  float it;
  float log_v;
  int64_t m0;                             // first m of the piece, in the vocabulary
  int64_t V;
  // out
  void* out;
  int64_t out_stride;                     // elements
  int64_t out_split;                      // elements between splits (kSums)
  int add;                                // kSums: add to what is there
};

constexpr int kLargest = 64;              // partial maxima of the gradients

// The power of two by which f16 derivatives are multiplied: the largest lies in
// [2^13, 2^14] by its bound, so that sums of two stay finite.
__device__ __forceinline__ int deriv_exponent(const float* largest) {
  float v = largest[threadIdx.x & 63];
#pragma unroll
  for (int off = 32; off; off >>= 1) v = fmaxf(v, __shfl_xor(v, off));
  if (!(v > 0.0f) || !(v < __builtin_huge_valf())) return 0;
  const int e = 13 - static_cast<int>((__float_as_uint(v) >> 23) & 0xFF) + 127;
  return e < -120 ? -120 : e > 120 ? 120 : e;
}
__device__ __forceinline__ float exp2i(int e) { return __uint_as_float(static_cast<unsigned>(e + 127) << 23); }

namespace tile {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr int kRowBytes = 128;            // of k in a tile's row

__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const void*)p));
}

// 16 bytes a lane from buffer + offset to LDS at `to` + 16 lane.
__device__ __forceinline__ void load_lds(u32x4 buffer, uint32_t offset, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
               :: "s"(to), "v"(offset), "s"(buffer) : "memory");
}

template <int N>
__device__ __forceinline__ void wait_loads() {     // all but the last N; and LDS reads
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" :: "n"(N) : "memory");
}

// One operand's tile: R rows of its own index, kRowBytes of k, loaded by WAVES
// waves.
template <int TYPE, bool ACROSS, int R, int WAVES>
struct Loader {
  static constexpr int kBytes = sizeof(typename Elem<TYPE>::T);
  static constexpr int kK = kRowBytes / kBytes;
  static constexpr int kLoads = R / 8 / WAVES;     // of a wave
  static_assert(kLoads * 8 * WAVES == R, "a tile is whole loads of every wave");
  uint64_t base;
  int64_t step, left;                              // bytes between k-tiles; bytes from base to the end
  uint32_t offset[kLoads];

  // (rows past a tensor's end may lie beyond 32 bits: out of range all the same)
  static constexpr int64_t kFar = 0x7FFFFFF0;
  static __device__ __forceinline__ uint32_t within(int64_t at) { return static_cast<uint32_t>(min(at, kFar)); }
  __device__ __forceinline__ void init(const void* p, int64_t stride, int64_t first, int64_t rows,
                                       int64_t K, int64_t kt) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if constexpr (!ACROSS) {
      const int64_t there = min<int64_t>(rows - first, R);
      step = kRowBytes;
      base = reinterpret_cast<uint64_t>(p) + first * stride + kt * step;
      left = (there - 1) * stride + K * kBytes - kt * step;
      const int g = (lane & 7) ^ (lane >> 3);      // (row & 7 is lane / 8)
#pragma unroll
      for (int q = 0; q < kLoads; ++q) {
        const int row = (wave * kLoads + q) * 8 + (lane >> 3);
        offset[q] = within(row * stride + g * 16);
      }
    } else {
      constexpr int kGranules = R * kBytes / 16;   // of a row
      step = kK * stride;
      base = reinterpret_cast<uint64_t>(p) + first * kBytes + kt * step;
      left = (K - 1) * stride + (rows - first) * kBytes - kt * step;
#pragma unroll
      for (int q = 0; q < kLoads; ++q) {
        const int slot = (wave * kLoads + q) * 64 + lane;
        const int k = slot / kGranules;
        int g = slot % kGranules;
        if constexpr (kBytes == 2) g ^= (k & 3) << 1;
        offset[q] = within(k * stride + g * 16);
      }
    }
  }
  // the next k-tile to LDS at `to`
  __device__ __forceinline__ void load(uint32_t to) {
    const int64_t n = (left + 3) & ~int64_t(3);    // (the word that holds the last element)
    u32x4 buffer;
    buffer[0] = static_cast<uint32_t>(base);
    buffer[1] = static_cast<uint32_t>(base >> 32) & 0xFFFF;
    buffer[2] = static_cast<uint32_t>(n < 0 ? 0 : n > kFar ? kFar : n);
    buffer[3] = 0x00020000;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
    for (int q = 0; q < kLoads; ++q) load_lds(buffer, offset[q], to + (wave * kLoads + q) * 1024);
    base += step;
    left -= step;
  }
};

// Fragments of one operand, 32 rows each, from a tile in LDS.
template <int TYPE, bool ACROSS, int R>
struct Reader {
  static constexpr int kBytes = sizeof(typename Elem<TYPE>::T);
  int row0;                                        // of the wave
  __device__ __forceinline__ u32x4 get(const char* lds, int block, int j) const {
    const int lane = threadIdx.x & 63;
    if constexpr (!ACROSS) {
      const int r = row0 + block * 32 + (lane & 31);
      const int g = (2 * j + (lane >> 5)) ^ (lane & 7);
      return *reinterpret_cast<const u32x4*>(lds + r * kRowBytes + g * 16);
    } else if constexpr (kBytes == 2) {
      const int i = lane & 15, k = 16 * j + 8 * (lane >> 5) + (i >> 2);
      const int unit = (row0 / 16 + block * 2 + ((lane >> 4) & 1)) ^ (i >> 2);
      const char* at = lds + k * (R * 2) + unit * 32 + (i & 3) * 8;
      typedef __attribute__((address_space(3))) s16x4 LdsVec;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsVec*)at);
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsVec*)(at + 4 * R * 2));
      u32x4 f;
      __builtin_memcpy(&f, &lo, 8);
      __builtin_memcpy(reinterpret_cast<char*>(&f) + 8, &hi, 8);
      return f;
    } else {
      u32x4 f;
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const int k = 8 * j + 4 * (lane >> 5) + s;
        f[s] = *reinterpret_cast<const uint32_t*>(lds + k * (R * 4) + (row0 + block * 32 + (lane & 31)) * 4);
      }
      return f;
    }
  }
};

// Elements of a fragment from `n` on cleared (n counted from its first).
template <int TYPE>
__device__ __forceinline__ u32x4 keep_first(u32x4 f, int n) {
  constexpr int kPer = 4 / sizeof(typename Elem<TYPE>::T);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (kPer == 1) f[i] = i < n ? f[i] : 0;
    else f[i] &= (2 * i < n ? 0xFFFFu : 0u) | (2 * i + 1 < n ? 0xFFFF0000u : 0u);
  }
  return f;
}

template <int TYPE>
__device__ __forceinline__ f32x16 mma(u32x4 a, u32x4 b, f32x16 c) {
  if constexpr (TYPE == BO_TYPE_BF16) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  } else if constexpr (TYPE == BO_TYPE_F16) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  } else {
#pragma unroll
    for (int s = 0; s < 4; ++s)
      c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[s]), __uint_as_float(b[s]), c, 0, 0, 0);
    return c;
  }
}

// Blocks go around the eight dies; a die takes consecutive tiles, four m-tiles
// beside each other before the next n-tile, so that those at work on a die share
// their operands in its cache.
__device__ __forceinline__ void place(const TileArgs& p, int& mt, int& nt, int& split) {
  const int b = blockIdx.x, nb = gridDim.x, die = b & 7, per = nb >> 3, rem = nb & 7;
  int i = die * per + (die < rem ? die : rem) + (b >> 3);
  const int tiles = p.m_tiles * p.n_tiles;
  split = i / tiles;
  i -= split * tiles;
  constexpr int kGroup = 4;
  const int group = i / (kGroup * p.n_tiles), in = i - group * kGroup * p.n_tiles;
  const int width = min(kGroup, p.m_tiles - group * kGroup);
  nt = in / width;
  mt = group * kGroup + in % width;
}

// BM x BN tiles, WM x WN waves, a ring of STAGES k-tiles in LDS.
template <int TYPE, bool AA, bool BA, Epilogue EPI, int BM, int BN, int WM, int WN, int STAGES>
__global__ __launch_bounds__(64 * WM * WN) void k_tile(TileArgs p) {
  using E = typename Elem<TYPE>::T;
  constexpr int kWaves = WM * WN, MI = BM / WM / 32, NI = BN / WN / 32;
  constexpr int kStage = (BM + BN) * kRowBytes;
  constexpr int kK = kRowBytes / static_cast<int>(sizeof(E));
  using LoadA = Loader<TYPE, AA, BM, kWaves>;
  using LoadB = Loader<TYPE, BA, BN, kWaves>;
  constexpr int kLoads = LoadA::kLoads + LoadB::kLoads;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / WN, wn = wave % WN;
  int mt, nt, split;
  place(p, mt, nt, split);
  const int64_t k_tiles = (p.K + kK - 1) / kK;
  const int64_t kt0 = split * p.split_k, kt1 = min(k_tiles, kt0 + p.split_k);
  if (EPI == kSums && p.add && kt0 >= kt1) return;
  LoadA la;
  LoadB lb;
  la.init(p.a, p.a_stride, static_cast<int64_t>(mt) * BM, p.M, p.K, kt0);
  lb.init(p.b, p.b_stride, static_cast<int64_t>(nt) * BN, p.N, p.K, kt0);
  const Reader<TYPE, AA, BM> ra{wm * MI * 32};
  const Reader<TYPE, BA, BN> rb{wn * NI * 32};
  f32x16 acc[MI][NI];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NI; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
  const uint32_t lds0 = lds_address(lds);
  const auto fetch = [&](int stage) {
    la.load(lds0 + stage * kStage);
    lb.load(lds0 + stage * kStage + BM * kRowBytes);
  };
  const auto multiply = [&](const char* stage, auto masked, int n) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      u32x4 a[MI], b[NI];
#pragma unroll
      for (int i = 0; i < MI; ++i) a[i] = ra.get(stage, i, j);
#pragma unroll
      for (int i = 0; i < NI; ++i) b[i] = rb.get(stage + BM * kRowBytes, i, j);
      if constexpr (decltype(masked)::value) {
        const int keep = n - (2 * j + (lane >> 5)) * (kK / 8);
#pragma unroll
        for (int i = 0; i < MI; ++i) a[i] = keep_first<TYPE>(a[i], keep);
#pragma unroll
        for (int i = 0; i < NI; ++i) b[i] = keep_first<TYPE>(b[i], keep);
      }
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int l = 0; l < NI; ++l) acc[i][l] = mma<TYPE>(a[i], b[l], acc[i][l]);
    }
  };
  // A k-tile is waited for, then (all waves being past the one before) the load
  // of a later one takes that one's place, then it is multiplied. Past the end
  // loads are issued all the same, out of range, so that counts stay the same.
  if (kt0 < kt1) {
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) fetch(s);
    int at = 0, next = STAGES - 1;
    // (products over tokens or d end in rows or columns of 0: nothing to clear)
    constexpr bool kLast = EPI == kLogprobs || EPI == kDerivs;
    for (int64_t kt = kt0; kt < kt1 - kLast; ++kt) {
      wait_loads<(STAGES - 2) * kLoads>();
      __builtin_amdgcn_s_barrier();
      fetch(next);
      multiply(lds + at * kStage, std::false_type(), 0);
      at = at + 1 == STAGES ? 0 : at + 1;
      next = next + 1 == STAGES ? 0 : next + 1;
    }
    if (kLast) {
      wait_loads<(STAGES - 2) * kLoads>();
      __builtin_amdgcn_s_barrier();
      multiply(lds + at * kStage, std::true_type(), static_cast<int>(p.K - (kt1 - 1) * kK));
    }
    wait_loads<0>();
  }

  const int64_t mw = static_cast<int64_t>(mt) * BM + wm * MI * 32;     // the wave's first m and n
  const int64_t nw = static_cast<int64_t>(nt) * BN + wn * NI * 32;
  const int half = lane >> 5;
  // element e of block i: m = mw + 32 i + 8 (e / 4) + 4 half + e % 4
  if constexpr (EPI == kLogprobs) {
    const int64_t slot = static_cast<int64_t>(mt) * WM + wm;
    const int rows = static_cast<int>(min<int64_t>(MI * 32, p.M - mw));
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      const int64_t n = nw + 32 * j + (lane & 31);
      const bool on = n < p.N;
      if (rows < MI * 32) {
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (32 * i + 8 * (e / 4) + 4 * half + e % 4 >= rows) acc[i][j][e] = -__builtin_huge_valf();
      }
      float m = acc[0][j][0];
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) m = fmaxf(m, acc[i][j][e]);
      m = fmaxf(m, __shfl_xor(m, 32));
      const float ref = m == -__builtin_huge_valf() ? 0.0f : m;
      float s = 0.0f, x = 0.0f;
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float d = (acc[i][j][e] - ref) * p.c;
          const float y = __builtin_amdgcn_exp2f(d);
          s += y;
          x = fmaf(y, fmaxf(d, -1e30f), x);       // (0 times what is masked)
        }
      s += __shfl_xor(s, 32);
      x += __shfl_xor(x, 32);
      if (on && half == 0) {
        float* to = p.part + slot * 3 * p.N + n;
        to[0] = m;
        to[p.N] = s;
        to[2 * p.N] = x;
      }
      const int64_t tok = on && p.tokens ? p.tokens[n] - mw : -1;
      const bool mine = tok >= 0 && tok < rows && ((tok >> 2) & 1) == half;
      if (__ballot(mine)) {
        float v = 0.0f;
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            v = 32 * i + 8 * (e / 4) + 4 * half + e % 4 == tok ? acc[i][j][e] : v;
        if (mine) p.given[n] = v;
      }
    }
  }
  if constexpr (EPI == kDerivs) {
    const float scale = TYPE == BO_TYPE_F16 ? exp2i(deriv_exponent(p.largest)) : 1.0f;
    const float c = p.c;
    E* out = static_cast<E*>(p.out);
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      const int64_t n = nw + 32 * j + (lane & 31);
      const bool on = n < p.N;
      const TokenCoef q = p.coef[on ? n : 0];
      const bool live = on && q.live;
      const float ref = q.m == -__builtin_huge_valf() ? 0.0f : q.m;
      const float is = p.it * scale;
      const int64_t tok = q.token - (p.m0 + mw);
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) {
          float d[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int r = 32 * i + 8 * e4 + 4 * half + e;
            const float u2 = (acc[i][j][4 * e4 + e] - ref) * c - q.ls * 1.44269504f;
            const float y = __builtin_amdgcn_exp2f(u2);
            const float lin = y == 0.0f ? 0.0f : fmaf(u2, 0.69314718f, q.entropy);
            float v = -y * fmaf(q.gh, lin, q.g);
            if (r == tok) v += q.g;
            d[e] = live && mw + r < p.M ? v * is : 0.0f;
          }
          if (on) {
            E h[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) h[e] = Elem<TYPE>::store(d[e]);
            __builtin_memcpy(out + n * p.out_stride + mw + 32 * i + 8 * e4 + 4 * half, h, sizeof(h));
          }
        }
    }
  }
  if constexpr (EPI == kSums) {
    float* out = static_cast<float*>(p.out) + split * p.out_split;
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      const int64_t n = nw + 32 * j + (lane & 31);
      if (n >= p.N) continue;
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) {
          const int64_t m = mw + 32 * i + 8 * e4 + 4 * half;
          if (m >= p.out_stride) continue;          // (rows are whole fours)
          float4* to = reinterpret_cast<float4*>(out + n * p.out_stride + m);
          float4 v = {acc[i][j][4 * e4], acc[i][j][4 * e4 + 1], acc[i][j][4 * e4 + 2], acc[i][j][4 * e4 + 3]};
          if (p.add) {
            const float4 o = *to;
            v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w;
          }
          *to = v;
        }
    }
  }
  if constexpr (EPI == kRows) {
    const float scale = TYPE == BO_TYPE_F16 ? exp2i(-deriv_exponent(p.largest)) : 1.0f;
    E* out = static_cast<E*>(p.out);
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      const int64_t n = nw + 32 * j + (lane & 31);
      if (n >= p.N) continue;
      const bool live = !p.coef || p.coef[n].live;
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) {
          const int64_t m = mw + 32 * i + 8 * e4 + 4 * half;
          E h[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) h[e] = Elem<TYPE>::store(live ? scale * acc[i][j][4 * e4 + e] : 0.0f);
          E* to = out + n * p.out_stride + m;
          if (m + 4 <= p.M) {
            __builtin_memcpy(to, h, sizeof(h));
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (m + e < p.M) to[e] = h[e];
          }
        }
    }
  }
}

template <int TYPE, bool AA, bool BA, Epilogue EPI, int BM, int BN, int WM, int WN, int STAGES>
hipError_t launch(const TileArgs& p, hipStream_t st) {
  constexpr size_t kLds = static_cast<size_t>(BM + BN) * kRowBytes * STAGES;
  const unsigned grid = static_cast<unsigned>(static_cast<int64_t>(p.m_tiles) * p.n_tiles * p.splits);
  k_tile<TYPE, AA, BA, EPI, BM, BN, WM, WN, STAGES><<<grid, 64 * WM * WN, kLds, st>>>(p);
  return hipGetLastError();
}

}  // namespace tile

// Shapes of tiles, m by n.
enum TileShape { kBig, kMiddle, kNarrow64, kNarrow32 };
constexpr int tile_m(TileShape s) { return s == kBig ? 256 : 128; }
constexpr int tile_n(TileShape s) { return s == kBig ? 256 : s == kMiddle ? 128 : s == kNarrow64 ? 64 : 32; }
constexpr int tile_wave_rows(TileShape s) { return s == kBig ? 2 : s == kMiddle ? 2 : 4; }    // waves along m

template <int TYPE, bool AA, bool BA, Epilogue EPI>
hipError_t launch_tile(TileArgs p, TileShape shape, hipStream_t st) {
  p.m_tiles = static_cast<int>((p.M + tile_m(shape) - 1) / tile_m(shape));
  p.n_tiles = static_cast<int>((p.N + tile_n(shape) - 1) / tile_n(shape));
  switch (shape) {
    case kBig: return tile::launch<TYPE, AA, BA, EPI, 256, 256, 2, 4, 2>(p, st);
    case kMiddle: return tile::launch<TYPE, AA, BA, EPI, 128, 128, 2, 2, 2>(p, st);
    default: break;
  }
  if constexpr (EPI == kLogprobs) {
    if (shape == kNarrow64) return tile::launch<TYPE, AA, BA, EPI, 128, 64, 4, 1, 3>(p, st);
    return tile::launch<TYPE, AA, BA, EPI, 128, 32, 4, 1, 3>(p, st);
  }
  return hipErrorInvalidValue;
}

enum TileProduct { kFormLogprobs, kFormDerivs, kHiddenSums, kHiddenRows, kWeightSums, kWeightRows };
template <int TYPE>
hipError_t launch_product(TileProduct what, const TileArgs& p, TileShape shape, hipStream_t st) {
  switch (what) {
    case kFormLogprobs: return launch_tile<TYPE, false, false, kLogprobs>(p, shape, st);
    case kFormDerivs: return launch_tile<TYPE, false, false, kDerivs>(p, shape, st);
    case kHiddenSums: return launch_tile<TYPE, true, false, kSums>(p, shape, st);
    case kHiddenRows: return launch_tile<TYPE, true, false, kRows>(p, shape, st);
    case kWeightSums: return launch_tile<TYPE, true, true, kSums>(p, shape, st);
    default: return launch_tile<TYPE, true, true, kRows>(p, shape, st);
  }
}
// one source file each
hipError_t launch_product_f32(TileProduct what, const TileArgs& p, TileShape shape, hipStream_t st);
hipError_t launch_product_bf16(TileProduct what, const TileArgs& p, TileShape shape, hipStream_t st);
hipError_t launch_product_f16(TileProduct what, const TileArgs& p, TileShape shape, hipStream_t st);

}  // namespace bo
