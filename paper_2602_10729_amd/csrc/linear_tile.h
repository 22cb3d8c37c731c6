// Tiled products of the log probabilities from hidden rows, with what each does
// to its tile: out[n][m] = sum_k A(m, k) B(n, k).
//
//   kLogprobs  A = weight, B = hidden, k over H: logits; a tile leaves each
//              token's maximum, sum of exponentials and sum of exponent times
//              exponential, and the given token's logit
//   kDerivs    the same product again; a tile becomes the logits' gradient, rounded
//   kSums      fp32 sums, added to what is there or not
//   kRows      rounded results
// The gradients are A = weight by k over the vocabulary and B = d (grad_hidden),
// and A = hidden, B = d, both by k over the tokens (grad_weight).
//
// m is the side that lies together in out: a lane holds four consecutive m of one n,
// and a token's logits stay within four lanes, so that the softmax exchanges little.
//
// An operand has k together in its rows, or its own index (ACROSS: rows are k).
// Tiles come by loads straight into LDS, 16 bytes a lane, range-checked by the
// buffer's size: rows and granules past the end are 0. A wave reads fragments of 16
// bytes a lane: its lane's row; or ACROSS, four rows at a time through the
// transposing read (16-bit types) or element by element (fp32). LDS rows hold their
// granules XORed with bits of the row's number, so that lanes which read together
// fall on different banks (no conflicts left).
//
// What bounds it: at 256 x 256 tiles of eight waves the matrix pipes are busy 61% of
// the time at 2.0 GHz, the clock that the power leaves; the products run at 1.28
// PFLOP/s (bf16, H = 4096, epilogues included) where a library's, of the same
// operands and no epilogue, reaches 1.36. Measured and not taken, for the training
// step of 8192 x 128000 x 4096 (26.9 ms): 32 x 32 matrix products 29.3, four waves
// of 128 x 128 33.7 (registers spilled), k-tiles of 64 bytes in a ring of four or
// five 28.3, raised wave priority around the products 30.1, a workgroup that stays and
// loads its next tile during a tile's end 27.5 (26.4 beside it), other orders of the
// tiles the same. With every operand in the nearest cache (not a right result) it takes
// 24.8: what memory costs.
#pragma once

#include <type_traits>

#include "serving.h"

namespace bo {

enum Epilogue { kLogprobs, kDerivs, kSums, kRows };

// What the gradient needs of a token, and whether it takes part.
struct TokenCoef {
  float m, ls, g, gh, entropy;            // stats; the gradients that come in
  int32_t token;                          // or -1
  int32_t live;
  int32_t exponent;                       // of the power of two by which f16 multiplies its derivatives
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
  float* part;                            // [m-tiles][3][N]
  float* given;                           // [N]
  // kDerivs
  const TokenCoef* coef;                  // (kRows: of out's rows, or nullptr)
  const float* largest;                   // [64], for the scale of f16 that all tokens share
  float it;
  void* out_rows;                         // f16: under each token's own scale, or nullptr
  int low;                                // rows N + n: what the rounding of rows n left
  int64_t m0;                             // first m of the piece, in the vocabulary
  // out (kDerivs in f16: under the common scale, or nullptr)
  void* out;
  int64_t out_stride;                     // elements
  int64_t out_split;                      // elements between splits (kSums)
  int add;                                // kSums: add to what is there
};

constexpr int kLargest = 64;              // partial maxima of the gradients

// The power of two by which f16 derivatives of at most `bound` are multiplied: the
// largest lies in [2^13, 2^14], so that sums of two stay finite.
__device__ __forceinline__ int exponent_of(float bound) {
  if (!(bound > 0.0f) || !(bound < __builtin_huge_valf())) return 0;
  const int e = 13 - static_cast<int>((__float_as_uint(bound) >> 23) & 0xFF) + 127;
  return e < -120 ? -120 : e > 120 ? 120 : e;
}
// That of all tokens, from partial maxima of their bounds.
__device__ __forceinline__ int common_exponent(const float* largest) {
  float v = largest[threadIdx.x & 63];
#pragma unroll
  for (int off = 32; off; off >>= 1) v = fmaxf(v, __shfl_xor(v, off));
  return exponent_of(v);
}
__device__ __forceinline__ float exp2i(int e) { return __uint_as_float(static_cast<unsigned>(e + 127) << 23); }

namespace tile {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr int kRowBytes = 128;            // of k in a tile's row

__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const void*)p));
}

// N times 16 bytes a lane from buffer + offset to LDS at `to` + 1024 i + 16 lane.
// The compiler does not see that this reads the buffer's registers as memory
// instructions do, so the five wait states after a vector instruction that wrote
// one of them (as a readfirstlane does) stand here, and the one after m0's write.
template <int N>
__device__ __forceinline__ void load_lds(u32x4 buffer, const uint32_t (&offset)[N], uint32_t to) {
  static_assert(N == 1 || N == 2 || N == 4, "loads of a wave");
  if constexpr (N == 1) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                 :: "s"(to), "v"(offset[0]), "s"(buffer) : "memory", "m0");
  } else if constexpr (N == 2) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %2, %4, 0 offen lds\n\t"
                 "s_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %3, %4, 0 offen lds"
                 :: "s"(to), "s"(to + 1024), "v"(offset[0]), "v"(offset[1]), "s"(buffer) : "memory", "m0");
  } else {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %4, %8, 0 offen lds\n\t"
                 "s_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %5, %8, 0 offen lds\n\t"
                 "s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %6, %8, 0 offen lds\n\t"
                 "s_mov_b32 m0, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %7, %8, 0 offen lds"
                 :: "s"(to), "s"(to + 1024), "s"(to + 2048), "s"(to + 3 * 1024), "v"(offset[0]), "v"(offset[1]),
                    "v"(offset[2]), "v"(offset[3]), "s"(buffer) : "memory", "m0");
  }
}

template <int N>
__device__ __forceinline__ void wait_loads() {     // all but the last N; and LDS reads
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" :: "n"(N) : "memory");
}

// LDS accesses of a wave are done in order; this keeps the compiler to it.
__device__ __forceinline__ void wave_order() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_wave_barrier();
}

// The transposing read takes 32 bytes of each of eight rows of k at once, four
// together and four eight further on: XORed into the number of those 32 bytes,
// these bits of k put them on all banks, of which a row of 64 columns spans half
// (with k % 4 alone, 9.9e7 of the 2.0e8 cycles that LDS was at work were conflicts).
template <int R>
__device__ __forceinline__ int across_swizzle(int k) {
  return R == 64 ? ((k >> 1) & 1) | ((k >> 2) & 2) : (k & 3) | ((k >> 1) & 4);
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
        if constexpr (kBytes == 2) g ^= across_swizzle<R>(k) << 1;
        offset[q] = within(k * stride + g * 16);
      }
    }
  }
  // the next k-tile to LDS at `to`
  __device__ __forceinline__ void load(uint32_t to) {
    const int64_t n = (left + 3) & ~int64_t(3);    // (the word that holds the last element)
    u32x4 buffer;
    buffer[0] = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(base));
    buffer[1] = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(base >> 32) & 0xFFFF);
    buffer[2] = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(n < 0 ? 0 : n > kFar ? kFar : n));
    buffer[3] = 0x00020000;
    load_lds(buffer, offset, to + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * (kLoads * 1024));
    base += step;
    left -= step;
  }
};

// Fragments of one operand, 16 rows and 64 bytes of k each, from a tile in LDS:
// lane l holds row l % 16 and the (l / 16)-th 16 bytes.
template <int TYPE, bool ACROSS, int R>
struct Reader {
  static constexpr int kBytes = sizeof(typename Elem<TYPE>::T);
  static constexpr int kReads = !ACROSS ? 1 : kBytes == 2 ? 2 : 4;       // of a fragment
  int row0;                                        // of the wave
  __device__ __forceinline__ u32x4 get(const char* lds, int block, int j) const {
    const int lane = threadIdx.x & 63, i = lane & 15, part = lane >> 4;
    if constexpr (!ACROSS) {
      const int r = row0 + block * 16 + i;
      const int g = (4 * j + part) ^ (lane & 7);
      return *reinterpret_cast<const u32x4*>(lds + r * kRowBytes + g * 16);
    } else if constexpr (kBytes == 2) {
      const int k = 32 * j + 8 * part + (i >> 2);
      const int unit = (row0 / 16 + block) ^ across_swizzle<R>(k);
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
        const int k = 16 * j + 4 * part + s;
        f[s] = *reinterpret_cast<const uint32_t*>(lds + k * (R * 4) + (row0 + block * 16 + i) * 4);
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

// 16 x 16 x 64 bytes. (32 x 32 products take as many operands from LDS for a wave's
// tile, but more time, also without bank conflicts: 29.3 against 26.8 ms for the
// training step of 8192 x 128000 x 4096.)
template <int TYPE>
__device__ __forceinline__ f32x4 mma(u32x4 a, u32x4 b, f32x4 c) {
  if constexpr (TYPE == BO_TYPE_BF16) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  } else if constexpr (TYPE == BO_TYPE_F16) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  } else {
#pragma unroll
    for (int s = 0; s < 4; ++s)
      c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[s]), __uint_as_float(b[s]), c, 0, 0, 0);
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

// Adds sums relative to a maximum mi to s and x, which are relative to ref.
__device__ __forceinline__ void join_sums(float mi, float si, float xi, float ref, float c, float& s, float& x) {
  const float d = (mi - ref) * c, y = __builtin_amdgcn_exp2f(d);
  s = fmaf(y, si, s);
  x = fmaf(y, fmaf(si, fmaxf(d, -1e30f), xi), x);
}

// BM x BN tiles, WM x WN waves, a ring of STAGES k-tiles in LDS.
template <int TYPE, bool AA, bool BA, Epilogue EPI, int BM, int BN, int WM, int WN, int STAGES>
__global__ __launch_bounds__(64 * WM * WN) void k_tile(TileArgs p) {
  using E = typename Elem<TYPE>::T;
  constexpr int kWaves = WM * WN, MI = BM / WM / 16, NI = BN / WN / 16;
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
  const Reader<TYPE, AA, BM> ra{wm * MI * 16};
  const Reader<TYPE, BA, BN> rb{wn * NI * 16};
  f32x4 acc[MI][NI];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NI; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  // Where registers allow, sums are carried on two levels: what kFlush k-tiles give is
  // added to the total, so that a long sum rounds partial sums of its own size less
  // often (errors of fp32 logits over 2048 columns: a third).
  constexpr bool kTwo = BM * BN <= 64 * 128;
  constexpr int kFlush = 8;
  f32x4 total[kTwo ? MI : 1][kTwo ? NI : 1];
  if constexpr (kTwo) {
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NI; ++j) total[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  const auto flush = [&]() {
    if constexpr (kTwo) {
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) {
          total[i][j] += acc[i][j];
          acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }
    }
  };
  const uint32_t lds0 = lds_address(lds);
  const auto fetch = [&](int stage) {
    la.load(lds0 + stage * kStage);
    lb.load(lds0 + stage * kStage + BM * kRowBytes);
  };
  // Fragments: all of B's and the latter half of A's twice, for a step and the
  // next; the first half of A's is replaced once its products are issued.
  constexpr int kHalf = MI / 2;
  u32x4 first[kHalf], second[2][kHalf], fb[2][NI];
  const auto read_most = [&](int stage, int j) {
    const char* at = lds + stage * kStage;
#pragma unroll
    for (int i = 0; i < NI; ++i) fb[j][i] = rb.get(at + BM * kRowBytes, i, j);
#pragma unroll
    for (int i = 0; i < kHalf; ++i) second[j][i] = ra.get(at, kHalf + i, j);
  };
  const auto read_first = [&](int stage, int j) {
#pragma unroll
    for (int i = 0; i < kHalf; ++i) first[i] = ra.get(lds + stage * kStage, i, j);
  };
  const auto multiply = [&](const u32x4 (&a)[kHalf], int j, int i0) {
#pragma unroll
    for (int i = 0; i < kHalf; ++i)
#pragma unroll
      for (int l = 0; l < NI; ++l) acc[i0 + i][l] = mma<TYPE>(a[i], fb[j][l], acc[i0 + i][l]);
  };
  constexpr int kProducts = kHalf * NI * (TYPE == BO_TYPE_F32 ? 4 : 1);
  const auto spread = [&](auto reads) {            // reads between products
    constexpr int kAll = decltype(reads)::value, kEach = kProducts / kAll > 2 ? 2 : 1;
#pragma unroll
    for (int i = 0; i < kAll; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x008, kEach, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, kProducts, 0);
  };
  using Most = std::integral_constant<int, NI * decltype(rb)::kReads + kHalf * decltype(ra)::kReads>;
  using First = std::integral_constant<int, kHalf * decltype(ra)::kReads>;
  // A k-tile is two steps of 64 bytes; a step's fragments are read during the
  // products of the one before. Between the two, every wave has all of the tile,
  // the next one has arrived, and a load of the tile STAGES further on takes this
  // one's place. Past the end loads are issued all the same, out of range, so
  // that counts stay the same.
  if (kt0 < kt1) {
#pragma unroll
    for (int s = 0; s < STAGES; ++s) fetch(s);
    wait_loads<(STAGES - 1) * kLoads>();
    __builtin_amdgcn_s_barrier();
    read_most(0, 0);
    read_first(0, 0);
    int at = 0;
    for (int64_t kt = kt0; kt < kt1 - 1; ++kt) {
      read_most(at, 1);
      multiply(first, 0, 0);
      spread(Most());
      read_first(at, 1);
      multiply(second[0], 0, kHalf);
      spread(First());
      wait_loads<(STAGES - 2) * kLoads>();
      __builtin_amdgcn_s_barrier();
      fetch(at);
      at = at + 1 == STAGES ? 0 : at + 1;
      read_most(at, 0);
      multiply(first, 1, 0);
      spread(Most());
      read_first(at, 0);
      multiply(second[1], 1, kHalf);
      spread(First());
      if (kTwo && (kt - kt0) % kFlush == kFlush - 1) flush();
    }
    // (products over tokens or d end in rows or columns of 0: nothing to clear)
    const int n = static_cast<int>(p.K - (kt1 - 1) * kK);
    const auto clear = [&](int j) {
      if constexpr (EPI == kLogprobs || EPI == kDerivs) {
        const int keep = n - (4 * j + (lane >> 4)) * (kK / 8);
#pragma unroll
        for (int i = 0; i < kHalf; ++i) first[i] = keep_first<TYPE>(first[i], keep);
#pragma unroll
        for (int i = 0; i < kHalf; ++i) second[j][i] = keep_first<TYPE>(second[j][i], keep);
#pragma unroll
        for (int i = 0; i < NI; ++i) fb[j][i] = keep_first<TYPE>(fb[j][i], keep);
      }
    };
    clear(0);
    read_most(at, 1);
    multiply(first, 0, 0);
    read_first(at, 1);
    multiply(second[0], 0, kHalf);
    clear(1);
    multiply(first, 1, 0);
    multiply(second[1], 1, kHalf);
    wait_loads<0>();
  }
  if constexpr (kTwo) {
    flush();
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NI; ++j) acc[i][j] = total[i][j];
  }

  const int64_t mw = static_cast<int64_t>(mt) * BM + wm * MI * 16;     // the wave's first m and n
  const int64_t nw = static_cast<int64_t>(nt) * BN + wn * NI * 16;
  const int part = lane >> 4;
  __builtin_amdgcn_s_barrier();                    // LDS is free
  // element e of block i, j: m = mw + 16 i + 4 part + e, n = nw + 16 j + lane % 16
  if constexpr (EPI == kLogprobs) {
    const int rows = static_cast<int>(min<int64_t>(MI * 16, p.M - mw));
    float* join = reinterpret_cast<float*>(lds);   // [WM][3][BN]
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      const int64_t n = nw + 16 * j + (lane & 15);
      const bool on = n < p.N;
      if (rows < MI * 16) {
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (16 * i + 4 * part + e >= rows) acc[i][j][e] = -__builtin_huge_valf();
      }
      float m = acc[0][j][0];
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) m = fmaxf(m, acc[i][j][e]);
      m = fmaxf(m, __shfl_xor(m, 16));
      m = fmaxf(m, __shfl_xor(m, 32));
      const float ref = m == -__builtin_huge_valf() ? 0.0f : m;
      float s = 0.0f, x = 0.0f;
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float d = (acc[i][j][e] - ref) * p.c;
          const float y = __builtin_amdgcn_exp2f(d);
          s += y;
          x = fmaf(y, d, x);
        }
      if (__ballot(!(x == x))) {                  // 0 times what is masked is 0
        x = 0.0f;
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float d = (acc[i][j][e] - ref) * p.c;
            x = fmaf(__builtin_amdgcn_exp2f(d), fmaxf(d, -1e30f), x);
          }
      }
      s += __shfl_xor(s, 16);
      x += __shfl_xor(x, 16);
      s += __shfl_xor(s, 32);
      x += __shfl_xor(x, 32);
      if (part == 0) {
        float* to = join + wm * 3 * BN + wn * NI * 16 + 16 * j + lane;
        to[0] = m;
        to[BN] = s;
        to[2 * BN] = x;
      }
      const int64_t tok = on && p.tokens ? p.tokens[n] - mw : -1;
      const bool mine = tok >= 0 && tok < rows && ((tok >> 2) & 3) == part;
      if (__ballot(mine)) {
        float v = 0.0f;
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) v = 16 * i + 4 * part + e == tok ? acc[i][j][e] : v;
        if (mine) p.given[n] = v;
      }
    }
    __syncthreads();
    const int64_t n = static_cast<int64_t>(nt) * BN + threadIdx.x;
    if (threadIdx.x < BN && n < p.N) {
      const float* from = join + threadIdx.x;
      float m = from[0];
#pragma unroll
      for (int w = 1; w < WM; ++w) m = fmaxf(m, from[w * 3 * BN]);
      const float ref = m == -__builtin_huge_valf() ? 0.0f : m;
      float s = 0.0f, x = 0.0f;
#pragma unroll
      for (int w = 0; w < WM; ++w) join_sums(from[w * 3 * BN], from[(w * 3 + 1) * BN], from[(w * 3 + 2) * BN], ref, p.c, s, x);
      float* to = p.part + static_cast<int64_t>(mt) * 3 * p.N + n;
      to[0] = m;
      to[p.N] = s;
      to[2 * p.N] = x;
    }
  } else {
    // A block of 16 n goes through the wave's own part of LDS, so that it leaves in
    // whole rows; granules are XORed with n against bank conflicts.
    using S = std::conditional_t<EPI == kSums, float, E>;
    constexpr int kGranules = MI * 16 * static_cast<int>(sizeof(S)) / 16, kSwizzle = kGranules < 16 ? kGranules - 1 : 15;
    static_assert(kWaves * 16 * kGranules * 16 <= STAGES * kStage, "a block of every wave fits");
    char* mine = lds + wave * (16 * kGranules * 16);
    // f16 derivatives are held twice: a token's sum over the vocabulary reads them under
    // a scale of its own, a word's sum over the tokens under one that all share (3.84
    // against 3.69 ms with that one alone at 8192 x 32000 x 2048, both gradients, where a
    // token 2^28 below another's lost what the softmax subtracts).
    constexpr int kScales = TYPE == BO_TYPE_F16 && EPI == kDerivs ? 2 : 1;
    int common = 0;
    if constexpr (TYPE == BO_TYPE_F16 && EPI != kSums) common = common_exponent(p.largest);
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      const int64_t n = nw + 16 * j + (lane & 15);
      const bool on = n < p.N;
      bool live = on;
      float to_common = 1.0f;
      if constexpr (EPI == kDerivs) {
        const TokenCoef q = p.coef[on ? n : 0];
        live = on && q.live;
        const float scale = kScales == 2 ? exp2i(q.exponent) : 1.0f;
        if constexpr (kScales == 2) to_common = exp2i(max(common - q.exponent, -126));
        const float ref = q.m == -__builtin_huge_valf() ? 0.0f : q.m;
        const float ls = q.ls * 1.44269504f, hot = q.g * p.it * scale, g = -hot, gh = -(q.gh * p.it * scale);
        // where a probability is 0: no product with what may be infinite (a masked
        // logit's u, or a large gradient times it), NaN only as the gradients' own
        const float own = fmaf(gh, q.entropy, g), none = own != own ? own : 0.0f;
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float u2 = fmaf(acc[i][j][e] - ref, p.c, -ls), y = __builtin_amdgcn_exp2f(u2);
            const float d = y * fmaf(gh, fmaf(u2, 0.69314718f, q.entropy), g);
            acc[i][j][e] = y == 0.0f ? none : d;
          }
        const int64_t tok = q.token - (p.m0 + mw);
        if (__ballot(q.token >= 0 && tok >= 0 && tok < MI * 16)) {
#pragma unroll
          for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i][j][e] += 16 * i + 4 * part + e == tok ? hot : 0.0f;
        }
        if (mw + MI * 16 > p.M) {
#pragma unroll
          for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (mw + 16 * i + 4 * part + e >= p.M) acc[i][j][e] = 0.0f;
        }
      }
      if constexpr (EPI == kRows) {
        live = on && (!p.coef || p.coef[n].live);
        if constexpr (TYPE == BO_TYPE_F16) {
          const float scale = exp2i(-(p.coef && on ? p.coef[n].exponent : common));
#pragma unroll
          for (int i = 0; i < MI; ++i) acc[i][j] *= scale;
        }
      }
      if (EPI != kSums && __ballot(on && !live)) {
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[i][j][e] = live ? acc[i][j][e] : 0.0f;
      }
      // every scale's values, then (p.low) what their rounding left
      const int halves = EPI == kDerivs && TYPE != BO_TYPE_F32 && p.low ? 2 : 1;
      for (int pass = 0; pass < kScales * halves; ++pass) {
        const bool shared = kScales == 2 && pass >= halves;
        const int half = shared ? pass - halves : pass;
        S* base = static_cast<S*>(kScales == 2 && !shared ? p.out_rows : p.out);
        if (kScales == 2 && !base) continue;
#pragma unroll
        for (int i = 0; i < MI; ++i) {
          S h[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float v = acc[i][j][e];
            if (shared) v *= to_common;
            if constexpr (EPI == kSums) {
              h[e] = v;
            } else {
              h[e] = Elem<TYPE>::store(v);
              if (half) h[e] = Elem<TYPE>::store(v - Elem<TYPE>::load(h[e]));
            }
          }
          const int byte = (16 * i + 4 * part) * static_cast<int>(sizeof(S));
          const int g = (byte >> 4) ^ (lane & kSwizzle);
          __builtin_memcpy(mine + (lane & 15) * (kGranules * 16) + g * 16 + (byte & 15), h, sizeof(h));
        }
        wave_order();
#pragma unroll
        for (int c = 0; c < kGranules / 4; ++c) {
          const int at = c * 64 + lane, r = at / kGranules, g = at % kGranules;
          const int64_t row = nw + 16 * j + r, m = mw + g * (16 / static_cast<int>(sizeof(S)));
          u32x4 v = *reinterpret_cast<const u32x4*>(mine + r * (kGranules * 16) + (g ^ (r & kSwizzle)) * 16);
          if (row >= p.N) continue;
          S* to = base + (EPI == kSums ? split * p.out_split : 0) + (row + half * p.N) * p.out_stride + m;
          if constexpr (EPI == kSums) {
            if (m >= p.out_stride) continue;          // (rows are whole granules)
            if (p.add) {
              const u32x4 o = *reinterpret_cast<const u32x4*>(to);
#pragma unroll
              for (int e = 0; e < 4; ++e) v[e] = __float_as_uint(__uint_as_float(v[e]) + __uint_as_float(o[e]));
            }
            *reinterpret_cast<u32x4*>(to) = v;
          } else if (EPI == kDerivs || m + 16 / static_cast<int>(sizeof(S)) <= p.M) {
            __builtin_memcpy(to, &v, 16);
          } else {
            S h[16 / sizeof(S)];
            __builtin_memcpy(h, &v, 16);
#pragma unroll
            for (int e = 0; e < 16 / static_cast<int>(sizeof(S)); ++e)
              if (m + e < p.M) to[e] = h[e];
          }
        }
        wave_order();
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
enum TileShape { kBig, kMiddle, kSmall, kNarrow64, kNarrow32 };
constexpr int tile_m(TileShape s) { return s == kBig ? 256 : s == kSmall || s == kNarrow32 ? 64 : 128; }
constexpr int tile_n(TileShape s) { return s == kBig ? 256 : s == kNarrow64 ? 64 : s == kNarrow32 ? 32 : 128; }
constexpr int tile_at_once(TileShape s) { return s == kBig ? 1 : s == kMiddle ? 2 : 3; }    // on a compute unit

template <int TYPE, bool AA, bool BA, Epilogue EPI>
hipError_t launch_tile(TileArgs p, TileShape shape, hipStream_t st) {
  p.m_tiles = static_cast<int>((p.M + tile_m(shape) - 1) / tile_m(shape));
  p.n_tiles = static_cast<int>((p.N + tile_n(shape) - 1) / tile_n(shape));
  switch (shape) {
    case kBig: return tile::launch<TYPE, AA, BA, EPI, 256, 256, 2, 4, 2>(p, st);
    case kMiddle: return tile::launch<TYPE, AA, BA, EPI, 128, 128, 2, 2, 2>(p, st);
    case kSmall: return tile::launch<TYPE, AA, BA, EPI, 64, 128, 2, 2, 2>(p, st);
    default: break;
  }
  if constexpr (EPI == kLogprobs) {
    if (shape == kNarrow64) return tile::launch<TYPE, AA, BA, EPI, 128, 64, 4, 1, 3>(p, st);
    return tile::launch<TYPE, AA, BA, EPI, 64, 32, 2, 2, 6>(p, st);
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
