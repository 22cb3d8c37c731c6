// Log probabilities straight from hidden rows and the output matrix, and the
// gradients of both: the plan of a call, and what happens beside the products of
// linear_tile.h.
//
// Forward: one product, whose tiles leave three numbers a token and tile of logits,
// and a join of them. Up to 64 tokens it reads the matrix once, through tiles as
// narrow as the tokens: 64 x 128000 x 4096 bf16 take 187 us, 5.6 TB/s; 1 x 32000 x
// 4096 53 us, 45 of them the matrix (262 MB).
//
// Backward: the vocabulary in pieces; a piece's d is formed by the same product (the
// logits are not kept, so their 2 T V H operations are done again: 8 T V H in all)
// and read twice: into fp32 sums of grad_hidden over all pieces, and into the piece's
// rows of grad_weight.
#include "linear_tile.h"

namespace bo {
namespace {

constexpr int kWg = 256;
// Of d held at once: what the last-level cache holds (four times as much takes 0.6%
// less time at 8192 x 128000 x 4096).
constexpr int64_t kPieceBytes = (int64_t)256 << 20;
constexpr int kUnits = 256;                             // compute units

int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

// Loads straight to LDS move whole 4-byte words, and a tile's rows are reached
// by 32-bit offsets.
bool fits(const void* p, int64_t stride, int64_t rows, int64_t es) {
  return reinterpret_cast<uintptr_t>(p) % 4 == 0 && (rows <= 1 || (stride * es) % 4 == 0) &&
         stride <= ((int64_t)1 << 30) / 256 / es;
}

struct Shape {
  int type;
  int64_t es, T, V, H;
  int64_t Hp;                             // elements of a copied row
  bool copy_hidden, copy_weight;
};
Shape shape_of(const LinearArgs& a) {
  Shape s;
  s.type = a.type;
  s.es = static_cast<int64_t>(type_bytes(a.type));
  s.T = a.T; s.V = a.V; s.H = a.H;
  s.Hp = up(a.H, 64);
  s.copy_hidden = !fits(a.hidden, a.hidden_stride, a.T, s.es);
  s.copy_weight = !fits(a.weight, a.weight_stride, a.V, s.es);
  return s;
}

int64_t tiles_of(TileShape t, int64_t M, int64_t N) {
  return up(M, tile_m(t)) / tile_m(t) * (up(N, tile_n(t)) / tile_n(t));
}

// Few tokens: what takes the time is the matrix, not the products, and their errors
// do not average out over many rows. Up to so many, logits go by small tiles, and d
// is held in two 16-bit parts, as twice the tokens (128 x 32000 x 4096 bf16: 289
// against 242 us; 16 x 32000 x 4096: 213 against 204).
constexpr int64_t kFewTokens = 128;

// The shape of the tiles and the splits of k that should take the least time: whole
// rounds of workgroups, and for split sums their way through memory (4 bytes a
// picosecond). A k-tile of as many tiles as a compute unit holds at once takes, in
// microseconds, measured with each shape alone (the small one before its sums had two
// levels); a tile's start and end are not counted:
constexpr double kTileTime[2][3] = {{1.65, 1.06, 0.96}, {7.2, 3.7, 2.86}};      // 16 bits, fp32; big, middle, small
struct Choice {
  TileShape tile;
  int64_t splits;
};
// `exact`: small tiles, which carry their sums on two levels (in fp32 these take 1.09
// to 1.14 times as long over many tokens).
Choice choose(int type, int64_t M, int64_t N, int64_t k_tiles, int64_t most_splits, bool exact) {
  Choice best{exact ? kSmall : kBig, 1};
  double least = 1e300;
  for (const TileShape t : {kBig, kMiddle, kSmall}) {
    if (exact && t != kSmall) continue;
    const int64_t tiles = tiles_of(t, M, N), at_once = kUnits * tile_at_once(t);
    const double k_tile = kTileTime[type == BO_TYPE_F32][t];
    if (t != kBig && !exact && tiles * most_splits >= (int64_t)1 << 24) continue;      // (a launch's threads)
    for (int64_t s = 1; s <= most_splits && (s == 1 || s <= k_tiles / 8); ++s) {
      const double rounds = static_cast<double>((tiles * s + at_once - 1) / at_once);
      const double sums = s == 1 ? 0.0 : 5.0 + 2e-6 * static_cast<double>(s * M) * static_cast<double>(N);
      const double cost = rounds * static_cast<double>((k_tiles + s - 1) / s) * k_tile + sums;
      if (cost < least) least = cost, best = {t, s};
    }
  }
  return best;
}

struct Forward {
  TileShape tile;
  int64_t slots;
  int64_t hidden, weight, part, given, total;      // offsets, bytes
};
Forward forward_plan(const Shape& s) {
  Forward f;
  f.tile = s.T <= 32 ? kNarrow32 : s.T <= 64 ? kNarrow64 : choose(s.type, s.V, s.T, 1, 1, s.T <= kFewTokens).tile;
  f.slots = up(s.V, tile_m(f.tile)) / tile_m(f.tile);
  int64_t at = 0;
  const auto take = [&](int64_t bytes) { const int64_t o = at; at += up(bytes, 256); return o; };
  f.hidden = take(s.copy_hidden ? s.T * s.Hp * s.es : 0);
  f.weight = take(s.copy_weight ? s.V * s.Hp * s.es : 0);
  f.part = take(f.slots * 3 * s.T * 4);
  f.given = take(s.T * 4);
  f.total = at;
  return f;
}

struct Backward {
  int64_t parts;                          // of d: 1 or 2
  int64_t piece, pieces;                  // columns
  TileShape derivs, rows, weight;
  int64_t h_splits, w_splits;
  bool h_direct;
  int64_t coef, largest, hidden, weight_copy, d, d_rows, h_sums, w_sums, total;
};
Backward backward_plan(const Shape& s) {
  Backward b;
  b.parts = s.es == 2 && s.T <= kFewTokens ? 2 : 1;
  const int64_t all = up(s.V, 256), T = b.parts * s.T, most = kPieceBytes / (T * s.es) / 256 * 256;
  b.piece = most < 256 ? 256 : most < all ? most : all;
  b.pieces = (all + b.piece - 1) / b.piece;
  const int64_t kK = 128 / s.es;
  const bool few = s.T <= kFewTokens;
  b.derivs = choose(s.type, b.piece, s.T, 1, 1, few).tile;
  const Choice h = choose(s.type, s.H, T, b.piece / kK, 16, few && b.parts == 1),
               w = choose(s.type, s.H, b.piece, up(T, kK) / kK, 16, false);
  b.rows = h.tile;
  b.h_splits = h.splits;
  b.weight = w.tile;
  b.w_splits = w.splits;
  b.h_direct = b.parts == 1 && b.pieces == 1 && b.h_splits == 1;
  int64_t at = 0;
  const auto take = [&](int64_t bytes) { const int64_t o = at; at += up(bytes, 256); return o; };
  b.coef = take(s.T * static_cast<int64_t>(sizeof(TokenCoef)));
  b.largest = take(4 * kLargest);
  b.hidden = take(T * s.Hp * s.es);
  b.weight_copy = take(s.copy_weight ? s.V * s.Hp * s.es : 0);
  b.d = take(T * b.piece * s.es);
  b.d_rows = take(s.type == BO_TYPE_F16 ? T * b.piece * s.es : 0);
  b.h_sums = take(b.h_direct ? 0 : b.h_splits * T * s.Hp * 4);
  b.w_sums = take(b.w_splits == 1 ? 0 : b.w_splits * b.piece * s.Hp * 4);
  b.total = at;
  return b;
}

hipError_t product(TileProduct what, const TileArgs& p, int type, TileShape t, hipStream_t st) {
  if (type == BO_TYPE_F32) return launch_product_f32(what, p, t, st);
  if (type == BO_TYPE_BF16) return launch_product_bf16(what, p, t, st);
  return launch_product_f16(what, p, t, st);
}

// ---- copies of rows: aligned, ended by zeros; rows that take no part are 0 ----

// The rows `copies` times, one after the other.
template <typename U>
__global__ __launch_bounds__(kWg) void k_copy_rows(const U* __restrict__ in, int64_t rows, int64_t copies,
                                                   int64_t H, int64_t stride,
                                                   const TokenCoef* __restrict__ coef,
                                                   U* __restrict__ out, int64_t Hp) {
  constexpr int kVec = 16 / sizeof(U);
  const int64_t per = Hp / kVec, n = rows * copies * per, all = static_cast<int64_t>(gridDim.x) * kWg;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * kWg + threadIdx.x; i < n; i += all) {
    const int64_t to = i / per, r = to < rows ? to : to - rows, h = i % per * kVec;
    U v[kVec];
    const bool live = !coef || coef[r].live;
    if (live && h + kVec <= H) {
      __builtin_memcpy(v, in + r * stride + h, 16);
    } else {
#pragma unroll
      for (int e = 0; e < kVec; ++e) v[e] = live && h + e < H ? in[r * stride + h + e] : 0;
    }
    __builtin_memcpy(out + to * Hp + h, v, 16);
  }
}
hipError_t copy_rows(const void* in, int64_t rows, int64_t copies, int64_t stride, const TokenCoef* coef,
                     void* out, const Shape& s, hipStream_t st) {
  const int64_t blocks = (rows * copies * s.Hp * s.es / 16 + kWg - 1) / kWg;
  const unsigned grid = static_cast<unsigned>(blocks < 16384 ? blocks : 16384);
  if (s.es == 2)
    k_copy_rows<uint16_t><<<grid, kWg, 0, st>>>(static_cast<const uint16_t*>(in), rows, copies, s.H, stride, coef, static_cast<uint16_t*>(out), s.Hp);
  else
    k_copy_rows<uint32_t><<<grid, kWg, 0, st>>>(static_cast<const uint32_t*>(in), rows, copies, s.H, stride, coef, static_cast<uint32_t*>(out), s.Hp);
  return hipGetLastError();
}

// ---- the join of the forward pass ----

// A workgroup 2^log_n tokens, its other lanes over the slots: each takes every
// so-many'th, then neighbours are joined. Maxima first, so that sums need one
// reference. Many tokens take several launches, from n0 on each: a workgroup for every
// 64 of 2^28 would be 2^32 threads, more than a launch has.
constexpr int64_t kJoinTokens = (int64_t)1 << 27;       // of a launch
__global__ __launch_bounds__(1024) void k_linear_join(const float* __restrict__ part, int64_t slots,
                                                      const float* __restrict__ given, int64_t T, int64_t V,
                                                      const int64_t* __restrict__ tokens, float it, float c,
                                                      int log_n, int64_t n0, float* __restrict__ logprob,
                                                      float* __restrict__ entropy, float* __restrict__ stats) {
  __shared__ float red[1024];
  __shared__ float red2[1024];
  const int tid = threadIdx.x, tokens_here = 1 << log_n, shares = 1024 >> log_n;
  const int64_t n = n0 + (static_cast<int64_t>(blockIdx.x) << log_n) + (tid & (tokens_here - 1));
  const int share = tid >> log_n;
  const bool on = n < T;
  float m = -__builtin_huge_valf();
  if (on)
#pragma unroll 4
    for (int64_t i = share; i < slots; i += shares) m = fmaxf(m, part[i * 3 * T + n]);
  red[tid] = m;
  for (int s = 512; s >= tokens_here; s >>= 1) {
    __syncthreads();
    if (tid < s) red[tid] = fmaxf(red[tid], red[tid + s]);
  }
  __syncthreads();
  m = red[tid & (tokens_here - 1)];
  __syncthreads();
  const float ref = m == -__builtin_huge_valf() ? 0.0f : m;
  float s = 0.0f, x = 0.0f;
  if (on)
#pragma unroll 4
    for (int64_t i = share; i < slots; i += shares)
      tile::join_sums(part[i * 3 * T + n], part[(i * 3 + 1) * T + n], part[(i * 3 + 2) * T + n], ref, c, s, x);
  red[tid] = s;
  red2[tid] = x;
  for (int w = 512; w >= tokens_here; w >>= 1) {
    __syncthreads();
    if (tid < w) {
      red[tid] += red[tid + w];
      red2[tid] += red2[tid + w];
    }
  }
  if (tid < tokens_here && on) {
    s = red[tid];
    x = red2[tid];
    const float ls = logf(s);
    const int64_t tok = tokens ? tokens[n] : -1;
    float lp = 0.0f;
    if (tok >= V) {
      lp = __builtin_nanf("");
    } else if (tok >= 0) {
      const float g = given[n];
      lp = g == -__builtin_huge_valf() && ls == ls ? g : (g - m) * it - ls;
    }
    logprob[n] = lp;
    entropy[n] = s == 0.0f ? 0.0f : ls - 0.69314718f * x / s;
    stats[2 * n] = m;
    stats[2 * n + 1] = ls;
  }
}

// ---- the gradient's tokens ----

__global__ __launch_bounds__(kWg) void k_linear_coef(const int64_t* __restrict__ tokens, int64_t T, int64_t V,
                                                     const float* __restrict__ stats,
                                                     const float* __restrict__ entropy,
                                                     const float* __restrict__ g_logprob,
                                                     const float* __restrict__ g_entropy, float it,
                                                     float log_v, TokenCoef* __restrict__ coef,
                                                     float* __restrict__ largest) {
  __shared__ float wave_most[kWg / 64];
  float most = 0.0f;
  for (int64_t t = static_cast<int64_t>(blockIdx.x) * kWg + threadIdx.x; t < T; t += static_cast<int64_t>(gridDim.x) * kWg) {
    const int64_t tok = tokens ? tokens[t] : -1;
    TokenCoef q;
    q.m = stats[2 * t];
    q.ls = stats[2 * t + 1];
    q.g = tok >= 0 && g_logprob ? g_logprob[t] : 0.0f;
    q.gh = g_entropy ? g_entropy[t] : 0.0f;
    // (no probabilities where every logit is masked)
    q.live = (q.g != 0.0f || q.gh != 0.0f) && !(q.m == -__builtin_huge_valf() && q.ls == q.m);
    q.entropy = entropy[t];
    if (tok >= V && q.live) q.g = __builtin_nanf("");
    q.token = tok >= 0 && tok < V ? static_cast<int32_t>(tok) : -1;
    // |p (u + H)| < H + 1 <= log V + 1; what is no finite size scales nothing
    const float size = it * (fabsf(q.g) + (log_v + 1.0f) * fabsf(q.gh));
    const float bound = q.live && size < __builtin_huge_valf() ? size : 0.0f;
    q.exponent = exponent_of(bound);
    coef[t] = q;
    most = fmaxf(most, bound);
  }
#pragma unroll
  for (int off = 32; off; off >>= 1) most = fmaxf(most, __shfl_xor(most, off));
  if ((threadIdx.x & 63) == 0) wave_most[threadIdx.x >> 6] = most;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kWg / 64; ++w) most = fmaxf(most, wave_most[w]);
    largest[blockIdx.x] = most;
  }
}

// out = the splits' sums (and the parts', `rows` apart), scaled and rounded; rows
// that take no part are 0.
template <int TYPE>
__global__ __launch_bounds__(kWg) void k_linear_round(const float* __restrict__ sums, int64_t splits, int64_t parts,
                                                      int64_t split_stride, int64_t rows, int64_t H, int64_t Hp,
                                                      const TokenCoef* __restrict__ coef,
                                                      const float* __restrict__ largest,
                                                      typename Elem<TYPE>::T* __restrict__ out, int64_t stride) {
  const int common = TYPE == BO_TYPE_F16 ? common_exponent(largest) : 0;
  const int64_t per = Hp / 4, n = rows * per, all = static_cast<int64_t>(gridDim.x) * kWg;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * kWg + threadIdx.x; i < n; i += all) {
    const int64_t r = i / per, h = i % per * 4;
    if (h >= H) continue;
    float4 v = {0.0f, 0.0f, 0.0f, 0.0f};
    if (!coef || coef[r].live)
      for (int64_t s = 0; s < splits; ++s)
        for (int64_t d = 0; d < parts; ++d) {
          const float4 o = *reinterpret_cast<const float4*>(sums + s * split_stride + (d * rows + r) * Hp + h);
          v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w;
        }
    const float scale = TYPE == BO_TYPE_F16 ? exp2i(-(coef ? coef[r].exponent : common)) : 1.0f;
    const float f[4] = {v.x * scale, v.y * scale, v.z * scale, v.w * scale};
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (h + e < H) out[r * stride + h + e] = Elem<TYPE>::store(f[e]);
  }
}
hipError_t round_sums(const float* sums, int64_t splits, int64_t parts, int64_t split_stride, int64_t rows, const Shape& s,
                      const TokenCoef* coef, const float* largest, void* out, int64_t stride, hipStream_t st) {
  const int64_t blocks = (rows * s.Hp / 4 + kWg - 1) / kWg;
  const unsigned grid = static_cast<unsigned>(blocks < 16384 ? blocks : 16384);
  const auto go = [&](auto ty) {
    using E = typename Elem<decltype(ty)::value>::T;
    k_linear_round<decltype(ty)::value><<<grid, kWg, 0, st>>>(sums, splits, parts, split_stride, rows, s.H, s.Hp, coef, largest, static_cast<E*>(out), stride);
  };
  if (s.type == BO_TYPE_F32) go(std::integral_constant<int, BO_TYPE_F32>());
  else if (s.type == BO_TYPE_BF16) go(std::integral_constant<int, BO_TYPE_BF16>());
  else go(std::integral_constant<int, BO_TYPE_F16>());
  return hipGetLastError();
}

template <typename U>
__global__ __launch_bounds__(kWg) void k_clear_rows(U* __restrict__ out, int64_t rows, int64_t H, int64_t stride) {
  const int64_t all = static_cast<int64_t>(gridDim.x) * kWg;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * kWg + threadIdx.x; i < rows * H; i += all) out[i / H * stride + i % H] = 0;
}

}  // namespace

int64_t linear_workspace(const LinearArgs& a) { return forward_plan(shape_of(a)).total; }
int64_t linear_grad_workspace(const LinearArgs& a) { return backward_plan(shape_of(a)).total; }

hipError_t launch_linear(const LinearArgs& a, hipStream_t st) {
  const Shape s = shape_of(a);
  const Forward f = forward_plan(s);
  char* w = static_cast<char*>(a.ws);
  hipError_t e;
  TileArgs p{};
  p.a = a.weight; p.a_stride = (s.V > 1 ? a.weight_stride : s.H) * s.es;
  p.b = a.hidden; p.b_stride = (s.T > 1 ? a.hidden_stride : s.H) * s.es;
  if (s.copy_hidden) {
    if ((e = copy_rows(a.hidden, s.T, 1, a.hidden_stride, nullptr, w + f.hidden, s, st)) != hipSuccess) return e;
    p.b = w + f.hidden; p.b_stride = s.Hp * s.es;
  }
  if (s.copy_weight) {
    if ((e = copy_rows(a.weight, s.V, 1, a.weight_stride, nullptr, w + f.weight, s, st)) != hipSuccess) return e;
    p.a = w + f.weight; p.a_stride = s.Hp * s.es;
  }
  p.M = s.V; p.N = s.T; p.K = s.H;
  p.splits = 1; p.split_k = INT64_MAX / 2;
  p.tokens = a.tokens;
  p.c = static_cast<float>(1.4426950408889634 * static_cast<double>(a.it));
  p.part = reinterpret_cast<float*>(w + f.part);
  p.given = reinterpret_cast<float*>(w + f.given);
  if ((e = product(kFormLogprobs, p, s.type, f.tile, st)) != hipSuccess) return e;
  int log_n = 0;
  while (log_n < 6 && ((int64_t)64 << log_n) < s.T) ++log_n;
  for (int64_t n0 = 0; n0 < s.T; n0 += kJoinTokens) {
    const int64_t n = s.T - n0 < kJoinTokens ? s.T - n0 : kJoinTokens;
    const unsigned grid = static_cast<unsigned>((n + ((int64_t)1 << log_n) - 1) >> log_n);
    k_linear_join<<<grid, 1024, 0, st>>>(p.part, f.slots, p.given, s.T, s.V, a.tokens, a.it, p.c, log_n, n0,
                                         a.logprob, a.entropy, a.stats);
  }
  return hipGetLastError();
}

hipError_t launch_linear_grad(const LinearArgs& a, hipStream_t st) {
  if (!a.grad_hidden && !a.grad_weight) return hipSuccess;
  const Shape s = shape_of(a);
  if (s.T == 0) {
    if (!a.grad_weight) return hipSuccess;
    const int64_t blocks = (s.V * s.H + kWg - 1) / kWg;
    const unsigned grid = static_cast<unsigned>(blocks < 16384 ? blocks : 16384);
    if (s.es == 2) k_clear_rows<uint16_t><<<grid, kWg, 0, st>>>(static_cast<uint16_t*>(a.grad_weight), s.V, s.H, a.grad_weight_stride);
    else k_clear_rows<uint32_t><<<grid, kWg, 0, st>>>(static_cast<uint32_t*>(a.grad_weight), s.V, s.H, a.grad_weight_stride);
    return hipGetLastError();
  }
  const Backward b = backward_plan(s);
  char* w = static_cast<char*>(a.ws);
  hipError_t e;
  TokenCoef* coef = reinterpret_cast<TokenCoef*>(w + b.coef);
  float* largest = reinterpret_cast<float*>(w + b.largest);
  const float log_v = logf(static_cast<float>(s.V));
  k_linear_coef<<<kLargest, kWg, 0, st>>>(a.tokens, s.T, s.V, a.stats_in, a.entropy_in, a.g_logprob, a.g_entropy, a.it, log_v, coef, largest);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  if ((e = copy_rows(a.hidden, s.T, b.parts, a.hidden_stride, coef, w + b.hidden, s, st)) != hipSuccess) return e;
  const char* hidden = w + b.hidden;
  const char* weight = static_cast<const char*>(a.weight);
  int64_t weight_stride = (s.V > 1 ? a.weight_stride : s.H) * s.es;
  if (s.copy_weight) {
    if ((e = copy_rows(a.weight, s.V, 1, a.weight_stride, nullptr, w + b.weight_copy, s, st)) != hipSuccess) return e;
    weight = w + b.weight_copy;
    weight_stride = s.Hp * s.es;
  }
  float* h_sums = reinterpret_cast<float*>(w + b.h_sums);
  float* w_sums = reinterpret_cast<float*>(w + b.w_sums);
  const int64_t kK = 128 / s.es;
  const bool scaled = s.type == BO_TYPE_F16;
  char* d = w + b.d;                      // what grad_weight reads, and what grad_hidden does
  char* d_rows = scaled ? w + b.d_rows : d;
  for (int64_t i = 0; i < b.pieces; ++i) {
    const int64_t v0 = i * b.piece, cols = s.V - v0 < b.piece ? s.V - v0 : b.piece;
    TileArgs p{};
    p.a = weight + v0 * weight_stride; p.a_stride = weight_stride;
    p.b = hidden; p.b_stride = s.Hp * s.es;
    p.M = cols; p.N = s.T; p.K = s.H;
    p.splits = 1; p.split_k = INT64_MAX / 2;
    p.c = static_cast<float>(1.4426950408889634 * static_cast<double>(a.it));
    p.it = a.it;
    p.coef = coef; p.largest = largest;
    p.low = b.parts > 1;
    p.m0 = v0;
    p.out = scaled && !a.grad_weight ? nullptr : d;
    p.out_rows = scaled && a.grad_hidden ? d_rows : nullptr;
    p.out_stride = b.piece;
    if ((e = product(kFormDerivs, p, s.type, b.derivs, st)) != hipSuccess) return e;
    if (a.grad_hidden) {
      TileArgs q{};
      q.a = weight + v0 * weight_stride; q.a_stride = weight_stride;
      q.b = d_rows; q.b_stride = b.piece * s.es;
      q.M = s.H; q.N = b.parts * s.T; q.K = cols;
      q.splits = static_cast<int>(b.h_splits);
      q.split_k = (b.piece / kK + b.h_splits - 1) / b.h_splits;
      q.largest = largest;
      if (b.h_direct) {
        q.coef = coef;
        q.out = a.grad_hidden; q.out_stride = a.grad_hidden_stride;
      } else {
        q.out = h_sums; q.out_stride = s.Hp; q.out_split = b.parts * s.T * s.Hp;
        q.add = i > 0;
      }
      if ((e = product(b.h_direct ? kHiddenRows : kHiddenSums, q, s.type, b.rows, st)) != hipSuccess) return e;
    }
    if (a.grad_weight) {
      TileArgs q{};
      q.a = hidden; q.a_stride = s.Hp * s.es;
      q.b = d; q.b_stride = b.piece * s.es;
      q.M = s.H; q.N = cols; q.K = b.parts * s.T;
      q.splits = static_cast<int>(b.w_splits);
      q.split_k = (up(b.parts * s.T, kK) / kK + b.w_splits - 1) / b.w_splits;
      q.largest = largest;
      char* out = static_cast<char*>(a.grad_weight) + v0 * a.grad_weight_stride * s.es;
      if (b.w_splits == 1) {
        q.out = out; q.out_stride = a.grad_weight_stride;
      } else {
        q.out = w_sums; q.out_stride = s.Hp; q.out_split = b.piece * s.Hp;
      }
      if ((e = product(b.w_splits == 1 ? kWeightRows : kWeightSums, q, s.type, b.weight, st)) != hipSuccess) return e;
      if (b.w_splits > 1 &&
          (e = round_sums(w_sums, b.w_splits, 1, b.piece * s.Hp, cols, s, nullptr, largest, out, a.grad_weight_stride, st)) != hipSuccess)
        return e;
    }
  }
  if (a.grad_hidden && !b.h_direct)
    return round_sums(h_sums, b.h_splits, b.parts, b.parts * s.T * s.Hp, s.T, s, coef, largest, a.grad_hidden, a.grad_hidden_stride, st);
  return hipSuccess;
}

}  // namespace bo
