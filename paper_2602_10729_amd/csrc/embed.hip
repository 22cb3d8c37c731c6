// Rows of a table by token, scaled, and the gradient of the table by sorted
// tokens.
//
//   out[t] = scale table[tokens[t]]
//   grad_table[v] = scale sum over t with tokens[t] = v, t rising, of grad[t]
//
// The gradient sorts the tokens (stable, by digits of at most ten bits), then takes
// the sorted list in chunks: a wave adds up the rows of a chunk's runs of equal
// tokens in fp32. A run inside the chunk is written at once; what reaches over a
// chunk's ends leaves its sum in the workspace and is joined in order. Rows without
// a token are cleared beside that work, each row of the table being written once.
// Nothing depends on the order in which atomics arrive.
//
// Memory bounds it: the rows of grad once, the table once. 32768 tokens of text over
// a table of 128000 x 2048 bf16 take 50 us forward (268 MB, 5.4 TB/s) and 143 for the
// gradient: 4.6 marks cleared, 33 the sort with 100 MB of rows cleared beside it, 97
// the sums and the rest (0.5 GB), 10 the runs over chunks.
#include "rows.h"

namespace bo {
namespace {

// ---- rows of the table ----

// 2^split waves a token.
template <int TYPE>
__global__ __launch_bounds__(kRowWg) void k_embed(const int64_t* __restrict__ tokens, int64_t T,
                                                  const typename Elem<TYPE>::T* __restrict__ table,
                                                  int64_t V, int64_t H, int64_t stride, float scale,
                                                  typename Elem<TYPE>::T* __restrict__ out,
                                                  int64_t out_stride, int split) {
  constexpr int kVec = Vec<TYPE>::kVec;
  const int lane = threadIdx.x & 63;
  const int64_t vecs = vectors(H, kVec);
  for (int64_t unit = first_unit(); unit < T << split; unit += units()) {
    const int64_t t = unit >> split, id = tokens[t];
#pragma unroll 2
    for (int64_t i = (unit & ((1 << split) - 1)) * 64 + lane; i < vecs; i += static_cast<int64_t>(64) << split) {
      const RowVec<TYPE> r(i, H);
      float v[kVec];
      if (id >= 0 && id < V) {
        Vec<TYPE> in;
        r.load(in, table + id * stride);
#pragma unroll
        for (int e = 0; e < kVec; ++e) v[e] = scale * in.get(e);
      } else {
#pragma unroll
        for (int e = 0; e < kVec; ++e) v[e] = id < 0 ? 0.0f : __builtin_nanf("");
      }
      Vec<TYPE> o;
      o.set_all(v);
      r.store(o, out + t * out_stride);
    }
  }
}

// ---- rows without a token ----

constexpr int kFillRows = 8;
// The table's rows as bytes, and a mark for each that a token names.
struct Fill {
  char* out;
  int64_t V, row, stride;                 // bytes of a row, and between rows
  const uint8_t* named;
  int split;                              // log2 of the waves that share kFillRows rows
  int64_t first, last;                    // units of this launch: so many rows and a share of their columns
  bool stream;
};

__device__ __forceinline__ void fill_unit(const Fill& f, int64_t unit) {
  const int lane = threadIdx.x & 63;
  const int64_t v0 = (unit >> f.split) * kFillRows, share = unit & ((1 << f.split) - 1);
  unsigned long long bare = __ballot(lane < kFillRows && v0 + lane < f.V && !f.named[min(v0 + lane, f.V - 1)]);
  const int64_t vecs = vectors(f.row, 16);
  typedef uint32_t Any __attribute__((ext_vector_type(4), aligned(2)));
  const Any zero = {0, 0, 0, 0};
  for (; bare; bare &= bare - 1) {
    const int64_t v = v0 + __ffsll(bare) - 1;
    char* to = f.out + v * f.stride;
    if (f.row >= 16) {
      for (int64_t i = share * 64 + lane; i < vecs; i += static_cast<int64_t>(64) << f.split) {
        Any* at = reinterpret_cast<Any*>(to + min(i * 16, f.row - 16));
        if (f.stream) __builtin_nontemporal_store(zero, at);
        else *at = zero;
      }
    } else if (share == 0 && lane * 2 < f.row) {
      *reinterpret_cast<uint16_t*>(to + lane * 2) = 0;
    }
  }
}
// The waves of block b of `blocks` take the launch's units in turn.
__device__ __forceinline__ void fill_part(const Fill& f, int64_t b, int64_t blocks) {
  const int waves = blockDim.x >> 6;
  for (int64_t u = f.first + b * waves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); u < f.last; u += blocks * waves)
    fill_unit(f, u);
}

__global__ __launch_bounds__(kRowWg) void k_embed_begin(uint4* __restrict__ named, int64_t n,
                                                        int32_t* __restrict__ runs) {
  const int64_t all = static_cast<int64_t>(gridDim.x) * kRowWg;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * kRowWg + threadIdx.x; i < n; i += all) named[i] = uint4{0, 0, 0, 0};
  if (blockIdx.x == 0 && threadIdx.x == 0) *runs = 0;
}

// No token at all.
__global__ __launch_bounds__(kRowWg) void k_embed_none(uint16_t* __restrict__ out, int64_t V, int64_t row,
                                                       int64_t stride) {
  const int64_t all = static_cast<int64_t>(gridDim.x) * kRowWg;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * kRowWg + threadIdx.x; i < V * row; i += all)
    out[i / row * stride + i % row] = 0;
}

// ---- sorting ----

constexpr int kSortWg = 1024;
constexpr int kSortWaves = kSortWg / 64;
constexpr int kSortBlocks = 256;
constexpr int kDigits = 1024;             // a digit's values, at most
constexpr int kSortItems = 4;             // tokens a lane holds where one workgroup sorts all

__device__ __forceinline__ uint32_t key_of(int64_t id, int64_t V) {
  return static_cast<uint32_t>(id >= 0 && id < V ? id : V);       // V: none, sorted last
}
// (a byte a row: many waves may mark the same one)
__device__ __forceinline__ void note(uint8_t* named, uint32_t key, int64_t V) {
  if (key < V) named[key] = 1;
}

// The lanes of the wave with this lane's digit.
__device__ __forceinline__ unsigned long long alike(unsigned digit, int bits, bool on) {
  unsigned long long same = __ballot(on);
  for (int b = 0; b < bits; ++b) {
    const bool set = (digit >> b) & 1;
    const unsigned long long v = __ballot(set);
    same &= set ? v : ~v;
  }
  return same;
}
__device__ __forceinline__ int lower(unsigned long long lanes) {
  return __builtin_amdgcn_mbcnt_hi(static_cast<unsigned>(lanes >> 32), __builtin_amdgcn_mbcnt_lo(static_cast<unsigned>(lanes), 0));
}
// Thread i's n summed over the threads before it. Two barriers.
__device__ __forceinline__ int sum_before(int n, int32_t* wave_total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int s = n;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int o = __shfl_up(s, off);
    s += lane >= off ? o : 0;
  }
  if (lane == 63) wave_total[wave] = s;
  __syncthreads();
  int below = s - n;
  for (int w = 0; w < kSortWaves; ++w) below += w < wave ? wave_total[w] : 0;
  __syncthreads();
  return below;
}

// Up to kSortWg * kSortItems tokens, all passes in one workgroup.
__global__ __launch_bounds__(kSortWg) void k_sort_all(const int64_t* __restrict__ tokens, int64_t V, int T,
                                                      int bits, int passes, uint8_t* __restrict__ named,
                                                      uint32_t* __restrict__ keys_out,
                                                      uint32_t* __restrict__ from_out) {
  extern __shared__ int32_t cnt[];                  // [kSortWaves][digits], then keys and origins
  __shared__ int32_t wave_total[kSortWaves];
  const int digits = 1 << bits, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint32_t* keys = reinterpret_cast<uint32_t*>(cnt + kSortWaves * digits);
  uint16_t* from = reinterpret_cast<uint16_t*>(keys + kSortWg * kSortItems);
  const int w0 = wave * 64 * kSortItems + lane;
  uint32_t key[kSortItems];
  unsigned src[kSortItems];
#pragma unroll
  for (int i = 0; i < kSortItems; ++i) {
    const int at = w0 + 64 * i;
    src[i] = static_cast<unsigned>(at);
    key[i] = at < T ? key_of(tokens[at], V) : 0;
    if (at < T) note(named, key[i], V);
  }
  for (int pass = 0; pass < passes; ++pass) {
    for (int i = tid; i < kSortWaves * digits; i += kSortWg) cnt[i] = 0;
    __syncthreads();
    int32_t* mine = cnt + wave * digits;
    unsigned digit[kSortItems];
    int rank[kSortItems];
#pragma unroll
    for (int i = 0; i < kSortItems; ++i) {
      const bool on = w0 + 64 * i < T;
      digit[i] = (key[i] >> (pass * bits)) & static_cast<unsigned>(digits - 1);
      const unsigned long long same = alike(digit[i], bits, on);
      const int before = lower(same);
      rank[i] = (on ? mine[digit[i]] : 0) + before;
      // all lanes have read before the first of each digit writes; a wave's LDS
      // accesses stay in order
      __builtin_amdgcn_wave_barrier();
      if (on && before == 0) mine[digit[i]] = rank[i] + __popcll(same);
      __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    int total = 0;
    if (tid < digits)
#pragma unroll
      for (int w = 0; w < kSortWaves; ++w) total += cnt[w * digits + tid];
    int run = sum_before(total, wave_total);
    if (tid < digits)
#pragma unroll
      for (int w = 0; w < kSortWaves; ++w) {
        const int c = cnt[w * digits + tid];
        cnt[w * digits + tid] = run;
        run += c;
      }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kSortItems; ++i)
      if (w0 + 64 * i < T) {
        const int place = mine[digit[i]] + rank[i];
        keys[place] = key[i];
        from[place] = static_cast<uint16_t>(src[i]);
      }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kSortItems; ++i)
      if (w0 + 64 * i < T) {
        key[i] = keys[w0 + 64 * i];
        src[i] = from[w0 + 64 * i];
      }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < kSortItems; ++i)
    if (w0 + 64 * i < T) {
      keys_out[w0 + 64 * i] = key[i];
      from_out[w0 + 64 * i] = src[i];
    }
}

// FIRST: keys are read from the tokens, and the rows that they name are noted.
// Blocks past the sort's clear rows.
template <bool FIRST>
__global__ __launch_bounds__(kSortWg) void k_sort_count(const int64_t* __restrict__ tokens, int64_t V,
                                                        const uint32_t* __restrict__ keys, int64_t T,
                                                        int64_t chunk, int blocks, int shift, int digits,
                                                        int32_t* __restrict__ hist,
                                                        uint8_t* __restrict__ named, Fill fill) {
  __shared__ int32_t cnt[kDigits];
  if (!FIRST && static_cast<int>(blockIdx.x) >= blocks) return fill_part(fill, blockIdx.x - blocks, gridDim.x - blocks);
  if (threadIdx.x < digits) cnt[threadIdx.x] = 0;
  __syncthreads();
  const int64_t p0 = blockIdx.x * chunk, p1 = min(T, p0 + chunk);
#pragma unroll 4
  for (int64_t p = p0 + threadIdx.x; p < p1; p += kSortWg) {
    const uint32_t k = FIRST ? key_of(tokens[p], V) : keys[p];
    if (FIRST) note(named, k, V);
    atomicAdd(&cnt[(k >> shift) & (digits - 1)], 1);
  }
  __syncthreads();
  if (threadIdx.x < digits) hist[static_cast<int64_t>(blockIdx.x) * digits + threadIdx.x] = cnt[threadIdx.x];
}

// Places a block's keys: a digit's keys of all blocks before it, then its own in
// order. A wave takes 64 at a time; the lanes with a lane's digit come from one
// ballot a bit. Blocks past the sort's clear rows.
template <bool FIRST>
__global__ __launch_bounds__(kSortWg) void k_sort_place(
    const int64_t* __restrict__ tokens, int64_t V, const uint32_t* __restrict__ keys,
    const uint32_t* __restrict__ from, int64_t T, int64_t chunk, int blocks, int shift, int bits,
    const int32_t* __restrict__ hist, uint32_t* __restrict__ keys_out, uint32_t* __restrict__ from_out,
    Fill fill) {
  extern __shared__ int32_t cnt[];                  // [kSortWaves][digits]
  __shared__ int32_t start[kDigits];
  __shared__ int32_t wave_total[kSortWaves];
  if (static_cast<int>(blockIdx.x) >= blocks) return fill_part(fill, blockIdx.x - blocks, gridDim.x - blocks);
  const int digits = 1 << bits;
  const int tid = threadIdx.x, wave = tid >> 6;
  {
    int before = 0, total = 0;
    if (tid < digits)
#pragma unroll 8
      for (int b = 0; b < blocks; ++b) {
        const int n = hist[static_cast<int64_t>(b) * digits + tid];
        total += n;
        before += b < static_cast<int>(blockIdx.x) ? n : 0;
      }
    const int below = sum_before(total, wave_total);
    if (tid < digits) start[tid] = below + before;
  }
  const int64_t p0 = blockIdx.x * chunk, p1 = min(T, p0 + chunk);
  for (int64_t t0 = p0; t0 < p1; t0 += kSortWg) {
    for (int i = tid; i < kSortWaves * digits; i += kSortWg) cnt[i] = 0;
    __syncthreads();
    const int64_t p = t0 + tid;
    const bool on = p < p1;
    uint32_t key = 0, src = 0;
    if (on) {
      key = FIRST ? key_of(tokens[p], V) : keys[p];
      src = FIRST ? static_cast<uint32_t>(p) : from[p];
    }
    const unsigned digit = (key >> shift) & static_cast<unsigned>(digits - 1);
    const unsigned long long same = alike(digit, bits, on);
    const int rank = lower(same);
    if (on && rank == 0) cnt[wave * digits + digit] = __popcll(same);
    __syncthreads();
    if (tid < digits) {
      int run = start[tid];
#pragma unroll
      for (int w = 0; w < kSortWaves; ++w) {
        const int c = cnt[w * digits + tid];
        cnt[w * digits + tid] = run;
        run += c;
      }
      start[tid] = run;
    }
    __syncthreads();
    if (on) {
      const int64_t place = cnt[wave * digits + digit] + rank;
      keys_out[place] = key;
      from_out[place] = src;
    }
    __syncthreads();
  }
}

// ---- sums ----

// 2^split waves a chunk of sorted tokens, 64 of them in the lanes at a time, eight
// rows on their way at once. part [chunks][2][H, in whole fours]: the sum of the run that came in
// over the chunk's start, and of the one that goes on past its end (one that does
// both: the first). runs: how many begin in a chunk and go on, then those chunks.
// The blocks past the sums clear rows (among them, one block of each in turn: 114
// against 97 us at 32768 tokens and 128000 x 2048 bf16).
template <int TYPE>
__global__ __launch_bounds__(kRowWg) void k_embed_sum(
    const uint32_t* __restrict__ keys, const uint32_t* __restrict__ from, int64_t T, int64_t V,
    int64_t chunk, const typename Elem<TYPE>::T* __restrict__ grad, int64_t H, int64_t grad_stride,
    float scale, typename Elem<TYPE>::T* __restrict__ out, int64_t out_stride,
    float* __restrict__ part, int32_t* __restrict__ runs, int split, int sum_blocks, Fill fill) {
  constexpr int kVec = Vec<TYPE>::kVec;
  if (static_cast<int>(blockIdx.x) >= sum_blocks) return fill_part(fill, blockIdx.x - sum_blocks, gridDim.x - sum_blocks);
  const int lane = threadIdx.x & 63;
  const int64_t vecs = vectors(H, kVec), all = (T + chunk - 1) / chunk, Hp = (H + 3) / 4 * 4;
  const int64_t step = static_cast<int64_t>(sum_blocks) * kRowWaves;
  for (int64_t unit = first_unit();
       unit < all << split; unit += step) {
    const int64_t c = unit >> split, i0 = c * chunk, i1 = min(T, i0 + chunk);
    const int64_t share = unit & ((1 << split) - 1);
    const bool came = i0 > 0 && keys[i0 - 1] == keys[i0];
    for (int64_t col = share * 64; col < vecs; col += static_cast<int64_t>(64) << split) {
      const bool on = col + lane < vecs;
      const RowVec<TYPE> r(on ? col + lane : 0, H);
      float sum[kVec];
#pragma unroll
      for (int e = 0; e < kVec; ++e) sum[e] = 0.0f;
      bool in = came;
      for (int64_t base = i0; base < i1; base += 64) {
        const int64_t at = base + lane;
        const uint32_t key = at < i1 ? keys[at] : 0xFFFFFFFFu;
        const uint32_t next = at + 1 < T ? keys[min(at + 1, T - 1)] : 0xFFFFFFFFu;
        const int src = static_cast<int>(at < i1 ? from[at] : 0);
        // (keys of V and above have no token and stand last)
        const int n = __popcll(__ballot(key < V));
        const unsigned long long ends = __ballot(key != next || at + 1 == i1);
        const unsigned long long over = __ballot(key == next && at + 1 == i1);
        const auto take = [&](int first, auto count) {
          constexpr int N = decltype(count)::value;
          Vec<TYPE> g[N];
#pragma unroll
          for (int j = 0; j < N; ++j) {
            const int64_t t = static_cast<uint32_t>(__builtin_amdgcn_readlane(src, first + j));
            if (on) r.template load<true>(g[j], grad + t * grad_stride);
          }
#pragma unroll
          for (int j = 0; j < N; ++j) {
#pragma unroll
            for (int e = 0; e < kVec; ++e) sum[e] += g[j].get(e);
            if (!((ends >> (first + j)) & 1)) continue;
            const bool goes_on = (over >> (first + j)) & 1;
            if (in || goes_on) {
              if (on) {
                float* to = part + (2 * c + (in ? 0 : 1)) * Hp + r.h;
#pragma unroll
                for (int e = 0; e < kVec; ++e)
                  if (e < r.n) to[e] = sum[e];
              }
              if (!in && col == 0 && lane == 0) runs[1 + atomicAdd(runs, 1)] = static_cast<int32_t>(c);
            } else if (on) {
              const int64_t v = static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(key), first + j));
              float f[kVec];
#pragma unroll
              for (int e = 0; e < kVec; ++e) f[e] = scale * sum[e];
              Vec<TYPE> o;
              o.set_all(f);
              r.store(o, out + v * out_stride);
            }
            in = false;
#pragma unroll
            for (int e = 0; e < kVec; ++e) sum[e] = 0.0f;
          }
        };
        int first = 0;
        for (; first + 8 <= n; first += 8) take(first, std::integral_constant<int, 8>());
        if ((n - first) & 4) take(first, std::integral_constant<int, 4>()), first += 4;
        if ((n - first) & 2) take(first, std::integral_constant<int, 2>()), first += 2;
        if ((n - first) & 1) take(first, std::integral_constant<int, 1>());
      }
    }
  }
}

// Joins the runs that reach over chunks: a workgroup a run and 256 columns, its
// waves equal shares of the run's chunks.
template <int TYPE>
__global__ __launch_bounds__(kRowWg) void k_embed_join(const uint32_t* __restrict__ keys, int64_t T,
                                                       int64_t H, int64_t chunk, float scale,
                                                       const float* __restrict__ part,
                                                       const int32_t* __restrict__ runs,
                                                       typename Elem<TYPE>::T* __restrict__ out,
                                                       int64_t out_stride) {
  __shared__ float4 sums[kRowWaves][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t columns = (H + 255) / 256, all = *runs * columns, chunks = (T + chunk - 1) / chunk;
  const int64_t Hp = (H + 3) / 4 * 4;
  for (int64_t unit = blockIdx.x; unit < all; unit += gridDim.x) {
    const int64_t c = runs[1 + unit / columns], h = unit % columns * 256 + lane * 4;
    const uint32_t key = keys[(c + 1) * chunk - 1];
    int64_t last = c;                                // its last chunk: the lanes look ahead
    for (;;) {
      const int64_t b = last + 1 + lane;
      const unsigned long long other = __ballot(b >= chunks || keys[min(b * chunk, T - 1)] != key);
      last += other ? __ffsll(other) - 1 : 64;
      if (other) break;
    }
    const int64_t each = (last - c + kRowWaves - 1) / kRowWaves;
    float4 s = {0.0f, 0.0f, 0.0f, 0.0f};
    const auto add = [&](const float4 o) {
      s.x += o.x;
      s.y += o.y;
      s.z += o.z;
      s.w += o.w;
    };
    if (h < H) {
      const auto at = [&](int64_t row) { return *reinterpret_cast<const float4*>(part + row * Hp + h); };
      if (wave == 0) s = at(2 * c + 1);
      const int64_t b1 = min(last + 1, c + 1 + (wave + 1) * each);
#pragma unroll 8
      for (int64_t b = c + 1 + wave * each; b < b1; ++b) add(at(2 * b));
    }
    __syncthreads();
    sums[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && h < H) {
      for (int w = 1; w < kRowWaves; ++w) add(sums[w][lane]);
      const float f[4] = {scale * s.x, scale * s.y, scale * s.z, scale * s.w};
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (h + e < H) out[static_cast<int64_t>(key) * out_stride + h + e] = Elem<TYPE>::store(f[e]);
    }
  }
}

// Workspace of the gradient: two lists of keys and origins, the blocks' counts, the
// named rows, the runs over chunks, the partial sums.
struct Plan {
  bool one;                               // one workgroup sorts
  int bits, passes;                       // of a digit; digits
  int64_t chunk, blocks;                  // of the sort
  int64_t sums, sum_chunks;               // sorted tokens of a chunk; chunks
  int64_t keys, hist, named, runs, part, total;        // bytes: one list, counts, ..
};
Plan plan_of(int64_t T, int64_t V, int64_t H) {
  Plan p;
  int all = 1;
  while (all < 32 && (V >> all) > 0) ++all;
  p.one = T <= kSortWg * kSortItems;
  p.passes = (all + 9) / 10;
  p.bits = (all + p.passes - 1) / p.passes;
  const int64_t each = (T + kSortBlocks - 1) / kSortBlocks;
  p.chunk = (each + kSortWg - 1) / kSortWg * kSortWg;
  p.blocks = p.one ? 1 : (T + p.chunk - 1) / p.chunk;
  // chunks long enough that a run over all of them is joined in few steps
  p.sums = 32;
  while (p.sums * 2048 < T) p.sums *= 2;
  p.sum_chunks = (T + p.sums - 1) / p.sums;
  const auto up = [](int64_t b) { return (b + 255) / 256 * 256; };
  p.keys = up(4 * T);
  p.hist = up(4 * p.blocks << p.bits);
  p.named = up(V);
  p.runs = up(4 * (p.sum_chunks + 1));
  p.part = up(8 * p.sum_chunks * ((H + 3) / 4 * 4));
  p.total = 4 * p.keys + p.hist + p.named + p.runs + p.part;
  return p;
}

constexpr int64_t kStreamBytes = (int64_t)160 << 20;    // a gradient above this passes the caches by

}  // namespace

hipError_t launch_embed(const EmbedArgs& a, hipStream_t st) {
  const int split = row_split(a.type, a.T, a.H);
  by_type(a.type, [&](auto ty) {
    using E = typename Elem<decltype(ty)::value>::T;
    k_embed<decltype(ty)::value><<<row_blocks(a.T << split), kRowWg, 0, st>>>(
        a.tokens, a.T, static_cast<const E*>(a.in), a.V, a.H, a.stride, a.scale,
        static_cast<E*>(a.out), a.out_stride, split);
  });
  return hipGetLastError();
}

int64_t embed_grad_workspace(int64_t T, int64_t V, int64_t H) { return T ? plan_of(T, V, H).total : 0; }

hipError_t launch_embed_grad(const EmbedArgs& a, hipStream_t st) {
  const int64_t es = static_cast<int64_t>(type_bytes(a.type));
  if (a.T == 0) {
    const int64_t blocks = (a.V * ((a.H * es + 15) / 16) + kRowWg - 1) / kRowWg;
    k_embed_none<<<static_cast<unsigned>(blocks < 16384 ? blocks : 16384), kRowWg, 0, st>>>(
        static_cast<uint16_t*>(a.out), a.V, a.H * es / 2, a.out_stride * es / 2);
    return hipGetLastError();
  }
  const Plan p = plan_of(a.T, a.V, a.H);
  char* w = static_cast<char*>(a.ws);
  uint32_t* keys[2] = {reinterpret_cast<uint32_t*>(w), reinterpret_cast<uint32_t*>(w + p.keys)};
  uint32_t* from[2] = {reinterpret_cast<uint32_t*>(w + 2 * p.keys), reinterpret_cast<uint32_t*>(w + 3 * p.keys)};
  w += 4 * p.keys;
  int32_t* hist = reinterpret_cast<int32_t*>(w);
  uint8_t* named = reinterpret_cast<uint8_t*>(w + p.hist);
  int32_t* runs = reinterpret_cast<int32_t*>(w + p.hist + p.named);
  float* part = reinterpret_cast<float*>(w + p.hist + p.named + p.runs);

  Fill fill{};
  fill.out = static_cast<char*>(a.out);
  fill.V = a.V;
  fill.row = a.H * es;
  fill.stride = (a.V > 1 ? a.out_stride : a.H) * es;
  fill.named = named;
  fill.stream = a.V * fill.row > kStreamBytes;
  const int64_t groups = (a.V + kFillRows - 1) / kFillRows;
  while (fill.split < 10 && ((int64_t)1024 << fill.split) < fill.row) ++fill.split;
  const int64_t fills = groups << fill.split;
  // what a launch of the sort has time for beside it: 32 MB (of 5 to 7 us, it then
  // takes 7 to 11)
  const int64_t beside = ((int64_t)32 << 20) / (kFillRows * fill.row) << fill.split;
  const auto share = [&](int64_t units) {
    fill.first = fill.last;
    fill.last = fill.first + units < fills ? fill.first + units : fills;
    const int64_t n = (fill.last - fill.first + kSortWaves - 1) / kSortWaves;
    return static_cast<unsigned>(n < 256 ? n : 256);
  };
  const int64_t clear = (p.named / 16 + kRowWg - 1) / kRowWg;
  k_embed_begin<<<static_cast<unsigned>(clear < 1024 ? clear : 1024), kRowWg, 0, st>>>(reinterpret_cast<uint4*>(named), p.named / 16, runs);
  int last = 0;
  if (p.one) {
    const size_t lds = (static_cast<size_t>(4 * kSortWaves) << p.bits) + kSortWg * kSortItems * 6;
    k_sort_all<<<1, kSortWg, lds, st>>>(a.tokens, a.V, static_cast<int>(a.T), p.bits, p.passes, named, keys[0], from[0]);
  } else {
    const unsigned grid = static_cast<unsigned>(p.blocks);
    const size_t lds = static_cast<size_t>(4 * kSortWaves) << p.bits;
    for (int i = 0; i < p.passes; ++i) {
      const int in = (i + 1) & 1, shift = i * p.bits, n = static_cast<int>(grid);
      last = i & 1;
      if (i == 0) {
        k_sort_count<true><<<grid, kSortWg, 0, st>>>(a.tokens, a.V, nullptr, a.T, p.chunk, n, 0, 1 << p.bits, hist, named, fill);
        const unsigned more = share(beside);
        k_sort_place<true><<<grid + more, kSortWg, lds, st>>>(a.tokens, a.V, nullptr, nullptr, a.T, p.chunk, n, 0, p.bits, hist, keys[last], from[last], fill);
      } else {
        unsigned more = share(beside);
        k_sort_count<false><<<grid + more, kSortWg, 0, st>>>(a.tokens, a.V, keys[in], a.T, p.chunk, n, shift, 1 << p.bits, hist, named, fill);
        more = share(beside);
        k_sort_place<false><<<grid + more, kSortWg, lds, st>>>(a.tokens, a.V, keys[in], from[in], a.T, p.chunk, n, shift, p.bits, hist, keys[last], from[last], fill);
      }
    }
  }
  share(fills);
  const int64_t rest = (fill.last - fill.first + kRowWaves - 1) / kRowWaves;
  const unsigned fill_blocks = static_cast<unsigned>(rest < 4096 ? rest : 4096);
  by_type(a.type, [&](auto ty) {
    constexpr int TYPE = decltype(ty)::value;
    using E = typename Elem<TYPE>::T;
    E* out = static_cast<E*>(a.out);
    const int split = row_split(a.type, p.sum_chunks, a.H);
    const unsigned sum_blocks = row_blocks(p.sum_chunks << split);
    k_embed_sum<TYPE><<<sum_blocks + fill_blocks, kRowWg, 0, st>>>(
        keys[last], from[last], a.T, a.V, p.sums, static_cast<const E*>(a.in), a.H, a.stride, a.scale, out,
        a.out_stride, part, runs, split, static_cast<int>(sum_blocks), fill);
    if (p.sum_chunks > 1) {
      const int64_t most = p.sum_chunks * ((a.H + 255) / 256);
      k_embed_join<TYPE><<<static_cast<unsigned>(most < 2048 ? most : 2048), kRowWg, 0, st>>>(
          keys[last], a.T, a.H, p.sums, a.scale, part, runs, out, a.out_stride);
    }
  });
  return hipGetLastError();
}

}  // namespace bo
