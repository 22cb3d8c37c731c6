// Rows of a table by token, scaled, and the gradient of the table by sorted
// tokens.
//
//   out[t] = scale table[tokens[t]]
//   grad_table[v] = scale sum over t with tokens[t] = v, t rising, of grad[t]
//
// The gradient sorts the tokens (stable, by digits of at most ten bits: a count
// and a placing launch each), then takes the sorted list in chunks of kChunk
// tokens: a wave adds up the rows of a chunk's runs of equal tokens in fp32. A
// run inside the chunk is written at once; what reaches over a chunk's ends
// leaves its sum in the workspace and is joined in order. Nothing depends on
// the order in which atomics arrive.
#include "rows.h"

namespace bo {
namespace {

constexpr int kChunk = 32;                // sorted tokens a wave adds up

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
  for (int64_t unit = first_unit(); unit < T << split; unit += units()) {
    const int64_t t = unit >> split, id = tokens[t];
    for (int64_t h = ((unit & ((1 << split) - 1)) * 64 + lane) * kVec; h < H; h += (64 * kVec) << split) {
      const int n = static_cast<int>(min<int64_t>(kVec, H - h));
      float v[kVec];
      if (id >= 0 && id < V) {
        Vec<TYPE> r;
        if (n == kVec) r.load(table + id * stride + h);
        else r.load_part(table + id * stride + h, n);
#pragma unroll
        for (int e = 0; e < kVec; ++e) v[e] = scale * r.get(e);
      } else {
#pragma unroll
        for (int e = 0; e < kVec; ++e) v[e] = id < 0 ? 0.0f : __builtin_nanf("");
      }
      Vec<TYPE> o;
      o.set_all(v);
      if (n == kVec) o.store(out + t * out_stride + h);
      else o.store_part(out + t * out_stride + h, n);
    }
  }
}

// ---- sorting ----

constexpr int kSortWg = 1024;
constexpr int kSortWaves = kSortWg / 64;
constexpr int kSortBlocks = 256;
constexpr int kDigits = 1024;             // a digit's values, at most

__device__ __forceinline__ uint32_t key_of(int64_t id, int64_t V) {
  return static_cast<uint32_t>(id >= 0 && id < V ? id : V);       // V: none, sorted last
}

// FIRST: keys are read from the tokens.
template <bool FIRST>
__global__ __launch_bounds__(kSortWg) void k_sort_count(const int64_t* __restrict__ tokens, int64_t V,
                                                        const uint32_t* __restrict__ keys, int64_t T,
                                                        int64_t chunk, int shift, int digits,
                                                        int32_t* __restrict__ hist) {
  __shared__ int32_t cnt[kDigits];
  if (threadIdx.x < digits) cnt[threadIdx.x] = 0;
  __syncthreads();
  const int64_t p0 = blockIdx.x * chunk, p1 = min(T, p0 + chunk);
#pragma unroll 4
  for (int64_t p = p0 + threadIdx.x; p < p1; p += kSortWg) {
    const uint32_t k = FIRST ? key_of(tokens[p], V) : keys[p];
    atomicAdd(&cnt[(k >> shift) & (digits - 1)], 1);
  }
  __syncthreads();
  if (threadIdx.x < digits) hist[static_cast<int64_t>(blockIdx.x) * digits + threadIdx.x] = cnt[threadIdx.x];
}

// Places a block's keys: a digit's keys of all blocks before it, then its own in
// order. A wave takes 64 at a time; the lanes with a lane's digit come from one
// ballot a bit.
template <bool FIRST>
__global__ __launch_bounds__(kSortWg) void k_sort_place(
    const int64_t* __restrict__ tokens, int64_t V, const uint32_t* __restrict__ keys,
    const uint32_t* __restrict__ from, int64_t T, int64_t chunk, int shift, int bits,
    const int32_t* __restrict__ hist, uint32_t* __restrict__ keys_out, uint32_t* __restrict__ from_out) {
  extern __shared__ int32_t cnt[];                  // [kSortWaves][digits]
  __shared__ int32_t start[kDigits];
  __shared__ int32_t wave_total[kSortWaves];
  const int digits = 1 << bits;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  {
    int before = 0, total = 0;
    if (tid < digits)
#pragma unroll 8
      for (int b = 0; b < static_cast<int>(gridDim.x); ++b) {
        const int n = hist[static_cast<int64_t>(b) * digits + tid];
        total += n;
        before += b < static_cast<int>(blockIdx.x) ? n : 0;
      }
    int s = total;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int o = __shfl_up(s, off);
      s += lane >= off ? o : 0;
    }
    if (lane == 63) wave_total[wave] = s;
    __syncthreads();
    int below = s - total;
    for (int w = 0; w < kSortWaves; ++w) below += w < wave ? wave_total[w] : 0;
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
    unsigned long long same = __ballot(on);
    for (int b = 0; b < bits; ++b) {
      const bool set = (digit >> b) & 1;
      const unsigned long long v = __ballot(set);
      same &= set ? v : ~v;
    }
    const int rank = __popcll(same & ((1ull << lane) - 1));
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

// 2^split waves a row.
template <int TYPE>
__global__ __launch_bounds__(kRowWg) void k_embed_zero(typename Elem<TYPE>::T* __restrict__ out, int64_t V,
                                                       int64_t H, int64_t stride, int split) {
  constexpr int kVec = Vec<TYPE>::kVec;
  const int lane = threadIdx.x & 63;
  Vec<TYPE> zero;
  zero.q[0] = zero.q[1] = zero.q[2] = zero.q[3] = 0;
  for (int64_t unit = first_unit(); unit < V << split; unit += units()) {
    const int64_t v = unit >> split;
    for (int64_t h = ((unit & ((1 << split) - 1)) * 64 + lane) * kVec; h < H; h += (64 * kVec) << split) {
      const int n = static_cast<int>(min<int64_t>(kVec, H - h));
      if (n == kVec) zero.store(out + v * stride + h);
      else zero.store_part(out + v * stride + h, n);
    }
  }
}

// 2^split waves a chunk of sorted tokens. part [chunks][2][H]: the sum of the run
// that came in over the chunk's start, and of the one that goes on past its end
// (one that does both: the first).
template <int TYPE>
__global__ __launch_bounds__(kRowWg) void k_embed_sum(
    const uint32_t* __restrict__ keys, const uint32_t* __restrict__ from, int64_t T, int64_t V,
    const typename Elem<TYPE>::T* __restrict__ grad, int64_t H, int64_t grad_stride, float scale,
    typename Elem<TYPE>::T* __restrict__ out, int64_t out_stride, float* __restrict__ part, int split) {
  constexpr int kVec = Vec<TYPE>::kVec;
  const int lane = threadIdx.x & 63;
  const int64_t all = (T + kChunk - 1) / kChunk;
  for (int64_t unit = first_unit(); unit < all << split; unit += units()) {
    const int64_t c = unit >> split, i0 = c * kChunk, i1 = min(T, i0 + kChunk);
    const uint32_t prev = i0 > 0 ? keys[i0 - 1] : 0xFFFFFFFFu, next = i1 < T ? keys[i1] : 0xFFFFFFFFu;
    for (int64_t h = ((unit & ((1 << split) - 1)) * 64 + lane) * kVec; h < H; h += (64 * kVec) << split) {
      const int n = static_cast<int>(min<int64_t>(kVec, H - h));
      float sum[kVec];
#pragma unroll
      for (int e = 0; e < kVec; ++e) sum[e] = 0.0f;
      bool in = keys[i0] == prev;
      for (int64_t i = i0; i < i1; ++i) {
        const uint32_t key = keys[i];
        if (key >= V) break;                         // the rest has no token
        Vec<TYPE> g;
        const typename Elem<TYPE>::T* row = grad + static_cast<int64_t>(from[i]) * grad_stride + h;
        if (n == kVec) g.load(row);
        else g.load_part(row, n);
#pragma unroll
        for (int e = 0; e < kVec; ++e) sum[e] += g.get(e);
        const bool last = i + 1 == i1;
        if (!last && keys[i + 1] == key) continue;
        const bool over = last && next == key;
        if (in || over) {
          float* to = part + (2 * c + (in ? 0 : 1)) * H + h;
#pragma unroll
          for (int e = 0; e < kVec; ++e)
            if (e < n) to[e] = sum[e];
        } else {
          float r[kVec];
#pragma unroll
          for (int e = 0; e < kVec; ++e) r[e] = scale * sum[e];
          Vec<TYPE> o;
          o.set_all(r);
          if (n == kVec) o.store(out + static_cast<int64_t>(key) * out_stride + h);
          else o.store_part(out + static_cast<int64_t>(key) * out_stride + h, n);
        }
        in = false;
#pragma unroll
        for (int e = 0; e < kVec; ++e) sum[e] = 0.0f;
      }
    }
  }
}

// Joins the runs that reach over chunks: a workgroup the run that begins in
// chunk c and 64 columns; its waves take equal shares of the run's chunks.
template <int TYPE>
__global__ __launch_bounds__(kRowWg) void k_embed_join(const uint32_t* __restrict__ keys, int64_t T, int64_t V,
                                                       int64_t H, float scale,
                                                       const float* __restrict__ part,
                                                       typename Elem<TYPE>::T* __restrict__ out,
                                                       int64_t out_stride) {
  __shared__ float sums[kRowWaves][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int64_t c = blockIdx.x; (c + 1) * kChunk < T; c += gridDim.x) {
    const int64_t i1 = (c + 1) * kChunk;
    const uint32_t key = keys[i1 - 1];
    if (key >= V || keys[i1] != key) continue;         // nothing goes on
    if (c > 0 && keys[c * kChunk - 1] == key) continue;   // it began earlier
    // the run's end: the first sorted token past it
    int64_t lo = i1, hi = T;
    while (lo < hi) {
      const int64_t mid = (lo + hi) / 2;
      if (keys[mid] == key) lo = mid + 1;
      else hi = mid;
    }
    const int64_t last = (lo - 1) / kChunk;            // its last chunk
    const int64_t each = (last - c + kRowWaves - 1) / kRowWaves;
    for (int64_t h0 = static_cast<int64_t>(blockIdx.y) * 64; h0 < H; h0 += gridDim.y * 64) {
      const int64_t h = h0 + lane;
      float s = 0.0f;
      if (h < H) {
        if (wave == 0) s = part[(2 * c + 1) * H + h];
        const int64_t b1 = min(last + 1, c + 1 + (wave + 1) * each);
#pragma unroll 8
        for (int64_t b = c + 1 + wave * each; b < b1; ++b) s += part[2 * b * H + h];
      }
      __syncthreads();
      sums[wave][lane] = s;
      __syncthreads();
      if (wave == 0 && h < H) {
        for (int w = 1; w < kRowWaves; ++w) s += sums[w][lane];
        out[static_cast<int64_t>(key) * out_stride + h] = Elem<TYPE>::store(scale * s);
      }
    }
  }
}

// Workspace of the gradient: two lists of keys and origins, the blocks' counts,
// the partial sums.
struct Plan {
  int bits, passes;                       // of a digit; digits
  int64_t chunk, blocks;                  // of the sort
  int64_t token_chunks;
  int64_t keys, hist, part, total;        // bytes: one list, counts, partial sums
};
Plan plan_of(int64_t T, int64_t V, int64_t H) {
  Plan p;
  int all = 1;
  while (all < 32 && (V >> all) > 0) ++all;
  p.passes = (all + 9) / 10;
  p.bits = (all + p.passes - 1) / p.passes;
  const int64_t each = (T + kSortBlocks - 1) / kSortBlocks;
  p.chunk = (each + kSortWg - 1) / kSortWg * kSortWg;
  p.blocks = (T + p.chunk - 1) / p.chunk;
  p.token_chunks = (T + kChunk - 1) / kChunk;
  const auto up = [](int64_t b) { return (b + 255) / 256 * 256; };
  p.keys = up(4 * T);
  p.hist = up(4 * p.blocks << p.bits);
  p.part = up(8 * p.token_chunks * H);
  p.total = 4 * p.keys + p.hist + p.part;
  return p;
}

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
  by_type(a.type, [&](auto ty) {
    constexpr int TYPE = decltype(ty)::value;
    using E = typename Elem<TYPE>::T;
    const E* grad = static_cast<const E*>(a.in);
    E* out = static_cast<E*>(a.out);
    int split = row_split(a.type, a.V, a.H);
    k_embed_zero<TYPE><<<row_blocks(a.V << split), kRowWg, 0, st>>>(out, a.V, a.H, a.out_stride, split);
    if (a.T == 0) return;
    const Plan p = plan_of(a.T, a.V, a.H);
    char* w = static_cast<char*>(a.ws);
    uint32_t* keys[2] = {reinterpret_cast<uint32_t*>(w), reinterpret_cast<uint32_t*>(w + p.keys)};
    uint32_t* from[2] = {reinterpret_cast<uint32_t*>(w + 2 * p.keys), reinterpret_cast<uint32_t*>(w + 3 * p.keys)};
    int32_t* hist = reinterpret_cast<int32_t*>(w + 4 * p.keys);
    float* part = reinterpret_cast<float*>(w + 4 * p.keys + p.hist);
    const unsigned grid = static_cast<unsigned>(p.blocks);
    const size_t lds = static_cast<size_t>(4 * kSortWaves) << p.bits;
    for (int i = 0; i < p.passes; ++i) {
      const int in = (i + 1) & 1, to = i & 1, shift = i * p.bits;
      if (i == 0) {
        k_sort_count<true><<<grid, kSortWg, 0, st>>>(a.tokens, a.V, nullptr, a.T, p.chunk, 0, 1 << p.bits, hist);
        k_sort_place<true><<<grid, kSortWg, lds, st>>>(a.tokens, a.V, nullptr, nullptr, a.T, p.chunk, 0, p.bits, hist, keys[to], from[to]);
      } else {
        k_sort_count<false><<<grid, kSortWg, 0, st>>>(a.tokens, a.V, keys[in], a.T, p.chunk, shift, 1 << p.bits, hist);
        k_sort_place<false><<<grid, kSortWg, lds, st>>>(a.tokens, a.V, keys[in], from[in], a.T, p.chunk, shift, p.bits, hist, keys[to], from[to]);
      }
    }
    const uint32_t* k = keys[(p.passes + 1) & 1];
    const uint32_t* f = from[(p.passes + 1) & 1];
    split = row_split(a.type, p.token_chunks, a.H);
    k_embed_sum<TYPE><<<row_blocks(p.token_chunks << split), kRowWg, 0, st>>>(
        k, f, a.T, a.V, grad, a.H, a.stride, a.scale, out, a.out_stride, part, split);
    if (p.token_chunks > 1) {
      const dim3 g(static_cast<unsigned>(p.token_chunks - 1 < 65536 ? p.token_chunks - 1 : 65536),
                   static_cast<unsigned>((a.H + 63) / 64 < 64 ? (a.H + 63) / 64 : 64));
      k_embed_join<TYPE><<<g, kRowWg, 0, st>>>(k, a.T, a.V, a.H, a.scale, part, out, a.out_stride);
    }
  });
  return hipGetLastError();
}

}  // namespace bo
