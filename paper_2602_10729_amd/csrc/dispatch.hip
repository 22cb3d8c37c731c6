// Dispatch: the (row, choice) pairs grouped by expert, each expert's in rising
// order: a stable counting sort.
//
// At most kMaxBlocks blocks of whole tiles. One launch counts each block's
// pairs per expert; the second sums the blocks before its own for itself
// (kMaxBlocks rows of counts from L2 cost less than a third launch between),
// and places the pairs. A wave takes 64 pairs at a time in order: the pairs
// with a lane's expert are a mask, built from one ballot per bit of the
// expert's number, and a pair's rank is the wave's count so far plus the lower
// lanes of the mask. Counts of the waves of a tile are then summed in order.
// A tile is put in order in LDS first, so that an expert's pairs are written in
// runs (32 of a popular tile's 8192 over 256 experts) rather than four bytes
// here and there: 23 -> 19 us for 2.1M pairs.
// What bounds it: a tile's chain of ballots, LDS counts and barriers, one tile a
// compute unit: 2.1M pairs over 256 experts take 5.0 + 18.4 us (25 MB, 5.3 us at
// a copy's rate).
// What fits one tile takes one launch. Nothing depends on the order in which
// atomics arrive: they only add integers.
#include <algorithm>
#include <type_traits>

#include "serving.h"

namespace bo {
namespace {

constexpr int kWg = 1024;
constexpr int kWaves = kWg / 64;
constexpr int kMaxItems = 8;              // pairs a lane holds, at most
constexpr int kMaxBlocks = 256;

// Words of a block's counts: whole 16-byte groups.
__host__ __device__ constexpr int row_of(int E) { return (E + 3) & ~3; }

__global__ __launch_bounds__(kWg) void k_dispatch_count(const int32_t* __restrict__ ids, int64_t N,
                                                        int64_t chunk, int E,
                                                        int32_t* __restrict__ hist) {
  __shared__ int32_t cnt[BO_MAX_EXPERTS];
  if (threadIdx.x < E) cnt[threadIdx.x] = 0;
  __syncthreads();
  const int64_t p0 = blockIdx.x * chunk, p1 = min(N, p0 + chunk);
#pragma unroll 8
  for (int64_t p = p0 + threadIdx.x; p < p1; p += kWg) {
    const int id = ids[p];
    if (id >= 0 && id < E) atomicAdd(&cnt[id], 1);
  }
  __syncthreads();
  const int row = row_of(E);
  if (threadIdx.x < row) hist[blockIdx.x * row + threadIdx.x] = threadIdx.x < E ? cnt[threadIdx.x] : 0;
}

// Thread e's `kept` summed over the threads before it. Two barriers.
__device__ int scan_before(int kept, int* wave_sum) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int s = kept;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int o = __shfl_up(s, off);
    s += lane >= off ? o : 0;
  }
  if (lane == 63) wave_sum[wave] = s;
  __syncthreads();
  int before = s - kept;
  for (int w = 0; w < kWaves; ++w) before += w < wave ? wave_sum[w] : 0;
  __syncthreads();
  return before;
}

// Dynamic LDS: the waves' counts [kWaves][E]; unless ONE, the tile's places in
// `order` and pairs, sorted by expert.
// ITEMS: pairs a lane holds; a tile is kWg times as many.
template <bool ONE, int ITEMS>
__global__ __launch_bounds__(kWg) void k_dispatch_place(const int32_t* __restrict__ ids, int64_t N,
                                                        int64_t chunk, int E, int64_t capacity,
                                                        const int32_t* __restrict__ hist,
                                                        int32_t* __restrict__ load,
                                                        int32_t* __restrict__ offsets,
                                                        int32_t* __restrict__ order,
                                                        int32_t* __restrict__ position) {
  constexpr int kTile = kWg * ITEMS;
  extern __shared__ int32_t cnt[];
  int32_t* places = cnt + kWaves * E;
  uint16_t* pairs = reinterpret_cast<uint16_t*>(places + kTile);
  __shared__ int32_t all[BO_MAX_EXPERTS];     // pairs of an expert
  __shared__ int32_t seen[BO_MAX_EXPERTS];    // of them before this tile
  __shared__ int32_t start[BO_MAX_EXPERTS];   // where the expert's pairs begin
  __shared__ int32_t slot0[BO_MAX_EXPERTS];   // its first slot in the tile, less `seen` before it
  __shared__ int wave_sum[kWaves];
  __shared__ int kept_total;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t cap = capacity > 0 ? capacity : N;
  const auto offsets_of = [&]() {
    const int n = tid < E ? all[tid] : 0;
    const int kept = n < cap ? n : static_cast<int>(cap);
    const int at = scan_before(kept, wave_sum);
    if (tid < E) {
      start[tid] = at;
      if (blockIdx.x == 0) {
        load[tid] = n;
        offsets[tid] = at;
      }
    }
    if (tid == kWg - 1) {                     // (threads past E keep nothing)
      kept_total = at + kept;
      if (blockIdx.x == 0) offsets[E] = at + kept;
    }
    __syncthreads();
  };
  if (tid < E) {
    all[tid] = 0;
    seen[tid] = 0;
  }
  // a tile: wave after wave, 64 pairs at a time (past its end the last pair
  // again); the first is on its way while the counts are summed
  const int64_t p0 = blockIdx.x * chunk, p1 = min(N, p0 + chunk);
  const int w0 = wave * 64 * ITEMS + lane;
  int id[ITEMS];
  const auto fetch = [&](int64_t t0) {
    const int n = static_cast<int>(min<int64_t>(kTile, p1 - t0));
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) id[i] = ids[t0 + min(w0 + 64 * i, n - 1)];
  };
  fetch(p0);
  __syncthreads();
  if (!ONE) {
    // every thread sums some blocks' counts of four experts, all loads at once
    const int quads = row_of(E) / 4;
    int width = 16;
    while (width < quads) width <<= 1;
    const int e = (tid & (width - 1)) * 4, parts = kWg / width, nb = static_cast<int>(gridDim.x);
    if (e < E) {
      const int4* rows = reinterpret_cast<const int4*>(hist + e);
      int4 before = {0, 0, 0, 0}, total = {0, 0, 0, 0};
#pragma unroll 16
      for (int b = tid / width; b < nb; b += parts) {
        const int4 n = rows[b * quads];
        const int on = b < static_cast<int>(blockIdx.x) ? -1 : 0;
        total.x += n.x; total.y += n.y; total.z += n.z; total.w += n.w;
        before.x += n.x & on; before.y += n.y & on; before.z += n.z & on; before.w += n.w & on;
      }
      const int t[4] = {total.x, total.y, total.z, total.w}, f[4] = {before.x, before.y, before.z, before.w};
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (e + i < E) {
          atomicAdd(&all[e + i], t[i]);
          atomicAdd(&seen[e + i], f[i]);
        }
    }
    __syncthreads();
    offsets_of();
  }
  int bits = 0;
  while ((1 << bits) < E) ++bits;
  for (int64_t t0 = p0; t0 < p1; t0 += kTile) {
    const int n = static_cast<int>(min<int64_t>(kTile, p1 - t0));
    for (int i = tid; i < kWaves * E; i += kWg) cnt[i] = 0;
    __syncthreads();
    int32_t* mine = cnt + wave * E;
    int e[ITEMS], rank[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) e[i] = w0 + 64 * i < n && id[i] >= 0 && id[i] < E ? id[i] : E;
    if (t0 + kTile < p1) fetch(t0 + kTile);
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const bool on = e[i] < E;
      const unsigned long long live = __ballot(on);
      unsigned lo = static_cast<unsigned>(live), hi = static_cast<unsigned>(live >> 32);
      for (int b = 0; b < bits; ++b) {
        const unsigned set = -((static_cast<unsigned>(e[i]) >> b) & 1u);
        const unsigned long long v = __ballot(set != 0);
        lo &= ~(static_cast<unsigned>(v) ^ set);
        hi &= ~(static_cast<unsigned>(v >> 32) ^ set);
      }
      const int before = __builtin_amdgcn_mbcnt_hi(hi, __builtin_amdgcn_mbcnt_lo(lo, 0));
      rank[i] = (on ? mine[e[i]] : 0) + before;
      // all lanes have read before the first of each expert writes; a wave's
      // LDS accesses stay in order
      __builtin_amdgcn_wave_barrier();
      if (on && before == 0) mine[e[i]] = rank[i] + __popc(lo) + __popc(hi);
      __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    int run = tid < E ? seen[tid] : 0;
    const int prior = run;
    if (tid < E) {
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const int c = cnt[w * E + tid];
        cnt[w * E + tid] = run;
        run += c;
      }
      seen[tid] = run;
      if (ONE) all[tid] = run;
    }
    if (ONE) {
      __syncthreads();
      offsets_of();
    } else {
      const int at = scan_before(run - prior, wave_sum);
      if (tid < E) slot0[tid] = at - prior;
      __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int at = w0 + 64 * i;
      if (at < n) {
        const int64_t p = t0 + at;
        int place = -1;
        if (e[i] < E) {
          const int r = mine[e[i]] + rank[i];
          if (r < cap) place = start[e[i]] + r;
          if (ONE) {
            if (place >= 0) order[place] = static_cast<int32_t>(p);
          } else {
            places[slot0[e[i]] + r] = place;
            pairs[slot0[e[i]] + r] = static_cast<uint16_t>(at);
          }
        }
        position[p] = place;
        if (p >= kept_total) order[p] = -1;
      }
    }
    __syncthreads();
    if (!ONE) {
      const int sorted = slot0[E - 1] + seen[E - 1];
      for (int i = tid; i < sorted; i += kWg)
        if (places[i] >= 0) order[places[i]] = static_cast<int32_t>(t0 + pairs[i]);
      __syncthreads();
    }
  }
}

__global__ __launch_bounds__(kWg) void k_dispatch_none(int E, int32_t* load, int32_t* offsets) {
  if (threadIdx.x < E) load[threadIdx.x] = offsets[threadIdx.x + 1] = 0;
  if (threadIdx.x == 0) offsets[0] = 0;
}

// Pairs a lane holds (1, 2, 4 or 8): the fewest that keep the blocks to
// kMaxBlocks, or hold everything in one.
int items_of(int64_t N) {
  int items = 1;
  while (items < kMaxItems && N > (int64_t)kWg * items * (N > kWg * kMaxItems ? kMaxBlocks : 1)) items *= 2;
  return items;
}
// Pairs a block takes: whole tiles (2^21 pairs are 256 blocks of one and take
// 22 us, 2^21 + 1 are 129 blocks of two and take 33).
int64_t chunk_of(int64_t N) {
  const int64_t tile = (int64_t)kWg * items_of(N), each = (N + kMaxBlocks - 1) / kMaxBlocks;
  return N <= kWg * kMaxItems ? tile : (each + tile - 1) / tile * tile;
}
int64_t blocks_of(int64_t N) { return (N + chunk_of(N) - 1) / chunk_of(N); }

}  // namespace

int64_t dispatch_workspace(int64_t N, int E) {
  return blocks_of(N) <= 1 ? 0 : 4 * blocks_of(N) * row_of(E);
}

hipError_t launch_dispatch(const int32_t* ids, int64_t N, int E, int64_t capacity, int32_t* load,
                           int32_t* offsets, int32_t* order, int32_t* position, void* ws,
                           hipStream_t st) {
  if (N == 0) {
    k_dispatch_none<<<1, kWg, 0, st>>>(E, load, offsets);
    return hipGetLastError();
  }
  int32_t* hist = static_cast<int32_t*>(ws);
  const int64_t chunk = chunk_of(N);
  const unsigned grid = static_cast<unsigned>(blocks_of(N));
  const auto place = [&](auto items) {
    constexpr int I = decltype(items)::value;
    const size_t counts = static_cast<size_t>(4) * kWaves * E;
    if (grid == 1)
      k_dispatch_place<true, I><<<1, kWg, counts, st>>>(ids, N, chunk, E, capacity, hist, load, offsets, order, position);
    else
      k_dispatch_place<false, I><<<grid, kWg, counts + kWg * I * 6, st>>>(ids, N, chunk, E, capacity, hist, load, offsets, order, position);
  };
  if (grid > 1) k_dispatch_count<<<grid, kWg, 0, st>>>(ids, N, chunk, E, hist);
  switch (items_of(N)) {
    case 1: place(std::integral_constant<int, 1>()); break;
    case 2: place(std::integral_constant<int, 2>()); break;
    case 4: place(std::integral_constant<int, 4>()); break;
    default: place(std::integral_constant<int, 8>());
  }
  return hipGetLastError();
}

}  // namespace bo
