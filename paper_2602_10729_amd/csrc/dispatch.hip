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
// What fits one tile takes one launch. Nothing depends on the order in which
// atomics arrive: they only add integers.
#include <algorithm>

#include "serving.h"

namespace bo {
namespace {

constexpr int kWg = 1024;
constexpr int kWaves = kWg / 64;
constexpr int kItems = 8;                 // pairs a lane holds
constexpr int kTile = kWg * kItems;
constexpr int kMaxBlocks = 256;

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
  if (threadIdx.x < E) hist[(int64_t)blockIdx.x * E + threadIdx.x] = cnt[threadIdx.x];
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

// Dynamic LDS: the waves' counts [kWaves][E].
template <bool ONE>
__global__ __launch_bounds__(kWg) void k_dispatch_place(const int32_t* __restrict__ ids, int64_t N,
                                                        int64_t chunk, int E, int64_t capacity,
                                                        const int32_t* __restrict__ hist,
                                                        int32_t* __restrict__ load,
                                                        int32_t* __restrict__ offsets,
                                                        int32_t* __restrict__ order,
                                                        int32_t* __restrict__ position) {
  extern __shared__ int32_t cnt[];
  __shared__ int32_t all[BO_MAX_EXPERTS];     // pairs of an expert
  __shared__ int32_t seen[BO_MAX_EXPERTS];    // of them before this tile
  __shared__ int32_t start[BO_MAX_EXPERTS];   // where the expert's pairs begin
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
  __syncthreads();
  if (!ONE) {
    // every thread sums some blocks' counts of one expert
    int width = 64;
    while (width < E) width <<= 1;
    const int e = tid & (width - 1), parts = kWg / width;
    int before = 0, total = 0;
    if (e < E) {
#pragma unroll 8
      for (int b = tid / width; b < static_cast<int>(gridDim.x); b += parts) {
        const int n = hist[b * E + e];
        total += n;
        before += b < static_cast<int>(blockIdx.x) ? n : 0;
      }
      atomicAdd(&all[e], total);
      atomicAdd(&seen[e], before);
    }
    __syncthreads();
    offsets_of();
  }
  int bits = 0;
  while ((1 << bits) <= E) ++bits;
  const int64_t p0 = blockIdx.x * chunk, p1 = min(N, p0 + chunk);
  for (int64_t t0 = p0; t0 < p1; t0 += kTile) {
    const int n = static_cast<int>(min<int64_t>(kTile, p1 - t0));
    const int items = (n + kWg - 1) / kWg;    // pairs of a lane in this tile
    for (int i = tid; i < kWaves * E; i += kWg) cnt[i] = 0;
    __syncthreads();
    int32_t* mine = cnt + wave * E;
    const int w0 = wave * 64 * items + lane;
    int e[kItems], rank[kItems];
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int at = w0 + 64 * i;
      e[i] = E;
      if (i < items && at < n) {
        const int id = ids[t0 + at];
        if (id >= 0 && id < E) e[i] = id;
      }
    }
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      rank[i] = 0;
      if (i < items) {
        unsigned long long same = ~0ull;
        for (int b = 0; b < bits; ++b) {
          const bool set = (e[i] >> b) & 1;
          const unsigned long long v = __ballot(set);
          same &= set ? v : ~v;
        }
        const int before = __popcll(same & ((1ull << lane) - 1));
        const bool on = e[i] < E;
        rank[i] = (on ? mine[e[i]] : 0) + before;
        // all lanes have read before the first of each expert writes; a wave's
        // LDS accesses stay in order
        __builtin_amdgcn_wave_barrier();
        if (on && before == 0) mine[e[i]] = rank[i] + __popcll(same);
        __builtin_amdgcn_wave_barrier();
      }
    }
    __syncthreads();
    if (tid < E) {
      int run = seen[tid];
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const int c = cnt[w * E + tid];
        cnt[w * E + tid] = run;
        run += c;
      }
      seen[tid] = run;
      if (ONE) all[tid] = run;
    }
    __syncthreads();
    if (ONE) offsets_of();
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int at = w0 + 64 * i;
      if (i < items && at < n) {
        const int64_t p = t0 + at;
        int place = -1;
        if (e[i] < E) {
          const int r = mine[e[i]] + rank[i];
          if (r < cap) {
            place = start[e[i]] + r;
            order[place] = static_cast<int32_t>(p);
          }
        }
        position[p] = place;
        if (p >= kept_total) order[p] = -1;
      }
    }
    __syncthreads();
  }
}

__global__ __launch_bounds__(kWg) void k_dispatch_none(int E, int32_t* load, int32_t* offsets) {
  if (threadIdx.x < E) load[threadIdx.x] = offsets[threadIdx.x + 1] = 0;
  if (threadIdx.x == 0) offsets[0] = 0;
}

// Pairs a block takes: whole waves' worth, whole tiles once it is more than one.
int64_t chunk_of(int64_t N) {
  const int64_t each = (N + kMaxBlocks - 1) / kMaxBlocks;
  const int64_t unit = each <= kTile ? kWg : kTile;
  return (each + unit - 1) / unit * unit;
}
int64_t blocks_of(int64_t N) { return N <= kTile ? 1 : (N + chunk_of(N) - 1) / chunk_of(N); }

}  // namespace

int64_t dispatch_workspace(int64_t N, int E) { return N <= kTile ? 0 : 4 * blocks_of(N) * E; }

hipError_t launch_dispatch(const int32_t* ids, int64_t N, int E, int64_t capacity, int32_t* load,
                           int32_t* offsets, int32_t* order, int32_t* position, void* ws,
                           hipStream_t st) {
  const size_t lds = static_cast<size_t>(4) * kWaves * E;
  if (N == 0) {
    k_dispatch_none<<<1, kWg, 0, st>>>(E, load, offsets);
  } else if (N <= kTile) {
    k_dispatch_place<true><<<1, kWg, lds, st>>>(ids, N, N, E, capacity, nullptr, load, offsets, order, position);
  } else {
    int32_t* hist = static_cast<int32_t*>(ws);
    const unsigned grid = static_cast<unsigned>(blocks_of(N));
    k_dispatch_count<<<grid, kWg, 0, st>>>(ids, N, chunk_of(N), E, hist);
    k_dispatch_place<false><<<grid, kWg, lds, st>>>(ids, N, chunk_of(N), E, capacity, hist, load, offsets, order, position);
  }
  return hipGetLastError();
}

}  // namespace bo
