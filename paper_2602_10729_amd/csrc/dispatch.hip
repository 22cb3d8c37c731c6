// Dispatch: the (row, choice) pairs grouped by expert, each expert's in rising
// order: a stable counting sort.
//
// Blocks of kBlock pairs. One launch counts each block's pairs per expert,
// one sums the counts (over earlier blocks, then over lower experts), and one
// places the pairs: a wave takes its 64 pairs in order, and a pair's place
// among its wave's equals comes from a mask of the lanes with the same expert.
// Nothing depends on the order in which atomics arrive.
#include "serving.h"

namespace bo {
namespace {

constexpr int kWg = 256;
constexpr int kBlock = 2048;

__global__ __launch_bounds__(kWg) void k_dispatch_count(const int32_t* __restrict__ ids, int64_t N,
                                                        int E, int32_t* __restrict__ hist) {
  __shared__ int32_t cnt[BO_MAX_EXPERTS];
  for (int e = threadIdx.x; e < E; e += kWg) cnt[e] = 0;
  __syncthreads();
  const int64_t p0 = (int64_t)blockIdx.x * kBlock;
  for (int i = threadIdx.x; i < kBlock; i += kWg) {
    const int64_t p = p0 + i;
    const int id = p < N ? ids[p] : -1;
    if (id >= 0 && id < E) atomicAdd(&cnt[id], 1);
  }
  __syncthreads();
  for (int e = threadIdx.x; e < E; e += kWg) hist[(int64_t)blockIdx.x * E + e] = cnt[e];
}

// One workgroup: per expert the blocks' counts become the counts of the blocks
// before, then loads and offsets.
__global__ __launch_bounds__(1024) void k_dispatch_scan(int32_t* __restrict__ hist, int64_t blocks,
                                                        int E, int64_t capacity,
                                                        int32_t* __restrict__ load,
                                                        int32_t* __restrict__ offsets) {
  __shared__ int32_t kept[1024];
  const int e = threadIdx.x;
  int32_t run = 0;
  if (e < E) {
    for (int64_t b = 0; b < blocks; ++b) {
      const int32_t c = hist[b * E + e];
      hist[b * E + e] = run;
      run += c;
    }
    load[e] = run;
  }
  kept[e] = e < E ? (capacity > 0 && run > capacity ? static_cast<int32_t>(capacity) : run) : 0;
  for (int off = 1; off < 1024; off <<= 1) {
    __syncthreads();
    const int32_t v = e >= off ? kept[e - off] : 0;
    __syncthreads();
    kept[e] += v;
  }
  if (e < E) offsets[e + 1] = kept[e];
  if (e == 0) offsets[0] = 0;
}

__global__ __launch_bounds__(64) void k_dispatch_place(const int32_t* __restrict__ ids, int64_t N,
                                                       int E, int64_t capacity,
                                                       const int32_t* __restrict__ hist,
                                                       const int32_t* __restrict__ offsets,
                                                       int32_t* __restrict__ order,
                                                       int32_t* __restrict__ position) {
  __shared__ int32_t seen[BO_MAX_EXPERTS];
  const int lane = threadIdx.x;
  for (int e = lane; e < E; e += 64) seen[e] = hist[(int64_t)blockIdx.x * E + e];
  __syncthreads();
  const int64_t p0 = (int64_t)blockIdx.x * kBlock;
  const int64_t total = offsets[E];
  int bits = 0;
  while ((1 << bits) <= E) ++bits;
  for (int i = 0; i < kBlock; i += 64) {
    const int64_t p = p0 + i + lane;
    const int id = p < N ? ids[p] : -1;
    const bool on = id >= 0 && id < E;
    const int e = on ? id : E;
    unsigned long long same = ~0ull;
    for (int b = 0; b < bits; ++b) {
      const unsigned long long v = __ballot((e >> b) & 1);
      same &= ((e >> b) & 1) ? v : ~v;
    }
    const int before = __popcll(same & ((1ull << lane) - 1));
    const int base = on ? seen[e] : 0;
    __syncthreads();
    if (on && before == 0) seen[e] = base + __popcll(same);
    __syncthreads();
    if (p < N) {
      const int64_t rank = (int64_t)base + before;
      const bool goes = on && (capacity == 0 || rank < capacity);
      const int64_t at = goes ? offsets[e] + rank : -1;
      position[p] = static_cast<int32_t>(at);
      if (goes) order[at] = static_cast<int32_t>(p);
      if (p >= total) order[p] = -1;
    }
  }
}

int64_t blocks_of(int64_t N) { return (N + kBlock - 1) / kBlock; }

}  // namespace

int64_t dispatch_workspace(int64_t N, int E) { return N > 0 ? 4 * blocks_of(N) * E : 0; }

hipError_t launch_dispatch(const int32_t* ids, int64_t N, int E, int64_t capacity, int32_t* load,
                           int32_t* offsets, int32_t* order, int32_t* position, void* ws,
                           hipStream_t st) {
  int32_t* hist = static_cast<int32_t*>(ws);
  const int64_t nb = blocks_of(N);
  const dim3 grid(static_cast<unsigned>(nb));
  if (nb > 0) k_dispatch_count<<<grid, kWg, 0, st>>>(ids, N, E, hist);
  k_dispatch_scan<<<1, 1024, 0, st>>>(hist, nb, E, capacity, load, offsets);
  if (nb > 0)
    k_dispatch_place<<<grid, 64, 0, st>>>(ids, N, E, capacity, hist, offsets, order, position);
  return hipGetLastError();
}

}  // namespace bo
