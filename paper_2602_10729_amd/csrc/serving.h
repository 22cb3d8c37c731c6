// Internal declarations of the served-output operators: log probabilities
// (logprobs.hip), routing (route.hip) and dispatch (dispatch.hip).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "bo_internal.h"

namespace bo {

// Element types of logits: conversion to fp32 and one rounding back.
template <int TYPE>
struct Elem;
template <>
struct Elem<BO_TYPE_F32> {
  using T = float;
  static __device__ __forceinline__ float load(T v) { return v; }
  static __device__ __forceinline__ T store(float v) { return v; }
};
template <>
struct Elem<BO_TYPE_BF16> {
  using T = __bf16;
  static __device__ __forceinline__ float load(T v) { return static_cast<float>(v); }
  static __device__ __forceinline__ T store(float v) { return static_cast<__bf16>(v); }
};
template <>
struct Elem<BO_TYPE_F16> {
  using T = _Float16;
  static __device__ __forceinline__ float load(T v) { return static_cast<float>(v); }
  static __device__ __forceinline__ T store(float v) { return static_cast<_Float16>(v); }
};

// Sixteen bytes of logits in registers: kVec elements.
template <int TYPE>
struct Vec {
  using T = typename Elem<TYPE>::T;
  static constexpr int kVec = 16 / sizeof(T);
  uint32_t q[4];
  // Any alignment: rows start where their stride puts them, and the memory
  // system takes a 16-byte access at every address. STREAM: past the caches.
  typedef uint32_t Any __attribute__((ext_vector_type(4), aligned(2)));
  template <bool STREAM = false>
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (STREAM) {
      const Any v = __builtin_nontemporal_load(reinterpret_cast<const Any*>(p));
#pragma unroll
      for (int i = 0; i < 4; ++i) q[i] = v[i];
    } else {
      __builtin_memcpy(q, p, 16);
    }
  }
  template <bool STREAM = false>
  __device__ __forceinline__ void store(T* p) const {
    if constexpr (STREAM) __builtin_nontemporal_store(Any{q[0], q[1], q[2], q[3]}, reinterpret_cast<Any*>(p));
    else __builtin_memcpy(p, q, 16);
  }
  // the first n elements, the rest -inf (the first one read again)
  __device__ __forceinline__ void load_part(const T* p, int n) {
    fill_masked();
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
      const uint32_t b = bits_of(p[e < n ? e : 0]);
      if (e < n) {
        if constexpr (kVec == 4) q[e] = b;
        else q[e / 2] = (e & 1) ? (q[e / 2] & 0xFFFFu) | (b << 16) : (q[e / 2] & 0xFFFF0000u) | b;
      }
    }
  }
  __device__ __forceinline__ void store_part(T* p, int n) const {
#pragma unroll
    for (int e = 0; e < kVec; ++e)
      if (e < n) {
        if constexpr (kVec == 4) {
          __builtin_memcpy(p + e, &q[e], 4);
        } else {
          const uint16_t h = static_cast<uint16_t>(q[e / 2] >> (16 * (e & 1)));
          __builtin_memcpy(p + e, &h, 2);
        }
      }
  }
  // Drops the first n elements and fills with -inf from behind (n >= 0; all of
  // them from kVec on).
  __device__ __forceinline__ void drop(int n) {
    const uint32_t b = bits_of(Elem<TYPE>::store(-__builtin_huge_valf()));
    const uint32_t f = kVec == 4 ? b : b | (b << 16);
    if constexpr (kVec == 8) {
      const bool one = n & 1;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t s = __builtin_amdgcn_alignbit(i < 3 ? q[i + 1] : f, q[i], 16);
        q[i] = one ? s : q[i];
      }
      n >>= 1;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = (n & 1) ? (i < 3 ? q[i + 1] : f) : q[i];
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = (n & 2) ? (i < 2 ? q[i + 2] : f) : q[i];
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = n >= 4 ? f : q[i];
  }
  __device__ __forceinline__ void fill_masked() {
    const uint32_t b = bits_of(Elem<TYPE>::store(-__builtin_huge_valf()));
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = kVec == 4 ? b : b | (b << 16);
  }
  __device__ __forceinline__ float get(int e) const {
    if constexpr (TYPE == BO_TYPE_F32) return __uint_as_float(q[e]);
    if constexpr (TYPE == BO_TYPE_BF16)
      return __uint_as_float((e & 1) ? (q[e / 2] & 0xFFFF0000u) : (q[e / 2] << 16));
    const uint16_t h = static_cast<uint16_t>(q[e / 2] >> (16 * (e & 1)));
    _Float16 f;
    __builtin_memcpy(&f, &h, 2);
    return static_cast<float>(f);
  }
  // every element, each rounded once
  __device__ __forceinline__ void set_all(const float (&v)[kVec]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (kVec == 4) {
        q[i] = __float_as_uint(v[i]);
      } else {
        typedef T T2 __attribute__((ext_vector_type(2)));
        const T2 h = {Elem<TYPE>::store(v[2 * i]), Elem<TYPE>::store(v[2 * i + 1])};
        __builtin_memcpy(&q[i], &h, 4);
      }
    }
  }

 private:
  static __device__ __forceinline__ uint32_t bits_of(T v) {
    if constexpr (kVec == 4) {
      return __float_as_uint(v);
    } else {
      uint16_t h;
      __builtin_memcpy(&h, &v, 2);
      return h;
    }
  }
};

// A value's order as an unsigned number (-0 and +0 are equal).
__device__ __forceinline__ unsigned code_of(float v) {
  const unsigned u = __float_as_uint(v + 0.0f);
  return u ^ (static_cast<unsigned>(static_cast<int>(u) >> 31) | 0x80000000u);
}
// Larger value first, the lower index among equals, as the unsigned order of
// one 64-bit key; 0 is below every key of a value.
__device__ __forceinline__ unsigned long long pack_key(float v, unsigned j) {
  return (static_cast<unsigned long long>(code_of(v)) << 32) | (0xFFFFFFFFu - j);
}
__device__ __forceinline__ float ordered_value(unsigned o) {
  return __uint_as_float((o & 0x80000000u) ? (o & 0x7FFFFFFFu) : ~o);
}
__device__ __forceinline__ float key_value(unsigned long long k) {
  return ordered_value(static_cast<unsigned>(k >> 32));
}
__device__ __forceinline__ int key_index(unsigned long long k) {
  return static_cast<int>(0xFFFFFFFFu - static_cast<unsigned>(k));
}

// max of three, NaN if one of them is
__device__ __forceinline__ float max3_nan(float a, float b, float c) {
  float d;
  asm("v_maximum3_f32 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "v"(c));
  return d;
}
// max of two; a quiet NaN operand is dropped (a signalling one comes through quiet)
__device__ __forceinline__ float max2(float a, float b) {
  float d;
  asm("v_max_f32 %0, %1, %2" : "=v"(d) : "v"(a), "v"(b));
  return d;
}

inline size_t type_bytes(int type) { return type == BO_TYPE_F32 ? 4 : 2; }

struct LogprobArgs {
  const void* logits;
  int type;
  int64_t T, V, stride;
  const int64_t* tokens;       // or nullptr
  float it;                    // inverse temperature
  float c, slack;              // log2(e) it; how far a reference may lag, in logits
  int top;
  float* logprob;
  int32_t* rank;
  float* entropy;
  float* stats;                // [T][2]
  int32_t* top_ids;
  float* top_logprobs;
  void* ws;
};
int64_t logprob_workspace(int64_t T, int64_t V, int top);
hipError_t launch_logprobs(const LogprobArgs& a, hipStream_t st);

struct LogprobGradArgs {
  const void* logits;
  int type;
  int64_t T, V, stride;
  const int64_t* tokens;       // or nullptr
  float it;
  const float* stats;
  const float* entropy;
  const float* g_logprob;      // or nullptr
  const float* g_entropy;      // or nullptr
  int top;
  const int32_t* top_ids;
  const float* g_top;
  void* out;
  int64_t out_stride;
};
hipError_t launch_logprobs_grad(const LogprobGradArgs& a, hipStream_t st);

struct RouteArgs {
  const void* logits;
  int type;
  int64_t T;
  int E;
  int64_t stride;
  const float* bias;           // or nullptr
  int score, top, groups, top_groups, group_best, renorm;
  float scale;
  int32_t* ids;
  float* weights;
};
hipError_t launch_route(const RouteArgs& a, hipStream_t st);

struct RouteGradArgs {
  const void* logits;
  int type;
  int64_t T;
  int E;
  int64_t stride;
  int score, top, renorm;
  float scale;
  const int32_t* ids;
  const float* g;
  void* out;
  int64_t out_stride;
};
hipError_t launch_route_grad(const RouteGradArgs& a, hipStream_t st);

int64_t dispatch_workspace(int64_t N, int E);
hipError_t launch_dispatch(const int32_t* ids, int64_t N, int E, int64_t capacity, int32_t* load,
                           int32_t* offsets, int32_t* order, int32_t* position, void* ws,
                           hipStream_t st);

}  // namespace bo
