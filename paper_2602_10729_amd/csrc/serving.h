// Internal declarations of the served-output operators: log probabilities
// (logprobs.hip), routing (route.hip) and dispatch (dispatch.hip).
#pragma once

#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>
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
  using T = __hip_bfloat16;
  static __device__ __forceinline__ float load(T v) { return __bfloat162float(v); }
  static __device__ __forceinline__ T store(float v) { return __float2bfloat16(v); }
};
template <>
struct Elem<BO_TYPE_F16> {
  using T = __half;
  static __device__ __forceinline__ float load(T v) { return __half2float(v); }
  static __device__ __forceinline__ T store(float v) { return __float2half(v); }
};

inline size_t type_bytes(int type) { return type == BO_TYPE_F32 ? 4 : 2; }

struct LogprobArgs {
  const void* logits;
  int type;
  int64_t T, V, stride;
  const int64_t* tokens;       // or nullptr
  float it;                    // inverse temperature
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
