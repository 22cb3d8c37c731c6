// C ABI entry points of the served-output operators: validation and launch.
// They keep no state and allocate nothing on the device.
#include <hip/hip_runtime.h>

#include <cmath>
#include <string>

#include "serving.h"

namespace {

using bo::check_dev;
using bo::fail;

// Nothing may leave a C entry as an exception; the only ones here come from
// the host allocator, under the strings of error messages.
template <typename F>
bo_status guarded(F&& f) {
  try {
    return f();
  } catch (...) {
    return BO_ERR_OUT_OF_MEMORY;
  }
}

bool bad_type(int32_t type) {
  return type != BO_TYPE_F32 && type != BO_TYPE_BF16 && type != BO_TYPE_F16;
}

// Bytes from the first to the last element of T rows of `cols`, `stride` apart,
// or -1 when the count overflows.
int64_t span_bytes(int64_t T, int64_t cols, int64_t stride, size_t es) {
  if (T <= 1) return cols * static_cast<int64_t>(es);
  int64_t n = 0;
  if (__builtin_mul_overflow(T - 1, stride, &n) || __builtin_add_overflow(n, cols, &n) ||
      __builtin_mul_overflow(n, static_cast<int64_t>(es), &n))
    return -1;
  return n;
}

// A matrix of `type` on the device: its pointer, alignment, stride and extent.
bo_status check_rows(const void* p, int32_t type, int64_t T, int64_t cols, int64_t stride,
                     const char* where, const char* name) {
  const size_t es = bo::type_bytes(type);
  const std::string W = std::string(where) + ": " + name;
  if (T > 1 && stride < cols) return fail(BO_ERR_INVALID_ARGUMENT, W + "'s stride is below its columns");
  const int64_t n = span_bytes(T, cols, stride, es);
  if (n < 0) return fail(BO_ERR_CAPACITY, W + " is too large");
  if (reinterpret_cast<uintptr_t>(p) % es) return fail(BO_ERR_INVALID_ARGUMENT, W + " is not aligned to its type");
  return check_dev(p, static_cast<size_t>(n), name);
}

// A gradient may take its input's place exactly, or must lie apart from it.
bo_status check_overlap(const void* in, int64_t in_stride, const void* out, int64_t out_stride,
                        int32_t type, int64_t T, int64_t cols, const char* where) {
  if (in == out && (T <= 1 || in_stride == out_stride)) return BO_OK;
  const size_t es = bo::type_bytes(type);
  const uintptr_t a = reinterpret_cast<uintptr_t>(in), b = reinterpret_cast<uintptr_t>(out);
  const uintptr_t ae = a + static_cast<uintptr_t>(span_bytes(T, cols, in_stride, es));
  const uintptr_t be = b + static_cast<uintptr_t>(span_bytes(T, cols, out_stride, es));
  if (a < be && b < ae)
    return fail(BO_ERR_INVALID_ARGUMENT, std::string(where) + ": grad_logits overlaps logits");
  return BO_OK;
}

bo_status check_workspace(const void* p, int64_t have, int64_t need, const char* where) {
  if (need == 0) return BO_OK;
  if (have < need) return fail(BO_ERR_INVALID_ARGUMENT, std::string(where) + ": workspace too small");
  if (reinterpret_cast<uintptr_t>(p) % 16)
    return fail(BO_ERR_INVALID_ARGUMENT, std::string(where) + ": workspace is not aligned to 16 bytes");
  return check_dev(p, static_cast<size_t>(need), "workspace");
}

constexpr int64_t kMaxRows = (int64_t)1 << 40;

// The sizes that bo_token_logprobs and its gradient share.
bo_status check_logprob_sizes(int32_t type, int64_t T, int64_t V, float it, int32_t top,
                              const char* where) {
  const std::string W(where);
  if (bad_type(type)) return fail(BO_ERR_INVALID_ARGUMENT, W + ": unknown type");
  if (T < 0 || V < 1) return fail(BO_ERR_INVALID_ARGUMENT, W + ": T < 0 or V < 1");
  if (!(it > 0.0f) || !(it <= 1e30f))     // (beyond, a product with log2(e) or a logit is no number)
    return fail(BO_ERR_INVALID_ARGUMENT, W + ": inv_temperature must be in (0, 1e30]");
  if (top < 0) return fail(BO_ERR_INVALID_ARGUMENT, W + ": top < 0");
  if (V >= ((int64_t)1 << 31) || T > kMaxRows) return fail(BO_ERR_CAPACITY, W + ": T or V beyond limit");
  if (top > BO_MAX_ALTERNATIVES) return fail(BO_ERR_CAPACITY, W + ": top beyond BO_MAX_ALTERNATIVES");
  return BO_OK;
}

bo_status check_route_sizes(int32_t type, int64_t T, int32_t E, int32_t score, int32_t top,
                            float scale, const char* where) {
  const std::string W(where);
  if (bad_type(type)) return fail(BO_ERR_INVALID_ARGUMENT, W + ": unknown type");
  if (T < 0 || E < 1) return fail(BO_ERR_INVALID_ARGUMENT, W + ": T < 0 or E < 1");
  if (score != BO_SCORE_SOFTMAX && score != BO_SCORE_SIGMOID)
    return fail(BO_ERR_INVALID_ARGUMENT, W + ": unknown score");
  if (top < 1) return fail(BO_ERR_INVALID_ARGUMENT, W + ": top < 1");
  if (!std::isfinite(scale)) return fail(BO_ERR_INVALID_ARGUMENT, W + ": scale is not finite");
  if (E > BO_MAX_EXPERTS) return fail(BO_ERR_CAPACITY, W + ": E beyond BO_MAX_EXPERTS");
  if (top > BO_MAX_CHOICES) return fail(BO_ERR_CAPACITY, W + ": top beyond BO_MAX_CHOICES");
  if (T > kMaxRows) return fail(BO_ERR_CAPACITY, W + ": T beyond limit");
  return BO_OK;
}

}  // namespace

extern "C" {

int64_t bo_token_logprobs_workspace(int64_t T, int64_t V, int32_t top) {
  if (T < 1 || V < 1 || top < 0 || top > BO_MAX_ALTERNATIVES || T > kMaxRows || V >= ((int64_t)1 << 31))
    return 0;
  return bo::logprob_workspace(T, V, top);
}

bo_status bo_token_logprobs(const void* logits, int32_t type, int64_t T, int64_t V, int64_t stride,
                            const int64_t* tokens, float inv_temperature, int32_t top,
                            float* logprob, int32_t* rank, float* entropy, float* stats,
                            int32_t* top_ids, float* top_logprobs, void* workspace,
                            int64_t workspace_bytes, void* stream) {
  return guarded([&]() -> bo_status {
    const char* W = "bo_token_logprobs";
    bo_status s = check_logprob_sizes(type, T, V, inv_temperature, top, W);
    if (s != BO_OK) return s;
    if (top > V) return fail(BO_ERR_INVALID_ARGUMENT, "bo_token_logprobs: top > V");
    if (T == 0) return BO_OK;
    if ((s = check_rows(logits, type, T, V, stride, W, "logits")) != BO_OK) return s;
    const size_t n = static_cast<size_t>(T);
    if (tokens && (s = check_dev(tokens, 8 * n, "tokens")) != BO_OK) return s;
    if ((s = check_dev(logprob, 4 * n, "logprob")) != BO_OK) return s;
    if ((s = check_dev(rank, 4 * n, "rank")) != BO_OK) return s;
    if ((s = check_dev(entropy, 4 * n, "entropy")) != BO_OK) return s;
    if ((s = check_dev(stats, 8 * n, "stats")) != BO_OK) return s;
    if (top > 0) {
      if ((s = check_dev(top_ids, 4 * n * top, "top_ids")) != BO_OK) return s;
      if ((s = check_dev(top_logprobs, 4 * n * top, "top_logprobs")) != BO_OK) return s;
    }
    if ((s = check_workspace(workspace, workspace_bytes, bo::logprob_workspace(T, V, top), W)) != BO_OK)
      return s;
    bo::LogprobArgs a{logits, type, T, V, stride, tokens, inv_temperature, 0.0f, 0.0f, top, logprob, rank,
                      entropy, stats, top_ids, top_logprobs, workspace};
    hipStream_t st = static_cast<hipStream_t>(stream);
    return bo::after_launch(bo::launch_logprobs(a, st), st, W);
  });
}

bo_status bo_token_logprobs_grad(const void* logits, int32_t type, int64_t T, int64_t V,
                                 int64_t stride, const int64_t* tokens, float inv_temperature,
                                 const float* stats, const float* entropy,
                                 const float* grad_logprob, const float* grad_entropy, int32_t top,
                                 const int32_t* top_ids, const float* grad_top, void* grad_logits,
                                 int64_t grad_stride, void* stream) {
  return guarded([&]() -> bo_status {
    const char* W = "bo_token_logprobs_grad";
    bo_status s = check_logprob_sizes(type, T, V, inv_temperature, top, W);
    if (s != BO_OK) return s;
    if (T == 0) return BO_OK;
    if ((s = check_rows(logits, type, T, V, stride, W, "logits")) != BO_OK) return s;
    if ((s = check_rows(grad_logits, type, T, V, grad_stride, W, "grad_logits")) != BO_OK) return s;
    if ((s = check_overlap(logits, stride, grad_logits, grad_stride, type, T, V, W)) != BO_OK) return s;
    const size_t n = static_cast<size_t>(T);
    if (tokens && (s = check_dev(tokens, 8 * n, "tokens")) != BO_OK) return s;
    if ((s = check_dev(stats, 8 * n, "stats")) != BO_OK) return s;
    if ((s = check_dev(entropy, 4 * n, "entropy")) != BO_OK) return s;
    if (grad_logprob && (s = check_dev(grad_logprob, 4 * n, "grad_logprob")) != BO_OK) return s;
    if (grad_entropy && (s = check_dev(grad_entropy, 4 * n, "grad_entropy")) != BO_OK) return s;
    if (top > 0) {
      if ((s = check_dev(top_ids, 4 * n * top, "top_ids")) != BO_OK) return s;
      if ((s = check_dev(grad_top, 4 * n * top, "grad_top")) != BO_OK) return s;
    }
    bo::LogprobGradArgs a{logits, type, T, V, stride, tokens, inv_temperature, stats, entropy,
                          grad_logprob, grad_entropy, top, top_ids, grad_top, grad_logits,
                          grad_stride};
    hipStream_t st = static_cast<hipStream_t>(stream);
    return bo::after_launch(bo::launch_logprobs_grad(a, st), st, W);
  });
}

bo_status bo_route(const void* logits, int32_t type, int64_t T, int32_t E, int64_t stride,
                   const float* bias, int32_t score, int32_t top, int32_t groups,
                   int32_t top_groups, int32_t group_best, int32_t renormalise, float scale,
                   int32_t* ids, float* weights, void* stream) {
  return guarded([&]() -> bo_status {
    const char* W = "bo_route";
    bo_status s = check_route_sizes(type, T, E, score, top, scale, W);
    if (s != BO_OK) return s;
    if (groups < 1 || groups > E || E % groups)
      return fail(BO_ERR_INVALID_ARGUMENT, "bo_route: groups must divide E");
    if (top_groups < 1 || top_groups > groups)
      return fail(BO_ERR_INVALID_ARGUMENT, "bo_route: top_groups out of range");
    if (group_best < 1 || group_best > 2 || group_best > E / groups)
      return fail(BO_ERR_INVALID_ARGUMENT, "bo_route: group_best out of range");
    if (top > E / groups * top_groups)
      return fail(BO_ERR_INVALID_ARGUMENT, "bo_route: top exceeds the experts of top_groups groups");
    if (T == 0) return BO_OK;
    if ((s = check_rows(logits, type, T, E, stride, W, "logits")) != BO_OK) return s;
    if (bias && (s = check_dev(bias, 4 * static_cast<size_t>(E), "bias")) != BO_OK) return s;
    const size_t n = static_cast<size_t>(T) * top;
    if ((s = check_dev(ids, 4 * n, "ids")) != BO_OK) return s;
    if ((s = check_dev(weights, 4 * n, "weights")) != BO_OK) return s;
    bo::RouteArgs a{logits, type, T, E, stride, bias, score, top, groups, top_groups, group_best,
                    renormalise != 0, scale, ids, weights};
    hipStream_t st = static_cast<hipStream_t>(stream);
    return bo::after_launch(bo::launch_route(a, st), st, W);
  });
}

bo_status bo_route_grad(const void* logits, int32_t type, int64_t T, int32_t E, int64_t stride,
                        int32_t score, int32_t top, int32_t renormalise, float scale,
                        const int32_t* ids, const float* grad_weights, void* grad_logits,
                        int64_t grad_stride, void* stream) {
  return guarded([&]() -> bo_status {
    const char* W = "bo_route_grad";
    bo_status s = check_route_sizes(type, T, E, score, top, scale, W);
    if (s != BO_OK) return s;
    if (top > E) return fail(BO_ERR_INVALID_ARGUMENT, "bo_route_grad: top > E");
    if (T == 0) return BO_OK;
    if ((s = check_rows(logits, type, T, E, stride, W, "logits")) != BO_OK) return s;
    if ((s = check_rows(grad_logits, type, T, E, grad_stride, W, "grad_logits")) != BO_OK) return s;
    if ((s = check_overlap(logits, stride, grad_logits, grad_stride, type, T, E, W)) != BO_OK) return s;
    const size_t n = static_cast<size_t>(T) * top;
    if ((s = check_dev(ids, 4 * n, "ids")) != BO_OK) return s;
    if ((s = check_dev(grad_weights, 4 * n, "grad_weights")) != BO_OK) return s;
    bo::RouteGradArgs a{logits, type, T, E, stride, score, top, renormalise != 0, scale, ids,
                        grad_weights, grad_logits, grad_stride};
    hipStream_t st = static_cast<hipStream_t>(stream);
    return bo::after_launch(bo::launch_route_grad(a, st), st, W);
  });
}

int64_t bo_dispatch_workspace(int64_t N, int32_t E) {
  if (N < 1 || N >= ((int64_t)1 << 31) - 65536 || E < 1 || E > BO_MAX_EXPERTS) return 0;
  return bo::dispatch_workspace(N, E);
}

bo_status bo_dispatch(const int32_t* ids, int64_t N, int32_t E, int64_t capacity, int32_t* load,
                      int32_t* offsets, int32_t* order, int32_t* position, void* workspace,
                      int64_t workspace_bytes, void* stream) {
  return guarded([&]() -> bo_status {
    const char* W = "bo_dispatch";
    if (N < 0 || E < 1 || capacity < 0)
      return fail(BO_ERR_INVALID_ARGUMENT, "bo_dispatch: N < 0, E < 1 or capacity < 0");
    if (N >= ((int64_t)1 << 31) - 65536) return fail(BO_ERR_CAPACITY, "bo_dispatch: N beyond limit");
    if (E > BO_MAX_EXPERTS) return fail(BO_ERR_CAPACITY, "bo_dispatch: E beyond BO_MAX_EXPERTS");
    bo_status s;
    const size_t n = static_cast<size_t>(N);
    if ((s = check_dev(load, 4 * static_cast<size_t>(E), "load")) != BO_OK) return s;
    if ((s = check_dev(offsets, 4 * (static_cast<size_t>(E) + 1), "offsets")) != BO_OK) return s;
    if (N > 0) {
      if ((s = check_dev(ids, 4 * n, "ids")) != BO_OK) return s;
      if ((s = check_dev(order, 4 * n, "order")) != BO_OK) return s;
      if ((s = check_dev(position, 4 * n, "position")) != BO_OK) return s;
      if ((s = check_workspace(workspace, workspace_bytes, bo::dispatch_workspace(N, E), W)) != BO_OK)
        return s;
    }
    hipStream_t st = static_cast<hipStream_t>(stream);
    return bo::after_launch(bo::launch_dispatch(ids, N, E, capacity, load, offsets, order, position,
                                                workspace, st),
                            st, W);
  });
}

}  // extern "C"
