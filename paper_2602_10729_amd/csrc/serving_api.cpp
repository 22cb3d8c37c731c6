// C ABI entry points of the served-output operators: validation and launch.
// They keep no state and allocate nothing on the device.
#include <hip/hip_runtime.h>

#include <cmath>
#include <initializer_list>
#include <string>

#include "serving.h"
#include "spans.h"

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

// A matrix of `type`, for what may not share memory.
bo::Span matrix(const void* p, int32_t type, int64_t rows, int64_t cols, int64_t stride) {
  const int64_t es = static_cast<int64_t>(bo::type_bytes(type));
  return {p, rows, cols * es, rows > 1 ? stride * es : 0};
}
// `n` elements of `es` bytes beside each other.
bo::Span vec(const void* p, size_t n, size_t es = 4) { return {p, 1, static_cast<int64_t>(n * es), 0}; }
// An output lies apart from what the call reads and from its other outputs.
bo_status check_apart(const bo::Span& out, std::initializer_list<bo::Span> others, const char* where,
                      const char* name) {
  for (const bo::Span& o : others)
    if (bo::share(out, o))
      return fail(BO_ERR_INVALID_ARGUMENT, std::string(where) + ": " + name + " overlaps an input or another output");
  return BO_OK;
}

constexpr int64_t kMaxPairs = ((int64_t)1 << 31) - 65536;
constexpr int64_t kMaxElems = (int64_t)1 << 31;
constexpr int64_t kMaxScores = (int64_t)1 << 38;      // (a launch's blocks and threads)

bo_status check_expert_sizes(int32_t type, int64_t T, int64_t H, int32_t top, int64_t R,
                             const char* where) {
  const std::string W(where);
  if (bad_type(type)) return fail(BO_ERR_INVALID_ARGUMENT, W + ": unknown type");
  if (T < 0 || H < 1 || top < 1) return fail(BO_ERR_INVALID_ARGUMENT, W + ": T < 0, H < 1 or top < 1");
  if (top > BO_MAX_CHOICES) return fail(BO_ERR_CAPACITY, W + ": top beyond BO_MAX_CHOICES");
  if (T >= kMaxPairs / top || H >= kMaxElems) return fail(BO_ERR_CAPACITY, W + ": T or H beyond limit");
  if (R < 0 || R > T * top) return fail(BO_ERR_INVALID_ARGUMENT, W + ": R must be in [0, T top]");
  return BO_OK;
}

bo_status check_linear_sizes(int32_t type, int64_t T, int64_t V, int64_t H, float it, const char* where) {
  const std::string W(where);
  if (bad_type(type)) return fail(BO_ERR_INVALID_ARGUMENT, W + ": unknown type");
  if (T < 0 || V < 1 || H < 1) return fail(BO_ERR_INVALID_ARGUMENT, W + ": T < 0, V < 1 or H < 1");
  if (!(it > 0.0f) || !(it <= 1e30f))
    return fail(BO_ERR_INVALID_ARGUMENT, W + ": inv_temperature must be in (0, 1e30]");
  if (T > kMaxElems / 8 || V > kMaxElems / 4 || T > kMaxScores / V)
    return fail(BO_ERR_CAPACITY, W + ": T, V or T times V beyond limit");
  if (H > BO_MAX_WIDTH) return fail(BO_ERR_CAPACITY, W + ": H beyond BO_MAX_WIDTH");
  return BO_OK;
}

bo::LinearArgs linear_args(const void* hidden, int64_t hidden_stride, const void* weight,
                           int64_t weight_stride, int32_t type, int64_t T, int64_t V, int64_t H) {
  bo::LinearArgs a{};
  a.hidden = hidden; a.hidden_stride = hidden_stride;
  a.weight = weight; a.weight_stride = weight_stride;
  a.type = type;
  a.T = T; a.V = V; a.H = H;
  return a;
}

bo_status check_embed_sizes(int32_t type, int64_t T, int64_t V, int64_t H, float scale,
                            const char* where) {
  const std::string W(where);
  if (bad_type(type)) return fail(BO_ERR_INVALID_ARGUMENT, W + ": unknown type");
  if (T < 0 || V < 1 || H < 1) return fail(BO_ERR_INVALID_ARGUMENT, W + ": T < 0, V < 1 or H < 1");
  if (!std::isfinite(scale)) return fail(BO_ERR_INVALID_ARGUMENT, W + ": scale is not finite");
  if (T >= kMaxPairs || V >= kMaxElems || H >= kMaxElems)
    return fail(BO_ERR_CAPACITY, W + ": T, V or H beyond limit");
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

bo_status bo_expert_gather(const void* x, int32_t type, int64_t T, int64_t H, int64_t stride,
                           int32_t top, const int32_t* order, int64_t R, const int32_t* position,
                           void* out, int64_t out_stride, void* stream) {
  return guarded([&]() -> bo_status {
    const char* W = "bo_expert_gather";
    bo_status s = check_expert_sizes(type, T, H, top, R, W);
    if (s != BO_OK) return s;
    if (T == 0 || R == 0) return BO_OK;
    if ((s = check_rows(x, type, T, H, stride, W, "x")) != BO_OK) return s;
    if ((s = check_rows(out, type, R, H, out_stride, W, "out")) != BO_OK) return s;
    const size_t n = static_cast<size_t>(T) * top, r = static_cast<size_t>(R);
    if ((s = check_dev(order, 4 * r, "order")) != BO_OK) return s;
    if ((s = check_dev(position, 4 * n, "position")) != BO_OK) return s;
    if ((s = check_apart(matrix(out, type, R, H, out_stride),
                         {matrix(x, type, T, H, stride), vec(order, r), vec(position, n)}, W, "out")) != BO_OK)
      return s;
    bo::ExpertArgs a{x, nullptr, type, T, H, R, stride, 0, top, order, position, nullptr, out,
                     out_stride, nullptr};
    hipStream_t st = static_cast<hipStream_t>(stream);
    return bo::after_launch(bo::launch_expert_gather(a, st), st, W);
  });
}

bo_status bo_expert_combine(const void* rows, int32_t type, int64_t R, int64_t H, int64_t stride,
                            const int32_t* position, int64_t T, int32_t top, const float* weights,
                            void* out, int64_t out_stride, void* stream) {
  return guarded([&]() -> bo_status {
    const char* W = "bo_expert_combine";
    bo_status s = check_expert_sizes(type, T, H, top, R, W);
    if (s != BO_OK) return s;
    if (T == 0) return BO_OK;
    if (R > 0 && (s = check_rows(rows, type, R, H, stride, W, "rows")) != BO_OK) return s;
    if ((s = check_rows(out, type, T, H, out_stride, W, "out")) != BO_OK) return s;
    const size_t n = static_cast<size_t>(T) * top;
    if ((s = check_dev(position, 4 * n, "position")) != BO_OK) return s;
    if (weights && (s = check_dev(weights, 4 * n, "weights")) != BO_OK) return s;
    if ((s = check_apart(matrix(out, type, T, H, out_stride),
                         {matrix(rows, type, R, H, stride), vec(position, n), vec(weights, n)}, W, "out")) != BO_OK)
      return s;
    bo::ExpertArgs a{nullptr, rows, type, T, H, R, 0, stride, top, nullptr, position, weights, out,
                     out_stride, nullptr};
    hipStream_t st = static_cast<hipStream_t>(stream);
    return bo::after_launch(bo::launch_expert_combine(a, st), st, W);
  });
}

bo_status bo_expert_combine_grad(const void* grad, int32_t type, int64_t T, int64_t H,
                                 int64_t grad_stride, const void* rows, int64_t R, int64_t stride,
                                 int32_t top, const int32_t* order, const int32_t* position,
                                 const float* weights, void* grad_rows, int64_t grad_rows_stride,
                                 float* grad_weights, void* stream) {
  return guarded([&]() -> bo_status {
    const char* W = "bo_expert_combine_grad";
    bo_status s = check_expert_sizes(type, T, H, top, R, W);
    if (s != BO_OK) return s;
    if (T == 0) return BO_OK;
    if ((s = check_rows(grad, type, T, H, grad_stride, W, "grad")) != BO_OK) return s;
    if (grad_weights && R > 0 && (s = check_rows(rows, type, R, H, stride, W, "rows")) != BO_OK) return s;
    const size_t n = static_cast<size_t>(T) * top, r = static_cast<size_t>(R);
    if (grad_rows && R > 0) {
      if ((s = check_rows(grad_rows, type, R, H, grad_rows_stride, W, "grad_rows")) != BO_OK) return s;
      if ((s = check_dev(order, 4 * r, "order")) != BO_OK) return s;
    }
    if ((s = check_dev(position, 4 * n, "position")) != BO_OK) return s;
    if (weights && (s = check_dev(weights, 4 * n, "weights")) != BO_OK) return s;
    if (grad_weights && (s = check_dev(grad_weights, 4 * n, "grad_weights")) != BO_OK) return s;
    const bo::Span gr = matrix(grad_rows, type, R, H, grad_rows_stride), gw = vec(grad_weights, n);
    const bo::Span in_g = matrix(grad, type, T, H, grad_stride);
    const bo::Span in_r = matrix(grad_weights ? rows : nullptr, type, R, H, stride);      // (else not read)
    const bo::Span in_o = vec(grad_rows ? order : nullptr, r), in_p = vec(position, n), in_w = vec(weights, n);
    if ((s = check_apart(gr, {in_g, in_r, in_o, in_p, in_w, gw}, W, "grad_rows")) != BO_OK) return s;
    if ((s = check_apart(gw, {in_g, in_r, in_o, in_p, in_w}, W, "grad_weights")) != BO_OK) return s;
    bo::ExpertArgs a{grad, rows, type, T, H, R, grad_stride, stride, top, order, position, weights,
                     R > 0 ? grad_rows : nullptr, grad_rows_stride, grad_weights};
    hipStream_t st = static_cast<hipStream_t>(stream);
    return bo::after_launch(bo::launch_expert_combine_grad(a, st), st, W);
  });
}

bo_status bo_embed(const int64_t* tokens, int64_t T, const void* table, int32_t type, int64_t V,
                   int64_t H, int64_t stride, float scale, void* out, int64_t out_stride,
                   void* stream) {
  return guarded([&]() -> bo_status {
    const char* W = "bo_embed";
    bo_status s = check_embed_sizes(type, T, V, H, scale, W);
    if (s != BO_OK) return s;
    if (T == 0) return BO_OK;
    if ((s = check_dev(tokens, 8 * static_cast<size_t>(T), "tokens")) != BO_OK) return s;
    if ((s = check_rows(table, type, V, H, stride, W, "table")) != BO_OK) return s;
    if ((s = check_rows(out, type, T, H, out_stride, W, "out")) != BO_OK) return s;
    if ((s = check_apart(matrix(out, type, T, H, out_stride),
                         {matrix(table, type, V, H, stride), vec(tokens, static_cast<size_t>(T), 8)}, W, "out")) != BO_OK)
      return s;
    bo::EmbedArgs a{tokens, table, type, T, V, H, stride, scale, out, out_stride, nullptr};
    hipStream_t st = static_cast<hipStream_t>(stream);
    return bo::after_launch(bo::launch_embed(a, st), st, W);
  });
}

int64_t bo_embed_grad_workspace(int64_t T, int64_t V, int64_t H) {
  if (T < 1 || T >= kMaxPairs || V < 1 || V >= kMaxElems || H < 1 || H >= kMaxElems) return 0;
  return bo::embed_grad_workspace(T, V, H);
}

bo_status bo_embed_grad(const int64_t* tokens, int64_t T, const void* grad, int32_t type, int64_t H,
                        int64_t stride, float scale, int64_t V, void* grad_table,
                        int64_t grad_table_stride, void* workspace, int64_t workspace_bytes,
                        void* stream) {
  return guarded([&]() -> bo_status {
    const char* W = "bo_embed_grad";
    bo_status s = check_embed_sizes(type, T, V, H, scale, W);
    if (s != BO_OK) return s;
    if ((s = check_rows(grad_table, type, V, H, grad_table_stride, W, "grad_table")) != BO_OK) return s;
    if (T > 0) {
      if ((s = check_dev(tokens, 8 * static_cast<size_t>(T), "tokens")) != BO_OK) return s;
      if ((s = check_rows(grad, type, T, H, stride, W, "grad")) != BO_OK) return s;
      if ((s = check_apart(matrix(grad_table, type, V, H, grad_table_stride),
                           {matrix(grad, type, T, H, stride), vec(tokens, static_cast<size_t>(T), 8)}, W,
                           "grad_table")) != BO_OK)
        return s;
      if ((s = check_workspace(workspace, workspace_bytes, bo::embed_grad_workspace(T, V, H), W)) != BO_OK)
        return s;
    }
    bo::EmbedArgs a{tokens, grad, type, T, V, H, stride, scale, grad_table, grad_table_stride, workspace};
    hipStream_t st = static_cast<hipStream_t>(stream);
    return bo::after_launch(bo::launch_embed_grad(a, st), st, W);
  });
}

int64_t bo_linear_logprobs_workspace(const void* hidden, int64_t hidden_stride, const void* weight,
                                     int64_t weight_stride, int32_t type, int64_t T, int64_t V,
                                     int64_t H) {
  if (T == 0 || check_linear_sizes(type, T, V, H, 1.0f, "bo_linear_logprobs_workspace") != BO_OK) return 0;
  return bo::linear_workspace(linear_args(hidden, hidden_stride, weight, weight_stride, type, T, V, H));
}

bo_status bo_linear_logprobs(const void* hidden, int64_t hidden_stride, const void* weight,
                             int64_t weight_stride, int32_t type, int64_t T, int64_t V, int64_t H,
                             const int64_t* tokens, float inv_temperature, float* logprob,
                             float* entropy, float* stats, void* workspace,
                             int64_t workspace_bytes, void* stream) {
  return guarded([&]() -> bo_status {
    const char* W = "bo_linear_logprobs";
    bo_status s = check_linear_sizes(type, T, V, H, inv_temperature, W);
    if (s != BO_OK) return s;
    if (T == 0) return BO_OK;
    if ((s = check_rows(hidden, type, T, H, hidden_stride, W, "hidden")) != BO_OK) return s;
    if ((s = check_rows(weight, type, V, H, weight_stride, W, "weight")) != BO_OK) return s;
    const size_t n = static_cast<size_t>(T);
    if (tokens && (s = check_dev(tokens, 8 * n, "tokens")) != BO_OK) return s;
    if ((s = check_dev(logprob, 4 * n, "logprob")) != BO_OK) return s;
    if ((s = check_dev(entropy, 4 * n, "entropy")) != BO_OK) return s;
    if ((s = check_dev(stats, 8 * n, "stats")) != BO_OK) return s;
    const bo::Span in_h = matrix(hidden, type, T, H, hidden_stride), in_w = matrix(weight, type, V, H, weight_stride);
    const bo::Span in_t = vec(tokens, n, 8), lp = vec(logprob, n), en = vec(entropy, n), sm = vec(stats, 2 * n);
    if ((s = check_apart(lp, {in_h, in_w, in_t, en, sm}, W, "logprob")) != BO_OK) return s;
    if ((s = check_apart(en, {in_h, in_w, in_t, sm}, W, "entropy")) != BO_OK) return s;
    if ((s = check_apart(sm, {in_h, in_w, in_t}, W, "stats")) != BO_OK) return s;
    bo::LinearArgs a = linear_args(hidden, hidden_stride, weight, weight_stride, type, T, V, H);
    if ((s = check_workspace(workspace, workspace_bytes, bo::linear_workspace(a), W)) != BO_OK) return s;
    a.tokens = tokens; a.it = inv_temperature;
    a.logprob = logprob; a.entropy = entropy; a.stats = stats;
    a.ws = workspace;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return bo::after_launch(bo::launch_linear(a, st), st, W);
  });
}

int64_t bo_linear_logprobs_grad_workspace(const void* hidden, int64_t hidden_stride,
                                          const void* weight, int64_t weight_stride, int32_t type,
                                          int64_t T, int64_t V, int64_t H) {
  if (T == 0 || check_linear_sizes(type, T, V, H, 1.0f, "bo_linear_logprobs_grad_workspace") != BO_OK) return 0;
  return bo::linear_grad_workspace(linear_args(hidden, hidden_stride, weight, weight_stride, type, T, V, H));
}

bo_status bo_linear_logprobs_grad(const void* hidden, int64_t hidden_stride, const void* weight,
                                  int64_t weight_stride, int32_t type, int64_t T, int64_t V,
                                  int64_t H, const int64_t* tokens, float inv_temperature,
                                  const float* stats, const float* entropy,
                                  const float* grad_logprob, const float* grad_entropy,
                                  void* grad_hidden, int64_t grad_hidden_stride, void* grad_weight,
                                  int64_t grad_weight_stride, void* workspace,
                                  int64_t workspace_bytes, void* stream) {
  return guarded([&]() -> bo_status {
    const char* W = "bo_linear_logprobs_grad";
    bo_status s = check_linear_sizes(type, T, V, H, inv_temperature, W);
    if (s != BO_OK) return s;
    if (grad_weight) {
      if ((s = check_rows(grad_weight, type, V, H, grad_weight_stride, W, "grad_weight")) != BO_OK) return s;
    }
    bo::LinearArgs a = linear_args(hidden, hidden_stride, weight, weight_stride, type, T, V, H);
    a.tokens = tokens; a.it = inv_temperature;
    a.stats_in = stats; a.entropy_in = entropy;
    a.g_logprob = grad_logprob; a.g_entropy = grad_entropy;
    a.grad_hidden = grad_hidden; a.grad_hidden_stride = grad_hidden_stride;
    a.grad_weight = grad_weight; a.grad_weight_stride = grad_weight_stride;
    a.ws = workspace;
    if (T > 0) {
      if ((s = check_rows(hidden, type, T, H, hidden_stride, W, "hidden")) != BO_OK) return s;
      if ((s = check_rows(weight, type, V, H, weight_stride, W, "weight")) != BO_OK) return s;
      if (grad_hidden && (s = check_rows(grad_hidden, type, T, H, grad_hidden_stride, W, "grad_hidden")) != BO_OK)
        return s;
      const size_t n = static_cast<size_t>(T);
      if (tokens && (s = check_dev(tokens, 8 * n, "tokens")) != BO_OK) return s;
      if ((s = check_dev(stats, 8 * n, "stats")) != BO_OK) return s;
      if ((s = check_dev(entropy, 4 * n, "entropy")) != BO_OK) return s;
      if (grad_logprob && (s = check_dev(grad_logprob, 4 * n, "grad_logprob")) != BO_OK) return s;
      if (grad_entropy && (s = check_dev(grad_entropy, 4 * n, "grad_entropy")) != BO_OK) return s;
      const bo::Span gh = matrix(grad_hidden, type, T, H, grad_hidden_stride);
      const bo::Span gw = matrix(grad_weight, type, V, H, grad_weight_stride);
      const bo::Span in_h = matrix(hidden, type, T, H, hidden_stride), in_w = matrix(weight, type, V, H, weight_stride);
      const bo::Span in_t = vec(tokens, n, 8), in_s = vec(stats, 2 * n), in_e = vec(entropy, n);
      const bo::Span in_gl = vec(grad_logprob, n), in_ge = vec(grad_entropy, n);
      if ((s = check_apart(gh, {in_h, in_w, in_t, in_s, in_e, in_gl, in_ge, gw}, W, "grad_hidden")) != BO_OK) return s;
      if ((s = check_apart(gw, {in_h, in_w, in_t, in_s, in_e, in_gl, in_ge}, W, "grad_weight")) != BO_OK) return s;
      if ((s = check_workspace(workspace, workspace_bytes, bo::linear_grad_workspace(a), W)) != BO_OK) return s;
    }
    hipStream_t st = static_cast<hipStream_t>(stream);
    return bo::after_launch(bo::launch_linear_grad(a, st), st, W);
  });
}

}  // extern "C"
