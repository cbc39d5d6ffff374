// Log probabilities of given tokens with entropy and top alternatives, and their gradient.
#include <cfloat>
#include <cmath>

#include "lopt_ops.h"

namespace lopt {
namespace {

// The order of the alternatives as one number: larger logit first, NaN above all, +0 and -0 alike, lower index first among equals.
// No element's number is 0 or all ones.
__device__ __forceinline__ uint64_t rank_key(float x, uint32_t index) {
  uint32_t u = __builtin_bit_cast(uint32_t, x + 0.f);
  u = x != x ? 0xfffffffeu : u & 0x80000000u ? ~u : u | 0x80000000u;
  return (uint64_t)u << 32 | (0xffffffffu - index);
}

__device__ __forceinline__ uint64_t block_max(uint64_t v, uint64_t* red) {
  for (int d = 32; d > 0; d >>= 1) {
    const uint64_t o = __shfl_xor((unsigned long long)v, d);
    v = o > v ? o : v;
  }
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  for (int i = 0; i < kBlock / kWave; ++i) v = red[i] > v ? red[i] : v;
  return v;
}

// One workgroup a row; an alternative is the largest key below the one before it.
template <typename T>
__global__ __launch_bounds__(kBlock) void k_logprobs(const T* __restrict__ x, int64_t ld, const int64_t* __restrict__ targets, int vocab, float scale,
                                                     int64_t ignore, int top, float* __restrict__ logp, float* __restrict__ entropy,
                                                     float* __restrict__ stats, float* __restrict__ top_logp, int64_t* __restrict__ top_index) {
  __shared__ float red[4];
  __shared__ uint64_t redk[4];
  const int64_t r = blockIdx.x;
  const T* xr = x + r * ld;
  float m = -INFINITY;
  for (int64_t i = threadIdx.x; i < vocab; i += kBlock) m = fmaxf(m, to_f32(xr[i]));
  for (int d = 32; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = m;
  __syncthreads();
  m = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  const float base = m == -INFINITY ? 0.f : m;
  float s = 0.f, h = 0.f;
  for (int64_t i = threadIdx.x; i < vocab; i += kBlock) {
    const float z = scale * (to_f32(xr[i]) - base), e = expf(z);
    s += e;
    h += e * fmaxf(z, -FLT_MAX);
  }
  s = block_sum<4>(s, red);
  h = block_sum<4>(h, red);
  const bool empty = s == 0.f;
  const float log_s = logf(s);
  if (threadIdx.x == 0) {
    if (logp) {
      const int64_t t = targets[r];
      float v = NAN;
      if (t == ignore) v = 0.f;
      else if (t >= 0 && t < vocab) v = empty ? -INFINITY : scale * (to_f32(xr[t]) - base) - log_s;
      logp[r] = v;
    }
    if (entropy) entropy[r] = empty ? 0.f : log_s - h / s;
    stats[2 * r] = m;
    stats[2 * r + 1] = log_s;
  }
  uint64_t before = ~(uint64_t)0;
  for (int k = 0; k < top; ++k) {
    uint64_t best = 0;
    for (int64_t i = threadIdx.x; i < vocab; i += kBlock) {
      const uint64_t key = rank_key(to_f32(xr[i]), (uint32_t)i);
      if (key < before && key > best) best = key;
    }
    before = best = block_max(best, redk);
    const uint32_t at = 0xffffffffu - (uint32_t)best;
    if (threadIdx.x == 0) {
      top_index[r * top + k] = at;
      top_logp[r * top + k] = empty ? -INFINITY : scale * (to_f32(xr[at]) - base) - log_s;
    }
  }
}

template <typename T>
__global__ __launch_bounds__(kBlock) void k_logprobs_back(const T* x, int64_t ld, const int64_t* __restrict__ targets, const float* __restrict__ stats,
                                                          const float* __restrict__ entropy, const float* __restrict__ dlogp,
                                                          const float* __restrict__ dentropy, T* dx, int64_t ld_d, int vocab, float scale, int64_t ignore) {
  const int64_t r = blockIdx.x;
  const float m = stats[2 * r], log_s = stats[2 * r + 1];
  const bool empty = log_s == -INFINITY;
  const int64_t t = dlogp ? targets[r] : ignore;
  float g = t == ignore ? 0.f : dlogp[r];
  if (t != ignore && (t < 0 || t >= vocab)) g = NAN;
  const float h = dentropy ? dentropy[r] : 0.f, ent = dentropy ? entropy[r] : 0.f;
  for (int64_t i = threadIdx.x; i < vocab; i += kBlock) {
    const float lp = fmaxf(scale * (to_f32(x[r * ld + i]) - m) - log_s, -FLT_MAX);
    const float p = expf(lp);
    float d = (i == t ? g : 0.f) - g * p - h * (p * (lp + ent));
    d = empty ? g * 0.f : scale * d;
    dx[r * ld_d + i] = from_f32<T>(d);
  }
}

}  // namespace
}  // namespace lopt

using namespace lopt;

extern "C" {

size_t lopt_token_logprobs_workspace(int64_t rows, int64_t vocab, uint32_t top) {
  (void)rows, (void)vocab, (void)top;
  return 0;
}

static lopt_status check_logits(const void* logits, int64_t ld, int64_t rows, int64_t vocab, uint32_t type, float scale) {
  LOPT_CHECK(check_type("type", type));
  LOPT_CHECK(check_matrix(rows, vocab, "vocab"));
  LOPT_CHECK(check_ld("ld", rows, vocab, ld, false));
  if (!(scale > 0.f) || std::isinf(scale)) return fail_call(LOPT_EINVAL, "scale must be finite and > 0");
  return check_array("logits", logits, type_bytes(type), rows > 0);
}

lopt_status lopt_token_logprobs(const void* logits, int64_t ld, const int64_t* targets, int64_t rows, int64_t vocab, uint32_t type, float scale,
                                int64_t ignore_index, uint32_t top, float* logp, float* entropy, float* stats, float* top_logp, int64_t* top_index,
                                void* workspace, size_t workspace_bytes, void* hip_stream) {
  LOPT_CHECK(check_logits(logits, ld, rows, vocab, type, scale));
  if (top > LOPT_TOP_MAX || (int64_t)top > vocab) return fail_call(LOPT_EINVAL, "top=%u is above %d or above vocab", top, LOPT_TOP_MAX);
  LOPT_CHECK(check_array("targets", targets, 8, rows > 0 && logp));
  LOPT_CHECK(check_array("logp", logp, 4, false));
  LOPT_CHECK(check_array("entropy", entropy, 4, false));
  LOPT_CHECK(check_array("stats", stats, 4, rows > 0));
  LOPT_CHECK(check_array("top_logp", top_logp, 4, rows > 0 && top > 0));
  LOPT_CHECK(check_array("top_index", top_index, 8, rows > 0 && top > 0));
  LOPT_CHECK(check_workspace(workspace, workspace_bytes, lopt_token_logprobs_workspace(rows, vocab, top)));
  if (rows == 0) return LOPT_OK;
  with_type(type, [&](auto t) {
    using T = decltype(t);
    hipLaunchKernelGGL(k_logprobs<T>, dim3((unsigned)rows), dim3(kBlock), 0, (hipStream_t)hip_stream, (const T*)logits, ld, targets, (int)vocab, scale,
                       ignore_index, (int)top, logp, entropy, stats, top_logp, top_index);
  });
  return launch_status("lopt_token_logprobs");
}

lopt_status lopt_token_logprobs_backward(const void* logits, int64_t ld, const int64_t* targets, const float* stats, const float* entropy,
                                         const float* dlogp, const float* dentropy, void* dlogits, int64_t ld_d, int64_t rows, int64_t vocab,
                                         uint32_t type, float scale, int64_t ignore_index, void* hip_stream) {
  LOPT_CHECK(check_logits(logits, ld, rows, vocab, type, scale));
  LOPT_CHECK(check_ld("ld_d", rows, vocab, ld_d, true));
  LOPT_CHECK(check_array("dlogits", dlogits, type_bytes(type), rows > 0));
  LOPT_CHECK(check_array("stats", stats, 4, rows > 0));
  LOPT_CHECK(check_array("dlogp", dlogp, 4, false));
  LOPT_CHECK(check_array("dentropy", dentropy, 4, false));
  LOPT_CHECK(check_array("targets", targets, 8, rows > 0 && dlogp));
  LOPT_CHECK(check_array("entropy", entropy, 4, rows > 0 && dentropy));
  if (dlogits == logits && ld_d != ld && rows > 1) return fail_call(LOPT_EINVAL, "dlogits is logits, but ld_d is not ld");
  if (rows == 0) return LOPT_OK;
  with_type(type, [&](auto t) {
    using T = decltype(t);
    hipLaunchKernelGGL(k_logprobs_back<T>, dim3((unsigned)rows), dim3(kBlock), 0, (hipStream_t)hip_stream, (const T*)logits, ld, targets, stats, entropy,
                       dlogp, dentropy, (T*)dlogits, ld_d, (int)vocab, scale, ignore_index);
  });
  return launch_status("lopt_token_logprobs_backward");
}

}  // extern "C"
