// What the calls without a context share: element types, host checks, small device helpers.
#pragma once

#include "lopt_device.h"

namespace lopt {

typedef __bf16 bf16_t;
typedef _Float16 f16_t;

template <typename T>
__device__ __forceinline__ float to_f32(T v) { return (float)v; }
template <typename T>
__device__ __forceinline__ T from_f32(float v) { return (T)v; }   // round to nearest even

// 16 bytes of consecutive elements, which may start at any element: the access needs no more than an element's alignment.
template <typename T> struct Pack;
template <> struct Pack<float> { static constexpr int n = 4; typedef float type __attribute__((ext_vector_type(4), aligned(4))); };
template <> struct Pack<bf16_t> { static constexpr int n = 8; typedef bf16_t type __attribute__((ext_vector_type(8), aligned(2))); };
template <> struct Pack<f16_t> { static constexpr int n = 8; typedef f16_t type __attribute__((ext_vector_type(8), aligned(2))); };

inline size_t type_bytes(uint32_t type) { return type == LOPT_F32 ? 4 : 2; }

// Calls `f` with a value of the element type.
template <typename F>
inline void with_type(uint32_t type, F&& f) {
  if (type == LOPT_F32) f(0.f);
  else if (type == LOPT_BF16) f(bf16_t{});
  else f(f16_t{});
}

// ---- host checks; each returns LOPT_OK or has recorded the message
inline lopt_status check_type(const char* what, uint32_t type) {
  return type <= LOPT_F16 ? LOPT_OK : fail_call(LOPT_EINVAL, "%s %u is not a lopt_type", what, type);
}
inline lopt_status check_array(const char* what, const void* p, size_t align, bool needed) {
  if (!p) return needed ? fail_call(LOPT_EINVAL, "%s is null", what) : LOPT_OK;
  return (uintptr_t)p % align ? fail_call(LOPT_EINVAL, "%s is not aligned to %zu bytes", what, align) : LOPT_OK;
}
// A matrix of rows x cols with `ld` elements from row to row; the last element's byte offset has to fit 62 bits.
inline lopt_status check_ld(const char* what, int64_t rows, int64_t cols, int64_t ld, bool written) {
  if (rows <= 1) return LOPT_OK;
  if (ld < (written ? cols : 0)) return fail_call(LOPT_ESHAPE, "%s=%lld is below %lld", what, (long long)ld, (long long)(written ? cols : 0));
  if (ld > ((int64_t)1 << 59) / rows) return fail_call(LOPT_ESHAPE, "%s=%lld: the matrix is larger than the address space", what, (long long)ld);
  return LOPT_OK;
}
inline lopt_status check_matrix(int64_t rows, int64_t cols, const char* cols_name) {
  if (rows < 0 || rows > 0x7fffffffLL) return fail_call(LOPT_ESHAPE, "rows=%lld outside [0, 2^31-1]", (long long)rows);
  if (cols < 1 || cols > 0x7fffffffLL) return fail_call(LOPT_ESHAPE, "%s=%lld outside [1, 2^31-1]", cols_name, (long long)cols);
  return LOPT_OK;
}
inline lopt_status check_workspace(const void* ws, size_t have, size_t need) {
  if (need == 0) return LOPT_OK;
  if (!ws) return fail_call(LOPT_EINVAL, "workspace is null");
  if ((uintptr_t)ws & 15) return fail_call(LOPT_EINVAL, "workspace is not 16-byte aligned");
  return have < need ? fail_call(LOPT_EINVAL, "workspace of %zu bytes, %zu are needed", have, need) : LOPT_OK;
}
inline lopt_status launch_status(const char* what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? LOPT_OK : fail_call(e == hipErrorOutOfMemory ? LOPT_ENOMEM : LOPT_EHIP, "%s: %s", what, hipGetErrorString(e));
}
#define LOPT_CHECK(call)                        \
  do {                                          \
    const lopt_status st_ = (call);             \
    if (st_ != LOPT_OK) return st_;             \
  } while (0)

// Largest value over the 64 lanes of a wavefront; every lane gets it. NaN is passed over.
__device__ __forceinline__ float wave_max(float v) {
  v = fmaxf(v, dpp_f<0xB1>(v));
  v = fmaxf(v, dpp_f<0x4E>(v));
  v = fmaxf(v, dpp_f<0x141>(v));
  v = fmaxf(v, dpp_f<0x140>(v));
  const float a = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 0));
  const float b = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 16));
  const float c = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 32));
  const float d = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 48));
  return fmaxf(fmaxf(a, b), fmaxf(c, d));
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, true));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, true));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xF, 0xF, true));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xF, 0xF, true));
  const uint32_t a = __builtin_amdgcn_readlane((int)v, 0), b = __builtin_amdgcn_readlane((int)v, 16);
  const uint32_t c = __builtin_amdgcn_readlane((int)v, 32), d = __builtin_amdgcn_readlane((int)v, 48);
  return max(max(a, b), max(c, d));
}
__device__ __forceinline__ uint64_t wave_max(uint64_t v) {
  const uint32_t hi = wave_max((uint32_t)(v >> 32));
  return (uint64_t)hi << 32 | wave_max((uint32_t)(v >> 32) == hi ? (uint32_t)v : 0u);
}
__device__ __forceinline__ uint64_t readlane(uint64_t v, int lane) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane), hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), lane);
  return (uint64_t)hi << 32 | lo;
}
// What the lanes of this wavefront wrote to LDS before is there for all of them after.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Sum over a workgroup of W wavefronts; every thread gets it. `red`: W values of LDS, free to use before and after.
template <int W, typename V>
__device__ __forceinline__ V block_sum(V v, V* red) {
  v = wave_sum(v);
  if (W == 1) return v;
  const int wave = threadIdx.x >> 6;
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[wave] = v;
  __syncthreads();
  V s = red[0];
#pragma unroll
  for (int i = 1; i < W; ++i) s += red[i];
  return s;
}

}  // namespace lopt
