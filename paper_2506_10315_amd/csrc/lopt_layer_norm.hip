// Layer norm and its gradient.
#include <cmath>

#include "lopt_ops.h"

namespace lopt {
namespace {

// One workgroup a row: mean, then the squares of what is left, then the row again.
template <typename T, typename W>
__global__ __launch_bounds__(kBlock) void k_norm(const T* __restrict__ x, int64_t ld_x, const W* __restrict__ w, const W* __restrict__ b, T* y,
                                                 int64_t ld_y, float* __restrict__ mean_out, float* __restrict__ rstd_out, int cols, float eps) {
  __shared__ float red[4];
  const int64_t r = blockIdx.x;
  const T* xr = x + r * ld_x;
  float s = 0.f;
  for (int64_t i = threadIdx.x; i < cols; i += kBlock) s += to_f32(xr[i]);
  const float mean = block_sum<4>(s, red) / (float)cols;
  float v = 0.f;
  for (int64_t i = threadIdx.x; i < cols; i += kBlock) {
    const float d = to_f32(xr[i]) - mean;
    v += d * d;
  }
  const float rstd = 1.f / sqrtf(block_sum<4>(v, red) / (float)cols + eps);
  for (int64_t i = threadIdx.x; i < cols; i += kBlock) {
    const float h = (to_f32(xr[i]) - mean) * rstd;
    y[r * ld_y + i] = from_f32<T>(h * (w ? to_f32(w[i]) : 1.f) + (b ? to_f32(b[i]) : 0.f));
  }
  if (threadIdx.x == 0) {
    if (mean_out) mean_out[r] = mean;
    if (rstd_out) rstd_out[r] = rstd;
  }
}

constexpr int kSlab = 128;   // rows whose column sums one wavefront adds up

// Partial sums of dy xh and dy over a slab of rows, a column a lane. Before dx, which may overwrite dy or x.
template <typename T>
__global__ __launch_bounds__(kWave) void k_norm_columns(const T* __restrict__ dy, int64_t ld_dy, const T* __restrict__ x, int64_t ld_x,
                                                        const float* __restrict__ mean, const float* __restrict__ rstd, int rows, int cols,
                                                        float* __restrict__ part) {
  const int64_t c = (int64_t)blockIdx.x * kWave + threadIdx.x;
  const int64_t r0 = (int64_t)blockIdx.y * kSlab, r1 = min(r0 + kSlab, (int64_t)rows);
  if (c >= cols) return;
  float sw = 0.f, sb = 0.f;
  for (int64_t r = r0; r < r1; ++r) {
    const float g = to_f32(dy[r * ld_dy + c]);
    sw += g * ((to_f32(x[r * ld_x + c]) - mean[r]) * rstd[r]);
    sb += g;
  }
  part[(int64_t)blockIdx.y * 2 * cols + c] = sw;
  part[((int64_t)blockIdx.y * 2 + 1) * cols + c] = sb;
}

template <typename W>
__global__ __launch_bounds__(kWave) void k_norm_columns_sum(const float* __restrict__ part, int slabs, int cols, W* __restrict__ dw, W* __restrict__ db) {
  const int64_t c = (int64_t)blockIdx.x * kWave + threadIdx.x;
  if (c >= cols) return;
  double sw = 0.0, sb = 0.0;
  for (int64_t k = 0; k < slabs; ++k) {
    sw += part[k * 2 * cols + c];
    sb += part[(k * 2 + 1) * cols + c];
  }
  if (dw) dw[c] = from_f32<W>((float)sw);
  if (db) db[c] = from_f32<W>((float)sb);
}

template <typename T, typename W>
__global__ __launch_bounds__(kBlock) void k_norm_rows(const T* dy, int64_t ld_dy, const T* x, int64_t ld_x, const W* __restrict__ w,
                                                      const float* __restrict__ mean, const float* __restrict__ rstd, T* dx, int64_t ld_dx, int cols) {
  __shared__ float red[4];
  const int64_t r = blockIdx.x;
  const float mu = mean[r], rs = rstd[r];
  float s1 = 0.f, s2 = 0.f;
  for (int64_t i = threadIdx.x; i < cols; i += kBlock) {
    const float a = to_f32(dy[r * ld_dy + i]) * (w ? to_f32(w[i]) : 1.f);
    s1 += a;
    s2 += a * ((to_f32(x[r * ld_x + i]) - mu) * rs);
  }
  const float m1 = block_sum<4>(s1, red) / (float)cols;
  const float m2 = block_sum<4>(s2, red) / (float)cols;
  for (int64_t i = threadIdx.x; i < cols; i += kBlock) {
    const float a = to_f32(dy[r * ld_dy + i]) * (w ? to_f32(w[i]) : 1.f);
    const float h = (to_f32(x[r * ld_x + i]) - mu) * rs;
    dx[r * ld_dx + i] = from_f32<T>(rs * (a - m1 - h * m2));
  }
}

unsigned slabs_of(int64_t rows) { return (unsigned)((rows + kSlab - 1) / kSlab); }

}  // namespace
}  // namespace lopt

using namespace lopt;

extern "C" {

lopt_status lopt_layer_norm(const void* x, int64_t ld_x, const void* weight, const void* bias, void* y, int64_t ld_y, float* mean, float* rstd,
                            int64_t rows, int64_t cols, float eps, uint32_t type, uint32_t weight_type, void* hip_stream) {
  LOPT_CHECK(check_type("type", type));
  LOPT_CHECK(check_type("weight_type", weight_type));
  LOPT_CHECK(check_matrix(rows, cols, "cols"));
  if (!(eps >= 0.f) || std::isinf(eps)) return fail_call(LOPT_EINVAL, "eps must be finite and >= 0");
  LOPT_CHECK(check_ld("ld_x", rows, cols, ld_x, y == x));
  LOPT_CHECK(check_ld("ld_y", rows, cols, ld_y, true));
  LOPT_CHECK(check_array("x", x, type_bytes(type), rows > 0));
  LOPT_CHECK(check_array("y", y, type_bytes(type), rows > 0));
  LOPT_CHECK(check_array("weight", weight, type_bytes(weight_type), false));
  LOPT_CHECK(check_array("bias", bias, type_bytes(weight_type), false));
  LOPT_CHECK(check_array("mean", mean, 4, false));
  LOPT_CHECK(check_array("rstd", rstd, 4, false));
  if (rows == 0) return LOPT_OK;
  if (y == x && ld_y != ld_x && rows > 1) return fail_call(LOPT_EINVAL, "y is x, but ld_y is not ld_x");
  with_type(type, [&](auto t) {
    with_type(weight_type, [&](auto u) {
      using T = decltype(t);
      using W = decltype(u);
      hipLaunchKernelGGL((k_norm<T, W>), dim3((unsigned)rows), dim3(kBlock), 0, (hipStream_t)hip_stream, (const T*)x, ld_x, (const W*)weight,
                         (const W*)bias, (T*)y, ld_y, mean, rstd, (int)cols, eps);
    });
  });
  return launch_status("lopt_layer_norm");
}

size_t lopt_layer_norm_workspace(int64_t rows, int64_t cols) {
  if (rows <= 0 || cols <= 0) return 0;
  return (size_t)slabs_of(rows) * 2 * (size_t)cols * sizeof(float);
}

lopt_status lopt_layer_norm_backward(const void* dy, int64_t ld_dy, const void* x, int64_t ld_x, const void* weight, const float* mean,
                                     const float* rstd, void* dx, int64_t ld_dx, void* dweight, void* dbias, int64_t rows, int64_t cols,
                                     uint32_t type, uint32_t weight_type, void* workspace, size_t workspace_bytes, void* hip_stream) {
  LOPT_CHECK(check_type("type", type));
  LOPT_CHECK(check_type("weight_type", weight_type));
  LOPT_CHECK(check_matrix(rows, cols, "cols"));
  LOPT_CHECK(check_ld("ld_dy", rows, cols, ld_dy, false));
  LOPT_CHECK(check_ld("ld_x", rows, cols, ld_x, false));
  if (dx) LOPT_CHECK(check_ld("ld_dx", rows, cols, ld_dx, true));
  LOPT_CHECK(check_array("dy", dy, type_bytes(type), rows > 0));
  LOPT_CHECK(check_array("x", x, type_bytes(type), rows > 0));
  LOPT_CHECK(check_array("mean", mean, 4, rows > 0));
  LOPT_CHECK(check_array("rstd", rstd, 4, rows > 0));
  LOPT_CHECK(check_array("weight", weight, type_bytes(weight_type), false));
  LOPT_CHECK(check_array("dx", dx, type_bytes(type), false));
  LOPT_CHECK(check_array("dweight", dweight, type_bytes(weight_type), false));
  LOPT_CHECK(check_array("dbias", dbias, type_bytes(weight_type), false));
  if (rows > 1 && dx && ((dx == dy && ld_dx != ld_dy) || (dx == x && ld_dx != ld_x)))
    return fail_call(LOPT_EINVAL, "dx is an input, but ld_dx is not that input's");
  const bool columns = dweight || dbias;
  if (columns) LOPT_CHECK(check_workspace(workspace, workspace_bytes, lopt_layer_norm_workspace(rows, cols)));
  if (rows == 0 && !columns) return LOPT_OK;
  hipStream_t stream = (hipStream_t)hip_stream;
  float* part = (float*)workspace;
  with_type(type, [&](auto t) {
    with_type(weight_type, [&](auto u) {
      using T = decltype(t);
      using W = decltype(u);
      const unsigned strips = (unsigned)((cols + kWave - 1) / kWave);
      if (columns) {
        if (rows > 0)
          hipLaunchKernelGGL(k_norm_columns<T>, dim3(strips, slabs_of(rows)), dim3(kWave), 0, stream, (const T*)dy, ld_dy, (const T*)x, ld_x, mean, rstd,
                             (int)rows, (int)cols, part);
        hipLaunchKernelGGL(k_norm_columns_sum<W>, dim3(strips), dim3(kWave), 0, stream, (const float*)part, (int)slabs_of(rows), (int)cols,
                           (W*)dweight, (W*)dbias);
      }
      if (dx && rows > 0)
        hipLaunchKernelGGL((k_norm_rows<T, W>), dim3((unsigned)rows), dim3(kBlock), 0, stream, (const T*)dy, ld_dy, (const T*)x, ld_x, (const W*)weight,
                           mean, rstd, (T*)dx, ld_dx, (int)cols);
    });
  });
  return launch_status("lopt_layer_norm_backward");
}

}  // extern "C"
