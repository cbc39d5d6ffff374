// Layer norm and its gradient. Forward, per row: mean = sum x / n, rstd = 1 / sqrt(sum (x - mean)^2 / n + eps), y = (x - mean) rstd w + b, in two
// sums over a row that is held, never sum x^2 - mean^2. Backward, with h = (x - mean) rstd and a = dy w: dx = rstd (a - sum(a) / n - h sum(a h) / n),
// dw = sum over the rows of dy h, db of dy. Both are bound by memory where there is enough of it (two and three arrays once each), by
// the launches below some 10 MB. Times below are of calls one behind the other in a graph, on the same inputs; those of a single kernel are from a kernel trace, where
// launches do not overlap, so that two of them add up to more than the call.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "lopt_rows.h"

namespace lopt {
namespace {

// Every group takes rows a grid apart and asks for the next before it works on the one it has. us (TB/s of one read and one write): 12608x768 bf16 9.5
// (4.1), 16384x2048 bf16 22.4 (6.0), 8192x4096 bf16 22.5 (6.0), 1024x16384 fp32 28 (4.8), 1x1024 2.8.
template <typename T, int G, int N>
__global__ __launch_bounds__(Group<G>::kThreads) void k_norm(const T* x, int64_t ld_x, Vectors wb, T* y, int64_t ld_y, float* __restrict__ mean_out,
                                                             float* __restrict__ rstd_out, int64_t rows, uint32_t cols, float eps) {
  typedef Share<T, G, N> S;
  constexpr int E = S::E, V = S::V, kRows = Group<G>::kRows;
  __shared__ float red[2][2][Group<G>::kWaves];
  const S s(cols);
  const int64_t step = (int64_t)gridDim.x * kRows;
  int64_t r = (int64_t)blockIdx.x * kRows + threadIdx.x / G;
  Row<T, G, N> next;
  if (kAhead<G> && r < rows) next.load(x + r * ld_x, s);
  float w[E], b[E];
  auto vectors = [&](int j) {
    load_vector(wb.w, wb.type, s, j, 1.f, w + j * V);
    load_vector(wb.b, wb.type, s, j, 0.f, b + j * V);
  };
  if (kAhead<G>) {
#pragma unroll
    for (int j = 0; j < S::P; ++j) vectors(j);
  }
  for (int odd = 0; r < rows; r += step, odd ^= 1) {
    if (!kAhead<G>) next.load(x + r * ld_x, s);
    const Row<T, G, N> row = next;
    if (kAhead<G> && r + step < rows) next.load(x + (r + step) * ld_x, s);
    float v[E], sum = 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      v[i] = row.get(i);
      if (s.mine(i)) sum += v[i];
    }
    const float mean = group_sum<G>(sum, red[odd][0]) / (float)cols;
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      v[i] -= mean;
      if (s.mine(i)) sum += v[i] * v[i];
    }
    const float rstd = 1.f / sqrtf(group_sum<G>(sum, red[odd][1]) / (float)cols + eps);
#pragma unroll
    for (int j = 0; j < S::P; ++j) {
      if (!kAhead<G>) vectors(j);
#pragma unroll
      for (int i = j * V; i < j * V + V; ++i) v[i] = v[i] * rstd * w[i] + b[i];
      Row<T, G, N>::store(y + r * ld_y, s, j, v + j * V);
    }
    if (threadIdx.x % G == 0) {
      if (mean_out) mean_out[r] = mean;
      if (rstd_out) rstd_out[r] = rstd;
    }
  }
}

// The gradient of the same rows. The columns' sums stay in each lane's registers over all of its rows; at the end the workgroup's groups add theirs
// up through LDS, half to half (one after the other: 100000x100 bf16 23 us, so 19), and the workgroup writes one row of partial sums:
// part[block][2][cols], 16 bytes a lane (single floats: 1024x16384 bf16 45 us, so 31). Both launches, us (TB/s of two reads and one write): 8192x1024 bf16
// 15.9 (3.2; the kernels 13.2 and 3.9), 16384x2048 bf16 38 (5.3), 8192x4096 bf16 38 (5.3), 5001x1531 fp16 18.3 (2.5; 15.8 and 3.9); dx alone 16384x2048 33.
template <typename T, int G, int N>
__global__ __launch_bounds__(Group<G>::kThreads) void k_norm_back(const T* dy, int64_t ld_dy, const T* x, int64_t ld_x, const void* __restrict__ weight,
                                                                  uint32_t weight_type, const float* __restrict__ mean, const float* __restrict__ rstd, T* dx,
                                                                  int64_t ld_dx, int64_t rows, uint32_t cols, float* __restrict__ part) {
  typedef Share<T, G, N> S;
  constexpr int E = S::E, kRows = Group<G>::kRows;
  __shared__ float red[2][2 * Group<G>::kWaves];
  const S s(cols);
  const int64_t step = (int64_t)gridDim.x * kRows;
  int64_t r = (int64_t)blockIdx.x * kRows + threadIdx.x / G;
  Row<T, G, N> next_x, next_dy;
  float next_mean = 0.f, next_rstd = 0.f;
  auto ask = [&](int64_t q) {
    next_x.load(x + q * ld_x, s);
    next_dy.load(dy + q * ld_dy, s);
    next_mean = mean[q];
    next_rstd = rstd[q];
  };
  if (kAhead<G> && r < rows) ask(r);
  float w[E], sw[E] = {}, sb[E] = {};
#pragma unroll
  for (int j = 0; j < S::P; ++j) load_vector(weight, weight_type, s, j, 1.f, w + j * S::V);
  for (int odd = 0; r < rows; r += step, odd ^= 1) {
    if (!kAhead<G>) ask(r);
    const Row<T, G, N> rx = next_x, rdy = next_dy;
    const float mu = next_mean, rs = next_rstd;
    if (kAhead<G> && r + step < rows) ask(r + step);
    float h[E], a[E], s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const float g = rdy.get(i);
      h[i] = (rx.get(i) - mu) * rs;
      a[i] = g * w[i];
      sw[i] += g * h[i];
      sb[i] += g;
      const float am = s.mine(i) ? a[i] : 0.f;
      s1 += am;
      s2 += am * h[i];
    }
    if (dx) {
      group_sums<G>(s1, s2, red[odd]);
      const float m1 = s1 / (float)cols, m2 = s2 / (float)cols;
#pragma unroll
      for (int i = 0; i < E; ++i) a[i] = rs * (a[i] - m1 - h[i] * m2);
#pragma unroll
      for (int j = 0; j < S::P; ++j) Row<T, G, N>::store(dx + r * ld_dx, s, j, a + j * S::V);
    }
  }
  if (part) columns_of_block<S, G, kRows>(s, sw, sb, part, cols);
}

// ---- rows too long for registers (above 32768 columns, backward 16384; fp32 the same): one workgroup a row, which reads it again (from L2) for every
// use. us: 200x65536 bf16 16, backward 53 (dx alone 22); 2000x20000 bf16 40, backward 87 (dx alone 52).
template <typename T>
__global__ __launch_bounds__(1024) void k_norm_long(const T* x, int64_t ld_x, Vectors wb, T* y, int64_t ld_y, float* __restrict__ mean_out,
                                                    float* __restrict__ rstd_out, int64_t rows, uint32_t cols, float eps) {
  constexpr int V = Pack<T>::n;
  __shared__ float red[16];
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
    const T* xr = x + r * ld_x;
    float s = 0.f;
    along_row<V>(cols, [&](uint32_t i, auto n) {
      float v[decltype(n)::value];
      load_run(xr + i, v);
#pragma unroll
      for (float a : v) s += a;
    });
    const float mean = block_sum<16>(s, red) / (float)cols;
    s = 0.f;
    along_row<V>(cols, [&](uint32_t i, auto n) {
      float v[decltype(n)::value];
      load_run(xr + i, v);
#pragma unroll
      for (float a : v) s += (a - mean) * (a - mean);
    });
    const float rstd = 1.f / sqrtf(block_sum<16>(s, red) / (float)cols + eps);
    along_row<V>(cols, [&](uint32_t i, auto n) {
      constexpr int N = decltype(n)::value;
      float v[N], w[N], b[N];
      load_run(xr + i, v);
      load_run_as(wb.w, i, wb.type, 1.f, w);
      load_run_as(wb.b, i, wb.type, 0.f, b);
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = (v[e] - mean) * rstd * w[e] + b[e];
      store_run(y + r * ld_y + i, v);
    });
    if (threadIdx.x == 0) {
      if (mean_out) mean_out[r] = mean;
      if (rstd_out) rstd_out[r] = rstd;
    }
  }
}

template <typename T>
__global__ __launch_bounds__(1024) void k_norm_long_rows(const T* dy, int64_t ld_dy, const T* x, int64_t ld_x, const void* __restrict__ w, uint32_t weight_type,
                                                         const float* __restrict__ mean, const float* __restrict__ rstd, T* dx, int64_t ld_dx, int64_t rows,
                                                         uint32_t cols) {
  constexpr int V = Pack<T>::n;
  __shared__ float red[16];
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
    const float mu = mean[r], rs = rstd[r];
    auto load = [&](uint32_t i, auto& a, auto& h) {
      constexpr int N = sizeof(a) / sizeof(float);
      float q[N];
      load_run(dy + r * ld_dy + i, a);
      load_run(x + r * ld_x + i, h);
      load_run_as(w, i, weight_type, 1.f, q);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        a[e] *= q[e];
        h[e] = (h[e] - mu) * rs;
      }
    };
    float s1 = 0.f, s2 = 0.f;
    along_row<V>(cols, [&](uint32_t i, auto n) {
      constexpr int N = decltype(n)::value;
      float a[N], h[N];
      load(i, a, h);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        s1 += a[e];
        s2 += a[e] * h[e];
      }
    });
    const float m1 = block_sum<16>(s1, red) / (float)cols;
    const float m2 = block_sum<16>(s2, red) / (float)cols;
    along_row<V>(cols, [&](uint32_t i, auto n) {
      constexpr int N = decltype(n)::value;
      float a[N], h[N];
      load(i, a, h);
#pragma unroll
      for (int e = 0; e < N; ++e) a[e] = rs * (a[e] - m1 - h[e] * m2);
      store_run(dx + r * ld_dx + i, a);
    });
  }
}

// Elements a lane holds at most: forward the row and two vectors, backward two rows, one vector and two sums. 32 and 16 leave
// every wavefront of a workgroup of 1024 the 128 registers that it can have; smaller groups, whose wavefronts could have more, keep to the same.
constexpr int kMostForward = 32, kMostBackward = 16;

// Workgroups of the backward pass over rows in registers, at most this many: each writes one row of partial sums. us with 128 / 256 / 512, before partial sums
// left in 16-byte accesses: groups of 64 and 256 lanes 16384x2048 bf16 110 / 62 / 44, 8192x4096 bf16 70 / 44 / 45; of 1024 lanes, where a row of partial sums is
// long beside the rows summed up, 4096x8192 bf16 67 / 49 / 59, 1024x16384 bf16 43 / 45 / 70, 2048x5504 fp32 38 / 32 / 36. The kernel alone on inputs
// that change, with 512 / 768 / 1024 workgroups, and of twice the lanes with 512 / 256: 8192x768 bf16 12.3 / 11.8 / 14.1, 15.6 / 12.4; 8192x1024 14.5 / 14.6 / 16.2, 18.2 /
// 14.6; 12608x768 15.2 / 14.8 / 17.4, 18.6 / 15.7; 100000x100 18.8 / 17.6 / 18.1, 18.9 / 20.0; 16384x2048 36.2 / 36.4 / 36.5; 8192x4096 36.5 / 36.6 / 40.1. The sums of the
// partial rows take 3.9 to 4.3 with 256 to 1024 of them at up to 1024 columns.
template <int G>
int64_t back_blocks(int64_t rows) { return std::min<int64_t>((rows + Group<G>::kRows - 1) / Group<G>::kRows, G == 1024 ? 256 : 512); }
template <int V>
int64_t back_parts(int64_t rows, int64_t cols) {
  int64_t parts = slabs_of(rows);
  with_group<V, kMostBackward>(cols, [&](auto g, auto) { parts = back_blocks<decltype(g)::value>(rows); });
  return parts;
}

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
  const Vectors wb{weight, bias, weight_type};
  with_type(type, [&](auto t) {
    using T = decltype(t);
    hipStream_t stream = (hipStream_t)hip_stream;
    const bool held = with_group<Pack<T>::n, kMostForward>(cols, [&](auto g, auto n) {
      constexpr int G = decltype(g)::value, N = decltype(n)::value;
      const int64_t blocks = std::min<int64_t>((rows + Group<G>::kRows - 1) / Group<G>::kRows, G == 1024 ? 512 : 2048);
      hipLaunchKernelGGL((k_norm<T, G, N>), dim3((unsigned)blocks), dim3(Group<G>::kThreads), 0, stream, (const T*)x, ld_x, wb, (T*)y, ld_y, mean, rstd,
                         rows, (uint32_t)cols, eps);
    });
    if (!held)
      hipLaunchKernelGGL(k_norm_long<T>, dim3((unsigned)std::min<int64_t>(rows, 1 << 16)), dim3(1024), 0, stream, (const T*)x, ld_x, wb, (T*)y, ld_y, mean,
                         rstd, rows, (uint32_t)cols, eps);
  });
  return launch_status("lopt_layer_norm");
}

size_t lopt_layer_norm_workspace(int64_t rows, int64_t cols) {
  if (rows <= 0 || cols <= 0 || rows > 0x7fffffffLL || cols > 0x7fffffffLL) return 0;
  return (size_t)std::max(back_parts<4>(rows, cols), back_parts<8>(rows, cols)) * 2 * (size_t)cols * sizeof(float);
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
  const uint32_t n_cols = (uint32_t)cols;
  with_type(type, [&](auto t) {
    using T = decltype(t);
    int64_t parts = 0;
    if (rows > 0) {
      parts = back_parts<Pack<T>::n>(rows, cols);
      const bool held = with_group<Pack<T>::n, kMostBackward>(cols, [&](auto g, auto n) {
        constexpr int G = decltype(g)::value, N = decltype(n)::value;
        hipLaunchKernelGGL((k_norm_back<T, G, N>), dim3((unsigned)parts), dim3(Group<G>::kThreads), 0, stream, (const T*)dy, ld_dy, (const T*)x, ld_x, weight,
                           weight_type, mean, rstd, (T*)dx, ld_dx, rows, n_cols, columns ? part : nullptr);
      });
      if (!held) {
        if (columns)
          launch_long_columns<T, T>((const T*)dy, ld_dy, (const T*)x, ld_x, mean, rstd, rows, n_cols, parts, part, stream);
        if (dx)
          hipLaunchKernelGGL(k_norm_long_rows<T>, dim3((unsigned)std::min<int64_t>(rows, 1 << 16)), dim3(1024), 0, stream, (const T*)dy, ld_dy, (const T*)x, ld_x,
                             weight, weight_type, mean, rstd, (T*)dx, ld_dx, rows, n_cols);
      }
    }
    if (columns) launch_columns_sum(part, parts, cols, weight_type, dweight, dbias, stream);
  });
  return launch_status("lopt_layer_norm_backward");
}

}  // extern "C"
