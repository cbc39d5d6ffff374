// Dropout, residual addition and layer norm in one pass, and its gradient. Forward: h = residual + dropout(x), rounded to the residual's type as it is
// stored, y = (h - mean) rstd w + b of the stored h, so that y is what the layer norm by itself makes of h and the backward pass, which has h,
// works with the same numbers. Backward, with xh = (h - mean) rstd and a = dy w: d = dh + rstd (a - sum(a) / n - xh sum(a xh) / n) is the residual's gradient,
// dropout(d) that of x, dw = sum over the rows of dy xh, db of dy. Bound by memory: four arrays once each forward, five backward.
#include <algorithm>
#include <cmath>

#include "lopt_random.h"
#include "lopt_rows.h"

namespace lopt {
namespace {

struct AddNorm {
  const void* weight;
  const void* bias;
  uint32_t weight_type;
  float eps;
  int64_t rows;
  uint32_t cols;
};

// The stay bits of a lane's packs. A pack that was moved back to the row's end takes the words of where it would begin: its elements before
// are not the lane's.
template <typename S>
__device__ __forceinline__ void stay_bits(const Dropout& d, const Words& words, const S& s, int64_t row, uint32_t (&bits)[S::P]) {
#pragma unroll
  for (int j = 0; j < S::P; ++j) bits[j] = d.on && s.have[j] ? words.template stay<S::V>((uint32_t)row, s.at[j] + s.skip[j]) << s.skip[j] : ~0u;
}

// A group of G lanes takes a row, which stays in its registers from the loads to y; the next row is asked for before this one's sums. 8192x1024 bf16 over fp32 18.5 us, 5.4 TB/s,
// vector units busy 52 %; one row 3.1.
template <typename T, typename R, int G, int N, bool NT>
__global__ __launch_bounds__(Group<G>::kThreads) void k_add_norm(const T* x, int64_t ld_x, const R* res, int64_t ld_res, T* y, int64_t ld_y, R* h, int64_t ld_h,
                                                                 float* __restrict__ mean_out, float* __restrict__ rstd_out, AddNorm a, Dropout d) {
  typedef Share<T, G, N> S;
  constexpr int E = S::E, V = S::V, kRows = Group<G>::kRows;
  __shared__ float red[2][2][Group<G>::kWaves];
  const S s(a.cols);
  const Words words(d);
  const int64_t step = (int64_t)gridDim.x * kRows;
  int64_t r = (int64_t)blockIdx.x * kRows + threadIdx.x / G;
  RowOf<T, S> next_x;
  RowOf<R, S> next_res;
  auto ask = [&](int64_t q) {
    next_x.template load<NT>(x + q * ld_x, s);
    next_res.template load<NT>(res + q * ld_res, s);
  };
  if (kAhead<G> && r < a.rows) ask(r);
  float w[E], b[E];
  auto vectors = [&](int j) {
    load_vector(a.weight, a.weight_type, s, j, 1.f, w + j * V);
    load_vector(a.bias, a.weight_type, s, j, 0.f, b + j * V);
  };
  if (kAhead<G>) {
#pragma unroll
    for (int j = 0; j < S::P; ++j) vectors(j);
  }
  for (int odd = 0; r < a.rows; r += step, odd ^= 1) {
    if (!kAhead<G>) ask(r);
    uint32_t bits[S::P];
    stay_bits(d, words, s, r, bits);
    float v[E], sum = 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const float in = where_bit(bits[i / V], i % V, next_x.get(i) * d.scale);
      v[i] = to_f32(from_f32<R>(next_res.get(i) + in));
      if (s.mine(i)) sum += v[i];
    }
    if (kAhead<G> && r + step < a.rows) ask(r + step);
#pragma unroll
    for (int j = 0; j < S::P; ++j) RowOf<R, S>::store(h + r * ld_h, s, j, v + j * V);
    const float mean = group_sum<G>(sum, red[odd][0]) / (float)a.cols;
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      v[i] -= mean;
      if (s.mine(i)) sum += v[i] * v[i];
    }
    const float rstd = 1.f / sqrtf(group_sum<G>(sum, red[odd][1]) / (float)a.cols + a.eps);
#pragma unroll
    for (int j = 0; j < S::P; ++j) {
      if (!kAhead<G>) vectors(j);
#pragma unroll
      for (int i = j * V; i < j * V + V; ++i) v[i] = v[i] * rstd * w[i] + b[i];
      RowOf<T, S>::store(y + r * ld_y, s, j, v + j * V);
    }
    if ((G > 64 ? threadIdx.x : threadIdx.x % G) == 0) {
      if (mean_out) mean_out[r] = mean;
      if (rstd_out) rstd_out[r] = rstd;
    }
  }
}

// The gradient of the same rows; the columns' sums as in the layer norm's, in registers over a workgroup's rows and then one row of partial sums each, or not at all. 5001x1531
// fp16 22.3 us, 3.4 TB/s, vector units busy 47 %: one round of 768 workgroups, two sums over three wavefronts a row; the columns 4.3.
template <typename T, typename R, int G, int N, bool COLUMNS, bool NT>
__global__ __launch_bounds__(Group<G>::kThreads) void k_add_norm_back(const T* dy, int64_t ld_dy, const R* dh, int64_t ld_dh, const R* h, int64_t ld_h,
                                                                      const float* __restrict__ mean, const float* __restrict__ rstd, T* dx, int64_t ld_dx, R* dres,
                                                                      int64_t ld_dres, AddNorm a, Dropout d, float* __restrict__ part) {
  typedef Share<T, G, N> S;
  constexpr int E = S::E, V = S::V, kRows = Group<G>::kRows;
  __shared__ float red[2][2 * Group<G>::kWaves];
  const S s(a.cols);
  const Words words(d);
  const int64_t step = (int64_t)gridDim.x * kRows;
  int64_t r = (int64_t)blockIdx.x * kRows + threadIdx.x / G;
  RowOf<R, S> next_h, next_dh;
  RowOf<T, S> next_dy;
  float next_mean = 0.f, next_rstd = 0.f;
  const bool rows_wanted = dx || dres;
  auto ask = [&](int64_t q) {
    next_h.template load<NT>(h + q * ld_h, s);
    next_dy.template load<NT>(dy + q * ld_dy, s);
    if (dh) next_dh.template load<NT>(dh + q * ld_dh, s);
    next_mean = mean[q];
    next_rstd = rstd[q];
  };
  if (kAhead<G> && r < a.rows) ask(r);
  float w[E], sw[E] = {}, sb[E] = {};
#pragma unroll
  for (int j = 0; j < S::P; ++j) load_vector(a.weight, a.weight_type, s, j, 1.f, w + j * V);
  for (int odd = 0; r < a.rows; r += step, odd ^= 1) {
    if (!kAhead<G>) ask(r);
    uint32_t bits[S::P];
    if (dx) stay_bits(d, words, s, r, bits);
    __builtin_amdgcn_sched_barrier(0);   // formed while the loads are under way: 16384x2048 bf16 73 -> 69 us, over fp32 115 -> 108
    const RowOf<R, S> rh = next_h, rdh = next_dh;
    const RowOf<T, S> rdy = next_dy;
    const float mu = next_mean, rs = next_rstd;
    if (kAhead<G> && r + step < a.rows) ask(r + step);
    float xh[E], v[E], s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const float g = rdy.get(i);
      xh[i] = (rh.get(i) - mu) * rs;
      v[i] = g * w[i];
      if (COLUMNS) {
        sw[i] += g * xh[i];
        sb[i] += g;
      }
      const float am = s.mine(i) ? v[i] : 0.f;
      s1 += am;
      s2 += am * xh[i];
    }
    if (rows_wanted) {
      group_sums<G>(s1, s2, red[odd]);
      const float m1 = s1 / (float)a.cols, m2 = s2 / (float)a.cols;
#pragma unroll
      for (int i = 0; i < E; ++i) {
        v[i] = rs * (v[i] - m1 - xh[i] * m2);
        if (dh) v[i] += rdh.get(i);
      }
      if (dres) {
#pragma unroll
        for (int j = 0; j < S::P; ++j) RowOf<R, S>::store(dres + r * ld_dres, s, j, v + j * V);
      }
      if (dx) {
#pragma unroll
        for (int i = 0; i < E; ++i) v[i] = where_bit(bits[i / V], i % V, v[i] * d.scale);
#pragma unroll
        for (int j = 0; j < S::P; ++j) RowOf<T, S>::store(dx + r * ld_dx, s, j, v + j * V);
      }
    }
  }
  if constexpr (COLUMNS)
    if (part) columns_of_block<S, G, kRows>(s, sw, sb, part, a.cols);
}

// ---- rows too long for registers: a workgroup a row, read again for every use, from the L2 as a rule.
template <typename T, typename R>
__global__ __launch_bounds__(1024) void k_add_norm_long(const T* x, int64_t ld_x, const R* res, int64_t ld_res, T* y, int64_t ld_y, R* h, int64_t ld_h,
                                                        float* __restrict__ mean_out, float* __restrict__ rstd_out, AddNorm a, Dropout d) {
  constexpr int V = Pack<T>::n;
  __shared__ float red[16];
  const Words words(d);
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    R* hr = h + r * ld_h;
    float s = 0.f;
    along_row<V>(a.cols, [&](uint32_t i, auto n) {
      constexpr int M = decltype(n)::value;
      float v[M], q[M];
      load_run(x + r * ld_x + i, v);
      load_run(res + r * ld_res + i, q);
      const uint32_t bits = d.on ? words.stay<M>((uint32_t)r, i) : ~0u;
#pragma unroll
      for (int e = 0; e < M; ++e) {
        v[e] = to_f32(from_f32<R>(q[e] + where_bit(bits, e, v[e] * d.scale)));
        s += v[e];
      }
      store_run(hr + i, v);
    });
    const float mean = block_sum<16>(s, red) / (float)a.cols;
    s = 0.f;
    along_row<V>(a.cols, [&](uint32_t i, auto n) {   // a thread reads what it has written itself
      float v[decltype(n)::value];
      load_run(hr + i, v);
#pragma unroll
      for (float e : v) s += (e - mean) * (e - mean);
    });
    const float rstd = 1.f / sqrtf(block_sum<16>(s, red) / (float)a.cols + a.eps);
    along_row<V>(a.cols, [&](uint32_t i, auto n) {
      constexpr int M = decltype(n)::value;
      float v[M], w[M], b[M];
      load_run(hr + i, v);
      load_run_as(a.weight, i, a.weight_type, 1.f, w);
      load_run_as(a.bias, i, a.weight_type, 0.f, b);
#pragma unroll
      for (int e = 0; e < M; ++e) v[e] = (v[e] - mean) * rstd * w[e] + b[e];
      store_run(y + r * ld_y + i, v);
    });
    if (threadIdx.x == 0) {
      if (mean_out) mean_out[r] = mean;
      if (rstd_out) rstd_out[r] = rstd;
    }
  }
}

template <typename T, typename R>
__global__ __launch_bounds__(1024) void k_add_norm_long_rows(const T* dy, int64_t ld_dy, const R* dh, int64_t ld_dh, const R* h, int64_t ld_h,
                                                             const float* __restrict__ mean, const float* __restrict__ rstd, T* dx, int64_t ld_dx, R* dres,
                                                             int64_t ld_dres, AddNorm a, Dropout d) {
  constexpr int V = Pack<T>::n;
  __shared__ float red[16];
  const Words words(d);
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const float mu = mean[r], rs = rstd[r];
    auto load = [&](uint32_t i, auto& v, auto& xh) {
      constexpr int M = sizeof(v) / sizeof(float);
      float q[M];
      load_run(dy + r * ld_dy + i, v);
      load_run(h + r * ld_h + i, xh);
      load_run_as(a.weight, i, a.weight_type, 1.f, q);
#pragma unroll
      for (int e = 0; e < M; ++e) {
        v[e] *= q[e];
        xh[e] = (xh[e] - mu) * rs;
      }
    };
    float s1 = 0.f, s2 = 0.f;
    along_row<V>(a.cols, [&](uint32_t i, auto n) {
      constexpr int M = decltype(n)::value;
      float v[M], xh[M];
      load(i, v, xh);
#pragma unroll
      for (int e = 0; e < M; ++e) {
        s1 += v[e];
        s2 += v[e] * xh[e];
      }
    });
    const float m1 = block_sum<16>(s1, red) / (float)a.cols;
    const float m2 = block_sum<16>(s2, red) / (float)a.cols;
    along_row<V>(a.cols, [&](uint32_t i, auto n) {
      constexpr int M = decltype(n)::value;
      float v[M], xh[M], g[M] = {};
      load(i, v, xh);
      if (dh) load_run(dh + r * ld_dh + i, g);
#pragma unroll
      for (int e = 0; e < M; ++e) v[e] = g[e] + rs * (v[e] - m1 - xh[e] * m2);
      if (dres) store_run(dres + r * ld_dres + i, v);
      if (dx) {
        const uint32_t bits = d.on ? words.stay<M>((uint32_t)r, i) : ~0u;
#pragma unroll
        for (int e = 0; e < M; ++e) v[e] = where_bit(bits, e, v[e] * d.scale);
        store_run(dx + r * ld_dx + i, v);
      }
    });
  }
}

// Elements a lane holds at most. Half as many, in groups of 128 and 512 lanes too, leave registers for twice the wavefronts and take as long or longer: backward 8192x1024 bf16 34 us
// over fp32 in place of 27.5, 35 over bf16 in place of 23, 16384x2048 117 / 116, 5001x1531 fp16 28 / 28.
constexpr int kMost = 16;

// with_group's, and 192 lanes a row where they suffice: 5001x1531 fp16 forward 17.2 -> 16.0 us, backward 28.5 -> 26.4, 20000x1280 bf16 47 -> 42, 72 -> 65.
template <int V, typename F>
bool with_rows(int64_t cols, F&& f) {
  constexpr int N = kMost / V / 2;
  const int64_t packs = (cols + V - 1) / V;
  if (packs > 128 * N && packs <= 192 * N) {
    f(std::integral_constant<int, 192>{}, std::integral_constant<int, N>{});
    return true;
  }
  return with_group<V, kMost>(cols, f);
}

// Rows of the widest group have no registers left for the columns' sums (1024x16384 bf16 over fp32 with spills 107 us, over bf16 76): theirs are
// a pass of their own, as those of longer rows (78, 59).
template <int V, int G, int N> constexpr bool kWide = G == 1024 && N * V == kMost;

// Workgroups, each of which leaves a row of partial sums; for 192 lanes 512 / 768 / 1024 of them: 5001x1531 fp16 30.6 / 26.4 / 27.4 us, 1000x1531 14.5 / 16.5 / 19.7.
template <int G>
int64_t back_blocks(int64_t rows) {
  return std::min<int64_t>((rows + Group<G>::kRows - 1) / Group<G>::kRows, G == 1024 ? 256 : G == 192 && rows >= 4096 ? 768 : 512);
}
template <int V>
int64_t back_parts(int64_t rows, int64_t cols) {
  int64_t parts = slabs_of(rows);
  with_rows<V>(cols, [&](auto g, auto n) {
    if (!kWide<V, decltype(g)::value, decltype(n)::value>) parts = back_blocks<decltype(g)::value>(rows);
  });
  return parts;
}

// Arrays that the Infinity Cache cannot hold are read past it: forward 16384x2048 bf16 over fp32 82 -> 77 us, backward 107 -> 101, over bf16 72 -> 65; but 8192x1024 bf16 over fp32, which
// it holds, 19 -> 24.
template <int G> constexpr bool kMayPass = G >= 64;   // narrower rows are hardly ever so many
// Calls f(whether to read past the cache).
template <int G, typename F>
void with_policy(int64_t bytes, F&& f) {
  if constexpr (kMayPass<G>)
    if (bytes > kCacheBytes) return f(std::true_type{});
  f(std::false_type{});
}

// Calls `f` with values of the two types; the residual's is the same, or float32.
template <typename F>
void with_types(uint32_t type, uint32_t residual_type, F&& f) {
  with_type(type, [&](auto t) {
    if (residual_type == LOPT_F32) f(t, 0.f);
    else f(t, t);
  });
}

lopt_status check_common(int64_t rows, int64_t cols, uint32_t type, uint32_t residual_type, uint32_t weight_type, float p, uint64_t seed, const uint64_t* seed_device,
                         uint64_t offset, Dropout* d) {
  LOPT_CHECK(check_type("type", type));
  LOPT_CHECK(check_type("residual_type", residual_type));
  LOPT_CHECK(check_type("weight_type", weight_type));
  if (residual_type != type && residual_type != LOPT_F32) return fail_call(LOPT_EINVAL, "residual_type %u is neither type %u nor float32", residual_type, type);
  LOPT_CHECK(check_matrix(rows, cols, "cols"));
  LOPT_CHECK(check_dropout(p, seed_device, d));
  d->seed = seed;
  d->offset = offset;
  return LOPT_OK;
}

// An output that is an input has that input's element size and distance of rows.
lopt_status check_in_place(const char* what, const void* out, int64_t ld_out, uint32_t out_type, const void* in, int64_t ld_in, uint32_t in_type, int64_t rows) {
  if (!out || out != in) return LOPT_OK;
  if (type_bytes(out_type) != type_bytes(in_type)) return fail_call(LOPT_EINVAL, "%s is an input of another type", what);
  if (ld_out != ld_in && rows > 1) return fail_call(LOPT_EINVAL, "%s is an input, but its ld is not that input's", what);
  return LOPT_OK;
}

}  // namespace
}  // namespace lopt

using namespace lopt;

extern "C" {

lopt_status lopt_dropout_add_layer_norm(const void* x, int64_t ld_x, const void* residual, int64_t ld_res, const void* weight, const void* bias, void* y,
                                        int64_t ld_y, void* h, int64_t ld_h, float* mean, float* rstd, int64_t rows, int64_t cols, float eps, uint32_t type,
                                        uint32_t residual_type, uint32_t weight_type, float p, uint64_t seed, const uint64_t* seed_device, uint64_t offset,
                                        void* hip_stream) {
  Dropout d{};
  LOPT_CHECK(check_common(rows, cols, type, residual_type, weight_type, p, seed, seed_device, offset, &d));
  if (!(eps >= 0.f) || std::isinf(eps)) return fail_call(LOPT_EINVAL, "eps must be finite and >= 0");
  LOPT_CHECK(check_ld("ld_x", rows, cols, ld_x, y == x));
  LOPT_CHECK(check_ld("ld_res", rows, cols, ld_res, h == residual));
  LOPT_CHECK(check_ld("ld_y", rows, cols, ld_y, true));
  LOPT_CHECK(check_ld("ld_h", rows, cols, ld_h, true));
  LOPT_CHECK(check_array("x", x, type_bytes(type), rows > 0));
  LOPT_CHECK(check_array("residual", residual, type_bytes(residual_type), rows > 0));
  LOPT_CHECK(check_array("y", y, type_bytes(type), rows > 0));
  LOPT_CHECK(check_array("h", h, type_bytes(residual_type), rows > 0));
  LOPT_CHECK(check_array("weight", weight, type_bytes(weight_type), false));
  LOPT_CHECK(check_array("bias", bias, type_bytes(weight_type), false));
  LOPT_CHECK(check_array("mean", mean, 4, false));
  LOPT_CHECK(check_array("rstd", rstd, 4, false));
  if (rows > 0 && y == h) return fail_call(LOPT_EINVAL, "y and h are the same memory");
  LOPT_CHECK(check_in_place("y", y, ld_y, type, x, ld_x, type, rows));
  LOPT_CHECK(check_in_place("h", h, ld_h, residual_type, residual, ld_res, residual_type, rows));
  LOPT_CHECK(check_in_place("y", y, ld_y, type, residual, ld_res, residual_type, rows));
  LOPT_CHECK(check_in_place("h", h, ld_h, residual_type, x, ld_x, type, rows));
  if (rows == 0) return LOPT_OK;
  const AddNorm a{weight, bias, weight_type, eps, rows, (uint32_t)cols};
  hipStream_t stream = (hipStream_t)hip_stream;
  with_types(type, residual_type, [&](auto t, auto u) {
    using T = decltype(t);
    using R = decltype(u);
    const bool held = with_rows<Pack<T>::n>(cols, [&](auto g, auto n) {
      constexpr int G = decltype(g)::value, N = decltype(n)::value;
      const int64_t blocks = std::min<int64_t>((rows + Group<G>::kRows - 1) / Group<G>::kRows, G == 1024 ? 512 : 2048);
      with_policy<G>(2 * rows * cols * (int64_t)(sizeof(T) + sizeof(R)), [&](auto nt) {
        hipLaunchKernelGGL((k_add_norm<T, R, G, N, decltype(nt)::value>), dim3((unsigned)blocks), dim3(Group<G>::kThreads), 0, stream, (const T*)x, ld_x, (const R*)residual, ld_res,
                           (T*)y, ld_y, (R*)h, ld_h, mean, rstd, a, d);
      });
    });
    if (!held)
      hipLaunchKernelGGL((k_add_norm_long<T, R>), dim3((unsigned)std::min<int64_t>(rows, 1 << 16)), dim3(1024), 0, stream, (const T*)x, ld_x, (const R*)residual,
                         ld_res, (T*)y, ld_y, (R*)h, ld_h, mean, rstd, a, d);
  });
  return launch_status("lopt_dropout_add_layer_norm");
}

size_t lopt_dropout_add_layer_norm_workspace(int64_t rows, int64_t cols) {
  if (rows <= 0 || cols <= 0 || rows > 0x7fffffffLL || cols > 0x7fffffffLL) return 0;
  return (size_t)std::max(back_parts<4>(rows, cols), back_parts<8>(rows, cols)) * 2 * (size_t)cols * sizeof(float);
}

lopt_status lopt_dropout_add_layer_norm_backward(const void* dy, int64_t ld_dy, const void* dh, int64_t ld_dh, const void* h, int64_t ld_h, const void* weight,
                                                 const float* mean, const float* rstd, void* dx, int64_t ld_dx, void* dresidual, int64_t ld_dres, void* dweight,
                                                 void* dbias, int64_t rows, int64_t cols, uint32_t type, uint32_t residual_type, uint32_t weight_type, float p,
                                                 uint64_t seed, const uint64_t* seed_device, uint64_t offset, void* workspace, size_t workspace_bytes,
                                                 void* hip_stream) {
  Dropout d{};
  LOPT_CHECK(check_common(rows, cols, type, residual_type, weight_type, p, seed, seed_device, offset, &d));
  LOPT_CHECK(check_ld("ld_dy", rows, cols, ld_dy, false));
  if (dh) LOPT_CHECK(check_ld("ld_dh", rows, cols, ld_dh, false));
  LOPT_CHECK(check_ld("ld_h", rows, cols, ld_h, false));
  if (dx) LOPT_CHECK(check_ld("ld_dx", rows, cols, ld_dx, true));
  if (dresidual) LOPT_CHECK(check_ld("ld_dres", rows, cols, ld_dres, true));
  LOPT_CHECK(check_array("dy", dy, type_bytes(type), rows > 0));
  LOPT_CHECK(check_array("dh", dh, type_bytes(residual_type), false));
  LOPT_CHECK(check_array("h", h, type_bytes(residual_type), rows > 0));
  LOPT_CHECK(check_array("mean", mean, 4, rows > 0));
  LOPT_CHECK(check_array("rstd", rstd, 4, rows > 0));
  LOPT_CHECK(check_array("weight", weight, type_bytes(weight_type), false));
  LOPT_CHECK(check_array("dx", dx, type_bytes(type), false));
  LOPT_CHECK(check_array("dresidual", dresidual, type_bytes(residual_type), false));
  LOPT_CHECK(check_array("dweight", dweight, type_bytes(weight_type), false));
  LOPT_CHECK(check_array("dbias", dbias, type_bytes(weight_type), false));
  if (rows > 0 && dx && dx == dresidual) return fail_call(LOPT_EINVAL, "dx and dresidual are the same memory");
  const struct { const char* name; void* out; int64_t ld; uint32_t type; } outs[2] = {{"dx", dx, ld_dx, type}, {"dresidual", dresidual, ld_dres, residual_type}};
  for (const auto& o : outs) {
    LOPT_CHECK(check_in_place(o.name, o.out, o.ld, o.type, dy, ld_dy, type, rows));
    LOPT_CHECK(check_in_place(o.name, o.out, o.ld, o.type, dh, ld_dh, residual_type, rows));
    LOPT_CHECK(check_in_place(o.name, o.out, o.ld, o.type, h, ld_h, residual_type, rows));
  }
  const bool columns = dweight || dbias;
  if (columns) LOPT_CHECK(check_workspace(workspace, workspace_bytes, lopt_dropout_add_layer_norm_workspace(rows, cols)));
  if (rows == 0 && !columns) return LOPT_OK;
  const AddNorm a{weight, nullptr, weight_type, 0.f, rows, (uint32_t)cols};
  hipStream_t stream = (hipStream_t)hip_stream;
  float* part = (float*)workspace;
  with_types(type, residual_type, [&](auto t, auto u) {
    using T = decltype(t);
    using R = decltype(u);
    int64_t parts = 0;
    if (rows > 0) {
      parts = back_parts<Pack<T>::n>(rows, cols);
      const bool held = with_rows<Pack<T>::n>(cols, [&](auto g, auto n) {
        constexpr int G = decltype(g)::value, N = decltype(n)::value;
        constexpr bool wide = kWide<Pack<T>::n, G, N>;
        if (wide && columns) launch_long_columns<T, R>((const T*)dy, ld_dy, (const R*)h, ld_h, mean, rstd, rows, a.cols, parts, part, stream);
        if (!wide || dx || dresidual)
          with_policy<G>(rows * cols * (int64_t)(2 * sizeof(T) + 3 * sizeof(R)), [&](auto nt) {
            hipLaunchKernelGGL((k_add_norm_back<T, R, G, N, !wide, decltype(nt)::value>), dim3((unsigned)(wide ? std::min<int64_t>(rows, 256) : parts)), dim3(Group<G>::kThreads), 0,
                               stream, (const T*)dy, ld_dy, (const R*)dh, ld_dh, (const R*)h, ld_h, mean, rstd, (T*)dx, ld_dx, (R*)dresidual, ld_dres, a, d,
                               columns && !wide ? part : nullptr);
          });
      });
      if (!held) {
        if (columns) launch_long_columns<T, R>((const T*)dy, ld_dy, (const R*)h, ld_h, mean, rstd, rows, a.cols, parts, part, stream);
        if (dx || dresidual)
          hipLaunchKernelGGL((k_add_norm_long_rows<T, R>), dim3((unsigned)std::min<int64_t>(rows, 1 << 16)), dim3(1024), 0, stream, (const T*)dy, ld_dy,
                             (const R*)dh, ld_dh, (const R*)h, ld_h, mean, rstd, (T*)dx, ld_dx, (R*)dresidual, ld_dres, a, d);
      }
    }
    if (columns) launch_columns_sum(part, parts, cols, weight_type, dweight, dbias, stream);
  });
  return launch_status("lopt_dropout_add_layer_norm_backward");
}

}  // extern "C"
