// Layer norm and its gradient. Forward, per row: mean = sum x / n, rstd = 1 / sqrt(sum (x - mean)^2 / n + eps), y = (x - mean) rstd w + b, in two
// sums over a row that is held, never sum x^2 - mean^2. Backward, with h = (x - mean) rstd and a = dy w: dx = rstd (a - sum(a) / n - h sum(a h) / n),
// dw = sum over the rows of dy h, db of dy. Both are bound by memory where there is enough of it (two and three arrays once each), by
// the launches below some 10 MB. Times below are of calls one behind the other in a graph, on the same inputs; those of a single kernel are from a kernel trace, where
// launches do not overlap, so that two of them add up to more than the call.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "lopt_ops.h"

namespace lopt {
namespace {

// ---- rows that one group of G lanes holds in registers. G = 8, 16, 32, 64: several rows a workgroup; G = 256, 1024: a workgroup a row. Against one
// workgroup of 256 for every row, which reads it three times: 12608x768 bf16 24 -> 9.5 us, backward of 8192x1024 bf16 74 -> 17.
template <int G> struct Group {
  static constexpr int kThreads = G <= 64 ? kBlock : G, kRows = kThreads / G, kWaves = G <= 64 ? 1 : G / 64;
};

// Sum over a group; every lane of it gets the same. Groups of several wavefronts: `red` has kWaves floats that no other sum uses until
// the group has passed another barrier.
template <int G>
__device__ __forceinline__ float group_sum(float v, float* red) {
  if (G >= 64) {
    v = wave_sum(v);
    if (G > 64) {
      if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
      __syncthreads();
      v = red[0];
#pragma unroll
      for (int i = 1; i < Group<G>::kWaves; ++i) v += red[i];
    }
    return v;
  }
  v += dpp_f<0xB1>(v);    // quad_perm [1,0,3,2]
  v += dpp_f<0x4E>(v);    // quad_perm [2,3,0,1]
  v += dpp_f<0x141>(v);   // row_half_mirror
  if (G >= 16) v += dpp_f<0x140>(v);   // row_mirror
  if (G >= 32) v += __shfl_xor(v, 16);
  return v;
}

// Two at once: `red` has 2 kWaves floats.
template <int G>
__device__ __forceinline__ void group_sums(float& v, float& w, float* red) {
  constexpr int W = Group<G>::kWaves;
  if (W == 1) {
    v = group_sum<G>(v, red);
    w = group_sum<G>(w, red);
    return;
  }
  v = wave_sum(v);
  w = wave_sum(w);
  if ((threadIdx.x & 63) == 0) {
    red[threadIdx.x >> 6] = v;
    red[W + (threadIdx.x >> 6)] = w;
  }
  __syncthreads();
  v = red[0];
  w = red[W];
#pragma unroll
  for (int i = 1; i < W; ++i) {
    v += red[i];
    w += red[W + i];
  }
}

// V floats that may start at any float.
template <int V> struct FloatPack { typedef float type __attribute__((ext_vector_type(V), aligned(4))); };

// A lane's share of a row: N packs of 16 bytes, G packs from one to the next. The pack that would pass the row's end is moved back to
// end with it; its first `skip` elements are the lane's before. Rows shorter than a
// pack (N = 0): one element a lane.
template <typename T, int G, int N>
struct Share {
  static constexpr int V = N ? Pack<T>::n : 1, P = N ? N : 1, E = P * V;
  uint32_t at[P];
  int skip[P];
  bool have[P];
  __device__ __forceinline__ Share(uint32_t cols) {
    const uint32_t lane = threadIdx.x & (G - 1);
#pragma unroll
    for (int j = 0; j < P; ++j) {
      const uint32_t k = (j * G + lane) * V;
      const bool full = j < P / 2;   // with_group takes no more packs than it has to
      have[j] = full || k < cols;
      at[j] = full ? k : min(k, cols - V);
      skip[j] = full ? 0 : have[j] ? (int)(k - at[j]) : V;
    }
  }
  __device__ __forceinline__ bool mine(int i) const { return i % V >= skip[i / V]; }
  // The lane's columns of an array, written from v or added to it; `v` has its own at the same places.
  __device__ __forceinline__ void write(float* a, const float (&v)[E]) const {
#pragma unroll
    for (int j = 0; j < P; ++j) {
      if (skip[j] == 0) {
        typename FloatPack<V>::type o;
#pragma unroll
        for (int e = 0; e < V; ++e) o[e] = v[j * V + e];
        *(typename FloatPack<V>::type*)(a + at[j]) = o;
      } else if (have[j]) {
#pragma unroll
        for (int e = 0; e < V; ++e)
          if (e >= skip[j]) a[at[j] + e] = v[j * V + e];
      }
    }
  }
  __device__ __forceinline__ void add(const float* a, float (&v)[E]) const {
#pragma unroll
    for (int j = 0; j < P; ++j)
      if (have[j]) {
        const typename FloatPack<V>::type o = *(const typename FloatPack<V>::type*)(a + at[j]);
#pragma unroll
        for (int e = 0; e < V; ++e) v[j * V + e] = o[e] + v[j * V + e];
      }
  }
};

template <typename T, int G, int N>
struct Row {
  typedef Share<T, G, N> S;
  typedef typename Pack<T>::type pack;
  pack raw[N ? N : 1];
  __device__ __forceinline__ void load(const T* row, const S& s) {
#pragma unroll
    for (int j = 0; j < S::P; ++j) {
      raw[j] = pack{};
      if (s.have[j]) {
        if (N) raw[j] = *(const pack*)(row + s.at[j]);
        else raw[j][0] = row[s.at[j]];
      }
    }
  }
  __device__ __forceinline__ float get(int i) const { return to_f32(raw[i / S::V][i % S::V]); }
  __device__ __forceinline__ static void store(T* row, const S& s, int j, const float* v) {
    if (!s.have[j]) return;
    if (N && s.skip[j]) {
#pragma unroll
      for (int e = 0; e < S::V; ++e)
        if (e >= s.skip[j]) row[s.at[j] + e] = from_f32<T>(v[e]);
    } else if (N) {
      pack o;
#pragma unroll
      for (int e = 0; e < S::V; ++e) o[e] = from_f32<T>(v[e]);
      *(pack*)(row + s.at[j]) = o;
    } else {
      row[s.at[j]] = from_f32<T>(v[0]);
    }
  }
};

// One pack of a lane's share of a weight or bias vector; `other` where there is none.
template <typename W, int V>
__device__ __forceinline__ void load_pack_as(const W* p, float* v) {
#pragma unroll
  for (int e = 0; e < V; ++e) v[e] = to_f32(p[e]);
}
template <typename S>
__device__ __forceinline__ void load_vector(const void* p, uint32_t type, const S& s, int j, float other, float* v) {
#pragma unroll
  for (int e = 0; e < S::V; ++e) v[e] = other;
  if (!p || !s.have[j]) return;
  if (type == LOPT_F32) load_pack_as<float, S::V>((const float*)p + s.at[j], v);
  else if (type == LOPT_BF16) load_pack_as<bf16_t, S::V>((const bf16_t*)p + s.at[j], v);
  else load_pack_as<f16_t, S::V>((const f16_t*)p + s.at[j], v);
}

// Groups of 1024 have 128 registers a lane: they ask for nothing ahead and read the vectors again for every row.
template <int G> constexpr bool kAhead = G < 1024;

struct Vectors { const void* w; const void* b; uint32_t type; };

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
  if (!part) return;
  float* out = part + (int64_t)blockIdx.x * 2 * cols;
  __shared__ __align__(16) float sums[kRows == 1 ? 1 : kRows / 2][2][kRows == 1 ? 4 : G * E];   // by column
  const int group = threadIdx.x / G;
#pragma unroll
  for (int half = kRows / 2; half >= 1; half /= 2) {   // the upper half hands over to the lower
    if (group >= half && group < 2 * half) {
      s.write(sums[group - half][0], sw);
      s.write(sums[group - half][1], sb);
    }
    __syncthreads();
    if (group < half) {
      s.add(sums[group][0], sw);
      s.add(sums[group][1], sb);
    }
    __syncthreads();
  }
  if (group == 0) {
    s.write(out, sw);
    s.write(out + cols, sb);
  }
}

// The partial sums of `parts` workgroups, added up in double: a workgroup takes 32 columns of one of the two sums, 32 lanes a row of partial sums. A launch
// has no more than 2^32 threads in a row: the workgroups of more than kMostColumnBlocks go round.
constexpr int64_t kMostColumnBlocks = 1 << 20;
template <typename W>
__global__ __launch_bounds__(1024) void k_norm_columns_sum(const float* __restrict__ part, int64_t parts, uint32_t cols, W* __restrict__ dw, W* __restrict__ db) {
  __shared__ double sums[32][33];
  const int col = threadIdx.x & 31, row = threadIdx.x >> 5;
  W* out = blockIdx.y ? db : dw;
  if (!out) return;
  for (uint64_t first = (uint64_t)blockIdx.x * 32; first < cols; first += (uint64_t)gridDim.x * 32) {
    const uint64_t c = first + col;
    double s = 0.0;
    if (c < cols) {
      const float* p = part + (uint64_t)blockIdx.y * cols + c;
      int64_t k = row;
      for (; k + 32 * 7 < parts; k += 32 * 8) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = p[2 * (k + 32 * i) * cols];
#pragma unroll
        for (int i = 0; i < 8; ++i) s += (double)v[i];
      }
      for (; k < parts; k += 32) s += (double)p[2 * k * cols];
    }
    sums[row][col] = s;
    __syncthreads();
    if (row == 0 && c < cols) {
      for (int i = 1; i < 32; ++i) s += sums[i][col];
      out[c] = from_f32<W>((float)s);
    }
    if (first + (uint64_t)gridDim.x * 32 < cols) __syncthreads();
  }
}

// ---- rows too long for registers (above 32768 columns, backward 16384; fp32 the same): one workgroup a row, which reads it again (from L2) for every
// use. us: 200x65536 bf16 16, backward 53 (dx alone 22); 2000x20000 bf16 40, backward 87 (dx alone 52).
// Calls f(first element, pack or element count) over a row: packs of 16 bytes, four in flight a thread, then what is left element by element.
template <int V, typename F>
__device__ __forceinline__ void along_row(uint32_t cols, F&& f) {
  using std::integral_constant;
  const uint32_t packs = cols / V;
  uint32_t k = threadIdx.x;
  for (; k + 3 * 1024 < packs; k += 4 * 1024) {
#pragma unroll
    for (int j = 0; j < 4; ++j) f((k + j * 1024) * V, integral_constant<int, V>{});
  }
  for (; k < packs; k += 1024) f(k * V, integral_constant<int, V>{});
  for (uint32_t i = packs * V + threadIdx.x; i < cols; i += 1024) f(i, integral_constant<int, 1>{});
}
template <typename T, int V>
__device__ __forceinline__ void load_run(const T* p, float (&v)[V]) {
  typedef T run __attribute__((ext_vector_type(V), aligned(sizeof(T))));
  const run x = *(const run*)p;
#pragma unroll
  for (int e = 0; e < V; ++e) v[e] = to_f32(x[e]);
}
template <typename T, int V>
__device__ __forceinline__ void store_run(T* p, const float (&v)[V]) {
  typedef T run __attribute__((ext_vector_type(V), aligned(sizeof(T))));
  run x;
#pragma unroll
  for (int e = 0; e < V; ++e) x[e] = from_f32<T>(v[e]);
  *(run*)p = x;
}
template <int V>
__device__ __forceinline__ void load_run_as(const void* p, uint32_t i, uint32_t type, float other, float (&v)[V]) {
#pragma unroll
  for (int e = 0; e < V; ++e) v[e] = other;
  if (!p) return;
  if (type == LOPT_F32) load_run((const float*)p + i, v);
  else if (type == LOPT_BF16) load_run((const bf16_t*)p + i, v);
  else load_run((const f16_t*)p + i, v);
}

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

// Rows whose column sums one lane adds up. With few rows that leaves few wavefronts: 200x65536 bf16 7 x 129 of them, which take 33 of the backward pass's 53 us.
constexpr int kSlab = 32;

// Partial sums of dy xh and dy over a slab of rows, a pack of columns a lane; the pack that would pass the row's end ends with it, and gives the columns that
// it shares the same sums. Runs before dx, which may overwrite dy or x.
template <typename T>
__global__ __launch_bounds__(kWave) void k_norm_long_columns(const T* __restrict__ dy, int64_t ld_dy, const T* __restrict__ x, int64_t ld_x,
                                                             const float* __restrict__ mean, const float* __restrict__ rstd, int64_t rows, uint32_t cols,
                                                             float* __restrict__ part) {
  constexpr int V = Pack<T>::n;
  const uint64_t k = ((uint64_t)blockIdx.x * kWave + threadIdx.x) * V;
  if (k >= cols) return;
  const uint32_t c = min((uint32_t)k, cols - V);
  for (int64_t slab = blockIdx.y; slab * kSlab < rows; slab += gridDim.y) {
    const int64_t r0 = slab * kSlab, r1 = min(r0 + kSlab, rows);
    float sw[V] = {}, sb[V] = {};
#pragma unroll 4
    for (int64_t r = r0; r < r1; ++r) {
      float g[V], h[V];
      load_run(dy + r * ld_dy + c, g);
      load_run(x + r * ld_x + c, h);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        sw[e] += g[e] * ((h[e] - mean[r]) * rstd[r]);
        sb[e] += g[e];
      }
    }
    store_run(part + slab * 2 * cols + c, sw);
    store_run(part + (slab * 2 + 1) * cols + c, sb);
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

// Calls f(group size, packs) as integral constants for the smallest group that holds a row with at most `most` elements a lane; false
// if none does. Of N >= 2 packs a lane the first N / 2 always lie in the row.
template <int V, int most, typename F>
bool with_group(int64_t cols, F&& f) {
  using std::integral_constant;
  const int64_t packs = (cols + V - 1) / V;
  auto take = [&](auto g, auto n) { f(g, n); return true; };
  if (cols < V) return take(integral_constant<int, 8>{}, integral_constant<int, 0>{});
  if (packs <= 8) return take(integral_constant<int, 8>{}, integral_constant<int, 1>{});
  if (packs <= 16) return take(integral_constant<int, 16>{}, integral_constant<int, 1>{});
  if (packs <= 32) return take(integral_constant<int, 32>{}, integral_constant<int, 1>{});
  if (packs <= 64) return take(integral_constant<int, 64>{}, integral_constant<int, 1>{});
  if (packs <= 128) return take(integral_constant<int, 64>{}, integral_constant<int, 2>{});
  constexpr int N = most / V;
  if (N >= 4 && packs <= 256) return take(integral_constant<int, 64>{}, integral_constant<int, N >= 4 ? 4 : 1>{});
  if (N > 4 && packs <= 64 * N) return take(integral_constant<int, 64>{}, integral_constant<int, N>{});
  if (packs <= 256 * N / 2) return take(integral_constant<int, 256>{}, integral_constant<int, N / 2>{});
  if (packs <= 256 * N) return take(integral_constant<int, 256>{}, integral_constant<int, N>{});
  if (packs <= 1024 * N / 2) return take(integral_constant<int, 1024>{}, integral_constant<int, N / 2>{});
  if (packs <= 1024 * N) return take(integral_constant<int, 1024>{}, integral_constant<int, N>{});
  return false;
}
// Elements a lane holds at most: forward the row and two vectors, backward two rows, one vector and two sums. 32 and 16 leave
// every wavefront of a workgroup of 1024 the 128 registers that it can have; smaller groups, whose wavefronts could have more, keep to the same.
constexpr int kMostForward = 32, kMostBackward = 16;

int64_t slabs_of(int64_t rows) { return (rows + kSlab - 1) / kSlab; }

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
          hipLaunchKernelGGL(k_norm_long_columns<T>, dim3((n_cols / Pack<T>::n + kWave) / kWave, (unsigned)std::min<int64_t>(parts, 1024)), dim3(kWave), 0, stream,
                             (const T*)dy, ld_dy, (const T*)x, ld_x, mean, rstd, rows, n_cols, part);
        if (dx)
          hipLaunchKernelGGL(k_norm_long_rows<T>, dim3((unsigned)std::min<int64_t>(rows, 1 << 16)), dim3(1024), 0, stream, (const T*)dy, ld_dy, (const T*)x, ld_x,
                             weight, weight_type, mean, rstd, (T*)dx, ld_dx, rows, n_cols);
      }
    }
    if (columns)
      with_type(weight_type, [&](auto u) {
        using W = decltype(u);
        hipLaunchKernelGGL(k_norm_columns_sum<W>, dim3((unsigned)std::min(((int64_t)cols + 31) / 32, kMostColumnBlocks), 2), dim3(1024), 0, stream, (const float*)part, parts, n_cols, (W*)dweight, (W*)dbias);
      });
  });
  return launch_status("lopt_layer_norm_backward");
}

}  // extern "C"
