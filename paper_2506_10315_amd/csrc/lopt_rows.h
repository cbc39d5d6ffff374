// Rows of matrices as groups of lanes hold them in registers, rows too long for that, and sums over their columns: what the layer norms share.
#pragma once

#include <algorithm>
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

// V elements that may start at any element.
template <typename T, int V> struct Run { typedef T type __attribute__((ext_vector_type(V), aligned(sizeof(T)))); };

// A lane's share of a row: N packs of 16 bytes, G packs from one to the next. The pack that would pass the row's end is moved back to
// end with it; its first `skip` elements are the lane's before. Rows shorter than a
// pack (N = 0): one element a lane.
template <typename T, int G, int N>
struct Share {
  static constexpr int V = N ? Pack<T>::n : 1, P = N ? N : 1, E = P * V;
  static constexpr bool kPacks = N > 0;
  uint32_t at[P];
  int skip[P];
  bool have[P];
  __device__ __forceinline__ Share(uint32_t cols) {
    const uint32_t lane = G > 64 ? threadIdx.x : threadIdx.x & (G - 1);   // groups of more than a wavefront are workgroups
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
        typename Run<float, V>::type o;
#pragma unroll
        for (int e = 0; e < V; ++e) o[e] = v[j * V + e];
        *(typename Run<float, V>::type*)(a + at[j]) = o;
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
        const typename Run<float, V>::type o = *(const typename Run<float, V>::type*)(a + at[j]);
#pragma unroll
        for (int e = 0; e < V; ++e) v[j * V + e] = o[e] + v[j * V + e];
      }
  }
};

// A row of elements of type T in the places of a share S, which may be that of a shorter type.
template <typename T, typename S>
struct RowOf {
  static constexpr bool N = S::kPacks;
  typedef typename Run<T, N ? S::V : 1>::type pack;
  pack raw[S::P];
  template <bool NT = false>
  __device__ __forceinline__ void load(const T* row, const S& s) {
#pragma unroll
    for (int j = 0; j < S::P; ++j) {
      raw[j] = pack{};
      if (s.have[j]) {
        if (N) raw[j] = NT ? __builtin_nontemporal_load((const pack*)(row + s.at[j])) : *(const pack*)(row + s.at[j]);
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

template <typename T, int G, int N> using Row = RowOf<T, Share<T, G, N>>;

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

// The end of a backward pass: the column sums of a workgroup's groups, added up half to half, become its row of partial sums.
template <typename S, int G, int kRows>
__device__ __forceinline__ void columns_of_block(const S& s, float (&sw)[S::E], float (&sb)[S::E], float* __restrict__ part, uint32_t cols) {
  constexpr int E = S::E;
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

inline void launch_columns_sum(const float* part, int64_t parts, int64_t cols, uint32_t weight_type, void* dw, void* db, hipStream_t stream) {
  with_type(weight_type, [&](auto u) {
    using W = decltype(u);
    hipLaunchKernelGGL(k_norm_columns_sum<W>, dim3((unsigned)std::min((cols + 31) / 32, kMostColumnBlocks), 2), dim3(1024), 0, stream, part, parts, (uint32_t)cols, (W*)dw,
                       (W*)db);
  });
}

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
// Rows whose column sums one lane adds up. With few rows that leaves few wavefronts: 200x65536 bf16 7 x 129 of them, which take 33 of the backward pass's 53 us.
constexpr int kSlab = 32;
inline int64_t slabs_of(int64_t rows) { return (rows + kSlab - 1) / kSlab; }

// Partial sums of dy xh and dy over a slab of rows, a pack of columns a lane; the pack that would pass the row's end ends with it, and gives the columns that
// it shares the same sums. Runs before dx, which may overwrite dy or x.
template <typename T, typename X>
__global__ __launch_bounds__(kWave) void k_norm_long_columns(const T* __restrict__ dy, int64_t ld_dy, const X* __restrict__ x, int64_t ld_x,
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

template <typename T, typename X>
inline void launch_long_columns(const T* dy, int64_t ld_dy, const X* x, int64_t ld_x, const float* mean, const float* rstd, int64_t rows, uint32_t cols, int64_t parts,
                                float* part, hipStream_t stream) {
  hipLaunchKernelGGL((k_norm_long_columns<T, X>), dim3((cols / Pack<T>::n + kWave) / kWave, (unsigned)std::min<int64_t>(parts, 1024)), dim3(kWave), 0, stream, dy, ld_dy, x,
                     ld_x, mean, rstd, rows, cols, part);
}

}  // namespace
}  // namespace lopt
