// Softmax over rows of logits: the base of the running sums, and pieces of a row in a wavefront's registers.
#pragma once

#include <cmath>

#include "lopt_ops.h"

namespace lopt {
namespace {

// Exponents are t = x c - b with c = scale / ln 2 and b = m c for the largest logit m, rounded and held within kMostBase: its rounding is
// in every exponent of the row alike. A row whose largest logit lies beyond is summed by differences from m.
constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.69314718055994531f;
constexpr float kMostBase = 268435456.f;

__device__ __forceinline__ float exp2_hw(float v) { return __builtin_amdgcn_exp2f(v); }
__device__ __forceinline__ float base_of(float m, float c) { return __builtin_amdgcn_fmed3f(m * c, -kMostBase, kMostBase); }
__device__ __forceinline__ bool beyond(float m, float c) { return fabsf(m * c) >= kMostBase && m != -INFINITY; }

// A wavefront, or a group of L of its lanes, takes a piece of a row at a time, E = 8 to 64 logits a lane in accesses of 16 bytes. Accesses are aligned: `off` elements ahead of the row
// begin a pack of 16 bytes, and pieces and packs are counted from there (rows at odd elements of 16 bits: 4096x50257 98 us, 83 at 50258; counted from
// their own start). The pack that would begin ahead of the row begins with it, the one that would pass the row's end ends
// with it, and the elements that they share with the pack beside them are masked.
template <typename T>
__device__ __forceinline__ int pack_offset(const T* row, uint32_t n) {
  return n >= (uint32_t)Pack<T>::n ? (int)((uintptr_t)row / sizeof(T) % Pack<T>::n) : 0;
}
template <typename T, int E, int L = kWave>
struct Piece {
  static constexpr int V = Pack<T>::n, N = E / V, kSize = E * L;
  typedef typename Pack<T>::type pack;
  pack raw[N];
  int first, off, n;
  // Where the lane's pack j would begin, in elements of the row, and where it does.
  __device__ __forceinline__ int place(int j) const { return first + (j * L + (int)(threadIdx.x % L)) * V - off; }
  __device__ __forceinline__ int begin(int j) const { return max(min(place(j), n - V), 0); }
  __device__ __forceinline__ int index(int i) const { return begin(i / V) + i % V; }
  // Whether an element is one, and this lane's.
  __device__ __forceinline__ bool mine(int i) const {
    const int p = place(i / V), k = index(i);
    return k >= p && k < min(p + V, n);
  }
  // Element of the first lane that the j-th packs begin with: below 0, they begin ahead of the row; n or above, they lie behind it.
  __device__ __forceinline__ int from(int j) const { return first + j * L * V - off; }
  template <bool NT = false>
  __device__ __forceinline__ void load(const T* row, int first_, int off_, int n_) {
    first = first_, off = off_, n = n_;
    if (n >= V) {
#pragma unroll
      for (int j = 0; j < N; ++j) raw[j] = NT ? __builtin_nontemporal_load((const pack*)(row + begin(j))) : *(const pack*)(row + begin(j));
    } else {
#pragma unroll
      for (int i = 0; i < E; ++i) raw[i / V][i % V] = mine(i) ? row[index(i)] : (T)-INFINITY;
    }
  }
  // Elements that are not the lane's become masked ones, where they lie. Of a row's packs one wavefront's first and one's last are mixed.
  __device__ __forceinline__ void mask() {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      if (from(j) >= 0 && from(j) + L * V <= n) continue;
      if (from(j) >= n) {
#pragma unroll
        for (int e = 0; e < V; ++e) raw[j][e] = (T)-INFINITY;
      } else {
        raw[j] = masked(raw[j], j);
      }
    }
  }
  __device__ __forceinline__ pack masked(pack v, int j) const {
    const int low = place(j) - begin(j), high = min(low + V, n - begin(j));   // of the pack's elements, the lane's
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = e >= low && e < high ? v[e] : (T)-INFINITY;
    return v;
  }
  __device__ __forceinline__ void unpack(float (&x)[E]) {
    mask();
#pragma unroll
    for (int i = 0; i < E; ++i) x[i] = to_f32(raw[i / V][i % V]);
  }
  // Pack j alone, read again (rows of a pack at least).
  __device__ __forceinline__ void values(const T* row, int j, float (&x)[V]) const {
    const pack v = masked(*(const pack*)(row + begin(j)), j);
#pragma unroll
    for (int e = 0; e < V; ++e) x[e] = to_f32(v[e]);
  }
};

template <int E>
__device__ __forceinline__ float most_of(const float (&x)[E]) {
  float m = x[0];
#pragma unroll
  for (int i = 1; i < E; ++i) m = fmaxf(m, x[i]);
  return m;
}

}  // namespace
}  // namespace lopt
