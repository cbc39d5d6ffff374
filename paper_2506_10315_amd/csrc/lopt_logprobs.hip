// Log probabilities of given tokens with entropy and top alternatives, and their gradient: softmax over rows of logits with a running
// maximum and sums, one pass over the logits in each direction.
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <type_traits>

#include "lopt_ops.h"

namespace lopt {
namespace {

// The order of the alternatives as one number: larger logit first, NaN above all, +0 and -0 alike, lower index first among equals.
// No element's number is 0 or all ones.
__device__ __forceinline__ uint32_t order_of(float x) {   // but for NaN
  const uint32_t u = __builtin_bit_cast(uint32_t, x + 0.f);
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ uint32_t full_order(float x) { return x != x ? 0xfffffffeu : order_of(x); }
__device__ __forceinline__ uint64_t rank_key(uint32_t order, uint32_t index) { return (uint64_t)order << 32 | (0xffffffffu - index); }
__device__ __forceinline__ uint32_t key_index(uint64_t key) { return 0xffffffffu - (uint32_t)key; }
__device__ __forceinline__ float key_value(uint64_t key) {
  const uint32_t u = (uint32_t)(key >> 32);
  return __builtin_bit_cast(float, u & 0x80000000u ? u ^ 0x80000000u : ~u);
}
// What to subtract from a logit so that the sign says whether it lies below a bound. Both zeros less -0 are +0, -0 less +0 would be -0; an infinite bound's
// difference from itself has no sign.
__device__ __forceinline__ float least_of(float bound) { return bound == 0.f ? -0.f : fminf(bound, FLT_MAX); }

// Running softmax sums of some logits x. With c = scale / ln 2, the hardware's 2^x, m = the largest of them and b = m c rounded:
//   s = sum 2^t,   h = sum 2^t t,   t = x c - b in one fused operation
// b's own rounding, m c - b = delta, is the same for every logit of the row and is taken out of ln S at the end:
//   ln S = ln s - delta ln 2,   entropy = ln s - ln 2 h / s
// which is one vector instruction a logit less than x - m, then times c. It adds delta to every exponent, so b is held within 2^28, where delta is 8
// at most (at 1.44e10 it would be 440, and 2^t infinite): logits of 1.8e8, or of 180 at a scale of 1e6. A lane or piece of logits below that (masks of -1e9 and
// less) adds 0; a row whose largest logit lies outside is summed again by extreme_sums.
// A masked logit has t = -infinity and 2^t = 0; for the product t is held to a finite value.
struct Soft { float m, s, h; };
constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.69314718055994531f;
constexpr float kMostBase = 268435456.f;

__device__ __forceinline__ float exp2_hw(float v) { return __builtin_amdgcn_exp2f(v); }
__device__ __forceinline__ float base_of(float m, float c) { return __builtin_amdgcn_fmed3f(m * c, -kMostBase, kMostBase); }

// a's sums seen from a larger m.
__device__ __forceinline__ Soft rebase(Soft a, float m, float c) {
  const float diff = base_of(a.m, c) - base_of(m, c), f = exp2_hw(diff), fs = f * a.s;
  return Soft{m, fs, f * a.h + (fs == 0.f ? 0.f : fs * diff)};
}
__device__ __forceinline__ Soft wave_join(Soft a, float c) {
  a = rebase(a, wave_max(a.m), c);
  return Soft{a.m, wave_sum(a.s), wave_sum(a.h)};
}

__device__ __forceinline__ bool beyond(float m, float c) { return fabsf(m * c) >= kMostBase && m != -INFINITY; }   // see extreme_sums

struct Outputs {
  float* logp;
  float* entropy;
  float* stats;
  float* top_logp;
  int64_t* top_index;
};
struct Target { int64_t t; float x; };

template <typename T>
__device__ __forceinline__ Target load_target(const T* row, const int64_t* targets, int64_t r, int vocab) {
  Target g{-1, 0.f};
  if (targets) {
    g.t = targets[r];
    if (g.t >= 0 && g.t < vocab) g.x = to_f32(row[g.t]);
  }
  return g;
}

// A row's outputs from its sums, which are by differences where `beyond` says so. Lane k of the wavefront holds the key of alternative k.
__device__ __forceinline__ void write_row(const Outputs& o, int64_t r, int lane, Soft a, float c, Target g, uint32_t vocab, float scale, int64_t ignore, int top, uint64_t key) {
  const float delta = fabsf(a.m * c) < kMostBase ? __builtin_fmaf(a.m, c, -base_of(a.m, c)) : 0.f;
  const bool empty = a.s == 0.f;
  const float ln_s = logf(a.s), log_s = ln_s - kLn2 * delta;
  if (lane == 0) {
    if (o.logp) {
      float v = NAN;
      if (g.t == ignore) v = 0.f;
      else if (g.t >= 0 && g.t < vocab) v = empty ? -INFINITY : scale * (g.x - a.m) - log_s;
      o.logp[r] = v;
    }
    if (o.entropy) o.entropy[r] = empty ? 0.f : ln_s - kLn2 * (a.h / a.s);
    o.stats[2 * r] = a.m;
    o.stats[2 * r + 1] = log_s;
  }
  if (lane < top) {
    o.top_index[r * top + lane] = key_index(key);
    o.top_logp[r * top + lane] = empty ? -INFINITY : scale * (key_value(key) - a.m) - log_s;
  }
}

// A wavefront takes a piece of a row at a time, E = 8 to 64 logits a lane in accesses of 16 bytes. Accesses are aligned: `off` elements ahead of the row
// begin a pack of 16 bytes, and pieces and packs are counted from there (rows at odd elements of 16 bits: 4096x50257 98 us, 83 at 50258; counted from
// their own start). The pack that would begin ahead of the row begins with it, the one that would pass the row's end ends
// with it, and the elements that they share with the pack beside them are masked.
template <typename T>
__device__ __forceinline__ int pack_offset(const T* row, uint32_t n) {
  return n >= (uint32_t)Pack<T>::n ? (int)((uintptr_t)row / sizeof(T) % Pack<T>::n) : 0;
}
template <typename T, int E>
struct Piece {
  static constexpr int V = Pack<T>::n, N = E / V, kSize = E * kWave;
  typedef typename Pack<T>::type pack;
  pack raw[N];
  int first, off, n;
  // Where the lane's pack j would begin, in elements of the row, and where it does.
  __device__ __forceinline__ int place(int j) const { return first + (j * kWave + (int)(threadIdx.x & 63)) * V - off; }
  __device__ __forceinline__ int begin(int j) const { return max(min(place(j), n - V), 0); }
  __device__ __forceinline__ int index(int i) const { return begin(i / V) + i % V; }
  // Whether an element is one, and this lane's.
  __device__ __forceinline__ bool mine(int i) const {
    const int p = place(i / V), k = index(i);
    return k >= p && k < min(p + V, n);
  }
  // Element of lane 0 that the wavefront's j-th packs begin with: below 0, they begin ahead of the row; n or above, they lie behind it.
  __device__ __forceinline__ int from(int j) const { return first + j * kWave * V - off; }
  __device__ __forceinline__ void load(const T* row, int first_, int off_, int n_) {
    first = first_, off = off_, n = n_;
    if (n >= V) {
#pragma unroll
      for (int j = 0; j < N; ++j) raw[j] = *(const pack*)(row + begin(j));
    } else {
#pragma unroll
      for (int i = 0; i < E; ++i) raw[i / V][i % V] = mine(i) ? row[index(i)] : (T)-INFINITY;
    }
  }
  // Elements that are not the lane's become masked ones, where they lie. Of a row's packs one wavefront's first and one's last are mixed.
  __device__ __forceinline__ void mask() {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      if (from(j) >= 0 && from(j) + kWave * V <= n) continue;
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
template <int E>
__device__ __forceinline__ void add_piece(Soft& a, const float (&x)[E], float most, float c) {
  const float m = fmaxf(a.m, most);
  a = rebase(a, m, c);
  const float b = base_of(m, c);
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const float t = __builtin_fmaf(x[i], c, -b), e = exp2_hw(t);
    a.s += e;
    a.h += e * fmaxf(t, -kMostBase);
  }
}

// Rows whose largest logit m is beyond kMostBase times 1 / c: summed again by differences from m, which may be as large as the type allows (+infinity: its
// difference from itself makes the sums NaN). By one wavefront of `waves`, in pieces as in the first pass: 4096x50257 bf16 at a scale of 1e8 119 us, 75 at 1.
template <typename T>
__device__ Soft extreme_sums(const T* row, uint32_t n, float m, float c, int wave, int waves) {
  typedef Piece<T, 16> P;
  const int off = pack_offset(row, n), end = (int)n + off;
  Soft a{m, 0.f, 0.f};
  for (int first = wave * P::kSize; first < end; first += waves * P::kSize) {
    P p;
    p.load(row, first, off, n);
    float v[16];
    p.unpack(v);
#pragma unroll
    for (float x : v) {
      const float t = (x - m) * c, e = exp2_hw(t);
      a.s += e;
      a.h += e * fmaxf(t, -FLT_MAX);
    }
  }
  return Soft{m, wave_sum(a.s), wave_sum(a.h)};
}
// By the whole workgroup; `sums`: what the wavefronts have, free for this on entry.
template <typename T>
__device__ Soft extreme_block(const T* row, uint32_t n, float m, float c, Soft* sums) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const Soft own = extreme_sums(row, n, m, c, wave, waves);
  __syncthreads();
  if (lane == 0) sums[wave] = own;
  __syncthreads();
  const Soft a = lane < waves ? sums[lane] : Soft{m, 0.f, 0.f};
  return Soft{m, wave_sum(a.s), wave_sum(a.h)};
}

// The largest number that at least `need` of the lanes' numbers reach, bit by bit from the top; 0 if fewer than that are not 0. With fewer than 32 `bits`
// what is left of it is 0, so that it is a little low: one vector instruction a bit.
__device__ __forceinline__ uint32_t reached_by(uint32_t v, int need, int bits) {
  uint32_t reached = 0;
  for (int b = 31; b >= 32 - bits; --b) {
    const uint32_t t = reached | 1u << b;
    if (__popcll(__ballot(v >= t)) >= need) reached = t;
  }
  return reached;
}
constexpr int kBoundBits = 16;   // of a bound that may be low: sign, exponent, seven bits
__device__ __forceinline__ int lanes_before(uint64_t mask) {
  return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}
// Sum of the lanes' n before this one, bit by bit (few are large); `all`: of all lanes.
__device__ __forceinline__ int count_before(int n, int* all) {
  int before = 0, sum = 0;
  for (int b = 0; __ballot(n >> b); ++b) {
    const uint64_t mask = __ballot(n >> b & 1);
    before += lanes_before(mask) << b;
    sum += __popcll(mask) << b;
  }
  *all = sum;
  return before;
}
// The `top` largest of `count` different keys in order, key k in lane k (0: there are fewer). Up to 64 keys: each goes to the place that the number of
// larger ones names (`place`: room for `top` keys beside the list); more: the largest is taken `top` times.
__device__ __forceinline__ uint64_t in_order(const uint64_t* list, int count, int top, uint64_t* place) {
  const int lane = threadIdx.x & 63;
  uint64_t out = 0;
  if (count <= kWave) {
    const uint64_t key = lane < count ? list[lane] : 0;
    int above = 0;
    for (int k = 0; k < count; ++k) above += readlane(key, k) > key;
    if (lane < count && above < top) place[above] = key;
    wave_sync();
    if (lane < top && lane < count) out = place[lane];
  } else {
    auto largest = [&](uint64_t below) {
      uint64_t best = 0;
      for (int i = lane; i < count; i += kWave) {
        const uint64_t key = list[i];
        if (key < below && key > best) best = key;
      }
      return best;
    };
    uint64_t mine = largest(~(uint64_t)0);
    for (int k = 0; k < top; ++k) {
      const uint64_t best = wave_max(mine);
      if (lane == k) out = best;
      if (mine == best) mine = largest(best);
    }
  }
  wave_sync();
  return out;
}

// The `top` largest keys of a piece in order, whatever its logits. At least `top` lanes' maxima reach a bound, which is found to its last bit: what lies above it
// belongs to fewer than `top` lanes, and of its equals, which may be many (masks, few different values), only the `top` of lowest index are taken. The
// values are read again, so that they take no registers. `list`: room for (E + 2) top keys.
template <typename T, int E>
__device__ __forceinline__ uint64_t exact_top(const T* row, const Piece<T, E>& p, int top, uint64_t* list) {
  typedef Piece<T, E> P;
  uint32_t ord[P::V], most = 0;   // 0: not an element
  auto read = [&](int j) {
    float y[P::V];
    if (p.n >= P::V) p.values(row, j, y);
#pragma unroll
    for (int e = 0; e < P::V; ++e) {
      const int i = j * P::V + e;
      if (p.n < P::V) y[e] = to_f32(row[min(p.index(i), p.n - 1)]);
      ord[e] = p.mine(i) ? full_order(y[e]) : 0;
    }
  };
#pragma unroll 1
  for (int j = 0; j < P::N; ++j) {
    read(j);
#pragma unroll
    for (int e = 0; e < P::V; ++e) most = max(most, ord[e]);
  }
  const uint32_t bound = max(reached_by(most, top, 32), 1u);
  int count = 0, taken = 0;
#pragma unroll 1
  for (int j = 0; j < P::N; ++j) {
    read(j);
#pragma unroll
    for (int e = 0; e < P::V; ++e) {
      const uint64_t mask = __ballot(ord[e] > bound);
      if (ord[e] > bound) list[count + lanes_before(mask)] = rank_key(ord[e], (uint32_t)p.index(j * P::V + e));
      count += __popcll(mask);
    }
  }
#pragma unroll 1
  for (int j = 0; j < P::N && taken < top; ++j) {   // in the order of the indices: packs, lanes, elements
    read(j);
    int pass = 0, all;
#pragma unroll
    for (int e = 0; e < P::V; ++e) pass += ord[e] == bound;
    int at = taken + count_before(pass, &all);
#pragma unroll
    for (int e = 0; e < P::V; ++e)
      if (ord[e] == bound) {
        if (at < top) list[count + at] = rank_key(bound, (uint32_t)p.index(j * P::V + e));
        ++at;
      }
    taken += all;
  }
  count += min(taken, top);
  wave_sync();
  return in_order(list, count, top, list + (E + 1) * top);
}

// The same from its values x, whose largest in the lane is `most`, by way of what reaches a bound that may be a little low; by exact_top where the list
// does not hold that, or masked logits are among it. `special`: there may be a NaN.
template <typename T, int E>
__device__ __forceinline__ uint64_t piece_top(const T* row, const Piece<T, E>& p, const float (&x)[E], float most, int top, bool special, uint64_t* list) {
  const uint32_t reached = reached_by(order_of(most), top, kBoundBits);
  if (!special && reached > order_of(-INFINITY)) {   // no masked logit reaches it, nor one that is not this lane's
    const float bound = key_value((uint64_t)reached << 32);
    int count = 0, at = 0;
#pragma unroll
    for (int i = 0; i < E; ++i) count += __popcll(__ballot(x[i] >= bound));
    if (count <= E * top) {
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const uint64_t mask = __ballot(x[i] >= bound);
        if (mask) {
          if (x[i] >= bound) list[at + lanes_before(mask)] = rank_key(order_of(x[i]), (uint32_t)p.index(i));
          at += __popcll(mask);
        }
      }
      wave_sync();
      return in_order(list, count, top, list + (E + 1) * top);
    }
  }
  return exact_top(row, p, top, list);
}

// The `top` largest of `count` lists of `top` ordered keys each, in order: a bound as in piece_top. `buffer`: room for count top keys. The
// lists are overwritten.
__device__ __forceinline__ uint64_t join_lists(uint64_t* lists, int count, int top, uint64_t* buffer) {
  const int lane = threadIdx.x & 63;
  // where `need` of the lists reach a bound with their `deep`-th key, `top` keys do
  const int deep = min((2 * top + count - 1) / count, top), need = (top + deep - 1) / deep;
  const uint32_t bound = max(reached_by(lane < count ? (uint32_t)(lists[lane * top + deep - 1] >> 32) : 0u, need, 32), 1u);
  int pass = 0, all;
  if (lane < count)
    while (pass < top && (uint32_t)(lists[lane * top + pass] >> 32) >= bound) ++pass;
  const int to = count_before(pass, &all);
  for (int k = 0; k < pass; ++k) buffer[to + k] = lists[lane * top + k];
  wave_sync();
  return in_order(buffer, all, top, lists);
}

// Workspace of one level of segments: the keys, then the sums.
inline size_t level_bytes(int64_t rows, int64_t segments, uint32_t top) {
  return (size_t)rows * (size_t)segments * (top * sizeof(uint64_t) + 3 * sizeof(float)) + 15 & ~(size_t)15;
}

// Rows of one piece of 8, 16 or 32 logits a lane: a wavefront each.
template <typename T, bool TOP, int E>
__global__ __launch_bounds__(kBlock) void k_logprobs_short(const T* __restrict__ x, int64_t ld, const int64_t* __restrict__ targets, int64_t rows, uint32_t vocab, float scale,
                                                           int64_t ignore, int top, Outputs o) {
  extern __shared__ uint64_t lists[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const float c = fminf(scale * kLog2e, FLT_MAX);
  for (int64_t r = (int64_t)blockIdx.x * 4 + wave; r < rows; r += (int64_t)gridDim.x * 4) {
    const T* row = x + r * ld;
    Piece<T, E> p;
    p.load(row, 0, pack_offset(row, vocab), vocab);
    const Target g = load_target(row, targets, r, vocab);
    float v[E];
    p.unpack(v);
    const float most = most_of(v);
    Soft a{-INFINITY, 0.f, 0.f};
    add_piece(a, v, most, c);
    a = wave_join(a, c);
    uint64_t key = 0;
    if (TOP) key = piece_top(row, p, v, most, top, a.s != a.s, lists + wave * (E + 2) * top);
    if (beyond(a.m, c)) a = extreme_sums(row, vocab, a.m, c, 0, 1);
    write_row(o, r, lane, a, c, g, vocab, scale, ignore, top, key);
  }
}

// A workgroup a row, its wavefronts a piece each in turn; the first wavefront joins what they have. Bound by memory and, nearly as much, by vector issue (9.9
// instructions for 64 logits, the power of two among them): 4096x50257 bf16 75 us, 5.5 TB/s with the vector units busy four fifths of the time;
// 12000x32000 bf16 135 us, 5.7; 3000x50257 fp32 101 us, 5.9. One pass with separate segments and a second launch to join them took 94 us.
template <typename T, int E>
__global__ __launch_bounds__(1024) void k_logprobs(const T* __restrict__ x, int64_t ld, const int64_t* __restrict__ targets, int64_t rows, uint32_t vocab, float scale,
                                                   int64_t ignore, Outputs o) {
  typedef Piece<T, E> P;
  __shared__ Soft sums[16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6, step = waves * P::kSize;
  const float c = fminf(scale * kLog2e, FLT_MAX);
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
    const T* row = x + r * ld;
    const int off = pack_offset(row, vocab), end = (int)vocab + off;
    P p;
    p.load(row, wave * P::kSize, off, vocab);   // every wavefront has a piece
    Target g{};
    if (wave == 0) g = load_target(row, targets, r, vocab);
    Soft a{-INFINITY, 0.f, 0.f};
    for (int first = wave * P::kSize; first < end; first += step) {
      float v[E];
      P next;
      if (first + step < end) next.load(row, first + step, off, vocab);
      p.unpack(v);
      add_piece(a, v, most_of(v), c);
      p = next;
    }
    a = wave_join(a, c);
    if (lane == 0) sums[wave] = a;
    __syncthreads();
    a = lane < waves ? sums[lane] : Soft{-INFINITY, 0.f, 0.f};
    const float most = wave_max(a.m);
    if (beyond(most, c)) a = extreme_block(row, vocab, most, c, sums);
    else if (wave == 0) a = wave_join(a, c);
    if (wave == 0) write_row(o, r, lane, a, c, g, vocab, scale, ignore, 0, 0);
    if (r + gridDim.x < rows) __syncthreads();
  }
}

// The `top` largest of `count` >= top different keys in LDS, in order, by one wavefront. `buffer`: room for `count` keys.
__device__ __forceinline__ uint64_t top_of_list(uint64_t* list, int count, int top, uint64_t* buffer) {
  const int lane = threadIdx.x & 63;
  if (count <= kWave) return in_order(list, count, top, buffer);
  uint64_t best = 0;
  for (int i = lane; i < count; i += kWave) best = max(best, list[i]);
  const uint32_t bound = reached_by((uint32_t)(best >> 32), top, kBoundBits);
  int pass = 0, all;
  for (int i = lane; i < count; i += kWave) pass += (uint32_t)(list[i] >> 32) >= bound;
  int at = count_before(pass, &all);
  for (int i = lane; i < count; i += kWave)
    if ((uint32_t)(list[i] >> 32) >= bound) buffer[at++] = list[i];
  wave_sync();
  return in_order(buffer, all, top, list);
}

// The same with alternatives: the workgroup holds the whole row, E logits a lane. Every wavefront's lanes' maxima give a bound that `top` of them
// reach; the largest of the wavefronts' bounds holds for the row. The few logits that reach it are gathered in LDS, and the first wavefront
// puts them in order. Fewer than `top` logits that are not masked: all of them, then the masked ones of lowest index. More than the list holds (few
// different values, masks of a low value): those above the bound, found to its last bit, then of its equals those of lowest index; a wavefront's
// logits are neighbours in the row. What is left, rows with a NaN among it, takes the largest key `top` times from memory. Bound by vector issue and, for one
// row, by one compute unit's: 1x50257 fp32 with 20 alternatives 10.1 us, 256x32000 bf16 with five 8.5, 1024x32000 bf16 with 20 24. One row spread over 13
// workgroups that a second launch joins: 6.3 + 8.7 us, and a launch and a workspace more on the host.
constexpr int kListed = 1024;
template <typename T, int E>
__global__ __launch_bounds__(1024) void k_logprobs_top(const T* __restrict__ x, int64_t ld, const int64_t* __restrict__ targets, int64_t rows, uint32_t vocab, float scale,
                                                       int64_t ignore, int top, Outputs o) {
  typedef Piece<T, E> P;
  __shared__ Soft sums[16];
  __shared__ uint32_t bounds[16];
  __shared__ uint64_t heads[2][16], list[kListed + LOPT_TOP_MAX], buffer[kListed + LOPT_TOP_MAX];
  __shared__ int listed[2], equals[16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const float c = fminf(scale * kLog2e, FLT_MAX);
  auto row_bound = [&] {   // masked logits do not reach it
    const uint32_t b = wave_max(lane < waves ? bounds[lane] : 0u);
    return b > order_of(-FLT_MAX) ? key_value((uint64_t)b << 32) : -FLT_MAX;
  };
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
    const T* row = x + r * ld;
    P p;
    p.load(row, wave * P::kSize, pack_offset(row, vocab), vocab);
    Target g{};
    if (wave == 0) g = load_target(row, targets, r, vocab);
    float v[E];
    p.unpack(v);
    const float most = most_of(v);
    const uint32_t own = reached_by(order_of(most), top, kBoundBits);
    if (lane == 0) bounds[wave] = own;
    if (threadIdx.x < 2) listed[threadIdx.x] = 0;
    Soft a{-INFINITY, 0.f, 0.f};
    add_piece(a, v, most, c);
    a = wave_join(a, c);
    if (lane == 0) sums[wave] = a;
    __syncthreads();
    float bound = row_bound();
    a = wave_join(lane < waves ? sums[lane] : Soft{-INFINITY, 0.f, 0.f}, c);
    const bool special = a.s != a.s;
    // Which logits reach the bound, a bit each: the sign of their distance, shifted in. There are few, and their values are read again.
    constexpr int kWords = E / 32;
    const float least = least_of(bound);
    uint32_t hits[kWords];
    int pass = 0, all, at;
#pragma unroll
    for (int w = 0; w < kWords; ++w) {
      uint32_t below = 0;
#pragma unroll
      for (int i = 0; i < 32; ++i) below = __builtin_amdgcn_alignbit(below, __builtin_bit_cast(uint32_t, v[w * 32 + i] - least), 31);
      hits[w] = ~below;   // logit i of the word is bit 31 - i
      pass += __popc(hits[w]);
    }
    at = count_before(pass, &all);
    if (all) {
      int begin = 0;
      if (lane == 0) begin = atomicAdd(&listed[0], all);
      begin = __builtin_amdgcn_readfirstlane(begin);
      if (begin + all <= kListed) {
        at += begin;
#pragma unroll
        for (int w = 0; w < kWords; ++w)
          while (hits[w]) {
            const int bit = __clz(hits[w]), k = p.index(w * 32 + bit);
            hits[w] &= ~(0x80000000u >> bit);
            list[at++] = rank_key(order_of(to_f32(row[k])), (uint32_t)k);
          }
      }
    }
    __syncthreads();
    int count = listed[0];
    bool found = count <= kListed && !special;
    if (!found && !special) {
      const uint32_t exact = reached_by(order_of(most), top, 32);
      if (lane == 0) bounds[wave] = exact;
      __syncthreads();
      bound = row_bound();
      float y[P::V];
      int above = 0, equal = 0, begin = 0;
      for (int j = 0; j < P::N; ++j) {
        p.values(row, j, y);
#pragma unroll
        for (int e = 0; e < P::V; ++e) {
          above += __popcll(__ballot(y[e] > bound));
          equal += __popcll(__ballot(y[e] == bound));
        }
      }
      if (lane == 0) {
        equals[wave] = equal;
        begin = atomicAdd(&listed[1], above);
      }
      begin = __builtin_amdgcn_readfirstlane(begin);
      if (begin + above <= kListed)
        for (int j = 0; j < P::N; ++j) {
          p.values(row, j, y);
#pragma unroll
          for (int e = 0; e < P::V; ++e) {
            const uint64_t mask = __ballot(y[e] > bound);
            if (y[e] > bound) list[begin + lanes_before(mask)] = rank_key(order_of(y[e]), (uint32_t)p.index(j * P::V + e));
            begin += __popcll(mask);
          }
        }
      __syncthreads();
      count = listed[1];
      found = count <= kListed;
      const int wanted = max(top - count, 0);
      int before = 0, have = 0;   // fewer than wanted where the bound keeps out masked logits
      for (int w = 0; w < waves; ++w) {
        before += w < wave ? equals[w] : 0;
        have += equals[w];
      }
      if (found)
        for (int j = 0; j < P::N && before < wanted; ++j) {   // in the order of the indices: packs, lanes, elements
          p.values(row, j, y);
          pass = 0;
#pragma unroll
          for (int e = 0; e < P::V; ++e) pass += y[e] == bound;
          at = before + count_before(pass, &all);
          before += all;
#pragma unroll
          for (int e = 0; e < P::V; ++e)
            if (y[e] == bound) {
              if (at < wanted) list[count + at] = rank_key(order_of(y[e]), (uint32_t)p.index(j * P::V + e));
              ++at;
            }
        }
      __syncthreads();
      count += min(wanted, have);
    }
    uint64_t key = 0, masked = 0;
    if (found && count < top) {   // at most 31 are not masked: the first 64 have to hold enough that are
      masked = __ballot(lane < vocab && to_f32(row[min(lane, (int)vocab - 1)]) == -INFINITY);
      found = __popcll(masked) >= top - count;
    }
    if (found) {
      if (wave == 0) {
        key = count >= top ? top_of_list(list, count, top, buffer) : in_order(list, count, top, buffer);
        if (lane >= count && lane < top) {
          for (int k = count; k < lane; ++k) masked &= masked - 1;
          key = rank_key(order_of(-INFINITY), __builtin_ctzll(masked));
        }
      }
    } else {
      auto largest = [&](uint64_t below) {
        uint64_t best = 0;
        for (uint32_t i = threadIdx.x; i < vocab; i += 8 * blockDim.x) {
          float y[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) y[j] = to_f32(row[min(i + j * blockDim.x, vocab - 1)]);
#pragma unroll
          for (int j = 0; j < 8; ++j) {   // the last logit may come more than once
            const uint64_t k = rank_key(full_order(y[j]), min(i + j * blockDim.x, vocab - 1));
            if (k < below && k > best) best = k;
          }
        }
        return best;
      };
      uint64_t mine = largest(~(uint64_t)0);
      for (int k = 0; k < top; ++k) {
        const uint64_t own_best = wave_max(mine);
        if (lane == 0) heads[k & 1][wave] = own_best;
        __syncthreads();
        uint64_t best = 0;
        for (int w = 0; w < waves; ++w) best = max(best, heads[k & 1][w]);
        if (lane == k) key = best;
        if (mine == best) mine = largest(best);
      }
    }
    if (beyond(a.m, c)) a = extreme_block(row, vocab, a.m, c, sums);
    if (wave == 0) write_row(o, r, lane, a, c, g, vocab, scale, ignore, top, key);
    if (r + gridDim.x < rows) __syncthreads();
  }
}

// The same for many long rows: as k_logprobs, and every wavefront lists the logits that may be among its `top` largest by their index: those that reach what
// `top` lanes' maxima of its pieces so far do (found again after 1, 2, 4, 8, ... pieces), later on without what only equals it, for `top` others come before
// that. A full list keeps what `top` of its lanes reach; a piece with more of them than the list has room for, with masked logits to take or with a NaN goes
// through exact_top. Bound by vector issue and by the search's dependent steps: 1024x50257 bf16 with 20 alternatives 34 us (20.6 without any), all but
// seven logits of the lowest value 38, 1024x131000 70. The bound found again with every piece that has hits: 36.5; and values read again as they are listed: 37.6.
constexpr int kKept = 128;
template <int E>
__host__ __device__ constexpr int many_scratch(int top) { return (E + 2) * top > 2 * kKept ? (E + 2) * top : 2 * kKept; }   // keys a wavefront
template <typename T, int E>
__global__ __launch_bounds__(512) void k_logprobs_many(const T* __restrict__ x, int64_t ld, const int64_t* __restrict__ targets, int64_t rows, uint32_t vocab, float scale,
                                                       int64_t ignore, int top, Outputs o) {
  typedef Piece<T, E> P;
  __shared__ Soft sums[8];
  __shared__ uint32_t bounds[8], lists[8][kKept];
  __shared__ int listed;
  extern __shared__ uint64_t keys[];   // a wavefront's for exact_top, then the row's list and room to order it
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6, step = waves * P::kSize;
  uint64_t* const scratch = keys + wave * many_scratch<E>(top);
  uint32_t* const kept = lists[wave];
  const float c = fminf(scale * kLog2e, FLT_MAX);
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
    const T* row = x + r * ld;
    const int off = pack_offset(row, vocab), end = (int)vocab + off;
    P p;
    p.load(row, wave * P::kSize, off, vocab);
    Target g{};
    if (wave == 0) g = load_target(row, targets, r, vocab);
    if (threadIdx.x == 0) listed = 0;
    Soft a{-INFINITY, 0.f, 0.f};
    int count = 0;
    uint32_t low = 0;   // order of the least logit that is wanted
    float high = -INFINITY;
    // The list's keys, two a lane, and what `top` lanes' reach.
    uint64_t k0, k1;
    auto kept_keys = [&] {
      auto key = [&](int i) {
        const uint32_t k = i < count ? kept[i] : 0u;
        const float v = to_f32(row[k]);
        return i < count ? rank_key(full_order(v), k) : 0;
      };
      k0 = key(lane), k1 = key(lane + kWave);
      return reached_by((uint32_t)(max(k0, k1) >> 32), top, kBoundBits);
    };
    // Puts those that reach a bound to list + the number of all before them, which the caller's `add` gives.
    auto put = [&](uint32_t bound, uint64_t* list, auto&& add) {
      const bool b0 = k0 && (uint32_t)(k0 >> 32) >= bound, b1 = k1 && (uint32_t)(k1 >> 32) >= bound;
      int all, at = count_before(b0 + b1, &all);
      at += add(all);
      if (b0) list[at++] = k0;
      if (b1) list[at] = k1;
      return all;
    };
    auto filter = [&] {
      const uint32_t bound = kept_keys();
      count = put(bound, scratch, [](int) { return 0; });
      low = max(low, bound + 1);
      wave_sync();
      uint64_t key = lane < count ? scratch[lane] : 0;
      if (count > kWave) {
        key = in_order(scratch, count, top, scratch);
        count = top;
      }
      if (lane < count) kept[lane] = key_index(key);
      wave_sync();
    };
    for (int first = wave * P::kSize, turn = 0; first < end; first += step, ++turn) {
      float v[E];
      P next;
      if (first + step < end) next.load(row, first + step, off, vocab);
      p.unpack(v);
      const float most = most_of(v);
      add_piece(a, v, most, c);
      high = fmaxf(high, most);
      const bool special = __ballot(a.s != a.s) != 0;
      if (special || low == 0 || __ballot(most >= key_value((uint64_t)low << 32))) {
        uint32_t bound = low;
        if ((turn & (turn - 1)) == 0) bound = max(low, reached_by(order_of(high), top, kBoundBits));
        bool whole = special || bound <= order_of(-INFINITY);
        if (!whole) {
          const float least = least_of(key_value((uint64_t)bound << 32));
          uint32_t below = 0;   // a bit each: the sign of the distance, shifted in
#pragma unroll
          for (int i = 0; i < E; ++i) below = __builtin_amdgcn_alignbit(below, __builtin_bit_cast(uint32_t, v[i] - least), 31);
          uint32_t hits = ~below << (32 - E);   // logit i is bit 31 - i
          int more, at = count_before(__popc(hits), &more);
          if (count + more > kKept && count) filter();
          whole = count + more > kKept;
          if (!whole) {
            if (bound > low) low = bound + 1;
            at += count;
            count += more;
            while (hits) {
              const int i = __clz(hits);
              hits &= ~(0x80000000u >> i);
              kept[at++] = (uint32_t)p.index(i);
            }
            wave_sync();
          }
        }
        if (whole) {
          const uint64_t key = exact_top(row, p, top, scratch);
          if (count > kKept - LOPT_TOP_MAX) filter();
          if (key) kept[count + lane] = key_index(key);   // the first lanes'
          wave_sync();
          count += __popcll(__ballot(key != 0));
          const uint64_t last = readlane(key, top - 1);
          if (last) low = max(low, (uint32_t)(last >> 32) + 1);
        }
      }
      p = next;
    }
    a = wave_join(a, c);
    const uint32_t own = kept_keys();
    if (lane == 0) {
      sums[wave] = a;
      bounds[wave] = own;
    }
    __syncthreads();
    put(wave_max(lane < waves ? bounds[lane] : 0u), keys, [&](int all) {
      int begin = 0;
      if (lane == 0) begin = atomicAdd(&listed, all);
      return __builtin_amdgcn_readfirstlane(begin);
    });
    a = lane < waves ? sums[lane] : Soft{-INFINITY, 0.f, 0.f};
    const float most = wave_max(a.m);
    __syncthreads();
    uint64_t key = 0;
    if (wave == 0) key = top_of_list(keys, listed, top, keys + waves * kKept);
    if (beyond(most, c)) a = extreme_block(row, vocab, most, c, sums);
    else if (wave == 0) a = wave_join(a, c);
    if (wave == 0) write_row(o, r, lane, a, c, g, vocab, scale, ignore, top, key);
    if (r + gridDim.x < rows) __syncthreads();
  }
}

// The same where a row is too long for one workgroup: segments of `pieces` pieces, a wavefront each, joined 64 at a time by k_logprobs_join.
// Alternatives: segments of one piece.
template <typename T, bool TOP>
__global__ __launch_bounds__(kBlock) void k_logprobs_split(const T* __restrict__ x, int64_t ld, int64_t rows, uint32_t vocab, float scale, int top, int64_t segments,
                                                           uint32_t pieces, float* __restrict__ part, uint64_t* __restrict__ keys) {
  typedef Piece<T, 32> P;
  extern __shared__ uint64_t lists[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const float c = fminf(scale * kLog2e, FLT_MAX);
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
    const T* row = x + r * ld;
    const int off = pack_offset(row, vocab);
    for (int64_t seg = (int64_t)blockIdx.y * 4 + wave; seg < segments; seg += (int64_t)gridDim.y * 4) {
      const int64_t from = seg * pieces * P::kSize, to = min(from + (int64_t)pieces * P::kSize, (int64_t)vocab + off);
      Soft a{-INFINITY, 0.f, 0.f};
      uint64_t key = 0;
      P p;
      if (from < to) p.load(row, (int)from, off, vocab);
      for (int64_t first = from; first < to; first += P::kSize) {
        float v[32];
        P next;
        if (first + P::kSize < to) next.load(row, (int)first + P::kSize, off, vocab);
        p.unpack(v);
        const float most = most_of(v);
        add_piece(a, v, most, c);
        if (TOP) key = piece_top(row, p, v, most, top, __ballot(a.s != a.s) != 0, lists + wave * 34 * top);
        p = next;
      }
      a = wave_join(a, c);
      const int64_t at = r * segments + seg;
      if (lane < 3) part[3 * at + lane] = lane == 0 ? a.m : lane == 1 ? a.s : a.h;
      if (TOP && lane < top) keys[at * top + lane] = key;
    }
  }
}

// Joins up to 64 neighbouring segments of a row, one wavefront. `last`: all of the row's are here, and its outputs are written; else one
// segment of the next level is.
template <typename T>
__global__ __launch_bounds__(kWave) void k_logprobs_join(const T* __restrict__ x, int64_t ld, const int64_t* __restrict__ targets, int64_t rows, uint32_t vocab, float scale,
                                                         int64_t ignore, int top, Outputs o, int64_t segments, const float* __restrict__ part,
                                                         const uint64_t* __restrict__ keys, float* __restrict__ part_out, uint64_t* __restrict__ keys_out) {
  extern __shared__ uint64_t lists[];
  const int lane = threadIdx.x;
  const float c = fminf(scale * kLog2e, FLT_MAX);
  const int64_t groups = (segments + kWave - 1) / kWave;
  const bool last = groups == 1;
  for (int64_t unit = blockIdx.x; unit < rows * groups; unit += gridDim.x) {
    const int64_t r = unit / groups, group = unit - r * groups, at = r * segments + group * kWave;
    const int count = (int)min(segments - group * kWave, (int64_t)kWave);
    Soft a{-INFINITY, 0.f, 0.f};
    if (lane < count) a = Soft{part[3 * (at + lane)], part[3 * (at + lane) + 1], part[3 * (at + lane) + 2]};
    for (int i = lane; i < count * top; i += kWave) lists[i] = keys[at * top + i];
    Target g{};
    if (last) g = load_target(x + r * ld, targets, r, vocab);
    uint64_t key = 0;
    if (top) {
      wave_sync();
      key = join_lists(lists, count, top, lists + kWave * top);
    }
    a = wave_join(a, c);
    if (last) {
      if (beyond(a.m, c)) a = extreme_sums(x + r * ld, vocab, a.m, c, 0, 1);
      write_row(o, r, lane, a, c, g, vocab, scale, ignore, top, key);
    } else {
      if (lane < 3) part_out[3 * unit + lane] = lane == 0 ? a.m : lane == 1 ? a.s : a.h;
      if (lane < top) keys_out[unit * top + lane] = key;
    }
  }
}

// Calls f(number of logits a lane, as an integral constant).
template <typename F>
inline void with_lane(int lane, F&& f) {
  if (lane == 8) f(std::integral_constant<int, 8>{});
  else if (lane == 16) f(std::integral_constant<int, 16>{});
  else if (lane == 32) f(std::integral_constant<int, 32>{});
  else f(std::integral_constant<int, 64>{});
}

// How rows are shared out. `lane`: logits a lane.
enum RowForm { kRowWave, kRowBlock, kRowMany, kRowSplit };
struct RowPlan {
  RowForm form;
  int lane, waves;
  int64_t pieces, segments;   // kRowSplit
};
inline RowPlan plan_rows(int64_t rows, int64_t vocab, uint32_t top) {
  const int64_t n = vocab + 7;   // a row counted from its pack
  if (n <= 2048) return RowPlan{kRowWave, n <= 512 ? 8 : n <= 1024 ? 16 : 32, 4, 0, 0};
  if (top) {
    // Fewer logits a lane are done sooner by a row alone, more cost less where rows queue for the units. us with 16 / 32 / 64 logits a lane: 1x3000 bf16
    // 4.3 / 4.4 / 5.0, 256x8000 6.9 / 7.3 / 7.8, 1024x8000 13.1 / 10.4 / 10.0, 1x16000 8.0 / 6.5 / 6.5, 256x16000 9.1 / 7.3 / 8.5, 1024x16000 25 / 16.3 / 14.1
    // (fp32 26 / 20.6 / 17.3), 1x32000 - / 8.6 / 7.7, 256x32000 - / 9.2 / 8.3 (fp32 - / 10.7 / 10.6), 1024x32000 - / 29 / 24 (fp32 - / 37 / 30).
    const int lane = n <= 8 * 1024 || (n <= 16 * 1024 && rows <= 256) ? 32 : 64;
    // Many long rows, eight wavefronts a row down to one, as many as make 4096 in all. us of it and of the other two: 256x32000 bf16 11 / 8.6, 300x33000 16.7 /
    // 16.0, 512x50257 22 / 26, 1024x50257 34 / 48 (fp32 40 / 56), 8192x50257 184 / 323, 1024x32000 26 / 24, 2048x32000 40 / 44, 2048x16000 25 / 23; 64x131000
    // 23 / 14, 128x70000 fp32 20 / 25, 128x131000 28 / 31, 1024x131000 70 / 153. 1024x50257 with 8 / 4 / 2: 39 / 34 / 40.
    if (n > 32 * 1024 ? rows > (n > 64 * 1024 ? 127 : 256) : n > 16 * 1024 && rows >= 2048)
      return RowPlan{kRowMany, 16, (int)std::clamp<int64_t>(4096 / rows, 1, 8), 0, 0};
    if (n <= 64 * 1024) return RowPlan{kRowBlock, lane, (int)((n + lane * kWave - 1) / (lane * kWave)), 0, 0};
    return RowPlan{kRowSplit, 32, 4, 1, (n + 2047) / 2048};
  }
  if (n <= 64 * 2048 || rows >= 256) {
    // Wavefronts: one for about five pieces up to four, eight for many rows of 32 pieces and more, whose wavefronts' accesses then lie closer together, and with
    // fewer than 1024 rows as many as make 4096 in all, 16 a compute unit. us with 1 / 2 / 4 / 8: 20000x5000 bf16 43 / 44 / 54, 16384x8191 56 / 55 / 62 / 89,
    // 8192x10007 37 / 36 / 37, 8192x16000 - / 54 / 52 / 58, 12000x32000 - / - / 135 / 135, 4096x50257 - / 88 / 77 / 75 (fp32 3000 rows 104 / 101), 2048x131000 - / - / 102 /
    // 96, 1024x50257 - / 29 / 23 / 25. With pieces of 8 logits a lane: 20000x5000 46, 16384x8191 58, 4096x50257 84, 256x8000 3.9 (3.5); of 32: 16384x8191 66.
    const int64_t pieces = (vocab + 1023) / 1024, long_rows = pieces >= 32 && rows >= 2048 ? 8 : std::clamp<int64_t>((pieces + 4) / 5, 1, 4);
    return RowPlan{kRowBlock, 16, (int)std::max(long_rows, std::min<int64_t>({16, pieces, 4096 / rows})), 0, 0};
  }
  const int64_t pieces = (n + 2047) / 2048, per = std::clamp<int64_t>(rows * pieces / 16384, 1, 8);
  return RowPlan{kRowSplit, 32, 4, per, (pieces + per - 1) / per};
}

// The gradient, element by element. With A = scale (g + h entropy), B = scale h:
//   dx = scale g [target] - p (A + B ln p),   ln p = scale (x - m) - ln S
// Bound by memory: one read and one write of the logits. Groups of G lanes, 16 or 64 for short rows and the workgroup for others (65536x100 fp32 68 -> 16
// us, 16384x1000 bf16 22 -> 15), take kBackPacks packs of 16 bytes a lane of a row, counted as in the forward pass from the pack in which the
// gradient's row begins, so that stores are aligned (4096x50257 bf16, odd rows at odd elements: 184 -> 174 us); a logit's row at
// another offset is read unaligned. Packs that reach out of the row go element by element. Accesses are nontemporal: nothing is read again here, and
// what both arrays would push out of the caches is (4096x50257 bf16 181 -> 172 us). Spans of a row are neighbours in the grid, so that what is in flight lies together:
// 4096x50257 bf16 172 -> 146 us, fp32 334 -> 284, 4096x32000 100 -> 87. Which span comes first turns every 64 rows, for a short last one would meet
// the same XCDs and units in every row (8000x10007 69 us with the rows as neighbours, 79 with the spans, 62 turned; 74 turned every eight rows). us of
// 4096x50257 bf16 with 2, 4, 8 packs: 159, 148, 158.
constexpr int kBackPacks = 4;
template <typename T, bool ENTROPY, int G>
__global__ __launch_bounds__(kBlock) void k_logprobs_back(const T* x, int64_t ld, const int64_t* __restrict__ targets, const float* __restrict__ stats,
                                                          const float* __restrict__ entropy, const float* __restrict__ dlogp,
                                                          const float* __restrict__ dentropy, T* dx, int64_t ld_d, int64_t rows, int vocab, float scale, int64_t ignore) {
  typedef typename Pack<T>::type pack;
  constexpr int V = Pack<T>::n, kSpan = kBackPacks * G * V, kRows = kBlock / G;
  const int lane = threadIdx.x % G;
  for (int64_t r = (int64_t)blockIdx.y * kRows + threadIdx.x / G; r < rows; r += (int64_t)gridDim.y * kRows) {
    const T* row = x + r * ld;
    T* out = dx + r * ld_d;
    const float m = stats[2 * r], log_s = stats[2 * r + 1];
    const int64_t t = dlogp ? targets[r] : ignore;
    float g = t == ignore ? 0.f : dlogp[r];
    if (t != ignore && (t < 0 || t >= vocab)) g = NAN;
    const float h = ENTROPY ? dentropy[r] : 0.f;
    const float at_target = scale * g, A = scale * (g + (ENTROPY ? h * entropy[r] : 0.f)), B = scale * h;
    const bool empty = log_s == -INFINITY;
    const int at = t != ignore && t >= 0 && t < vocab ? (int)t : -1;
    auto gradient = [&](float v) {
      float lp = scale * (v - m) - log_s;
      const float p = exp2_hw(lp * kLog2e);
      if (ENTROPY) lp = fmaxf(lp, -1e4f);   // p is 0 there
      const float d = -p * (ENTROPY ? A + B * lp : A);
      return empty ? 0.f * A : d;
    };
    const int off = (int)((uintptr_t)out / sizeof(T) % V);
    for (int64_t first = (int64_t)((blockIdx.x + blockIdx.y / 64) % gridDim.x) * kSpan; first < (int64_t)vocab + off; first += (int64_t)gridDim.x * kSpan) {
      const int begin = (int)first + lane * V - off;
      pack in[kBackPacks];
#pragma unroll
      for (int j = 0; j < kBackPacks; ++j) {
        const int k = begin + j * G * V;
        if (k >= 0 && k <= vocab - V) in[j] = __builtin_nontemporal_load((const pack*)(row + k));
      }
#pragma unroll
      for (int j = 0; j < kBackPacks; ++j) {
        const int k = begin + j * G * V;
        if (k >= 0 && k <= vocab - V) {
          float d[V];
#pragma unroll
          for (int e = 0; e < V; ++e) d[e] = gradient(to_f32(in[j][e]));
          if ((unsigned)(at - k) < (unsigned)V) {
#pragma unroll
            for (int e = 0; e < V; ++e)
              if (at == k + e) d[e] += empty ? 0.f : at_target;
          }
          pack o;
#pragma unroll
          for (int e = 0; e < V; ++e) o[e] = from_f32<T>(d[e]);
          __builtin_nontemporal_store(o, (pack*)(out + k));
        } else if (k > -V && k < vocab) {
          for (int i = max(k, 0); i < min(k + V, vocab); ++i) {
            const float d = gradient(to_f32(row[i]));
            out[i] = from_f32<T>(at == i && !empty ? d + at_target : d);
          }
        }
      }
    }
  }
}

}  // namespace
}  // namespace lopt

using namespace lopt;

extern "C" {

size_t lopt_token_logprobs_workspace(int64_t rows, int64_t vocab, uint32_t top) {
  if (rows <= 0 || vocab <= 0 || rows > 0x7fffffffLL || vocab > 0x7fffffffLL || top > LOPT_TOP_MAX) return 0;
  const RowPlan plan = plan_rows(rows, vocab, top);
  size_t bytes = 0;
  if (plan.form == kRowSplit)
    for (int64_t segments = plan.segments; segments > 1; segments = (segments + kWave - 1) / kWave) bytes += level_bytes(rows, segments, top);
  return bytes;
}

static lopt_status check_logits(const void* logits, int64_t ld, int64_t rows, int64_t vocab, uint32_t type, float scale) {
  LOPT_CHECK(check_type("type", type));
  LOPT_CHECK(check_matrix(rows, vocab, "vocab"));
  if (vocab > LOPT_VOCAB_MAX) return fail_call(LOPT_ESHAPE, "vocab=%lld is above %d", (long long)vocab, LOPT_VOCAB_MAX);
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
  const Outputs o{logp, entropy, stats, top_logp, top_index};
  const RowPlan plan = plan_rows(rows, vocab, top);
  const int64_t* tg = logp ? targets : nullptr;
  hipStream_t stream = (hipStream_t)hip_stream;
  const unsigned blocks = (unsigned)std::min<int64_t>(plan.form == kRowWave ? (rows + 3) / 4 : rows, 1 << 20);
  const uint32_t n = (uint32_t)vocab;
  with_type(type, [&](auto t) {
    using T = decltype(t);
    const T* x = (const T*)logits;
    if (plan.form != kRowSplit) {
      with_lane(plan.lane, [&](auto e) {
        constexpr int E = decltype(e)::value;
        const dim3 block(plan.waves * kWave);
        if constexpr (E <= 32)
          if (plan.form == kRowWave) {
            auto kernel = top ? k_logprobs_short<T, true, E> : k_logprobs_short<T, false, E>;
            hipLaunchKernelGGL(kernel, dim3(blocks), block, plan.waves * (E + 2) * top * sizeof(uint64_t), stream, x, ld, tg, rows, n, scale, ignore_index, (int)top, o);
            return;
          }
        if constexpr (E == 16)
          if (plan.form == kRowMany) {
            const size_t lds = plan.waves * many_scratch<E>((int)top) * sizeof(uint64_t);
            hipLaunchKernelGGL((k_logprobs_many<T, E>), dim3(blocks), block, lds, stream, x, ld, tg, rows, n, scale, ignore_index, (int)top, o);
            return;
          }
        if constexpr (E >= 32)
          if (top) {
            hipLaunchKernelGGL((k_logprobs_top<T, E>), dim3(blocks), block, 0, stream, x, ld, tg, rows, n, scale, ignore_index, (int)top, o);
            return;
          }
        if constexpr (E == 16) hipLaunchKernelGGL((k_logprobs<T, E>), dim3(blocks), block, 0, stream, x, ld, tg, rows, n, scale, ignore_index, o);
      });
      return;
    }
    char* ws = (char*)workspace;
    uint64_t* keys = (uint64_t*)ws;
    float* part = (float*)(ws + (size_t)rows * plan.segments * top * sizeof(uint64_t));
    const dim3 grid(blocks, (unsigned)std::min<int64_t>((plan.segments + 3) / 4, 1024));
    if (top)
      hipLaunchKernelGGL((k_logprobs_split<T, true>), grid, dim3(kBlock), 4 * 34 * top * sizeof(uint64_t), stream, x, ld, rows, n, scale, (int)top, plan.segments,
                         (uint32_t)plan.pieces, part, keys);
    else
      hipLaunchKernelGGL((k_logprobs_split<T, false>), grid, dim3(kBlock), 0, stream, x, ld, rows, n, scale, 0, plan.segments, (uint32_t)plan.pieces, part,
                         keys);
    for (int64_t segments = plan.segments; segments > 1;) {
      const int64_t groups = (segments + kWave - 1) / kWave;
      char* above = (char*)keys + level_bytes(rows, segments, top);
      uint64_t* keys_out = (uint64_t*)above;
      float* part_out = (float*)(above + (size_t)rows * groups * top * sizeof(uint64_t));
      hipLaunchKernelGGL(k_logprobs_join<T>, dim3((unsigned)std::min<int64_t>(rows * groups, 1 << 22)), dim3(kWave),
                         2 * kWave * top * sizeof(uint64_t), stream, x, ld, tg, rows, n, scale, ignore_index, (int)top, o,
                         segments, (const float*)part, (const uint64_t*)keys, part_out, keys_out);
      keys = keys_out;
      part = part_out;
      segments = groups;
    }
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
    const int64_t packs = (vocab + 2 * Pack<T>::n - 2) / Pack<T>::n;   // that a row may touch
    auto launch = [&](auto g) {
      constexpr int G = decltype(g)::value;
      // a rest of less than an eighth of a span goes to workgroups that have one (16384x8191 bf16 108 -> 96 us; rests of a quarter 18 -> 21)
      const int64_t spans = (packs + kBackPacks * G - kBackPacks * G / 8) / (kBackPacks * G);
      const dim3 grid((unsigned)std::clamp<int64_t>(spans, 1, 1024), (unsigned)std::min<int64_t>((rows + kBlock / G - 1) / (kBlock / G), 65535));
      auto kernel = dentropy ? k_logprobs_back<T, true, G> : k_logprobs_back<T, false, G>;
      hipLaunchKernelGGL(kernel, grid, dim3(kBlock), 0, (hipStream_t)hip_stream, (const T*)logits, ld, targets, stats, entropy, dlogp, dentropy, (T*)dlogits, ld_d,
                         rows, (int)vocab, scale, ignore_index);
    };
    if (packs <= kBackPacks * 16) launch(std::integral_constant<int, 16>{});
    else if (packs <= kBackPacks * 64) launch(std::integral_constant<int, 64>{});
    else launch(std::integral_constant<int, kBlock>{});
  });
  return launch_status("lopt_token_logprobs_backward");
}

}  // extern "C"
