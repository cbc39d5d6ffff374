// Log probabilities of given tokens with entropy and top alternatives, and their gradient.
#include <algorithm>
#include <cfloat>
#include <cmath>

#include "lopt_ops.h"

namespace lopt {
namespace {

// The order of the alternatives as one number: larger logit first, NaN above all, +0 and -0 alike, lower index first among equals.
// No element's number is 0 or all ones.
__device__ __forceinline__ uint32_t order_of(float x) {   // NaN: see piece_top
  const uint32_t u = __builtin_bit_cast(uint32_t, x + 0.f);
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ uint64_t rank_key(uint32_t order, uint32_t index) { return (uint64_t)order << 32 | (0xffffffffu - index); }
__device__ __forceinline__ uint32_t key_index(uint64_t key) { return 0xffffffffu - (uint32_t)key; }
__device__ __forceinline__ float key_value(uint64_t key) {
  const uint32_t u = (uint32_t)(key >> 32);
  return __builtin_bit_cast(float, u & 0x80000000u ? u ^ 0x80000000u : ~u);
}

// Running softmax sums of some logits x: base = the largest of them (-FLT_MAX where all are -infinity), s = sum e^(c (x - base)),
// h = sum e^(c (x - base)) (x - base). c = scale / ln 2 goes into the hardware's 2^x; x - base is formed before it is scaled, so that large
// logits lose nothing and a scale never makes a finite difference infinite twice. A masked logit has x - base = -infinity and
// e = 0; its term of h is 0 because the difference is held to -FLT_MAX.
struct Soft { float base, s, h; };
constexpr float kLog2e = 1.44269504088896341f;

__device__ __forceinline__ float exp2_hw(float v) { return __builtin_amdgcn_exp2f(v); }

// a's sums seen from a larger base.
__device__ __forceinline__ Soft rebase(Soft a, float base, float c) {
  const float diff = fmaxf(a.base - base, -FLT_MAX);
  const float f = exp2_hw((a.base - base) * c), fs = f * a.s;   // NaN where both are +infinity
  return Soft{base, fs, f * a.h + fs * diff};
}
__device__ __forceinline__ Soft wave_join(Soft a, float c) {
  a = rebase(a, wave_max(a.base), c);
  return Soft{a.base, wave_sum(a.s), wave_sum(a.h)};
}

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

// A row's outputs from its sums. Lane k of the wavefront holds the key of alternative k.
__device__ __forceinline__ void write_row(const Outputs& o, int64_t r, int lane, Soft a, Target g, int vocab, float scale, int64_t ignore, int top, uint64_t key) {
  const bool empty = a.s == 0.f;
  const float log_s = logf(a.s);
  if (lane == 0) {
    if (o.logp) {
      float v = NAN;
      if (g.t == ignore) v = 0.f;
      else if (g.t >= 0 && g.t < vocab) v = empty ? -INFINITY : scale * (g.x - a.base) - log_s;
      o.logp[r] = v;
    }
    if (o.entropy) o.entropy[r] = empty ? 0.f : log_s - scale * (a.h / a.s);
    o.stats[2 * r] = empty ? -INFINITY : a.base;
    o.stats[2 * r + 1] = log_s;
  }
  if (lane < top) {
    o.top_index[r * top + lane] = key_index(key);
    o.top_logp[r * top + lane] = empty ? -INFINITY : scale * (key_value(key) - a.base) - log_s;
  }
}

// A wavefront takes a piece of a row at a time, E = 16 or 32 logits a lane in accesses of 16 bytes. The access that would pass the row's end
// is moved back to end with it, and the elements that the lane before has are masked.
template <typename T, int E>
struct Piece {
  static constexpr int V = Pack<T>::n, N = E / V, kSize = E * kWave;
  typedef typename Pack<T>::type pack;
  pack raw[N];
  __device__ __forceinline__ static uint32_t place(uint32_t first, int j) { return first + (j * kWave + (threadIdx.x & 63)) * V; }
  __device__ __forceinline__ void load(const T* row, uint32_t first, uint32_t n) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      if (first + j * kWave * V >= n) break;
      const uint32_t at = place(first, j);
      if (n >= (uint32_t)V) {
        raw[j] = *(const pack*)(row + min(at, n - V));
      } else {
#pragma unroll
        for (int e = 0; e < V; ++e) raw[j][e] = at + e < n ? row[at + e] : (T)-INFINITY;
      }
    }
  }
  // Index of an element, and whether it is this lane's.
  __device__ __forceinline__ static uint32_t index(uint32_t first, int i, uint32_t n) {
    const uint32_t at = place(first, i / V);
    return (n >= (uint32_t)V ? min(at, n - V) : at) + i % V;
  }
  __device__ __forceinline__ static bool mine(uint32_t first, int i, uint32_t n) {
    const uint32_t k = index(first, i, n);
    return k >= place(first, i / V) && k < n;
  }
  __device__ __forceinline__ void unpack(float (&x)[E], uint32_t first, uint32_t n) const {
    if (first + kSize <= n) {
#pragma unroll
      for (int i = 0; i < E; ++i) x[i] = to_f32(raw[i / V][i % V]);
      return;
    }
#pragma unroll
    for (int i = 0; i < E; ++i) {
      x[i] = -INFINITY;
      if (first + i / V * kWave * V < n && mine(first, i, n)) x[i] = to_f32(raw[i / V][i % V]);
    }
  }
};

template <int E>
__device__ __forceinline__ void add_piece(Soft& a, const float (&x)[E], float c, bool first) {
  float base = a.base;
#pragma unroll
  for (int i = 0; i < E; ++i) base = fmaxf(base, x[i]);
  if (first) a.base = base;
  else a = rebase(a, base, c);
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const float d = x[i] - base, e = exp2_hw(d * c);
    a.s += e;
    a.h += e * fmaxf(d, -FLT_MAX);
  }
}

// The largest number that at least `need` of the lanes' numbers reach; 0 if fewer than that are not 0.
__device__ __forceinline__ uint32_t reached_by(uint32_t v, int need) {
  int reach = 0;
#pragma unroll
  for (int l = 0; l < kWave; ++l) reach += (uint32_t)__builtin_amdgcn_readlane((int)v, l) >= v;
  return wave_max(reach >= need ? v : 0u);
}
// Sum of the lanes' n (at most 63) before this one; `all`: of all lanes.
__device__ __forceinline__ int count_before(int n, int* all) {
  int before = 0, sum = 0;
#pragma unroll
  for (int b = 0; b < 6; ++b) {
    const uint64_t mask = __ballot(n >> b & 1);
    before += (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0)) << b;
    sum += __popcll(mask) << b;
  }
  *all = sum;
  return before;
}
// The `top` largest of `count` different keys in order, key k in lane k (0: there are fewer): each goes to the place that the number of larger ones
// names. `place`: room for `top` keys beside the list.
__device__ __forceinline__ uint64_t in_order(const uint64_t* list, int count, int top, uint64_t* place) {
  const int lane = threadIdx.x & 63;
  if (count <= kWave) {
    const uint64_t key = lane < count ? list[lane] : 0;
    int above = 0;
    for (int k = 0; k < count; ++k) above += readlane(key, k) > key;
    if (lane < count && above < top) place[above] = key;
  } else {
    for (int c = lane; c < count; c += kWave) {
      const uint64_t key = list[c];
      int above = 0;
      for (int k = 0; k < count; ++k) above += list[k] > key;
      if (above < top) place[above] = key;
    }
  }
  wave_sync();
  const uint64_t out = lane < top && lane < count ? place[lane] : 0;
  wave_sync();
  return out;
}

// The `top` largest keys of a piece in order; `most` is the largest of the lane's logits (-FLT_MAX if all are masked). At least `top`
// lanes' maxima reach `bound`, so nothing below it counts, and what lies above it belongs to fewer than `top` lanes. What equals it may be many
// (masks, few different values): where the list does not hold them all, only the `top` of lowest index are taken.
// `list`: room for (E + 2) top keys. `special`: there may be a NaN.
template <typename T, int E>
__device__ __forceinline__ uint64_t piece_top(const float (&x)[E], float most, uint32_t first, uint32_t n, int top, bool special, uint64_t* list) {
  typedef Piece<T, E> P;
  const int room = E * top;
  int pass = 0, count, at;
  if (!special) {
    const float bound = key_value((uint64_t)reached_by(order_of(most), top) << 32);
#pragma unroll
    for (int i = 0; i < E; ++i) pass += x[i] >= bound;
    at = count_before(pass, &count);
    if (count <= room && bound > -FLT_MAX) {   // no masked logit among them, nor one that is not this lane's
#pragma unroll
      for (int i = 0; i < E; ++i)
        if (x[i] >= bound) list[at++] = rank_key(order_of(x[i]), P::index(first, i, n));
      wave_sync();
      return in_order(list, count, top, list + (E + 1) * top);
    }
  }
  uint32_t ord[E], hi = 0;   // 0: not an element
#pragma unroll
  for (int i = 0; i < E; ++i) {
    ord[i] = x[i] != x[i] ? 0xfffffffeu : order_of(x[i]);
    ord[i] = P::mine(first, i, n) ? ord[i] : 0;
    hi = max(hi, ord[i]);
  }
  const uint32_t bound = max(reached_by(hi, top), 1u);
  pass = 0;
#pragma unroll
  for (int i = 0; i < E; ++i) pass += ord[i] > bound;
  at = count_before(pass, &count);
#pragma unroll
  for (int i = 0; i < E; ++i)
    if (ord[i] > bound) list[at++] = rank_key(ord[i], P::index(first, i, n));
  int taken = 0;
#pragma unroll
  for (int j = 0; j < P::N; ++j) {   // in the order of the indices: packs, lanes, elements
    pass = 0;
#pragma unroll
    for (int i = j * P::V; i < (j + 1) * P::V; ++i) pass += ord[i] == bound;
    int all;
    at = taken + count_before(pass, &all);
#pragma unroll
    for (int i = j * P::V; i < (j + 1) * P::V; ++i)
      if (ord[i] == bound) {
        if (at < top) list[count + at] = rank_key(ord[i], P::index(first, i, n));
        ++at;
      }
    taken += all;
  }
  count += min(taken, top);
  wave_sync();
  return in_order(list, count, top, list + (E + 1) * top);
}

// How a row is shared out: `segments` of `pieces` pieces, a wavefront each; a row of one segment is finished by that wavefront, more are
// joined 64 at a time by k_logprobs_join. Alternatives are found piece by piece.
struct RowPlan {
  int lane_elements;   // 16 or 32
  int64_t pieces, segments;
};
constexpr int64_t kFewPieces = 1024;
inline RowPlan plan_rows(int64_t rows, int64_t vocab, uint32_t top) {
  const int64_t all = (vocab + 2047) / 2048;
  if (top) {
    // few rows: pieces of half the size, as long as one join takes them all
    if (rows * all <= kFewPieces && all <= kWave / 2) return RowPlan{16, 1, (vocab + 1023) / 1024};
    return RowPlan{32, 1, all};
  }
  int64_t per = rows * all / 16384;
  per = per < 1 ? 1 : per > 8 ? 8 : per;
  int64_t segments = (all + per - 1) / per;
  if (segments > 1) segments = std::min((segments + 3) / 4 * 4, all);   // four a workgroup
  return RowPlan{32, (all + segments - 1) / segments, segments};
}

// Workspace of one level of segments: the keys, then the sums.
inline size_t level_bytes(int64_t rows, int64_t segments, uint32_t top) {
  return (size_t)rows * (size_t)segments * (top * sizeof(uint64_t) + 3 * sizeof(float)) + 15 & ~(size_t)15;
}

// One wavefront a segment: a workgroup takes four rows where they have one segment, else four segments of a row.
template <typename T, bool TOP, int E>
__global__ __launch_bounds__(kBlock) void k_logprobs(const T* __restrict__ x, int64_t ld, const int64_t* __restrict__ targets, int64_t rows, uint32_t vocab, float scale,
                                                     int64_t ignore, int top, Outputs o, int64_t segments, uint32_t pieces, float* __restrict__ part,
                                                     uint64_t* __restrict__ keys) {
  typedef Piece<T, E> P;
  extern __shared__ uint64_t lists[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const float c = fminf(scale * kLog2e, FLT_MAX);
  const bool whole = segments == 1;
  for (int64_t b = blockIdx.x;; b += gridDim.x) {
    const int64_t r = whole ? b * 4 + wave : b;
    if (r >= rows) break;
    const T* row = x + r * ld;
    for (int64_t seg = whole ? 0 : (int64_t)blockIdx.y * 4 + wave; seg < segments; seg += (int64_t)gridDim.y * 4) {
      const uint32_t first = (uint32_t)(seg * pieces) * (uint32_t)P::kSize;
      const uint32_t end = min((uint64_t)first + (uint64_t)pieces * P::kSize, (uint64_t)vocab);
      Soft a{-FLT_MAX, 0.f, 0.f};
      P p;
      p.load(row, first, vocab);
      Target g{};
      if (whole) g = load_target(row, targets, r, vocab);
      uint64_t key = 0;
      float v[E];
      if (TOP) {
        p.unpack(v, first, vocab);
        add_piece(a, v, c, true);
        const float most = a.base;
        a = wave_join(a, c);
        key = piece_top<T, E>(v, most, first, vocab, top, a.s != a.s, lists + wave * (E + 2) * top);
      } else {
        for (uint32_t f = first; f < end; f += P::kSize) {
          P next;
          if (f + P::kSize < end) next.load(row, f + P::kSize, vocab);
          p.unpack(v, f, vocab);
          add_piece(a, v, c, f == first);
          p = next;
        }
        a = wave_join(a, c);
      }
      if (whole) {
        write_row(o, r, lane, a, g, vocab, scale, ignore, top, key);
      } else {
        const int64_t at = r * segments + seg;
        if (lane < 3) part[3 * at + lane] = lane == 0 ? a.base : lane == 1 ? a.s : a.h;
        if (TOP && lane < top) keys[at * top + lane] = key;
      }
    }
  }
}

// Joins up to 64 neighbouring segments of a row, one wavefront: the sums lane by lane, the ordered lists of alternatives by a bound
// as in piece_top. `last`: all of the row's are here, and its outputs are written; else one segment of the next level is.
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
    Target g{};
    if (last && !top) g = load_target(x + r * ld, targets, r, vocab);
    Soft a{-FLT_MAX, 0.f, 0.f};
    if (lane < count) a = Soft{part[3 * (at + lane)], part[3 * (at + lane) + 1], part[3 * (at + lane) + 2]};
    uint64_t key = 0;
    if (top) {
      uint64_t* list = lists + kWave * top;
      for (int i = lane; i < count * top; i += kWave) lists[i] = keys[at * top + i];
      if (last) g = load_target(x + r * ld, targets, r, vocab);   // its two loads in a row run beside what follows
      wave_sync();
      // the lists are in order: where `need` of them reach a bound with their `deep`-th key, `top` keys do
      const int deep = min((2 * top + count - 1) / count, top), need = (top + deep - 1) / deep;
      const uint64_t bound = reached_by(lane < count ? (uint32_t)(lists[lane * top + deep - 1] >> 32) : 0u, need);
      int pass = 0, all;
      if (lane < count)
        while (pass < top && lists[lane * top + pass] >> 32 >= max(bound, (uint64_t)1)) ++pass;
      int to = count_before(pass, &all);
      for (int k = 0; k < pass; ++k) list[to + k] = lists[lane * top + k];
      wave_sync();
      key = in_order(list, all, top, lists);
    }
    a = wave_join(a, c);
    if (last) {
      write_row(o, r, lane, a, g, vocab, scale, ignore, top, key);
    } else {
      if (lane < 3) part_out[3 * unit + lane] = lane == 0 ? a.base : lane == 1 ? a.s : a.h;
      if (lane < top) keys_out[unit * top + lane] = key;
    }
  }
}

// The gradient, element by element: a workgroup takes kBackPacks packs of 16 bytes a thread of one row. With A = scale (g + h entropy), B = scale h:
//   dx = scale g [target] - p (A + B ln p)
// where ln p = scale (x - m) - ln S. Elements behind the last whole pack of a row go one a thread.
constexpr int kBackPacks = 4;
template <typename T, bool ENTROPY>
__global__ __launch_bounds__(kBlock) void k_logprobs_back(const T* x, int64_t ld, const int64_t* __restrict__ targets, const float* __restrict__ stats,
                                                          const float* __restrict__ entropy, const float* __restrict__ dlogp,
                                                          const float* __restrict__ dentropy, T* dx, int64_t ld_d, int64_t rows, uint32_t vocab, float scale, int64_t ignore) {
  typedef typename Pack<T>::type pack;
  constexpr int V = Pack<T>::n;
  constexpr uint32_t kSpan = kBackPacks * kBlock * V;
  const uint32_t whole = vocab / V * V;
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
    const T* row = x + r * ld;
    T* out = dx + r * ld_d;
    const float m = stats[2 * r], log_s = stats[2 * r + 1];
    const int64_t t = dlogp ? targets[r] : ignore;
    float g = t == ignore ? 0.f : dlogp[r];
    if (t != ignore && (t < 0 || t >= vocab)) g = NAN;
    const float h = ENTROPY ? dentropy[r] : 0.f;
    const float at_target = scale * g, A = scale * (g + (ENTROPY ? h * entropy[r] : 0.f)), B = scale * h;
    const bool empty = log_s == -INFINITY;
    const uint32_t at = t >= 0 && t < vocab ? (uint32_t)t : 0xffffffffu;
    auto gradient = [&](float v) {
      float lp = scale * (v - m) - log_s;
      const float p = exp2_hw(lp * kLog2e);
      if (ENTROPY) lp = fmaxf(lp, -1e4f);   // p is 0 there
      const float d = -p * (ENTROPY ? A + B * lp : A);
      return empty ? 0.f * A : d;
    };
    for (uint32_t first = blockIdx.y * kSpan; first < vocab; first += gridDim.y * kSpan) {
      pack in[kBackPacks];
#pragma unroll
      for (int j = 0; j < kBackPacks; ++j) {
        const uint32_t k = first + (j * kBlock + threadIdx.x) * V;
        if (k < whole) in[j] = *(const pack*)(row + k);
      }
#pragma unroll
      for (int j = 0; j < kBackPacks; ++j) {
        const uint32_t k = first + (j * kBlock + threadIdx.x) * V;
        if (k < whole) {
          float d[V];
#pragma unroll
          for (int e = 0; e < V; ++e) d[e] = gradient(to_f32(in[j][e]));
          if (at - k < (uint32_t)V) {
#pragma unroll
            for (int e = 0; e < V; ++e)
              if (at == k + e) d[e] += empty ? 0.f : at_target;
          }
          pack o;
#pragma unroll
          for (int e = 0; e < V; ++e) o[e] = from_f32<T>(d[e]);
          *(pack*)(out + k) = o;
        }
      }
      const uint32_t k = whole + threadIdx.x;
      if (first + kSpan >= vocab && k < vocab) {
        const float d = gradient(to_f32(row[k]));
        out[k] = from_f32<T>(at == k && !empty ? d + at_target : d);
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
  size_t bytes = 0;
  for (int64_t segments = plan_rows(rows, vocab, top).segments; segments > 1; segments = (segments + kWave - 1) / kWave)
    bytes += level_bytes(rows, segments, top);
  return bytes;
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
  const Outputs o{logp, entropy, stats, top_logp, top_index};
  const RowPlan plan = plan_rows(rows, vocab, top);
  const int64_t* tg = logp ? targets : nullptr;
  hipStream_t stream = (hipStream_t)hip_stream;
  const int64_t blocks = plan.segments == 1 ? (rows + 3) / 4 : rows;
  const dim3 grid((unsigned)std::min<int64_t>(blocks, 1 << 20), plan.segments == 1 ? 1 : (unsigned)std::min<int64_t>((plan.segments + 3) / 4, 1024));
  char* ws = (char*)workspace;
  with_type(type, [&](auto t) {
    using T = decltype(t);
    const T* x = (const T*)logits;
    const uint32_t n = (uint32_t)vocab;
    uint64_t* keys = (uint64_t*)ws;
    float* part = (float*)(ws + (size_t)rows * plan.segments * top * sizeof(uint64_t));
    auto launch = [&](auto kernel, size_t lds) {
      hipLaunchKernelGGL(kernel, grid, dim3(kBlock), lds, stream, x, ld, tg, rows, n, scale, ignore_index, (int)top, o, plan.segments, (uint32_t)plan.pieces, part, keys);
    };
    const size_t lds = 4 * (plan.lane_elements + 2) * top * sizeof(uint64_t);
    if (!top) launch(k_logprobs<T, false, 32>, 0);
    else if (plan.lane_elements == 16) launch(k_logprobs<T, true, 16>, lds);
    else launch(k_logprobs<T, true, 32>, lds);
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
    constexpr int64_t kSpan = (int64_t)kBackPacks * kBlock * Pack<T>::n;
    const dim3 grid((unsigned)std::min<int64_t>(rows, 1 << 20), (unsigned)std::min<int64_t>((vocab + kSpan - 1) / kSpan, 1024));
    if (dentropy)
      hipLaunchKernelGGL((k_logprobs_back<T, true>), grid, dim3(kBlock), 0, (hipStream_t)hip_stream, (const T*)logits, ld, targets, stats, entropy, dlogp,
                         dentropy, (T*)dlogits, ld_d, rows, (uint32_t)vocab, scale, ignore_index);
    else
      hipLaunchKernelGGL((k_logprobs_back<T, false>), grid, dim3(kBlock), 0, (hipStream_t)hip_stream, (const T*)logits, ld, targets, stats, entropy, dlogp,
                         dentropy, (T*)dlogits, ld_d, rows, (uint32_t)vocab, scale, ignore_index);
  });
  return launch_status("lopt_token_logprobs_backward");
}

}  // extern "C"
