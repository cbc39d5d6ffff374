// Losses made of tokens' log probabilities, and their gradients: the clipped policy loss with KL and entropy terms, and the loss of pairs of
// answers. A few operations a token, then sums over tokens, sequences and the batch in a fixed order, in 64 bits. Bound by memory where there are
// millions of tokens, else by the launches: one workgroup does a small batch in one launch, more leave partial sums to a second launch of one.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "lopt_flat.h"

namespace lopt {
namespace {

constexpr int kJoin = 1024;          // threads of the workgroup that joins, and of the one that does everything
constexpr int kQuad = 4;             // neighbouring tokens of a lane, where sequences have as many
constexpr int64_t kAlone = 16384;    // tokens up to which one workgroup may do everything, if it goes round no more often than that:
constexpr int64_t kAloneTrips = 2;
constexpr int64_t kPieces = 1024;     // that few sequences are cut into, about

// Sum over groups of G lanes, a power of two up to 64; every lane gets it.
template <typename V>
__device__ __forceinline__ V lanes_sum(V v, int G) {
  for (int d = 1; d < G; d *= 2) v += __shfl_xor(v, d);
  return v;
}

// Q = 4 neighbouring elements, or one where sequences have fewer than four tokens. The four that would pass a sequence's end are moved back to end with it.
template <int Q, typename T>
__device__ __forceinline__ void load_as(const T* p, float (&v)[Q]) {
  typedef T quad __attribute__((ext_vector_type(Q), aligned(sizeof(T))));
  const quad q = *(const quad*)p;
#pragma unroll
  for (int e = 0; e < Q; ++e) v[e] = to_f32(q[e]);
}
template <int Q>
__device__ __forceinline__ void load_of(const void* p, uint32_t type, int64_t i, float (&v)[Q]) {
  if (type == LOPT_F32) load_as<Q>((const float*)p + i, v);
  else if (type == LOPT_BF16) load_as<Q>((const bf16_t*)p + i, v);
  else load_as<Q>((const f16_t*)p + i, v);
}
__device__ __forceinline__ float load_one_of(const void* p, uint32_t type, int64_t i) {
  return type == LOPT_F32 ? ((const float*)p)[i] : type == LOPT_BF16 ? to_f32(((const bf16_t*)p)[i]) : to_f32(((const f16_t*)p)[i]);
}
// But for the first `skip`, which are another lane's.
template <int Q>
__device__ __forceinline__ void store(float* p, const float (&v)[Q], uint32_t skip) {
  typedef float quad __attribute__((ext_vector_type(Q), aligned(4)));
  if (skip) {
#pragma unroll
    for (int e = 1; e < Q; ++e)
      if (e >= (int)skip) p[e] = v[e];
    return;
  }
  quad q;
#pragma unroll
  for (int e = 0; e < Q; ++e) q[e] = v[e];
  *(quad*)p = q;
}
// Bit e: whether token e counts.
template <int Q>
__device__ __forceinline__ uint32_t load_mask(const uint8_t* mask, int64_t i) {
  if (!mask) return (1u << Q) - 1u;
  typedef uint8_t quad __attribute__((ext_vector_type(Q), aligned(1)));
  const quad q = *(const quad*)(mask + i);
  uint32_t bits = 0;
#pragma unroll
  for (int e = 0; e < Q; ++e) bits |= (q[e] ? 1u : 0u) << e;
  return bits;
}

// How sequences are shared out: a group of `lanes` lanes takes a sequence, four neighbouring tokens a lane in turn, or one of its `pieces`, every so many turns, so that
// padding, which costs nothing, falls to all of them (512x8192 tokens and their gradient 35.8 us, with neighbouring turns a piece 36.6).
// Of kMany sequences or more fewer lanes each go on more often, so that fewer are idle at the ends. us of the loss and its gradient with lanes for one time | for up to four:
// 60000x30 35 | 26, 30000x100 50 | 36, 14000x200 33.6 | 31, 8000x400 50 | 36, 4000x700 35.3 | 28.4; of few 1000x100 12.5 | 14, 300x900 12.9 | 17. 200000x10 by 16 lanes each
// 68, by 4 34.
// Few sequences are cut so that there are about kPieces pieces, a power of two of each, with which lanes of the join share out a sequence. us of k_policy and its join for
// 512x8192 tokens cut into 512, 1024, 2048, 4096: 23.8 + 4.0, 16.8 + 4.2, 19.0 + 5.1, 20.9 + 6.9.
constexpr int64_t kMany = 2048;
struct Plan {
  int lanes, threads, shift, quad;   // pieces: 2^shift; neighbouring tokens of a lane
  int64_t pieces, units, blocks;
  bool alone, cut;   // cut: into pieces that a join puts together
};
inline Plan plan_of(int64_t seqs, int64_t tokens) {
  Plan p{};
  p.quad = tokens < kQuad ? 1 : kQuad;
  const int most = seqs >= kMany ? 4 : 1;   // times that a lane goes on
  p.lanes = tokens <= (most > 1 ? 2 : 1) * 4 * kQuad ? 4 : tokens <= 16 * kQuad * most ? 16 : tokens <= 64 * kQuad * most ? 64 : kBlock;
  if (seqs * tokens <= kAlone) {   // all sequences at one time, if fewer lanes each can do that
    int lanes = p.lanes;
    while (lanes > 16 && seqs * lanes > kJoin) lanes /= 4;
    p.alone = (tokens + p.quad * lanes - 1) / (p.quad * lanes) * ((seqs * lanes + kJoin - 1) / kJoin) <= kAloneTrips;
    if (p.alone) p.lanes = lanes;
  }
  p.pieces = 1;
  if (!p.alone && p.lanes == kBlock)
    while (p.pieces < kPieces && p.pieces * seqs < kPieces && p.pieces * kQuad * kBlock < tokens) p.pieces *= 2;
  for (p.shift = 0; (int64_t)1 << p.shift < p.pieces;) ++p.shift;
  p.units = seqs * p.pieces;
  p.threads = p.alone ? kJoin : kBlock;
  const int64_t groups = p.threads / p.lanes;
  // units of whole sequences go round and leave one partial sum a workgroup, pieces one each
  p.blocks = p.alone ? 1 : p.pieces > 1 ? p.units : std::clamp<int64_t>((p.units + groups - 1) / groups, 1, 2048);
  return p;
}
// Calls f(lanes, threads, tokens of a lane) as integral constants.
template <typename F>
void with_plan(const Plan& p, F&& f) {
  using std::integral_constant;
  auto go = [&](auto g, auto q) {
    if (p.alone) f(g, integral_constant<int, kJoin>{}, q);
    else f(g, integral_constant<int, kBlock>{}, q);
  };
  if (p.quad == 1) go(integral_constant<int, 4>{}, integral_constant<int, 1>{});
  else if (p.lanes == 4) go(integral_constant<int, 4>{}, integral_constant<int, kQuad>{});
  else if (p.lanes == 16) go(integral_constant<int, 16>{}, integral_constant<int, kQuad>{});
  else if (p.lanes == 64) go(integral_constant<int, 64>{}, integral_constant<int, kQuad>{});
  else go(integral_constant<int, kBlock>{}, integral_constant<int, kQuad>{});
}

// Sum over a group of G lanes of a workgroup that is a multiple of it; `red` has a value for each wavefront. Every wavefront of the workgroup calls it.
template <int G, typename V>
__device__ __forceinline__ V group_total(V v, V* red) {
  if (G < kWave) return lanes_sum(v, G);
  v = wave_sum(v);
  if (G > kWave) {
    constexpr int W = G / kWave;
    const int wave = threadIdx.x >> 6, first = wave / W * W;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[wave] = v;
    __syncthreads();
    v = red[first];
#pragma unroll
    for (int i = 1; i < W; ++i) v += red[first + i];
  }
  return v;
}
// Eight sums over a wavefront at once: lanes hand each other the half of the sums that the other goes on with, so that ten exchanges do what
// forty-eight would. A lane gets the sum whose index is 4 (bit 3 of the lane's number) + 2 (bit 2) + bit 1.
__device__ __forceinline__ double eight_totals(const double (&v)[8]) {
  const int lane = threadIdx.x;
  auto half = [](bool high, double a, double b, auto exchange) {   // keeps a where low, b where high
    const double keep = high ? b : a, give = high ? a : b;
    return keep + exchange(give);
  };
  auto mirror = [](double x) { return dpp_d<0x140>(x); };        // lane i of a row of 16 has lane 15 - i's
  auto half_mirror = [](double x) { return dpp_d<0x141>(x); };   // of 8, lane 7 - i's
  auto pairs = [](double x) { return dpp_d<0x4E>(x); };          // quad_perm [2,3,0,1]
  double w[4], x[2];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = half(lane & 8, v[i], v[4 + i], mirror);
#pragma unroll
  for (int i = 0; i < 2; ++i) x[i] = half(lane & 4, w[i], w[2 + i], half_mirror);
  double y = half(lane & 2, x[0], x[1], pairs);
  y += dpp_d<0xB1>(y);                                           // quad_perm [1,0,3,2]
  y += __shfl_xor(y, 16);
  return y + __shfl_xor(y, 32);
}
// Eight sums over the workgroup, which thread 0 gets; `red` has eight values for each wavefront.
__device__ __forceinline__ void block_totals(double (&v)[8], double* red) {
  const int lane = threadIdx.x & 63, waves = blockDim.x / kWave;
  const double mine = eight_totals(v);
  __syncthreads();
  if (lane < 16 && (lane & 1) == 0) red[(threadIdx.x >> 6) * 8 + (lane >> 1 & 4) + (lane >> 1 & 2) + (lane >> 1 & 1)] = mine;
  __syncthreads();
  if (threadIdx.x >= kWave) return;
  double s = 0.0;   // lane i adds up the i-th
  if (lane < 8)
    for (int w = 0; w < waves; ++w) s += red[w * 8 + lane];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = readlane_d(s, i);
}

// ---------------------------------------------------------------------------------------------- policy loss

// e^v, e^v - 1 and e^v - 1 - v. Where NEAR, |v| < kNear: of half of v the last is its square times a polynomial that is off by 4e-9 of it, and with s = e^(v/2) - 1 that of v is
// s^2 + 2 (s - v / 2), in which nothing cancels. Else by the hardware's power of two, whose exponent's rounding is a unit of |v|. e^v itself is 1 + (rest + v): within a unit of 2^-24 of it for
// |v| <= 0.25, where most ratios lie, but 9e-7 of it, 15 units, near v = -2, where the sum cancels.
constexpr float kNear = 2.f;
struct Exp { float less_one, rest, value; };
template <bool NEAR>
__device__ __forceinline__ Exp exp_of(float v) {
  const float h = 0.5f * v;
  float r = 2.7659865e-6f;
  r = __builtin_fmaf(r, h, 2.5353789e-5f);
  r = __builtin_fmaf(r, h, 1.98451148e-4f);
  r = __builtin_fmaf(r, h, 1.38854675e-3f);
  r = __builtin_fmaf(r, h, 8.3333049e-3f);
  r = __builtin_fmaf(r, h, 4.1666734e-2f);
  r = __builtin_fmaf(r, h, 1.66666671e-1f);
  r = __builtin_fmaf(r, h, 4.99999998e-1f);
  r *= h * h;
  const float s = r + h, rest = __builtin_fmaf(s, s, 2.f * r);
  Exp x{rest + v, rest, 1.f + (rest + v)};
  if (!NEAR && !(fabsf(v) < kNear)) {
    x.value = __builtin_amdgcn_exp2f(v * 1.44269504088896341f);
    x.less_one = x.value - 1.f;
    x.rest = x.less_one - v;
  }
  return x;
}

// A token's terms. Which side of a bound the ratio lies on, which decides over the whole gradient, is found in 64 bits, where the difference of the logarithms has
// no rounding that matters; its values are in 32. NEAR: all logarithms of ratios at hand are within kNear.
struct Bounds { double low, high; float at_low, at_high; };   // ln(1 - clip_low), ln(1 + clip_high) and what they are the logarithms of
struct Terms { float surrogate, kl, beyond_one, drift, slope; bool clipped; };   // beyond_one: the ratio less 1
template <bool NEAR>
__device__ __forceinline__ Terms token_terms(float logp, float old, float adv, const Bounds& b, bool has_ref, float ref, float kl_coef) {
  Terms t{};
  const double d = (double)logp - (double)old;
  const Exp x = exp_of<NEAR>((float)d);
  t.drift = x.rest;
  t.beyond_one = x.less_one;
  t.clipped = adv > 0.f ? d > b.high : adv < 0.f && d < b.low;
  const float bound = adv > 0.f ? b.at_high : b.at_low;
  t.surrogate = adv == 0.f ? 0.f : -adv * (t.clipped ? bound : x.value);
  t.slope = t.clipped ? 0.f : t.surrogate;
  if (has_ref) {
    const Exp y = exp_of<NEAR>(ref - logp);
    t.kl = y.rest;
    t.slope -= kl_coef * y.less_one;   // d kl / d logp = 1 - e^u
  }
  return t;
}

// Tokens of a sequence. What does not count is 0 throughout, so that its ratio is 1 and its terms are 0.
template <int Q>
struct Tokens {
  float logp[Q], old[Q], adv[Q], ref[Q];
  uint32_t bits;
  // Padding, which comes in runs, is not read.
  __device__ __forceinline__ void load(const lopt_policy& a, int64_t seq, int64_t t, float adv_seq, uint32_t bits_) {
    bits = bits_;
    if (!bits) return;
    load_as<Q>(a.logp + seq * a.ld_logp + t, logp);
    load_of<Q>(a.old_logp, a.old_type, seq * a.ld_old + t, old);
    if (a.advantage_per_sequence) {
#pragma unroll
      for (int e = 0; e < Q; ++e) adv[e] = adv_seq;
    } else {
      load_of<Q>(a.advantages, a.advantage_type, seq * a.ld_advantages + t, adv);
    }
    if (a.ref_logp) load_of<Q>(a.ref_logp, a.ref_type, seq * a.ld_ref + t, ref);
  }
  // Whether all of a wavefront's are within kNear of each other.
  __device__ __forceinline__ bool choose(bool has_ref) {
    bool far = false;
#pragma unroll
    for (int e = 0; e < Q; ++e) {
      const bool in = bits >> e & 1;
      logp[e] = in ? logp[e] : 0.f;
      old[e] = in ? old[e] : 0.f;
      adv[e] = in ? adv[e] : 0.f;
      far |= !(fabsf(logp[e] - old[e]) < kNear);
      if (has_ref) {
        ref[e] = in ? ref[e] : 0.f;
        far |= !(fabsf(ref[e] - logp[e]) < kNear);
      }
    }
    return __ballot(far) == 0;
  }
};

// Sums in the order of the stats: surrogate, kl, entropy, clipped, ratio less 1, drift, tokens, sequences.
constexpr int kSums = 8;

__device__ __forceinline__ void write_policy(const double (&sum)[kSums], const lopt_policy& a, float* loss, float* stats) {
  const double n = a.per_sequence ? sum[7] : sum[6], w = n > 0.0 ? 1.0 / n : 0.0;
  double mean[6];
#pragma unroll
  for (int i = 0; i < 6; ++i) mean[i] = n > 0.0 ? sum[i] * w : 0.0;
  if (n > 0.0) mean[4] += 1.0;   // its terms are the ratios less 1
  double v = mean[0];
  if ((a.ref_logp || a.kl) && a.kl_coef != 0.0) v += a.kl_coef * mean[1];   // infinite or NaN, it is only reported where its coefficient is 0
  if (a.entropy && a.entropy_coef != 0.0) v -= a.entropy_coef * mean[2];
  *loss = (float)v;
#pragma unroll
  for (int i = 0; i < 6; ++i) stats[i] = (float)mean[i];
  stats[6] = (float)sum[6];
  stats[7] = (float)sum[7];
}

// The sums of units of whole sequences (`shift` is 0), one row of them a workgroup, or of pieces, one row each; with `alone` the loss.
// 512x8192 tokens, half of them padding, 16.5 us: 1.8 TB/s of what is read, vector units busy 37 % on the average and twice that where the sequences are long; 8x128 5.5.
template <int G, int kThreads, int Q>
__global__ __launch_bounds__(kThreads) void k_policy(lopt_policy a, Bounds b, int shift, int64_t units, double* __restrict__ part, bool alone,
                                                     float* __restrict__ loss, float* __restrict__ stats, float* __restrict__ counts) {
  __shared__ double red[kThreads / kWave * kSums];
  const int lane = threadIdx.x % G;
  constexpr int kGroups = kThreads / G;
  double sum[kSums] = {};
  const bool has_ref = a.ref_logp != nullptr;
  // every wavefront goes through the loop as often, for the barriers of the group's sums
  for (int64_t base = (int64_t)blockIdx.x * kGroups; base < units; base += (int64_t)gridDim.x * kGroups) {
    const int64_t unit = base + threadIdx.x / G;
    const bool have = unit < units;
    const int64_t seq = have ? unit >> shift : 0, from = (unit & (((int64_t)1 << shift) - 1)) * G * Q, to = have ? a.tokens : 0, step = (int64_t)G * Q << shift;
    double own[6] = {};   // [3] is formed at the end
    int clipped = 0, count_in = 0;
    const float adv_seq = have && a.advantage_per_sequence ? load_one_of(a.advantages, a.advantage_type, seq * a.ld_advantages) : 0.f;
    for (int64_t t = from + lane * Q; t < to; t += step) {
      const int64_t at = min(t, a.tokens - Q);
      const uint32_t bits = load_mask<Q>(a.mask, seq * a.ld_mask + at) & ~0u << (t - at);   // not those of the lane before
      if (__ballot(bits != 0) == 0) continue;
      Tokens<Q> q;
      q.load(a, seq, at, adv_seq, bits);
      float beyond_one = 0.f, drift = 0.f;   // of four, in 32 bits
      auto add = [&](auto near) {
#pragma unroll
        for (int e = 0; e < Q; ++e) {
          const Terms v = token_terms<decltype(near)::value>(q.logp[e], q.old[e], q.adv[e], b, has_ref, q.ref[e], 0.f);
          own[0] += (double)v.surrogate;
          if (has_ref) own[1] += (double)v.kl;
          clipped += v.clipped ? 1 : 0;
          beyond_one += v.beyond_one;
          drift += v.drift;
        }
      };
      if (q.choose(has_ref)) add(std::true_type{});
      else add(std::false_type{});
      own[4] += (double)beyond_one;
      own[5] += (double)drift;
      count_in += __popc(bits);
      auto given = [&](const float* p, double& to_sum) {
        if (!bits) return;
        float v[Q];
        load_as<Q>(p + at, v);
#pragma unroll
        for (int e = 0; e < Q; ++e) to_sum += bits >> e & 1 ? (double)v[e] : 0.0;
      };
      if (a.kl) given(a.kl + seq * a.ld_kl, own[1]);
      if (a.entropy) given(a.entropy + seq * a.ld_entropy, own[2]);
    }
    own[3] = (double)clipped;
    double w = 1.0;
    if (shift == 0) {   // the sequence is whole
      const double n = group_total<G>((double)count_in, red);
      if (a.per_sequence && n > 0.0) w = 1.0 / n;
      if (lane == 0 && have) {
        sum[7] += n > 0.0 ? 1.0 : 0.0;
        if (counts) counts[seq] = (float)n;
      }
    }
#pragma unroll
    for (int i = 0; i < 6; ++i) sum[i] += w * own[i];
    sum[6] += (double)count_in;
  }
  block_totals(sum, red);
  if (threadIdx.x != 0) return;
  if (alone) {
    write_policy(sum, a, loss, stats);
  } else {
#pragma unroll
    for (int i = 0; i < kSums; ++i) part[(int64_t)blockIdx.x * kSums + i] = sum[i];
  }
}

// Joins `rows` rows of sums. Of pieces, `lanes` lanes take a sequence.
__global__ __launch_bounds__(kJoin) void k_policy_join(lopt_policy a, int64_t rows, int64_t pieces, const double* __restrict__ part, float* __restrict__ loss,
                                                       float* __restrict__ stats, float* __restrict__ counts) {
  __shared__ double red[kJoin / kWave * kSums];
  double sum[kSums] = {};
  if (pieces == 1) {
    for (int64_t k = threadIdx.x; k < rows; k += kJoin) {
#pragma unroll
      for (int i = 0; i < kSums; ++i) sum[i] += part[k * kSums + i];
    }
  } else {
    const int lanes = (int)min(pieces, (int64_t)kWave), lane = threadIdx.x % lanes;
    for (int64_t base = 0; base < a.seqs; base += kJoin / lanes) {
      const int64_t seq = base + threadIdx.x / lanes;
      double own[7] = {};
      if (seq < a.seqs) {
        for (int64_t k = lane; k < pieces; k += lanes) {
#pragma unroll
          for (int i = 0; i < 7; ++i) own[i] += part[(seq * pieces + k) * kSums + i];
        }
      }
      const double n = lanes_sum(own[6], lanes), w = a.per_sequence && n > 0.0 ? 1.0 / n : 1.0;
#pragma unroll
      for (int i = 0; i < 6; ++i) sum[i] += w * own[i];
      sum[6] += own[6];
      if (lane == 0 && seq < a.seqs) {
        sum[7] += n > 0.0 ? 1.0 : 0.0;
        if (counts) counts[seq] = (float)n;
      }
    }
  }
  block_totals(sum, red);
  if (threadIdx.x == 0) write_policy(sum, a, loss, stats);
}

// Calls g(sequence, first token, how many of them are another lane's) for every Q tokens of all sequences; the last of a sequence end with it. One call a thread: two or four
// one after the other take 16.9 us for 512x8192 tokens of the policy loss, one 15.4.
template <int Q, typename F>
__device__ __forceinline__ void for_tokens(const Flat& f, F&& g) {
  for (int64_t first = (int64_t)blockIdx.x * kBlock; first < f.total; first += (int64_t)gridDim.x * kBlock) {
    int64_t seq;
    uint32_t t;
    if (!Chunk(f, first).at(f, Q, threadIdx.x, seq, t)) continue;
    const uint32_t at = min(t, f.cols - Q);
    g(seq, at, t - at);
  }
}

// The gradients, all terms formed again: 512x8192 tokens 15.2 us, 3 TB/s, 8x128 3.3.
template <int Q>
__global__ __launch_bounds__(kBlock) void k_policy_back(lopt_policy a, Bounds b, Flat f, const float* __restrict__ stats, const float* __restrict__ counts,
                                                        const float* __restrict__ dloss, float* __restrict__ dlogp, float* __restrict__ dkl, float* __restrict__ dentropy) {
  const float up = *dloss, whole = stats[a.per_sequence ? 7 : 6];
  const float kl_coef = (float)a.kl_coef, entropy_coef = (float)a.entropy_coef;
  const bool has_ref = a.ref_logp != nullptr;
  for_tokens<Q>(f, [&](int64_t seq, uint32_t t, uint32_t skip) {
    const uint32_t bits = load_mask<Q>(a.mask, seq * a.ld_mask + t);
    // of a token that counts there are a sequence that has one and a batch that has one
    const float w = up / (a.per_sequence ? whole * counts[seq] : whole);
    if (dlogp) {
      Tokens<Q> q;
      q.load(a, seq, t, a.advantage_per_sequence ? load_one_of(a.advantages, a.advantage_type, seq * a.ld_advantages) : 0.f, bits);
      float o[Q] = {};
      auto slopes = [&](auto near) {
#pragma unroll
        for (int e = 0; e < Q; ++e) {
          const float v = token_terms<decltype(near)::value>(q.logp[e], q.old[e], q.adv[e], b, has_ref, q.ref[e], kl_coef).slope;
          o[e] = q.bits >> e & 1 ? w * v : 0.f;
        }
      };
      if (__ballot(bits != 0) != 0) {
        if (q.choose(has_ref)) slopes(std::true_type{});
        else slopes(std::false_type{});
      }
      store<Q>(dlogp + seq * a.tokens + t, o, skip);
    }
    auto same = [&](float* out, float v) {
      float o[Q];
#pragma unroll
      for (int e = 0; e < Q; ++e) o[e] = bits >> e & 1 ? v : 0.f;
      store<Q>(out + seq * a.tokens + t, o, skip);
    };
    if (dkl) same(dkl, w * kl_coef);
    if (dentropy) same(dentropy, -w * entropy_coef);
  });
}

lopt_status check_policy(const lopt_policy* a) {
  if (!a) return fail_call(LOPT_EINVAL, "terms_host is null");
  LOPT_CHECK(check_matrix(a->seqs, a->tokens, "tokens"));
  LOPT_CHECK(check_type("old_type", a->old_type));
  LOPT_CHECK(check_type("advantage_type", a->advantage_type));
  LOPT_CHECK(check_type("ref_type", a->ref_type));
  const bool any = a->seqs > 0;
  LOPT_CHECK(check_array("logp", a->logp, 4, any));
  LOPT_CHECK(check_array("old_logp", a->old_logp, type_bytes(a->old_type), any));
  LOPT_CHECK(check_array("advantages", a->advantages, type_bytes(a->advantage_type), any));
  LOPT_CHECK(check_array("ref_logp", a->ref_logp, type_bytes(a->ref_type), false));
  LOPT_CHECK(check_array("kl", a->kl, 4, false));
  LOPT_CHECK(check_array("entropy", a->entropy, 4, false));
  LOPT_CHECK(check_ld("ld_logp", a->seqs, a->tokens, a->ld_logp, false));
  LOPT_CHECK(check_ld("ld_old", a->seqs, a->tokens, a->ld_old, false));
  LOPT_CHECK(check_ld("ld_advantages", a->seqs, a->tokens, a->ld_advantages, false));
  if (a->ref_logp) LOPT_CHECK(check_ld("ld_ref", a->seqs, a->tokens, a->ld_ref, false));
  if (a->kl) LOPT_CHECK(check_ld("ld_kl", a->seqs, a->tokens, a->ld_kl, false));
  if (a->entropy) LOPT_CHECK(check_ld("ld_entropy", a->seqs, a->tokens, a->ld_entropy, false));
  if (a->mask) LOPT_CHECK(check_ld("ld_mask", a->seqs, a->tokens, a->ld_mask, false));
  if (a->ref_logp && a->kl) return fail_call(LOPT_EINVAL, "ref_logp and kl are both given");
  if (!(a->clip_low >= 0.0 && a->clip_low <= 1.0)) return fail_call(LOPT_EINVAL, "clip_low must be in [0, 1]");
  if (!(a->clip_high >= 0.0)) return fail_call(LOPT_EINVAL, "clip_high must be >= 0");
  if (!std::isfinite(a->kl_coef) || !std::isfinite(a->entropy_coef)) return fail_call(LOPT_EINVAL, "kl_coef and entropy_coef must be finite");
  return LOPT_OK;
}
Bounds bounds_of(const lopt_policy& a) { return Bounds{std::log1p(-a.clip_low), std::log1p(a.clip_high), (float)(1.0 - a.clip_low), (float)(1.0 + a.clip_high)}; }

// ---------------------------------------------------------------------------------------------- preference loss

struct Answer { double sum, count; };   // of log ratios, and of the tokens that count

// What the join of a pair gives: loss and statistics added up over the pairs, what the backward pass needs written.
struct PairOutputs {
  float* loss;
  float* stats;
  float* rewards;
  float* coef;
};
constexpr int kPairSums = 8;   // loss, right ones, margins, rewards of the chosen, of the rejected, three of nothing

__device__ __forceinline__ void write_pair(const lopt_preference& a, int64_t pair, Answer chosen, Answer rejected, const PairOutputs& o, double (&sum)[kPairSums]) {
  if (a.ref && a.ref_sums) {
    if (chosen.count > 0.0) chosen.sum -= load_one_of(a.ref, a.ref_type, pair * a.ld_ref);
    if (rejected.count > 0.0) rejected.sum -= load_one_of(a.ref, a.ref_type, (a.pairs + pair) * a.ld_ref);
  }
  double per[2] = {1.0, 1.0};
  if (a.average) {
    per[0] = fmax(chosen.count, 1.0);
    per[1] = fmax(rejected.count, 1.0);
    chosen.sum /= per[0];
    rejected.sum /= per[1];
  }
  const double m = chosen.sum - rejected.sum, z = a.beta * m - a.margin;
  double loss, slope;   // slope: d loss / d m
  if (a.kind == LOPT_PREFERENCE_SIGMOID) {
    const double soft = log1p(exp(-fabs(z))), s = a.label_smoothing;
    loss = 0.0;   // an infinite z adds nothing where its weight is 0
    if (s != 1.0) loss += (1.0 - s) * (fmax(-z, 0.0) + soft);
    if (s != 0.0) loss += s * (fmax(z, 0.0) + soft);
    slope = a.beta * (1.0 / (1.0 + exp(-z)) - (1.0 - s));
  } else if (a.kind == LOPT_PREFERENCE_HINGE) {
    loss = fmax(1.0 - z, 0.0);
    slope = z < 1.0 ? -a.beta : 0.0;
  } else {
    const double off = m - 0.5 / a.beta;
    loss = off * off;
    slope = 2.0 * off;
  }
  if (z != z) loss = slope = z;   // a NaN is not less than a bound
  slope /= (double)a.pairs;
  const double rc = a.beta * chosen.sum, rr = a.beta * rejected.sum;
  o.rewards[pair] = (float)rc;
  o.rewards[a.pairs + pair] = (float)rr;
  o.coef[pair] = (float)(slope / per[0]);
  o.coef[a.pairs + pair] = (float)(-slope / per[1]);
  sum[0] += loss;
  sum[1] += m > 0.0 ? 1.0 : 0.0;
  sum[2] += a.beta * m;
  sum[3] += rc;
  sum[4] += rr;
}

// The loss and the statistics, by thread 0 of a workgroup whose threads have sums of pairs.
__device__ __forceinline__ void write_preference(const lopt_preference& a, double (&sum)[kPairSums], const PairOutputs& o, double* red) {
  block_totals(sum, red);
  if (threadIdx.x != 0) return;
  const double w = a.pairs > 0 ? 1.0 / (double)a.pairs : 0.0;
  *o.loss = (float)(sum[0] * w);
#pragma unroll
  for (int i = 1; i < 5; ++i) o.stats[i - 1] = (float)(sum[i] * w);
}

// What Q tokens add to an answer.
template <int Q>
__device__ __forceinline__ void add_tokens(const lopt_preference& a, int64_t row, int64_t at, uint32_t bits, bool has_ref, Answer& own) {
  if (!bits) return;   // padding is not read
  float logp[Q], ref[Q] = {};
  load_as<Q>(a.logp + row * a.ld_logp + at, logp);
  if (has_ref) load_of<Q>(a.ref, a.ref_type, row * a.ld_ref + at, ref);
#pragma unroll
  for (int e = 0; e < Q; ++e) own.sum += bits >> e & 1 ? (double)logp[e] - (double)ref[e] : 0.0;
  own.count += (double)__popc(bits);
}

// Whole answers: a group takes both of a pair and writes what it gives; workgroups leave one row of sums each, or with `alone` the loss. us of the loss and its gradient when
// one workgroup joined all pairs | so: 30000x100 56 | 18.4, 100 000 pairs of few tokens 147 | 20.
template <int G, int kThreads, int Q>
__global__ __launch_bounds__(kThreads) void k_preference(lopt_preference a, double* __restrict__ part, bool alone, PairOutputs o) {
  __shared__ double red[kThreads / kWave * kPairSums];
  const int lane = threadIdx.x % G;
  constexpr int kGroups = kThreads / G;
  const bool has_ref = a.ref && !a.ref_sums;
  double sum[kPairSums] = {};
  for (int64_t base = (int64_t)blockIdx.x * kGroups; base < a.pairs; base += (int64_t)gridDim.x * kGroups) {
    const int64_t pair = base + threadIdx.x / G;
    const bool have = pair < a.pairs;
    Answer own[2] = {};
    for (int64_t t = lane * Q; have && t < a.tokens; t += G * Q) {
      const int64_t at = min(t, a.tokens - Q);
      uint32_t bits[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) bits[i] = load_mask<Q>(a.mask, (i * a.pairs + pair) * a.ld_mask + at) & ~0u << (t - at);   // not those of the lane before
#pragma unroll
      for (int i = 0; i < 2; ++i) add_tokens<Q>(a, i * a.pairs + pair, at, bits[i], has_ref, own[i]);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      own[i].sum = group_total<G>(own[i].sum, red);
      own[i].count = group_total<G>(own[i].count, red);
    }
    if (lane == 0 && have) write_pair(a, pair, own[0], own[1], o, sum);
  }
  if (alone) return write_preference(a, sum, o, red);
  block_totals(sum, red);
  if (threadIdx.x != 0) return;
#pragma unroll
  for (int i = 0; i < kPairSums; ++i) part[(int64_t)blockIdx.x * kPairSums + i] = sum[i];
}
__global__ __launch_bounds__(kJoin) void k_preference_sums(lopt_preference a, int64_t rows, const double* __restrict__ part, PairOutputs o) {
  __shared__ double red[kJoin / kWave * kPairSums];
  double sum[kPairSums] = {};
  for (int64_t k = threadIdx.x; k < rows; k += kJoin) {
#pragma unroll
    for (int i = 0; i < kPairSums; ++i) sum[i] += part[k * kPairSums + i];
  }
  write_preference(a, sum, o, red);
}

// Few long answers: a workgroup takes a piece, and one workgroup joins them, `lanes` lanes a pair. 512 pairs of up to 4096 tokens 7.0 + 4.2 us.
__global__ __launch_bounds__(kBlock) void k_preference_pieces(lopt_preference a, int shift, Answer* __restrict__ part) {
  __shared__ double red[kBlock / kWave];
  const bool has_ref = a.ref && !a.ref_sums;
  const int64_t unit = blockIdx.x, row = unit >> shift, from = (unit & (((int64_t)1 << shift) - 1)) * kBlock * kQuad, step = (int64_t)kBlock * kQuad << shift;   // a workgroup for every piece
  Answer own{};
  for (int64_t t = from + threadIdx.x * kQuad; t < a.tokens; t += step) {
    const int64_t at = min(t, a.tokens - kQuad);
    add_tokens<kQuad>(a, row, at, load_mask<kQuad>(a.mask, row * a.ld_mask + at) & ~0u << (t - at), has_ref, own);
  }
  own.sum = group_total<kBlock>(own.sum, red);
  own.count = group_total<kBlock>(own.count, red);
  if (threadIdx.x == 0) part[unit] = own;
}
__global__ __launch_bounds__(kJoin) void k_preference_join(lopt_preference a, int64_t pieces, const Answer* __restrict__ part, PairOutputs o) {
  __shared__ double red[kJoin / kWave * kPairSums];
  double sum[kPairSums] = {};
  const int lanes = (int)min(pieces, (int64_t)kWave), lane = threadIdx.x % lanes;
  for (int64_t base = 0; base < a.pairs; base += kJoin / lanes) {
    const int64_t pair = base + threadIdx.x / lanes;
    Answer own[2] = {};
    if (pair < a.pairs) {
      for (int64_t k = lane; k < pieces; k += lanes) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const Answer q = part[(i * a.pairs + pair) * pieces + k];
          own[i].sum += q.sum;
          own[i].count += q.count;
        }
      }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      own[i].sum = lanes_sum(own[i].sum, lanes);
      own[i].count = lanes_sum(own[i].count, lanes);
    }
    if (lane == 0 && pair < a.pairs) write_pair(a, pair, own[0], own[1], o, sum);
  }
  write_preference(a, sum, o, red);
}

template <int Q>
__global__ __launch_bounds__(kBlock) void k_preference_back(const float* __restrict__ coef, const uint8_t* __restrict__ mask, int64_t ld_mask, const float* __restrict__ dloss,
                                                            float* __restrict__ dlogp, Flat f) {
  const float up = *dloss;
  for_tokens<Q>(f, [&](int64_t seq, uint32_t t, uint32_t skip) {
    const uint32_t bits = load_mask<Q>(mask, seq * ld_mask + t);
    const float v = up * coef[seq];
    float o[Q];
#pragma unroll
    for (int e = 0; e < Q; ++e) o[e] = bits >> e & 1 ? v : 0.f;
    store<Q>(dlogp + seq * (int64_t)f.cols + t, o, skip);
  });
}

unsigned flat_blocks(const Flat& f) { return (unsigned)std::min<int64_t>((f.total + kBlock - 1) / kBlock, 1 << 22); }

}  // namespace
}  // namespace lopt

using namespace lopt;

extern "C" {

size_t lopt_policy_loss_workspace(int64_t seqs, int64_t tokens) {
  if (seqs < 0 || tokens <= 0 || seqs > 0x7fffffffLL || tokens > 0x7fffffffLL) return 0;
  const Plan p = plan_of(seqs, tokens);
  return p.alone ? 0 : (size_t)p.blocks * kSums * sizeof(double);
}

lopt_status lopt_policy_loss(const lopt_policy* terms_host, float* loss, float* stats, float* counts, void* workspace, size_t workspace_bytes, void* hip_stream) {
  LOPT_CHECK(check_policy(terms_host));
  const lopt_policy a = *terms_host;
  LOPT_CHECK(check_array("loss", loss, 4, true));
  LOPT_CHECK(check_array("stats", stats, 4, true));
  LOPT_CHECK(check_array("counts", counts, 4, a.per_sequence && a.seqs > 0));
  LOPT_CHECK(check_workspace(workspace, workspace_bytes, lopt_policy_loss_workspace(a.seqs, a.tokens)));
  const Plan p = plan_of(a.seqs, a.tokens);
  hipStream_t stream = (hipStream_t)hip_stream;
  double* part = (double*)workspace;
  with_plan(p, [&](auto g, auto threads, auto q) {
    hipLaunchKernelGGL((k_policy<decltype(g)::value, decltype(threads)::value, decltype(q)::value>), dim3((unsigned)p.blocks), dim3(p.threads), 0, stream, a, bounds_of(a), p.shift,
                       p.units, part, p.alone, loss, stats, counts);
  });
  if (!p.alone) hipLaunchKernelGGL(k_policy_join, dim3(1), dim3(kJoin), 0, stream, a, p.blocks, p.pieces, (const double*)part, loss, stats, counts);
  return launch_status("lopt_policy_loss");
}

lopt_status lopt_policy_loss_backward(const lopt_policy* terms_host, const float* stats, const float* counts, const float* dloss, float* dlogp, float* dkl,
                                      float* dentropy, void* hip_stream) {
  LOPT_CHECK(check_policy(terms_host));
  lopt_policy a = *terms_host;
  LOPT_CHECK(check_array("stats", stats, 4, true));
  LOPT_CHECK(check_array("counts", counts, 4, a.per_sequence && a.seqs > 0));
  LOPT_CHECK(check_array("dloss", dloss, 4, true));
  LOPT_CHECK(check_array("dlogp", dlogp, 4, false));
  LOPT_CHECK(check_array("dkl", dkl, 4, false));
  LOPT_CHECK(check_array("dentropy", dentropy, 4, false));
  if (dkl && !a.kl) return fail_call(LOPT_EINVAL, "dkl without kl");
  if (dentropy && !a.entropy) return fail_call(LOPT_EINVAL, "dentropy without entropy");
  if (a.seqs == 0 || !(dlogp || dkl || dentropy)) return LOPT_OK;
  if (a.kl_coef == 0.0) a.ref_logp = nullptr;   // not in the loss
  const int quad = a.tokens < kQuad ? 1 : kQuad;
  const Flat f = flat_of(a.seqs, a.tokens, quad);
  auto kernel = quad == 1 ? k_policy_back<1> : k_policy_back<kQuad>;
  hipLaunchKernelGGL(kernel, dim3(flat_blocks(f)), dim3(kBlock), 0, (hipStream_t)hip_stream, a, bounds_of(a), f, stats, counts, dloss, dlogp, dkl, dentropy);
  return launch_status("lopt_policy_loss_backward");
}

static Plan preference_plan(int64_t pairs, int64_t tokens) {
  Plan p = plan_of(2 * pairs, tokens);
  // answers that a whole workgroup takes are pieces too while they are few: 512x4096 pairs 7.3 + 4.1 us, by pairs 11.4 + 3.9
  p.cut = p.pieces > 1 || (!p.alone && p.lanes == kBlock && pairs <= kMany);
  if (!p.cut && !p.alone) {   // units are pairs
    const int64_t groups = p.threads / p.lanes;
    p.blocks = std::clamp<int64_t>((pairs + groups - 1) / groups, 1, 2048);
  }
  return p;
}
size_t lopt_preference_loss_workspace(int64_t pairs, int64_t tokens) {
  if (pairs <= 0 || tokens <= 0 || pairs > 0x3fffffffLL || tokens > 0x7fffffffLL) return 0;
  const Plan p = preference_plan(pairs, tokens);
  return p.alone ? 0 : p.cut ? (size_t)p.units * sizeof(Answer) : (size_t)p.blocks * kPairSums * sizeof(double);
}

lopt_status lopt_preference_loss(const lopt_preference* terms_host, float* loss, float* stats, float* rewards, float* coef, void* workspace, size_t workspace_bytes,
                                 void* hip_stream) {
  if (!terms_host) return fail_call(LOPT_EINVAL, "terms_host is null");
  const lopt_preference a = *terms_host;
  if (a.pairs < 0 || a.pairs > 0x3fffffffLL) return fail_call(LOPT_ESHAPE, "pairs=%lld outside [0, 2^30-1]", (long long)a.pairs);
  LOPT_CHECK(check_matrix(2 * a.pairs, a.tokens, "tokens"));
  LOPT_CHECK(check_type("ref_type", a.ref_type));
  const bool any = a.pairs > 0;
  LOPT_CHECK(check_array("logp", a.logp, 4, any));
  LOPT_CHECK(check_array("ref", a.ref, type_bytes(a.ref_type), false));
  LOPT_CHECK(check_ld("ld_logp", 2 * a.pairs, a.tokens, a.ld_logp, false));
  if (a.ref) LOPT_CHECK(check_ld("ld_ref", 2 * a.pairs, a.tokens, a.ld_ref, false));
  if (a.mask) LOPT_CHECK(check_ld("ld_mask", 2 * a.pairs, a.tokens, a.ld_mask, false));
  if (a.kind > LOPT_PREFERENCE_SQUARED) return fail_call(LOPT_EINVAL, "kind %u is not a lopt_preference_kind", a.kind);
  if (!(a.beta > 0.0) || std::isinf(a.beta)) return fail_call(LOPT_EINVAL, "beta must be finite and > 0");
  if (!(a.label_smoothing >= 0.0 && a.label_smoothing <= 1.0)) return fail_call(LOPT_EINVAL, "label_smoothing must be in [0, 1]");
  if (a.label_smoothing != 0.0 && a.kind != LOPT_PREFERENCE_SIGMOID) return fail_call(LOPT_EINVAL, "label_smoothing goes with the sigmoid only");
  if (!std::isfinite(a.margin)) return fail_call(LOPT_EINVAL, "margin must be finite");
  if (a.margin != 0.0 && a.kind == LOPT_PREFERENCE_SQUARED) return fail_call(LOPT_EINVAL, "margin does not go with the squared loss");
  LOPT_CHECK(check_array("loss", loss, 4, true));
  LOPT_CHECK(check_array("stats", stats, 4, true));
  LOPT_CHECK(check_array("rewards", rewards, 4, any));
  LOPT_CHECK(check_array("coef", coef, 4, any));
  LOPT_CHECK(check_workspace(workspace, workspace_bytes, lopt_preference_loss_workspace(a.pairs, a.tokens)));
  const Plan p = preference_plan(a.pairs, a.tokens);
  hipStream_t stream = (hipStream_t)hip_stream;
  const PairOutputs o{loss, stats, rewards, coef};
  if (p.cut) {
    Answer* part = (Answer*)workspace;
    hipLaunchKernelGGL(k_preference_pieces, dim3((unsigned)p.units), dim3(kBlock), 0, stream, a, p.shift, part);
    hipLaunchKernelGGL(k_preference_join, dim3(1), dim3(kJoin), 0, stream, a, p.pieces, (const Answer*)part, o);
    return launch_status("lopt_preference_loss");
  }
  double* part = (double*)workspace;
  with_plan(p, [&](auto g, auto threads, auto q) {
    hipLaunchKernelGGL((k_preference<decltype(g)::value, decltype(threads)::value, decltype(q)::value>), dim3((unsigned)p.blocks), dim3(p.threads), 0, stream, a, part, p.alone, o);
  });
  if (!p.alone) hipLaunchKernelGGL(k_preference_sums, dim3(1), dim3(kJoin), 0, stream, a, p.blocks, (const double*)part, o);
  return launch_status("lopt_preference_loss");
}

lopt_status lopt_preference_loss_backward(const float* coef, const uint8_t* mask, int64_t ld_mask, const float* dloss, float* dlogp, int64_t pairs, int64_t tokens,
                                          void* hip_stream) {
  if (pairs < 0 || pairs > 0x3fffffffLL) return fail_call(LOPT_ESHAPE, "pairs=%lld outside [0, 2^30-1]", (long long)pairs);
  LOPT_CHECK(check_matrix(2 * pairs, tokens, "tokens"));
  if (mask) LOPT_CHECK(check_ld("ld_mask", 2 * pairs, tokens, ld_mask, false));
  LOPT_CHECK(check_array("coef", coef, 4, pairs > 0));
  LOPT_CHECK(check_array("dloss", dloss, 4, true));
  LOPT_CHECK(check_array("dlogp", dlogp, 4, pairs > 0));
  if (pairs == 0) return LOPT_OK;
  const int quad = tokens < kQuad ? 1 : kQuad;
  const Flat f = flat_of(2 * pairs, tokens, quad);
  auto kernel = quad == 1 ? k_preference_back<1> : k_preference_back<kQuad>;
  hipLaunchKernelGGL(kernel, dim3(flat_blocks(f)), dim3(kBlock), 0, (hipStream_t)hip_stream, coef, mask, ld_mask, dloss, dlogp, f);
  return launch_status("lopt_preference_loss_backward");
}

}  // extern "C"
