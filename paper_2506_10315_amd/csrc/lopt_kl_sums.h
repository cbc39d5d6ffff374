// The arithmetic of the KL divergence's running sums: what a lane does with its logits, and how sums are joined. Without lanes, so that the same lines run on the host, where tests hold
// them to 64 bits: a program that includes this there defines __device__, __forceinline__ and the three builtins.
#pragma once

#include <algorithm>
#include <cfloat>
#include <cmath>

namespace lopt {
namespace {

// Running sums of some pairs of logits, mx and mr the largest of either (the type's lowest where all are masked), e = 2^(c (x - mx)) and f = 2^(c (r - mr)) with
// c = scale / ln 2:
//   sx = sum e,   sr = sum f,   w = sum (f - e),   h = unit sum e d   with d = c ((x - r) - (mx - mr))
//   KL = ln 2 h / (unit sx) + ln(sr / sx)
// Differences from the maxima and between the two lose nothing where they are near, however large the logits are; where a constant of more than kOffset lies between the two
// rows, d goes by (x - mx) - (r - mr). Of two sharp distributions both terms
// are far smaller than the sums, which begin with the same 1: there ln(sr / sx) = ln(1 + w / sx), whose rounding goes with w (1x10 fp32 of KL 1e-4: off by 4e-5 with the
// sums alone; by 2e-4 with the maxima's products rounded as in the token log probabilities, for e and f are not 1 at them). `most`: the largest d that was
// not near; it is infinite where r masks a token that x does not (or where finite logits are 3.4e38 apart). A NaN makes the maximum and by it the sums NaN.
struct Apart { float mx, mr, sx, sr, w, h, most; };
// c, and a power of two by which it is 2^-26 to 2^-25. A lane whose tokens x masks all by a finite value has that value as its maximum and e = 1 for them, and r may have the type's
// lowest there, c d being beyond the type: in this unit the sum of 2^25 of them is finite until the row's maxima take it away. (From c = 2^75 on the unit stays, and fewer are: rebase
// drops what is nothing beside the row's maxima even if it is infinite.)
struct Scale { float c, unit, step; };   // step = c unit, which differences near the type's largest are multiplied by at once
inline Scale scale_of(float c) {
  const float unit = std::ldexp(1.f, -std::clamp(std::ilogb(c) + 26, -100, 100));
  return Scale{c, unit, c * unit};
}
__device__ __forceinline__ Apart nothing() { return Apart{-FLT_MAX, -FLT_MAX, 0.f, 0.f, 0.f, 0.f, -INFINITY}; }
__device__ __forceinline__ float shift_of(float mx, float mr, float c) { return __builtin_amdgcn_fmed3f(c * (mx - mr), -FLT_MAX, FLT_MAX); }
// The same of a wavefront or more. Lanes add up some hundred terms each in 32 bits, whose roundings are many and independent; the sums over the lanes and what is made of them
// are in 64, for KL is the small difference of its two terms (32 bits throughout: 1.6e-6 of the KL of 64 rows, so 2e-7).
struct Total { double sx, sr, w, h; float mx, mr, most; };

// 2^-d - 1 for |d| <= 4: that of a quarter of d, to 4e-8 of it, squared twice, by (1 + s)^2 - 1 = s (s + 2).
__device__ __forceinline__ float less_one(float d) {
  float s = -9.43454013e-10f;
  s = __builtin_fmaf(s, d, 3.81747935e-08f);
  s = __builtin_fmaf(s, d, -1.30198002e-06f);
  s = __builtin_fmaf(s, d, 3.75662583e-05f);
  s = __builtin_fmaf(s, d, -8.67252099e-04f);
  s = __builtin_fmaf(s, d, 1.50141658e-02f);
  s = __builtin_fmaf(s, d, -1.73286795e-01f) * d;
  s = __builtin_fmaf(s, s, s + s);
  return __builtin_fmaf(s, s, s + s);
}

// What a change to larger maxima makes of sums: factors of e and f, the second less the first, what d moves by in the unit. Near maxima's second factor goes by
// the move, as f went by d.
template <typename V> struct Move { V fx, fr, apart, moved; };
constexpr float kNear = 64.f, kOffset = 32.f;
template <typename V>
__device__ __forceinline__ Move<V> move_of(float mx0, float mr0, float mx, float mr, Scale s) {
  const bool close_by = fabsf(mx0 - mr0) <= kOffset && fabsf(mx - mr) <= kOffset;
  const float apart = (mx0 - mx) - (mr0 - mr);
  const float moved = close_by ? shift_of(mx0, mr0, s.c) - shift_of(mx, mr, s.c) : s.c * apart, held = close_by ? moved * s.unit : __builtin_amdgcn_fmed3f(apart * s.step, -FLT_MAX, FLT_MAX);
  const float fx = __builtin_amdgcn_exp2f((mx0 - mx) * s.c), less = fabsf(moved) <= 4.f ? less_one(moved) : __builtin_amdgcn_exp2f(-moved) - 1.f;
  if (fabsf(moved) <= kNear && fx > 0.f) return Move<V>{fx, (V)fx + (V)fx * less, (V)fx * less, held};
  const float fr = __builtin_amdgcn_exp2f((mr0 - mr) * s.c);
  return Move<V>{fx, fr, fr - fx, held};
}
// a's sums seen from larger maxima, beside which they may be nothing, whatever h is.
__device__ __forceinline__ Apart rebase(Apart a, float mx, float mr, Scale s) {
  const Move<float> m = move_of<float>(a.mx, a.mr, mx, mr, s);
  const float fs = m.fx * a.sx;
  return Apart{mx, mr, fs, m.fr * a.sr, m.fr * a.w + m.apart * a.sx, fs == 0.f ? 0.f : m.fx * a.h + fs * m.moved, a.most};
}
// The largest, NaN where there is one.
template <int E>
__device__ __forceinline__ float strict_most_of(const float (&x)[E], float m) {
#pragma unroll
  for (int i = 0; i < E; ++i) m = __builtin_elementwise_maximum(m, x[i]);
  return m;
}

// A lane's piece of logits beside the sums so far, which are seen from the new maxima: each d, and how far the largest lies from 0 (infinite where d has to go by the maxima).
// FIRST: there are no sums so far.
template <int E, bool FIRST>
__device__ __forceinline__ float differences_of(Apart& a, const float (&x)[E], const float (&r)[E], Scale s, float (&d)[E]) {
  const float mx = strict_most_of(x, a.mx), mr = strict_most_of(r, a.mr);
  if (FIRST) a.mx = mx, a.mr = mr;
  else a = rebase(a, mx, mr, s);
  const float shift = shift_of(a.mx, a.mr, s.c);
  float far = fabsf(a.mx - a.mr) <= kOffset ? 0.f : INFINITY;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    d[i] = __builtin_fmaf(x[i] - r[i], s.c, -shift);
    far = fmaxf(far, fabsf(d[i]));
  }
  return far;
}
// f = e 2^-d, so that what e was rounded by is in f too and cancels in KL: with an f by itself 1501 fp16 logits at a scale of 0.5 are off by 5e-7 of KL, so 2e-7. An e below 2^-126 has
// an f below 2^-62, which adds nothing. Of both logits masked there is no d. Here |d| <= 4: q - 1 goes by less_one, and not by q, whose rounding next to 1 is what remains of a KL that few
// unlikely tokens make up: of rows of some ten logits by 5e-6. It takes half as many instructions again as q; in long rows such roundings are many.
template <int E>
__device__ __forceinline__ void add_fine(Apart& a, const float (&x)[E], const float (&d)[E], Scale s) {
  float h = 0.f;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const float e = __builtin_amdgcn_exp2f((x[i] - a.mx) * s.c), near = __builtin_amdgcn_fmed3f(d[i], -4.f, 4.f), g = e * less_one(near);
    a.sx += e;
    a.sr += e + g;
    a.w += g;
    h = __builtin_fmaf(e, near, h);
  }
  a.h = __builtin_fmaf(h, s.unit, a.h);
}
// |d| <= kNear.
template <int E>
__device__ __forceinline__ void add_near(Apart& a, const float (&x)[E], const float (&d)[E], Scale s) {
  float h = 0.f;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const float e = __builtin_amdgcn_exp2f((x[i] - a.mx) * s.c), near = __builtin_amdgcn_fmed3f(d[i], -kNear, kNear), q = __builtin_amdgcn_exp2f(-near);
    a.sx += e;
    a.sr = __builtin_fmaf(e, q, a.sr);
    a.w = __builtin_fmaf(e, q - 1.f, a.w);
    h = __builtin_fmaf(e, near, h);
  }
  a.h = __builtin_fmaf(h, s.unit, a.h);
}
// Any d.
template <int E>
__device__ __forceinline__ void add_far(Apart& a, const float (&x)[E], const float (&r)[E], Scale s) {
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const float dx = x[i] - a.mx, dr = r[i] - a.mr, e = __builtin_amdgcn_exp2f(dx * s.c), f = __builtin_amdgcn_exp2f(dr * s.c), d = dx - dr;
    a.most = fmaxf(a.most, d);
    a.sx += e;
    a.sr += f;
    a.w += f - e;
    a.h = __builtin_fmaf(e, __builtin_amdgcn_fmed3f(d * s.step, -FLT_MAX, FLT_MAX), a.h);   // that of a masked token is finite, for e is 0
  }
}

// Sums of a segment seen from larger maxima, in 64 bits; the factors are rounded to 32, each for itself.
__device__ __forceinline__ void add_segment(Total& t, const Total& b, Scale s) {
  const Move<double> m = move_of<double>(b.mx, b.mr, t.mx, t.mr, s);
  const double fs = m.fx * b.sx;
  t.sx += fs;
  t.sr += m.fr * b.sr;
  t.w += m.fr * b.w + m.apart * b.sx;
  t.h += fs == 0.0 ? 0.0 : m.fx * b.h + fs * m.moved;
  t.most = fmaxf(t.most, b.most);
}

// A row's KL and stats from its sums. Sums that are 0 belong to a row that is masked whole; a NaN or +infinity is in the sum.
struct RowResult { float kl, stats[5]; };
__device__ __forceinline__ RowResult result_of(const Total& a, Scale s) {
  // what the shift of every d was rounded by is in sr as well, so that KL does not have it; the stats have it taken out
  constexpr double ln2 = 0.693147180559945309417;
  const double ratio = a.w / a.sx, mean = ln2 * a.h / ((double)s.unit * a.sx);
  const double rounded = fabsf(a.mx - a.mr) <= kOffset ? ln2 * ((double)shift_of(a.mx, a.mr, s.c) - (double)s.c * ((double)a.mx - (double)a.mr)) : 0.0;
  float kl = (float)(mean + (fabs(ratio) < 0.5 ? log1p(ratio) : log(a.sr / a.sx))), shifted = (float)(mean + rounded);
  if (kl < 0.f) kl = 0.f;   // a NaN stays one
  if (a.sr == 0.0 || a.most == INFINITY) kl = shifted = INFINITY;
  if (a.sx == 0.0) kl = shifted = 0.f;
  if (!(a.sx < INFINITY && a.sr < INFINITY)) kl = shifted = NAN;
  return RowResult{kl, {a.sx == 0.0 ? -INFINITY : a.mx, logf((float)a.sx), a.sr == 0.0 ? -INFINITY : a.mr, logf((float)a.sr) - (a.sr == 0.0 ? 0.f : (float)rounded), shifted}};
}

}  // namespace
}  // namespace lopt
