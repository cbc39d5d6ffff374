// KL divergence of rows by the kernels' own arithmetic (csrc/lopt_kl_sums.h), lane by lane on the CPU: built and run by tests/test_kl_sums_cpu.py.
// Arguments: lanes of a group, logits a lane and piece (8, 16 or 32), logits of a pack (4 or 8), wavefronts, pieces of a segment (0: the row is whole), scale.
// Standard input: rows and logits of a row as two int32, then x and r as float32. Standard output: kl and the five stats of each row as float32.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <vector>

#define __device__
#define __forceinline__ inline
static inline float exp2_of(float v) { return exp2f(v); }
static inline float med3(float a, float b, float c) { return std::isnan(a) ? b : std::max(std::min(a, c), b); }   // of b < c; of a NaN the least, as the instruction
static inline float most_strictly(float a, float b) { return std::isnan(a) || std::isnan(b) ? NAN : std::max(a, b); }
#define __builtin_amdgcn_exp2f exp2_of
#define __builtin_amdgcn_fmed3f med3
#define __builtin_elementwise_maximum most_strictly
#include "lopt_kl_sums.h"
using namespace lopt;

struct Shape { int lanes, pack, waves, pieces; Scale sc; };

// The sums of every wavefront's lanes over a segment from the logit `from` on, joined as a workgroup does. `fine`: rows of one piece.
template <int E>
static Total segment(const Shape& s, const float* x, const float* r, int n, int64_t from, int64_t end, bool fine) {
  const int size = s.lanes * E, W = s.waves;
  std::vector<Apart> all((size_t)W * s.lanes, nothing());
  for (int w = 0; w < W; ++w)
    for (int64_t first = from + (int64_t)w * size; first < end; first += (int64_t)W * size) {
      std::vector<float> d((size_t)s.lanes * E), u(d.size()), v(d.size());
      float far = 0.f;
      for (int lane = 0; lane < s.lanes; ++lane) {
        float (&a)[E] = *(float (*)[E])&u[lane * E], (&b)[E] = *(float (*)[E])&v[lane * E];
        for (int i = 0; i < E; ++i) {
          const int64_t k = first + ((int64_t)(i / s.pack) * s.lanes + lane) * s.pack + i % s.pack;
          a[i] = k < n ? x[k] : -INFINITY;
          b[i] = k < n ? r[k] : -INFINITY;
        }
        Apart& sums = all[w * s.lanes + lane];
        float (&t)[E] = *(float (*)[E])&d[lane * E];
        far = std::max(far, fine ? differences_of<E, true>(sums, a, b, s.sc, t) : differences_of<E, false>(sums, a, b, s.sc, t));
      }
      for (int lane = 0; lane < s.lanes; ++lane) {
        Apart& a = all[w * s.lanes + lane];
        float (&p)[E] = *(float (*)[E])&u[lane * E], (&q)[E] = *(float (*)[E])&v[lane * E], (&t)[E] = *(float (*)[E])&d[lane * E];
        if (fine && !(far > 4.f)) add_fine(a, p, t, s.sc);
        else if (!(far > kNear)) add_near(a, p, t, s.sc);
        else add_far(a, p, q, s.sc);
      }
    }
  float mx = -FLT_MAX, mr = -FLT_MAX;
  for (const Apart& a : all) mx = fmaxf(mx, a.mx), mr = fmaxf(mr, a.mr);
  Total t{0.0, 0.0, 0.0, 0.0, mx, mr, -INFINITY};
  for (Apart a : all) {
    a = rebase(a, mx, mr, s.sc);
    t.sx += a.sx, t.sr += a.sr, t.w += a.w, t.h += a.h;
    t.most = fmaxf(t.most, a.most);
  }
  return t;
}

template <int E>
static RowResult row_of(const Shape& s, const float* x, const float* r, int n) {
  if (!s.pieces) return result_of(segment<E>(s, x, r, n, 0, n, s.waves == 1 && n <= s.lanes * E), s.sc);
  std::vector<Total> parts;
  for (int64_t from = 0; from < n; from += (int64_t)s.pieces * s.lanes * E)
    parts.push_back(segment<E>(s, x, r, n, from, std::min<int64_t>(from + (int64_t)s.pieces * s.lanes * E, n), false));
  Total t{0.0, 0.0, 0.0, 0.0, -FLT_MAX, -FLT_MAX, -INFINITY};
  for (const Total& p : parts) t.mx = fmaxf(t.mx, p.mx), t.mr = fmaxf(t.mr, p.mr);
  for (const Total& p : parts) add_segment(t, p, s.sc);
  return result_of(t, s.sc);
}

int main(int argc, char** argv) {
  if (argc != 7) return 2;
  const int E = atoi(argv[2]);
  const Shape s{atoi(argv[1]), atoi(argv[3]), atoi(argv[4]), atoi(argv[5]), scale_of(fminf((float)atof(argv[6]) * 1.44269504088896341f, FLT_MAX))};
  int32_t size[2];
  if (fread(size, 4, 2, stdin) != 2) return 2;
  const size_t count = (size_t)size[0] * size[1];
  std::vector<float> x(count), r(count);
  if (fread(x.data(), 4, count, stdin) != count || fread(r.data(), 4, count, stdin) != count) return 2;
  for (int row = 0; row < size[0]; ++row) {
    const float *a = &x[(size_t)row * size[1]], *b = &r[(size_t)row * size[1]];
    const RowResult o = E == 8 ? row_of<8>(s, a, b, size[1]) : E == 16 ? row_of<16>(s, a, b, size[1]) : row_of<32>(s, a, b, size[1]);
    fwrite(&o, 4, 6, stdout);
  }
  return 0;
}
