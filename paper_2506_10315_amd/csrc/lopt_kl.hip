// KL divergence of each row's softmax(scale x) from softmax(scale r), and its gradient for both: running maxima and sums, one pass over both rows of logits.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "lopt_softmax.h"

#include "lopt_kl_sums.h"

namespace lopt {
namespace {

// Over a wavefront or each 16 of its lanes.
template <int G>
__device__ __forceinline__ float group_max(float v) {
  if (G == kWave) return wave_max(v);
  v = fmaxf(v, dpp_f<0xB1>(v));
  v = fmaxf(v, dpp_f<0x4E>(v));
  v = fmaxf(v, dpp_f<0x141>(v));
  return fmaxf(v, dpp_f<0x140>(v));
}
template <int G>
__device__ __forceinline__ double group_sum(double v) {
  if (G == kWave) return wave_sum(v);
  v += dpp_d<0xB1>(v);
  v += dpp_d<0x4E>(v);
  v += dpp_d<0x141>(v);
  return v + dpp_d<0x140>(v);
}
template <int G>
__device__ __forceinline__ bool none_of_group(bool v) {
  const uint64_t bits = __ballot(v);
  return G == kWave ? bits == 0 : (bits >> (threadIdx.x & 48) & 0xffff) == 0;
}
// Seen from maxima that none of the lanes exceeds.
template <int G>
__device__ __forceinline__ Total total_of(Apart a, float mx, float mr, Scale sc) {
  a = rebase(a, mx, mr, sc);
  return Total{group_sum<G>((double)a.sx), group_sum<G>((double)a.sr), group_sum<G>((double)a.w), group_sum<G>((double)a.h), mx, mr, group_max<G>(a.most)};
}

// Adds a piece, by the way that all lanes of the group can take. FINE: rows of one piece.
template <int E, bool FINE, int G = kWave>
__device__ __forceinline__ void add_piece(Apart& a, const float (&x)[E], const float (&r)[E], Scale sc) {
  float d[E];
  const float far = differences_of<E, FINE>(a, x, r, sc, d);
  if (FINE && none_of_group<G>(far > 4.f)) return add_fine(a, x, d, sc);
  if (none_of_group<G>(far > kNear)) return add_near(a, x, d, sc);
  add_far(a, x, r, sc);
}

template <typename T>
struct Rows {
  const T* x;
  const T* r;
  int64_t ld_x, ld_r, rows;
  uint32_t n;
  float scale;
  Scale sc;
  const uint8_t* keep;   // null: every row counts
};
struct Outputs {
  float* kl;
  float* stats;
};

// A row's outputs, by one lane.
__device__ __forceinline__ void write_row(const Outputs& o, int64_t row, const Total& a, Scale sc) {
  const RowResult r = result_of(a, sc);
  o.kl[row] = r.kl;
#pragma unroll
  for (int i = 0; i < 5; ++i) o.stats[5 * row + i] = r.stats[i];
}
__device__ __forceinline__ void write_nothing(const Outputs& o, int64_t row) {
  o.kl[row] = 0.f;
#pragma unroll
  for (int i = 0; i < 5; ++i) o.stats[5 * row + i] = 0.f;
}

// Rows of one piece: G lanes each, `batch` <= G neighbouring ones in turn. Lane k of the group keeps the sums of the k-th, and all lanes make their rows' outputs at once.
// Bound by vector issue, some 500 instructions a row of 64 lanes: batches, of which 8192 wavefronts have one each, spare most rows those of the outputs. us with a row a batch | so:
// 20000x1000 bf16 34.0 | 30.6 to 32.1, 100000x100 fp32 26.6 | 24.4, with 64 lanes a row 89.
template <typename T, int E, int G>
__global__ __launch_bounds__(kBlock) void k_kl_short(Rows<T> a, int batch, Outputs o) {
  constexpr int kGroups = kBlock / G;
  const int lane = threadIdx.x % G;
  const int64_t group = (int64_t)blockIdx.x * kGroups + threadIdx.x / G, first = group * batch;   // a group for every batch
  const int count = (int)max(min((int64_t)batch, a.rows - first), (int64_t)0);
  Total own{};
  for (int k = 0; k < count; ++k) {
    const int64_t row = first + k;
    if (a.keep && !a.keep[row]) continue;
    const T *x = a.x + row * a.ld_x, *r = a.r + row * a.ld_r;
    const int off = pack_offset(x, a.n);
    Piece<T, E, G> p, q;
    p.load(x, 0, off, a.n);
    q.load(r, 0, off, a.n);
    float u[E], v[E];
    p.unpack(u);
    q.unpack(v);
    Apart s = nothing();
    add_piece<E, true, G>(s, u, v, a.sc);
    const Total t = total_of<G>(s, group_max<G>(s.mx), group_max<G>(s.mr), a.sc);
    if (lane == k) own = t;
  }
  if (lane >= count) return;
  if (a.keep && !a.keep[first + lane]) write_nothing(o, first + lane);
  else write_row(o, first + lane, own, a.sc);
}

// A wavefront's sums over every `step`-th element's piece of a row, from `first` to `end`, counted from the pack in which the row of x begins.
template <typename T, int E, bool NT>
__device__ __forceinline__ Apart sums_of(const Rows<T>& a, const T* x, const T* r, int off, int64_t first, int64_t end, int64_t step) {
  typedef Piece<T, E> P;
  Apart s = nothing();
  P p, q;
  if (first < end) {
    p.template load<NT>(x, (int)first, off, a.n);
    q.template load<NT>(r, (int)first, off, a.n);
  }
  for (; first < end; first += step) {
    float u[E], v[E];
    P next_p, next_q;
    if (first + step < end) {
      next_p.template load<NT>(x, (int)(first + step), off, a.n);
      next_q.template load<NT>(r, (int)(first + step), off, a.n);
    }
    p.unpack(u);
    q.unpack(v);
    add_piece<E, false>(s, u, v, a.sc);
    p = next_p;
    q = next_q;
  }
  return s;
}

// Joins what the wavefronts of a workgroup have, from common maxima; thread 0 gets it. `room`: free before, and after another barrier.
constexpr int kMostWaves = 8;
struct Room { float mx[16], mr[16]; Total total[16]; };   // 16 for the join of segments
__device__ __forceinline__ Total block_total(const Apart& s, Scale sc, Room& room) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  float mx = wave_max(s.mx), mr = wave_max(s.mr);
  if (lane == 0) room.mx[wave] = mx, room.mr[wave] = mr;
  __syncthreads();
  mx = wave_max(lane < waves ? room.mx[lane] : -FLT_MAX);
  mr = wave_max(lane < waves ? room.mr[lane] : -FLT_MAX);
  Total t = total_of<kWave>(s, mx, mr, sc);
  if (lane == 0) room.total[wave] = t;
  __syncthreads();
  if (threadIdx.x == 0)
    for (int i = 1; i < waves; ++i) {
      const Total& o = room.total[i];
      t = Total{t.sx + o.sx, t.sr + o.sr, t.w + o.w, t.h + o.h, mx, mr, fmaxf(t.most, o.most)};
    }
  return t;
}

// A workgroup a row, its wavefronts a piece each in turn. Bound by memory and by vector issue (24 instructions for a pair of logits, two powers of two among them, as 4 each): 4096x50257
// bf16 of which an eighth does not count 140 us in a graph, 5.1 TB/s, where loads alone take 127; 3000x50257 fp32 190 us, 6.3 TB/s. Registers for four wavefronts a unit; fp32, whose packs
// take twice as many, for three (spilled for four: 234 us), bf16 for three 155.
template <typename T, int E, bool NT>
__global__ __launch_bounds__(kMostWaves * kWave, sizeof(T) == 4 ? 3 : 4) void k_kl(Rows<T> a, Outputs o) {
  typedef Piece<T, E> P;
  __shared__ Room room;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    if (a.keep && !a.keep[row]) {
      if (threadIdx.x == 0) write_nothing(o, row);
      continue;
    }
    const T *x = a.x + row * a.ld_x, *r = a.r + row * a.ld_r;
    const int off = pack_offset(x, a.n);
    const Apart s = sums_of<T, E, NT>(a, x, r, off, wave * P::kSize, (int64_t)a.n + off, (int64_t)waves * P::kSize);
    const Total t = block_total(s, a.sc, room);
    if (threadIdx.x == 0) write_row(o, row, t, a.sc);
    if (row + gridDim.x < a.rows) __syncthreads();
  }
}

// Few rows too long for one workgroup: segments of `pieces` pieces, a workgroup of four wavefronts each, and a workgroup a row that joins them.
template <typename T>
__global__ __launch_bounds__(kBlock) void k_kl_split(Rows<T> a, int64_t segments, uint32_t pieces, Total* __restrict__ part) {
  typedef Piece<T, 16> P;
  __shared__ Room room;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  for (int64_t unit = blockIdx.x; unit < a.rows * segments; unit += gridDim.x) {
    const int64_t row = unit / segments, from = (unit - row * segments) * pieces * P::kSize;
    if (a.keep && !a.keep[row]) continue;
    const T *x = a.x + row * a.ld_x, *r = a.r + row * a.ld_r;
    const int off = pack_offset(x, a.n);
    const int64_t end = min(from + (int64_t)pieces * P::kSize, (int64_t)a.n + off);
    const Apart s = sums_of<T, 16, false>(a, x, r, off, from + wave * P::kSize, end, 4 * P::kSize);
    const Total t = block_total(s, a.sc, room);
    if (threadIdx.x == 0) part[unit] = t;
    __syncthreads();
  }
}
template <typename T>
__global__ __launch_bounds__(1024) void k_kl_join(Rows<T> a, Outputs o, int64_t segments, const Total* __restrict__ part) {
  __shared__ Room room;
  const int64_t row = blockIdx.x;   // a workgroup for every row
  if (a.keep && !a.keep[row]) {
    if (threadIdx.x == 0) write_nothing(o, row);
    return;
  }
  float mx = -FLT_MAX, mr = -FLT_MAX;
  for (int64_t i = threadIdx.x; i < segments; i += 1024) {
    mx = fmaxf(mx, part[row * segments + i].mx);
    mr = fmaxf(mr, part[row * segments + i].mr);
  }
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  mx = wave_max(mx);
  mr = wave_max(mr);
  if (lane == 0) room.mx[wave] = mx, room.mr[wave] = mr;
  __syncthreads();
  mx = wave_max(room.mx[lane & 15]);
  mr = wave_max(room.mr[lane & 15]);
  Total t{0.0, 0.0, 0.0, 0.0, mx, mr, -INFINITY};
  for (int64_t i = threadIdx.x; i < segments; i += 1024) add_segment(t, part[row * segments + i], a.sc);
  t = Total{wave_sum(t.sx), wave_sum(t.sr), wave_sum(t.w), wave_sum(t.h), mx, mr, wave_max(t.most)};
  if (lane == 0) room.total[wave] = t;
  __syncthreads();
  if (threadIdx.x != 0) return;
  for (int i = 1; i < 16; ++i) {
    const Total& b = room.total[i];
    t = Total{t.sx + b.sx, t.sr + b.sr, t.w + b.w, t.h + b.h, mx, mr, fmaxf(t.most, b.most)};
  }
  write_row(o, row, t, a.sc);
}

// How rows are shared out.
enum RowForm { kRowWave, kRowBlock, kRowSplit };
struct RowPlan {
  RowForm form;
  int lane, waves;              // logits a lane, wavefronts
  int lanes;                    // a row, kRowWave
  int64_t pieces, segments;     // kRowSplit
};
inline RowPlan plan_rows(int64_t rows, int64_t vocab) {
  const int64_t n = vocab + 7;   // a row counted from its pack
  // us with 64 lanes a row / 16: 1024x100 fp32 4.8 / 4.8, 16384x100 17.4 / 7.0, 100000x300 bf16 91 / 58, 16384x500 fp16 19.1 / 13.9, 4096x500 bf16 7.8 / 6.6, but 1024x500 4.8 / 6.4
  if (n <= 128 || (n <= 512 && rows >= 4096)) return RowPlan{kRowWave, n <= 128 ? 8 : n <= 256 ? 16 : 32, 4, 16, 0, 0};
  if (n <= 2048) return RowPlan{kRowWave, n <= 512 ? 8 : n <= 1024 ? 16 : 32, 4, kWave, 0, 0};
  const int64_t pieces = (n + 1023) / 1024;
  // Few long rows in segments, which costs a launch and a workspace more on the host, some 5 us. us in a graph, a workgroup a row / segments: 1x50257 fp32 12.9 / 8.5, 1x100000 bf16
  // 21 / 8.2, 12x99760 fp32 21.9 / 9.6, 64x100000 bf16 22 / 16.7, 128x70000 18.6 / 19.1, 200x100000 25 / 30, 200x131000 fp32 37 / 42, but 70x262300 bf16 52 / 27.
  if (rows <= 64 ? n > 64 * 1024 : rows < 256 && n > 256 * 1024) {
    const int64_t per = std::clamp<int64_t>(rows * pieces / 2048, 4, 32);
    return RowPlan{kRowSplit, 16, 4, kWave, per, (pieces + per - 1) / per};
  }
  // Wavefronts: one for about five pieces up to four, with fewer than 1024 rows as many as make 4096 in all, up to eight. us with 1 / 2 / 4 / 8: 20000x5000 bf16 85 / 98 / 120,
  // 8192x16000 101 / 100 / 104 / 132, 4096x50257 159 / 164 / 152 / 167, 2048x131000 255 / 198 / 191 / 197, 512x50257 62 / 43 / 27 / 26, 256x32000 38 / 22 / 14 / 12.
  return RowPlan{kRowBlock, 16, (int)std::max(std::clamp<int64_t>((pieces + 4) / 5, 1, 4), std::min<int64_t>({kMostWaves, pieces, 4096 / rows})), kWave, 0, 0};
}

// The gradients, element by element, with d = scale ((x - r) - (mx - mr)) and g = dkl:
//   dx = g scale p (d - mean d under p),   dr = g scale (q - p)
// Bound by memory: two reads and one or two writes of the logits. Laid out as the gradient of the token log probabilities. Reads and writes go past the cache whatever the size. us together
// with a sum that reads dx, so / stores by the cache / loads too: 4096x50257 bf16 339 / 352 / 353; smaller ones lose by it, 1024x50257 91 / 85 / 98, 512x50257 48 / 45 / 46, 64x50257 13.8 / 13.1 / 12.4.
template <typename T, bool DX, bool DR, int G>
__global__ __launch_bounds__(kBlock) void k_kl_back(Rows<T> a, float lift, float drop, const float* __restrict__ stats, const float* __restrict__ dkl, T* dx, int64_t ld_dx,
                                                    T* dr, int64_t ld_dr) {
  typedef typename Pack<T>::type pack;
  constexpr int V = Pack<T>::n, kPacks = 2, kSpan = kPacks * G * V, kRows = kBlock / G;
  const int lane = threadIdx.x % G, vocab = (int)a.n;
  for (int64_t row = (int64_t)blockIdx.y * kRows + threadIdx.x / G; row < a.rows; row += (int64_t)gridDim.y * kRows) {
    const T *x = a.x + row * a.ld_x, *r = a.r + row * a.ld_r;
    T *out_x = DX ? dx + row * ld_dx : nullptr, *out_r = DR ? dr + row * ld_dr : nullptr;
    const float* s = stats + 5 * row;
    const float mx = s[0], ln_sx = s[1], mr = s[2], ln_sr = s[3], mean = s[4], g = a.keep && !a.keep[row] ? 0.f : dkl[row];
    const bool zero = g == 0.f || (mx == -INFINITY && ln_sx == -INFINITY);
    const bool r_empty = mr == -INFINITY;
    const float A = zero ? 0.f : mean < INFINITY ? g * a.scale : NAN;   // an infinite mean or none makes the whole row NaN
    // d - mean under an unlikely token may be beyond the type where the token's gradient is not: for dx a power of two goes from the scale over to g
    float Ax = A, scale_d = a.scale, mean_d = mean;
    if (lift != 1.f && fabsf(A * lift) < INFINITY) Ax *= lift, scale_d *= drop, mean_d *= drop;
    // d by way of x - r, or of the maxima where a constant lies between the rows
    const bool close_by = fabsf(mx - mr) <= kOffset;
    const float ux = close_by ? 0.f : mx, ur = close_by ? 0.f : mr, dm = close_by ? mx - mr : 0.f;
    auto gradient = [&](float u, float v, float& gx, float& gr) {
      const float p = exp2_hw((a.scale * (u - mx) - ln_sx) * kLog2e);
      if (DX) gx = Ax * (p * __builtin_amdgcn_fmed3f(__builtin_fmaf(((u - ux) - (v - ur)) - dm, scale_d, -mean_d), -FLT_MAX, FLT_MAX));   // finite, for p may be 0
      if (DR) gr = A * ((r_empty ? 0.f : exp2_hw((a.scale * (v - mr) - ln_sr) * kLog2e)) - p);
    };
    const T* grid_row = DX ? out_x : out_r;
    const int off = (int)((uintptr_t)grid_row / sizeof(T) % V);
    for (int64_t first = (int64_t)((blockIdx.x + blockIdx.y / 64) % gridDim.x) * kSpan; first < (int64_t)vocab + off; first += (int64_t)gridDim.x * kSpan) {
      const int begin = (int)first + lane * V - off;
      pack in_x[kPacks], in_r[kPacks];
#pragma unroll
      for (int j = 0; j < kPacks; ++j) {
        const int k = begin + j * G * V;
        if (!zero && k >= 0 && k <= vocab - V) {
          in_x[j] = __builtin_nontemporal_load((const pack*)(x + k));
          in_r[j] = __builtin_nontemporal_load((const pack*)(r + k));
        }
      }
#pragma unroll
      for (int j = 0; j < kPacks; ++j) {
        const int k = begin + j * G * V;
        if (k >= 0 && k <= vocab - V) {
          pack o_x = {}, o_r = {};
          if (!zero) {
#pragma unroll
            for (int e = 0; e < V; ++e) {
              float gx = 0.f, gr = 0.f;
              gradient(to_f32(in_x[j][e]), to_f32(in_r[j][e]), gx, gr);
              o_x[e] = from_f32<T>(gx);
              o_r[e] = from_f32<T>(gr);
            }
          }
          if (DX) __builtin_nontemporal_store(o_x, (pack*)(out_x + k));
          if (DR) __builtin_nontemporal_store(o_r, (pack*)(out_r + k));
        } else if (k > -V && k < vocab) {
          for (int i = max(k, 0); i < min(k + V, vocab); ++i) {
            float gx = 0.f, gr = 0.f;
            if (!zero) gradient(to_f32(x[i]), to_f32(r[i]), gx, gr);
            if (DX) out_x[i] = from_f32<T>(gx);
            if (DR) out_r[i] = from_f32<T>(gr);
          }
        }
      }
    }
  }
}

lopt_status check_logits(const void* logits, int64_t ld, const void* ref, int64_t ld_ref, int64_t rows, int64_t vocab, uint32_t type, float scale) {
  LOPT_CHECK(check_type("type", type));
  LOPT_CHECK(check_matrix(rows, vocab, "vocab"));
  if (vocab > LOPT_VOCAB_MAX) return fail_call(LOPT_ESHAPE, "vocab=%lld is above %d", (long long)vocab, LOPT_VOCAB_MAX);
  LOPT_CHECK(check_ld("ld", rows, vocab, ld, false));
  LOPT_CHECK(check_ld("ld_ref", rows, vocab, ld_ref, false));
  if (!(scale > 0.f) || std::isinf(scale)) return fail_call(LOPT_EINVAL, "scale must be finite and > 0");
  LOPT_CHECK(check_array("logits", logits, type_bytes(type), rows > 0));
  return check_array("ref", ref, type_bytes(type), rows > 0);
}

}  // namespace
}  // namespace lopt

using namespace lopt;

extern "C" {

size_t lopt_token_kl_workspace(int64_t rows, int64_t vocab) {
  if (rows <= 0 || vocab <= 0 || rows > 0x7fffffffLL || vocab > 0x7fffffffLL) return 0;
  const RowPlan plan = plan_rows(rows, vocab);
  return plan.form == kRowSplit ? (size_t)rows * (size_t)plan.segments * sizeof(Total) : 0;
}

lopt_status lopt_token_kl(const void* logits, int64_t ld, const void* ref, int64_t ld_ref, const uint8_t* mask, int64_t rows, int64_t vocab, uint32_t type,
                          float scale, float* kl, float* stats, void* workspace, size_t workspace_bytes, void* hip_stream) {
  LOPT_CHECK(check_logits(logits, ld, ref, ld_ref, rows, vocab, type, scale));
  LOPT_CHECK(check_array("kl", kl, 4, rows > 0));
  LOPT_CHECK(check_array("stats", stats, 4, rows > 0));
  LOPT_CHECK(check_workspace(workspace, workspace_bytes, lopt_token_kl_workspace(rows, vocab)));
  if (rows == 0) return LOPT_OK;
  const Outputs o{kl, stats};
  const RowPlan plan = plan_rows(rows, vocab);
  hipStream_t stream = (hipStream_t)hip_stream;
  with_type(type, [&](auto t) {
    using T = decltype(t);
    const Rows<T> a{(const T*)logits, (const T*)ref, ld, ld_ref, rows, (uint32_t)vocab, scale, scale_of(std::fmin(scale * kLog2e, FLT_MAX)), mask};
    const dim3 block(plan.waves * kWave);
    if (plan.form == kRowWave) {
      // so many rows that there would be 2^32 threads: as large batches as there can be
      const int lanes = plan.lanes, batch = rows >> 26 ? lanes : (int)std::clamp<int64_t>(rows * lanes / kWave / 8192, 1, 16), per = kBlock / lanes * batch;
      auto kernel = lanes == 16 ? plan.lane == 8 ? k_kl_short<T, 8, 16> : plan.lane == 16 ? k_kl_short<T, 16, 16> : k_kl_short<T, 32, 16>
                                : plan.lane == 8 ? k_kl_short<T, 8, 64> : plan.lane == 16 ? k_kl_short<T, 16, 64> : k_kl_short<T, 32, 64>;
      hipLaunchKernelGGL(kernel, dim3((unsigned)((rows + per - 1) / per)), block, 0, stream, a, batch, o);
    } else if (plan.form == kRowBlock) {
      // what the Infinity Cache cannot hold is not left there: 4096x50257 bf16 157 -> 150 us, 20000x5000 87 -> 84, 3000x50257 fp32 212 -> 189, but 1024x50257, which fits, 43 -> 44.5
      const bool large = 2 * rows * vocab * (int64_t)sizeof(T) > kCacheBytes;
      auto kernel = large ? k_kl<T, 16, true> : k_kl<T, 16, false>;
      hipLaunchKernelGGL(kernel, dim3((unsigned)std::min<int64_t>(rows, 1 << 20)), block, 0, stream, a, o);
    } else {
      Total* part = (Total*)workspace;
      hipLaunchKernelGGL(k_kl_split<T>, dim3((unsigned)std::min<int64_t>(rows * plan.segments, 1 << 22)), block, 0, stream, a, plan.segments, (uint32_t)plan.pieces, part);
      hipLaunchKernelGGL(k_kl_join<T>, dim3((unsigned)rows), dim3(1024), 0, stream, a, o, plan.segments, (const Total*)part);
    }
  });
  return launch_status("lopt_token_kl");
}

lopt_status lopt_token_kl_backward(const void* logits, int64_t ld, const void* ref, int64_t ld_ref, const uint8_t* mask, const float* stats, const float* dkl,
                                   void* dlogits, int64_t ld_d, void* dref, int64_t ld_dref, int64_t rows, int64_t vocab, uint32_t type, float scale,
                                   void* hip_stream) {
  LOPT_CHECK(check_logits(logits, ld, ref, ld_ref, rows, vocab, type, scale));
  LOPT_CHECK(check_array("stats", stats, 4, rows > 0));
  LOPT_CHECK(check_array("dkl", dkl, 4, rows > 0));
  LOPT_CHECK(check_array("dlogits", dlogits, type_bytes(type), false));
  LOPT_CHECK(check_array("dref", dref, type_bytes(type), false));
  if (dlogits) LOPT_CHECK(check_ld("ld_d", rows, vocab, ld_d, true));
  if (dref) LOPT_CHECK(check_ld("ld_dref", rows, vocab, ld_dref, true));
  if (dlogits && dlogits == dref && rows > 0) return fail_call(LOPT_EINVAL, "dlogits and dref are the same memory");
  const struct { const char* name; const void* out; int64_t ld; } outs[2] = {{"dlogits", dlogits, ld_d}, {"dref", dref, ld_dref}};
  for (const auto& q : outs)
    if (q.out && rows > 1 && ((q.out == logits && q.ld != ld) || (q.out == ref && q.ld != ld_ref)))
      return fail_call(LOPT_EINVAL, "%s is an input, but its ld is not that input's", q.name);
  if (rows == 0 || (!dlogits && !dref)) return LOPT_OK;
  with_type(type, [&](auto t) {
    using T = decltype(t);
    const Rows<T> a{(const T*)logits, (const T*)ref, ld, ld_ref, rows, (uint32_t)vocab, scale, scale_of(std::fmin(scale * kLog2e, FLT_MAX)), mask};
    const int64_t packs = (vocab + 2 * Pack<T>::n - 2) / Pack<T>::n;   // that a row may touch
    const float lift = scale > 1.f ? std::ldexp(1.f, std::min(std::ilogb(scale) + 1, 16)) : 1.f;
    auto launch = [&](auto g) {
      constexpr int G = decltype(g)::value, kSpan = 2 * G;
      const int64_t spans = (packs + kSpan - kSpan / 8) / kSpan;
      const dim3 grid((unsigned)std::clamp<int64_t>(spans, 1, 1024), (unsigned)std::min<int64_t>((rows + kBlock / G - 1) / (kBlock / G), 65535));
      auto kernel = !dref ? k_kl_back<T, true, false, G> : !dlogits ? k_kl_back<T, false, true, G> : k_kl_back<T, true, true, G>;
      hipLaunchKernelGGL(kernel, grid, dim3(kBlock), 0, (hipStream_t)hip_stream, a, lift, 1.f / lift, stats, dkl, (T*)dlogits, ld_d, (T*)dref, ld_dref);
    };
    if (packs <= 2 * 16) launch(std::integral_constant<int, 16>{});
    else if (packs <= 2 * 64) launch(std::integral_constant<int, 64>{});
    else launch(std::integral_constant<int, kBlock>{});
  });
  return launch_status("lopt_token_kl_backward");
}

}  // extern "C"
