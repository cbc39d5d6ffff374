// Global gradient norm over a list of tensors, and clipping: norm = sqrt(sum g^2), out = min(1, max_norm / (norm + eps)) g.
// Two sweeps over the list with the norm between them; the list travels in the kernels' arguments, so that a call uploads and keeps
// nothing.
#include <algorithm>
#include <cmath>
#include <memory>
#include <new>

#include "lopt_ops.h"

namespace lopt {
namespace {

constexpr int kChunk = 4096;      // elements of one tensor that a workgroup takes at a time: 16 a thread
constexpr int kBatch = 160;       // tensors of one launch: 24 bytes each, within the 4 KB of kernel arguments
constexpr int kGrid = 2048;       // workgroups that share out a list, eight a compute unit; each leaves one partial sum

struct ClipTensor {
  const void* in;
  void* out;
  uint32_t first;      // this tensor's first chunk among those of the launch
  uint32_t last : 16;  // elements of its last chunk, minus one
  uint32_t type : 4, out_type : 4;
};
struct ClipBatch {
  ClipTensor t[kBatch];
  int n;
  uint32_t chunks;     // of all of them
};

// A workgroup's neighbouring chunks of the batch, and the tensor that the one at hand belongs to.
struct Walk {
  uint32_t begin, end;
  int k;
  __device__ __forceinline__ Walk(const ClipBatch& b, bool backwards) {
    begin = (uint32_t)((uint64_t)b.chunks * blockIdx.x / gridDim.x);
    end = (uint32_t)((uint64_t)b.chunks * (blockIdx.x + 1) / gridDim.x);
    const uint32_t at = backwards ? end - 1 : begin;   // every workgroup has a chunk
    k = __syncthreads_count(threadIdx.x < (unsigned)b.n && b.t[threadIdx.x].first <= at) - 1;
  }
  __device__ __forceinline__ void seek(const ClipBatch& b, uint32_t chunk) {
    while (k + 1 < b.n && b.t[k + 1].first <= chunk) ++k;
    while (b.t[k].first > chunk) --k;
  }
  __device__ __forceinline__ static int count(const ClipBatch& b, int k, uint32_t chunk) {
    const uint32_t next = k + 1 == b.n ? b.chunks : b.t[k + 1].first;
    return chunk + 1 == next ? (int)b.t[k].last + 1 : kChunk;
  }
};

// A thread's 16 elements of a chunk of `count`, in groups of V neighbours, 256 V apart.
template <typename T, int V, bool NT>
__device__ __forceinline__ void load_chunk(const T* p, int count, float (&v)[16]) {
  typedef T vec __attribute__((ext_vector_type(V), aligned(sizeof(T))));
#pragma unroll
  for (int j = 0; j < 16 / V; ++j) {
    const int k = (j * kBlock + (int)threadIdx.x) * V;
    if (k + V <= count) {
      const vec x = NT ? __builtin_nontemporal_load((const vec*)(p + k)) : *(const vec*)(p + k);
#pragma unroll
      for (int e = 0; e < V; ++e) v[j * V + e] = to_f32(x[e]);
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) v[j * V + e] = k + e < count ? to_f32(p[k + e]) : 0.f;
    }
  }
}
template <typename T, int V>
__device__ __forceinline__ void store_chunk(T* p, int count, const float (&v)[16]) {
  typedef T vec __attribute__((ext_vector_type(V), aligned(sizeof(T))));
#pragma unroll
  for (int j = 0; j < 16 / V; ++j) {
    const int k = (j * kBlock + (int)threadIdx.x) * V;
    if (k + V <= count) {
      vec x;
#pragma unroll
      for (int e = 0; e < V; ++e) x[e] = from_f32<T>(v[j * V + e]);
      __builtin_nontemporal_store(x, (vec*)(p + k));
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e)
        if (k + e < count) p[k + e] = from_f32<T>(v[j * V + e]);
    }
  }
}
template <int V, bool NT>
__device__ __forceinline__ void load_chunk_as(const void* p, int64_t at, uint32_t type, int count, float (&v)[16]) {
  if (type == LOPT_F32) load_chunk<float, V, NT>((const float*)p + at, count, v);
  else if (type == LOPT_BF16) load_chunk<bf16_t, V, NT>((const bf16_t*)p + at, count, v);
  else load_chunk<f16_t, V, NT>((const f16_t*)p + at, count, v);
}

__global__ __launch_bounds__(kBlock) void k_clip_squares(const ClipBatch b, double* __restrict__ part) {
  __shared__ double red[4];
  Walk w(b, false);
  double s = 0.0;
  for (uint32_t c = w.begin; c < w.end; ++c) {
    w.seek(b, c);
    const int count = Walk::count(b, w.k, c);
    const int64_t at = (int64_t)(c - b.t[w.k].first) * kChunk;
    float v[16];
    if (b.t[w.k].type == LOPT_F32) load_chunk<float, 4, false>((const float*)b.t[w.k].in + at, count, v);
    else load_chunk_as<8, false>(b.t[w.k].in, at, b.t[w.k].type, count, v);
#pragma unroll
    for (int i = 0; i < 16; ++i) s += (double)v[i] * (double)v[i];
  }
  s = block_sum<4>(s, red);
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}

// The norm from the partial sums of every launch of the first sweep, in every thread, and the factor.
struct Norm { float norm, factor; };
__device__ __forceinline__ Norm join_norm(const double* __restrict__ part, int parts, float max_norm, double* red) {
  double s = 0.0;
  for (int i = threadIdx.x; i < parts; i += kBlock) s += part[i];
  const double v = sqrt(block_sum<4>(s, red)), c = (double)max_norm / (v + (double)LOPT_CLIP_EPS);
  return Norm{(float)v, c > 1.0 ? 1.f : (float)c};   // NaN stays
}
__global__ __launch_bounds__(kBlock) void k_clip_norm(const double* __restrict__ part, int parts, float* __restrict__ norm) {
  __shared__ double red[4];
  const Norm n = join_norm(part, parts, 0.f, red);
  if (threadIdx.x == 0) norm[0] = n.norm;
}

// V neighbours a lane: 16 bytes of the wider type, so that every access of a wavefront is one run of memory.
template <int V>
__device__ __forceinline__ void scale_chunk(const ClipTensor& t, int64_t at, int count, float f) {
  float v[16];
  load_chunk_as<V, true>(t.in, at, t.type, count, v);
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] *= f;
  if (t.out_type == LOPT_F32) store_chunk<float, V>((float*)t.out + at, count, v);
  else if (t.out_type == LOPT_BF16) store_chunk<bf16_t, V>((bf16_t*)t.out + at, count, v);
  else store_chunk<f16_t, V>((f16_t*)t.out + at, count, v);
}

// Every workgroup joins the partial sums for itself, which takes the place of a launch in between, and goes through its chunks from the last to
// the first: what the first sweep read last is still in the Infinity Cache (355 M elements fp32 771 -> 747 us). That is also why the
// first sweep's loads are ordinary ones, and this one's loads and stores nontemporal: what will not be read again pushes nothing out. us, ordinary / stores
// nontemporal / stores and this sweep's loads / all: 86 M fp32 212 / 182 / 165 / 188, 54 M bf16 to fp32 105 / 79 / 74 / 93, 20 M bf16 31 / 28 / 26 / 31. Both sweeps
// are bound by memory: 86 M fp32 are two reads and one write of 344 MB, 6.2 TB/s.
__global__ __launch_bounds__(kBlock) void k_clip_scale(const ClipBatch b, const double* __restrict__ part, int parts, float max_norm, float* __restrict__ norm) {
  __shared__ double red[4];
  const Norm n = join_norm(part, parts, max_norm, red);
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) norm[0] = n.norm;
  const float f = n.factor;
  Walk w(b, true);
  for (uint32_t c = w.end; c-- > w.begin;) {
    w.seek(b, c);
    const ClipTensor& t = b.t[w.k];
    if (f == 1.f && t.in == t.out) continue;
    const int count = Walk::count(b, w.k, c);
    const int64_t at = (int64_t)(c - t.first) * kChunk;
    if (t.type == LOPT_F32 || t.out_type == LOPT_F32) scale_chunk<4>(t, at, count, f);
    else scale_chunk<8>(t, at, count, f);
  }
}

int64_t chunks_of(int64_t count) { return (count + kChunk - 1) / kChunk; }
// Workgroups of a launch that has `here` of the list's `all` chunks: its share of kGrid, but no fewer than kLeast (1346 M elements with 2000 tiny tensors,
// twelve launches of those: 7.7 -> 3.6 ms).
constexpr int kLeast = 128;
int grid_of(int64_t here, int64_t all) { return (int)std::min<int64_t>(here, std::max<int64_t>((here * kGrid + all - 1) / all, kLeast)); }
// Partial sums of n tensors at most: kGrid and, for rounding up, kLeast for every launch; no more than one a chunk. A launch ends after kBatch tensors, or
// with more than 0.75 * 2^30 chunks.
size_t most_parts(size_t n, int64_t chunks) { return (size_t)std::min<int64_t>(chunks, kGrid + kLeast * ((int64_t)((n + kBatch - 1) / kBatch) + (chunks >> 29))); }

// Workgroups read and write the tensors in no order: an output that shares memory with another one, or with a gradient that is not its own, would come
// out differently from call to call. Lists whose outputs lie in ascending order, as in one flat buffer, are not sorted.
lopt_status check_overlap(size_t n, const int64_t* counts, const void* const* grads, const uint32_t* types, void* const* out, const uint32_t* out_types) {
  struct Span { uintptr_t begin, end; };
  const std::unique_ptr<Span[]> spans(new (std::nothrow) Span[n]);
  if (!spans) return fail_call(LOPT_ENOMEM, "out of host memory");
  size_t m = 0;
  bool sorted = true;
  for (size_t i = 0; i < n; ++i) {
    if (counts[i] == 0) continue;
    const uintptr_t begin = (uintptr_t)out[i];
    sorted = sorted && (m == 0 || spans[m - 1].begin < begin);
    spans[m++] = Span{begin, begin + (uintptr_t)counts[i] * type_bytes(out_types[i])};
  }
  if (!sorted) std::sort(spans.get(), spans.get() + m, [](const Span& a, const Span& b) { return a.begin < b.begin; });
  for (size_t k = 1; k < m; ++k)
    if (spans[k].begin < spans[k - 1].end) return fail_call(LOPT_EINVAL, "two outputs overlap");
  for (size_t i = 0; i < n; ++i) {
    if (counts[i] == 0 || out[i] == grads[i]) continue;
    const uintptr_t begin = (uintptr_t)grads[i], end = begin + (uintptr_t)counts[i] * type_bytes(types[i]);
    const Span* next = std::lower_bound(spans.get(), spans.get() + m, end, [](const Span& a, uintptr_t e) { return a.begin < e; });
    if (next != spans.get() && next[-1].end > begin) return fail_call(LOPT_EINVAL, "tensor %zu: an output overlaps this gradient", i);
  }
  return LOPT_OK;
}

}  // namespace
}  // namespace lopt

using namespace lopt;

extern "C" {

size_t lopt_clip_workspace(size_t n, const int64_t* counts) {
  int64_t chunks = 0;
  for (size_t i = 0; counts && i < n; ++i) chunks += counts[i] > 0 && counts[i] < (int64_t)1 << 40 ? chunks_of(counts[i]) : 0;
  return std::max<size_t>(16, most_parts(n, chunks) * sizeof(double));
}

lopt_status lopt_clip_grads(size_t n, const int64_t* counts, const void* const* grads, const uint32_t* types, void* const* out,
                            const uint32_t* out_types, float max_norm, float* norm, void* workspace, size_t workspace_bytes,
                            void* hip_stream) {
  LOPT_CHECK(check_array("norm", norm, 4, true));
  if (!(max_norm >= 0.f)) return fail_call(LOPT_EINVAL, "max_norm must be >= 0");
  if (n > 0 && (!counts || !grads || !types)) return fail_call(LOPT_EINVAL, "counts_host, grads_host or types_host is null");
  if (n > 0 && out && !out_types) return fail_call(LOPT_EINVAL, "out_types_host is null");
  if (n > (size_t)1 << 24) return fail_call(LOPT_EINVAL, "too many tensors");
  int64_t chunks = 0;
  for (size_t i = 0; i < n; ++i) {
    if (counts[i] < 0 || counts[i] >= (int64_t)1 << 40) return fail_call(LOPT_ESHAPE, "counts_host[%zu]=%lld outside [0, 2^40)", i, (long long)counts[i]);
    if (types[i] > LOPT_F16 || (out && out_types[i] > LOPT_F16)) return fail_call(LOPT_EINVAL, "tensor %zu: not a lopt_type", i);
    if (counts[i] == 0) continue;
    if (!grads[i] || (out && !out[i])) return fail_call(LOPT_EINVAL, "tensor %zu: null pointer", i);
    if ((uintptr_t)grads[i] % type_bytes(types[i]) || (out && (uintptr_t)out[i] % type_bytes(out_types[i])))
      return fail_call(LOPT_EINVAL, "tensor %zu is not aligned to its elements", i);
    if (out && out[i] == grads[i] && types[i] != out_types[i]) return fail_call(LOPT_EINVAL, "tensor %zu: in place, but of another type", i);
    chunks += chunks_of(counts[i]);
  }
  if (n > 0 && out) LOPT_CHECK(check_overlap(n, counts, grads, types, out, out_types));
  LOPT_CHECK(check_workspace(workspace, workspace_bytes, std::max<size_t>(16, most_parts(n, chunks) * sizeof(double))));
  hipStream_t stream = (hipStream_t)hip_stream;
  double* part = (double*)workspace;
  int parts = 0;
  for (int pass = 0; pass < (out ? 2 : 1); ++pass) {
    for (size_t i = 0; i < n;) {
      ClipBatch b;
      b.n = 0;
      int64_t here = 0;
      for (; i < n && b.n < kBatch; ++i) {
        if (counts[i] == 0) continue;
        const int64_t c = chunks_of(counts[i]);
        if (here + c > (int64_t)1 << 30) break;   // one tensor has 2^28 at most
        b.t[b.n++] = ClipTensor{grads[i], out ? out[i] : nullptr, (uint32_t)here, (uint32_t)(counts[i] - (c - 1) * kChunk - 1), types[i], out ? out_types[i] : 0};
        here += c;
      }
      if (!here) break;
      b.chunks = (uint32_t)here;
      const dim3 grid(grid_of(here, chunks));
      if (pass == 0) {
        hipLaunchKernelGGL(k_clip_squares, grid, dim3(kBlock), 0, stream, b, part + parts);
        parts += grid.x;
      } else {
        hipLaunchKernelGGL(k_clip_scale, grid, dim3(kBlock), 0, stream, b, (const double*)part, parts, max_norm, norm);
        norm = nullptr;   // the first launch writes it
      }
    }
  }
  if (norm) hipLaunchKernelGGL(k_clip_norm, dim3(1), dim3(kBlock), 0, stream, (const double*)part, parts, norm);
  return launch_status("lopt_clip_grads");
}

}  // extern "C"
