// Global gradient norm over a list of tensors, and clipping: norm = sqrt(sum g^2), out = min(1, max_norm / (norm + eps)) g.
// Two sweeps over the list with the norm between them; the list travels in the kernels' arguments, so that a call uploads and keeps
// nothing.
#include <cmath>

#include "lopt_ops.h"

namespace lopt {
namespace {

constexpr int kChunk = 16384;     // elements one workgroup takes of one tensor
constexpr int kBatch = 160;       // tensors of one launch: 24 bytes each, within the 4 KB of kernel arguments

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
};

__device__ __forceinline__ void store_as(void* p, int64_t i, uint32_t type, float v) {
  if (type == LOPT_F32) ((float*)p)[i] = v;
  else if (type == LOPT_BF16) ((bf16_t*)p)[i] = from_f32<bf16_t>(v);
  else ((f16_t*)p)[i] = from_f32<f16_t>(v);
}

// Which tensor of the batch this workgroup's chunk belongs to, and the chunk's elements.
struct Chunk { int tensor; int64_t at; int count; };
__device__ __forceinline__ Chunk find_chunk(const ClipBatch& b) {
  const int below = threadIdx.x < (unsigned)b.n ? b.t[threadIdx.x].first <= blockIdx.x : 0;
  const int k = __syncthreads_count(below) - 1;
  const uint32_t c = blockIdx.x - b.t[k].first;
  const bool last = k + 1 == b.n ? blockIdx.x + 1 == gridDim.x : blockIdx.x + 1 == b.t[k + 1].first;
  return Chunk{k, (int64_t)c * kChunk, last ? (int)b.t[k].last + 1 : kChunk};
}

__global__ __launch_bounds__(kBlock) void k_clip_squares(const ClipBatch b, double* __restrict__ part) {
  __shared__ double red[4];
  const Chunk c = find_chunk(b);
  const uint32_t type = b.t[c.tensor].type;
  double s = 0.0;
  for (int i = threadIdx.x; i < c.count; i += kBlock) {
    const double g = (double)load_as(b.t[c.tensor].in, c.at + i, type);
    s += g * g;
  }
  s = block_sum<4>(s, red);
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}

// norm[0] for the caller, coef[0] for the second sweep.
__global__ __launch_bounds__(kBlock) void k_clip_norm(const double* __restrict__ part, int64_t n, float max_norm, float* __restrict__ norm,
                                                      float* __restrict__ coef) {
  __shared__ double red[4];
  double s = 0.0;
  for (int64_t i = threadIdx.x; i < n; i += kBlock) s += part[i];
  s = block_sum<4>(s, red);
  if (threadIdx.x == 0) {
    const float v = (float)sqrt(s);
    norm[0] = v;
    const float c = max_norm / (v + LOPT_CLIP_EPS);
    coef[0] = c > 1.f ? 1.f : c;   // NaN stays
  }
}

__global__ __launch_bounds__(kBlock) void k_clip_scale(const ClipBatch b, const float* __restrict__ coef) {
  const Chunk c = find_chunk(b);
  const ClipTensor& t = b.t[c.tensor];
  const float f = coef[0];
  if (f == 1.f && t.in == t.out) return;
  for (int i = threadIdx.x; i < c.count; i += kBlock) store_as(t.out, c.at + i, t.out_type, f * load_as(t.in, c.at + i, t.type));
}

int64_t chunks_of(int64_t count) { return (count + kChunk - 1) / kChunk; }

}  // namespace
}  // namespace lopt

using namespace lopt;

extern "C" {

size_t lopt_clip_workspace(size_t n, const int64_t* counts) {
  size_t chunks = 0;
  for (size_t i = 0; counts && i < n; ++i) chunks += counts[i] > 0 ? (size_t)chunks_of(counts[i]) : 0;
  return 16 + chunks * sizeof(double);
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
  if (chunks >= (int64_t)1 << 31) return fail_call(LOPT_ESHAPE, "more than 2^45 elements");
  LOPT_CHECK(check_workspace(workspace, workspace_bytes, 16 + (size_t)chunks * sizeof(double)));
  hipStream_t stream = (hipStream_t)hip_stream;
  float* coef = (float*)workspace;
  double* part = (double*)((char*)workspace + 16);
  for (int pass = 0; pass < (out ? 2 : 1); ++pass) {
    size_t i = 0;
    int64_t done = 0;
    while (i < n) {
      ClipBatch b;
      b.n = 0;
      int64_t here = 0;
      for (; i < n && b.n < kBatch; ++i) {
        if (counts[i] == 0) continue;
        const int64_t c = chunks_of(counts[i]);
        if (here > 0 && here + c > 0x7fffffff / kBlock) break;   // a grid's threads fit 31 bits
        b.t[b.n++] = ClipTensor{grads[i], out ? out[i] : nullptr, (uint32_t)here, (uint32_t)(counts[i] - (c - 1) * kChunk - 1), types[i], out ? out_types[i] : 0};
        here += c;
      }
      if (!here) break;
      if (pass == 0) hipLaunchKernelGGL(k_clip_squares, dim3((unsigned)here), dim3(kBlock), 0, stream, b, part + done);
      else hipLaunchKernelGGL(k_clip_scale, dim3((unsigned)here), dim3(kBlock), 0, stream, b, (const float*)coef);
      done += here;
    }
    if (pass == 0) hipLaunchKernelGGL(k_clip_norm, dim3(1), dim3(kBlock), 0, stream, (const double*)part, chunks, max_norm, norm, coef);
  }
  return launch_status("lopt_clip_grads");
}

}  // extern "C"
