// Dropout of rows, the mask formed where it is needed and stored nowhere: y = x / (1 - p) where the element's word of the generator stays, else 0.
// The gradient is the same call on the gradient. Bound by memory, one read and one write.
#include <algorithm>

#include "lopt_flat.h"
#include "lopt_random.h"

namespace lopt {
namespace {

// A workgroup takes kChunk neighbouring packs of 16 bytes, four a thread.
constexpr int kPacks = 4, kChunk = kPacks * kBlock;

template <typename T>
__global__ __launch_bounds__(kBlock) void k_dropout(const T* x, int64_t ld_x, T* y, int64_t ld_y, Flat f, Dropout d) {
  constexpr int V = Pack<T>::n;
  typedef typename Pack<T>::type pack;
  const Words words(d);
  const uint32_t cols = f.cols;
  for (int64_t first = (int64_t)blockIdx.x * kChunk; first < f.total; first += (int64_t)gridDim.x * kChunk) {
    const Chunk chunk(f, first);
    pack in[kPacks];
    int64_t row[kPacks];
    uint32_t col[kPacks];
    bool have[kPacks];
#pragma unroll
    for (int j = 0; j < kPacks; ++j) {
      have[j] = chunk.at(f, V, j * kBlock + threadIdx.x, row[j], col[j]);
      in[j] = pack{};
      if (have[j] && col[j] + V <= cols) in[j] = __builtin_nontemporal_load((const pack*)(x + row[j] * ld_x + col[j]));
    }
#pragma unroll
    for (int j = 0; j < kPacks; ++j) {
      if (!have[j]) continue;
      const uint32_t bits = d.on ? words.stay<V>((uint32_t)row[j], col[j]) : ~0u;
      T* out = y + row[j] * ld_y + col[j];
      if (col[j] + V <= cols) {
        pack o;
#pragma unroll
        for (int e = 0; e < V; ++e) o[e] = from_f32<T>(where_bit(bits, e, to_f32(in[j][e]) * d.scale));
        __builtin_nontemporal_store(o, (pack*)out);
      } else {
        const T* p = x + row[j] * ld_x + col[j];
        for (uint32_t e = 0; e < cols - col[j]; ++e) out[e] = bits >> e & 1 ? from_f32<T>(to_f32(p[e]) * d.scale) : (T)0.f;
      }
    }
  }
}

}  // namespace
}  // namespace lopt

using namespace lopt;

extern "C" lopt_status lopt_dropout(const void* x, int64_t ld_x, void* y, int64_t ld_y, int64_t rows, int64_t cols, uint32_t type, float p, uint64_t seed,
                                    const uint64_t* seed_device, uint64_t offset, void* hip_stream) {
  Dropout d{};
  d.seed = seed;
  d.offset = offset;
  LOPT_CHECK(check_type("type", type));
  LOPT_CHECK(check_matrix(rows, cols, "cols"));
  LOPT_CHECK(check_dropout(p, seed_device, &d));
  LOPT_CHECK(check_ld("ld_x", rows, cols, ld_x, y == x));
  LOPT_CHECK(check_ld("ld_y", rows, cols, ld_y, true));
  LOPT_CHECK(check_array("x", x, type_bytes(type), rows > 0));
  LOPT_CHECK(check_array("y", y, type_bytes(type), rows > 0));
  if (y == x && ld_y != ld_x && rows > 1) return fail_call(LOPT_EINVAL, "y is x, but ld_y is not ld_x");
  if (rows == 0) return LOPT_OK;
  with_type(type, [&](auto t) {
    using T = decltype(t);
    const Flat f = flat_of(rows, cols, Pack<T>::n);
    const unsigned blocks = (unsigned)std::min<int64_t>((f.total + kChunk - 1) / kChunk, 1 << 22);
    hipLaunchKernelGGL(k_dropout<T>, dim3(blocks), dim3(kBlock), 0, (hipStream_t)hip_stream, (const T*)x, ld_x, (T*)y, ld_y, f, d);
  });
  return launch_status("lopt_dropout");
}
