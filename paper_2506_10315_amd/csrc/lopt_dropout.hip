// Dropout of rows, the mask formed where it is needed and stored nowhere: y = x / (1 - p) where the element's word of the generator stays, else 0.
// The gradient is the same call on the gradient. Bound by memory, one read and one write.
#include <algorithm>

#include "lopt_random.h"

namespace lopt {
namespace {

// A row's packs of 16 bytes are counted from its first element, those of all rows through; a workgroup takes kChunk neighbouring packs, four a thread, which
// may be of many short rows or a part of a long one. `magic`: 2^32 / packs rounded up, with which a 32-bit product divides what a workgroup has to
// divide (below packs + kChunk) exactly while packs <= 2^15; longer rows have the quotient 0 or 1.
constexpr int kPacks = 4, kChunk = kPacks * kBlock;
constexpr uint32_t kShortPacks = 1 << 15;

template <typename T>
__global__ __launch_bounds__(kBlock) void k_dropout(const T* x, int64_t ld_x, T* y, int64_t ld_y, int64_t total, uint32_t packs, uint32_t magic, uint32_t cols, Dropout d) {
  constexpr int V = Pack<T>::n;
  typedef typename Pack<T>::type pack;
  const Words words(d);
  for (int64_t first = (int64_t)blockIdx.x * kChunk; first < total; first += (int64_t)gridDim.x * kChunk) {
    const int64_t row0 = first / packs;
    const uint32_t rest = (uint32_t)(first - row0 * packs);
    pack in[kPacks];
    int64_t row[kPacks];
    uint32_t col[kPacks];
#pragma unroll
    for (int j = 0; j < kPacks; ++j) {
      const uint32_t local = j * kBlock + threadIdx.x, n = rest + local;
      const uint32_t q = packs > kShortPacks ? (n >= packs ? 1u : 0u) : packs == 1 ? n : __umulhi(n, magic);
      row[j] = row0 + q;
      col[j] = first + local < total ? (n - q * packs) * V : cols;   // cols: there is no such pack
      in[j] = pack{};
      if (col[j] + V <= cols) in[j] = __builtin_nontemporal_load((const pack*)(x + row[j] * ld_x + col[j]));
    }
#pragma unroll
    for (int j = 0; j < kPacks; ++j) {
      if (col[j] >= cols) continue;
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
    const int64_t packs = (cols + Pack<T>::n - 1) / Pack<T>::n, total = rows * packs;
    const uint32_t magic = packs > 1 ? (uint32_t)((((uint64_t)1 << 32) + packs - 1) / packs) : 0;
    const unsigned blocks = (unsigned)std::min<int64_t>((total + kChunk - 1) / kChunk, 1 << 22);
    hipLaunchKernelGGL(k_dropout<T>, dim3(blocks), dim3(kBlock), 0, (hipStream_t)hip_stream, (const T*)x, ld_x, (T*)y, ld_y, total, (uint32_t)packs, magic,
                       (uint32_t)cols, d);
  });
  return launch_status("lopt_dropout");
}
