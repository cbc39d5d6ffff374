// Dropout of rows, the mask formed where it is needed and stored nowhere: y = x / (1 - p) where the element's word of the generator stays, else 0.
// The gradient is the same call on the gradient. Bound by memory, one read and one write.
#include <algorithm>

#include "lopt_flat.h"
#include "lopt_random.h"

namespace lopt {
namespace {

// A workgroup takes kChunk neighbouring packs of 16 bytes, four a thread.
constexpr int kPacks = 4, kChunk = kPacks * kBlock;

// WHOLE: rows are whole packs, and a word is compared where it is needed. Else the pack that would pass a row's end ends with it, and its bits are moved with it. us: 5001x1531
// fp16 11.2, with the elements of such packs loaded one by one 12.8; 8192x4096 bf16 26.5 in a graph (28.3 with inputs that change, 4.7 TB/s), with two exclusive ors each in the
// ten rounds in place of one of three inputs 31. Reads and writes go past the cache whatever the size. us together with a sum that reads y, so / stores by the cache: 16384x8192 bf16 183 / 197,
// 8192x4096 53 / 51, 8192x1024 16.1 / 16.7, 2048x1024 9.2 / 9.1, 197x768 8.6 / 7.9.
template <typename T, bool WHOLE>
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
      if (have[j]) in[j] = __builtin_nontemporal_load((const pack*)(x + row[j] * ld_x + (WHOLE ? col[j] : min(col[j], cols - V))));
    }
#pragma unroll
    for (int j = 0; j < kPacks; ++j) {
      if (!have[j]) continue;
      const uint32_t at = WHOLE ? col[j] : min(col[j], cols - V), skip = col[j] - at;
      T* out = y + row[j] * ld_y + at;
      pack o;
      if (WHOLE && d.on && !d.none) {
#pragma unroll
        for (int e = 0; e < V; e += 4) {
          uint32_t w[4];
          words.four((uint32_t)row[j], col[j] / 4 + e / 4, w);
#pragma unroll
          for (int i = 0; i < 4; ++i) o[e + i] = from_f32<T>(w[i] >= d.least ? to_f32(in[j][e + i]) * d.scale : 0.f);
        }
      } else {
        const uint32_t bits = d.on ? words.stay<V>((uint32_t)row[j], col[j]) << skip : ~0u;
#pragma unroll
        for (int e = 0; e < V; ++e) o[e] = from_f32<T>(where_bit(bits, e, to_f32(in[j][e]) * d.scale));
      }
      if (skip == 0) {
        __builtin_nontemporal_store(o, (pack*)out);
      } else {
#pragma unroll
        for (int e = 1; e < V; ++e)
          if (e >= (int)skip) out[e] = o[e];
      }
    }
  }
}

// Rows shorter than a pack: an element a thread.
template <typename T>
__global__ __launch_bounds__(kBlock) void k_dropout_narrow(const T* x, int64_t ld_x, T* y, int64_t ld_y, Flat f, Dropout d) {
  const Words words(d);
  for (int64_t first = (int64_t)blockIdx.x * kBlock; first < f.total; first += (int64_t)gridDim.x * kBlock) {
    int64_t row;
    uint32_t col;
    if (!Chunk(f, first).at(f, 1, threadIdx.x, row, col)) continue;
    const uint32_t bits = d.on ? words.stay<1>((uint32_t)row, col) : 1u;
    y[row * ld_y + col] = from_f32<T>(where_bit(bits, 0, to_f32(x[row * ld_x + col]) * d.scale));
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
    constexpr int V = Pack<T>::n;
    const Flat f = flat_of(rows, cols, cols < V ? 1 : V);
    const int chunk = cols < V ? kBlock : kChunk;
    const unsigned blocks = (unsigned)std::min<int64_t>((f.total + chunk - 1) / chunk, 1 << 22);
    auto kernel = cols < V ? k_dropout_narrow<T> : cols % V == 0 ? k_dropout<T, true> : k_dropout<T, false>;
    hipLaunchKernelGGL(kernel, dim3(blocks), dim3(kBlock), 0, (hipStream_t)hip_stream, (const T*)x, ld_x, (T*)y, ld_y, f, d);
  });
  return launch_status("lopt_dropout");
}
