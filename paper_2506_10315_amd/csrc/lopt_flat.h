// Packs of V neighbouring elements of a matrix's rows, counted from each row's first element, those of all rows through: element-wise passes
// hand them out in chunks, which may be of many short rows or a part of a long one.
#pragma once

#include "lopt_ops.h"

namespace lopt {
namespace {

struct Flat {
  int64_t total;             // packs in all
  uint32_t packs, magic;     // of a row; 2^32 / packs rounded up
  uint32_t cols;
};
constexpr uint32_t kShortPacks = 1 << 15;
inline Flat flat_of(int64_t rows, int64_t cols, int V) {
  const int64_t packs = (cols + V - 1) / V;
  return Flat{rows * packs, (uint32_t)packs, packs > 1 ? (uint32_t)((((uint64_t)1 << 32) + packs - 1) / packs) : 0, (uint32_t)cols};
}

// Where the packs of a chunk of at most 2^15 packs lie. A 32-bit product with `magic` divides what there is to divide, below packs + 2^15, exactly while packs <= 2^15;
// longer rows have the quotient 0 or 1.
struct Chunk {
  int64_t first, row0;
  uint32_t rest;
  __device__ __forceinline__ Chunk(const Flat& f, int64_t first_) : first(first_) {
    if (first_ >> 32 == 0) row0 = (uint32_t)first_ / f.packs;   // a quarter of the instructions
    else row0 = first_ / f.packs;
    rest = (uint32_t)(first_ - row0 * f.packs);
  }
  // Row and first column of the chunk's pack `local`; false if there is no such pack.
  __device__ __forceinline__ bool at(const Flat& f, int V, uint32_t local, int64_t& row, uint32_t& col) const {
    const uint32_t n = rest + local, q = f.packs > kShortPacks ? (n >= f.packs ? 1u : 0u) : f.packs == 1 ? n : __umulhi(n, f.magic);
    row = row0 + q;
    col = (n - q * f.packs) * V;
    return first + local < f.total;
  }
};

}  // namespace
}  // namespace lopt
