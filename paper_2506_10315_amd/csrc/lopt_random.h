// The counter-based generator of dropout: Philox4x32 of ten rounds (Salmon, Moraes, Dror, Shaw 2011, "Parallel random numbers: as easy as
// 1, 2, 3"). Key: the seed; counter: (column / 4, row, offset); the four words belong to four neighbouring columns of a row, counted from the
// row's first element, so that a lane's pack of 16 bytes takes whole blocks wherever the row lies in memory, and forward and backward
// passes of any split form the same mask.
#pragma once

#include <cmath>

#include "lopt_ops.h"

namespace lopt {
namespace {

// An element stays if its word reaches `least`, which is p 2^32; `none`: p is 1. `on`: p is not 0.
struct Dropout {
  uint32_t least;
  float scale;   // 1 / (1 - p)
  bool on, none;
  uint64_t seed, offset;
  const uint64_t* seed_device;   // in place of `seed`, read when the kernel runs
};

inline lopt_status check_dropout(float p, const uint64_t* seed_device, Dropout* d) {
  if (!(p >= 0.f && p <= 1.f)) return fail_call(LOPT_EINVAL, "p must be in [0, 1]");
  LOPT_CHECK(check_array("seed_device", seed_device, 8, false));
  const uint64_t least = (uint64_t)std::llrint((double)p * 4294967296.0);   // 2^32 only for p = 1, a float32
  d->on = least > 0;
  d->none = p == 1.f;
  d->least = (uint32_t)std::min<uint64_t>(least, 0xffffffffu);
  d->scale = d->none ? 0.f : (float)(1.0 / (1.0 - (double)p));
  d->seed_device = seed_device;
  return LOPT_OK;
}

// One instruction, which the compiler does not find by itself.
__device__ __forceinline__ uint32_t xor3(uint32_t a, uint32_t b, uint32_t c) { return __builtin_amdgcn_bitop3_b32(a, b, c, 0x96); }

// The generator of one launch, its key read.
struct Words {
  uint32_t key0, key1, offset0, offset1, least;
  bool none;
  __device__ __forceinline__ explicit Words(const Dropout& d) {
    const uint64_t key = d.on && d.seed_device ? *d.seed_device : d.seed;
    key0 = (uint32_t)key, key1 = (uint32_t)(key >> 32);
    offset0 = (uint32_t)d.offset, offset1 = (uint32_t)(d.offset >> 32);
    least = d.least;
    none = d.none;
  }
  // The words of columns 4 block to 4 block + 3 of the row.
  __device__ __forceinline__ void four(uint32_t row, uint32_t block, uint32_t (&w)[4]) const {
    uint32_t c0 = block, c1 = row, c2 = offset0, c3 = offset1, k0 = key0, k1 = key1;
#pragma unroll
    for (int i = 0; i < 10; ++i) {
      const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
      c0 = xor3((uint32_t)(b >> 32), c1, k0);
      c2 = xor3((uint32_t)(a >> 32), c3, k1);
      c1 = (uint32_t)b;
      c3 = (uint32_t)a;
      k0 += 0x9E3779B9u;
      k1 += 0xBB67AE85u;
    }
    w[0] = c0, w[1] = c1, w[2] = c2, w[3] = c3;
  }
  // Bit e: whether column `col` + e of the row stays, of V columns from a multiple of 4 on (of one column, any).
  template <int V>
  __device__ __forceinline__ uint32_t stay(uint32_t row, uint32_t col) const {
    uint32_t bits = 0, w[4];
#pragma unroll
    for (int e = 0; e < V; e += 4) {
      four(row, col / 4 + e / 4, w);
#pragma unroll
      for (int i = 0; i < 4; ++i) bits |= (w[i] >= least ? 1u : 0u) << (e + i);
    }
    if (none) bits = 0;
    return V == 1 ? bits >> (col & 3) & 1u : bits;
  }
};

// v where bit e is set, else 0 (whatever v is).
__device__ __forceinline__ float where_bit(uint32_t bits, int e, float v) {
  const int32_t all = (int32_t)(bits << (31 - e)) >> 31;
  return __builtin_bit_cast(float, __builtin_bit_cast(int32_t, v) & all);
}

}  // namespace
}  // namespace lopt
