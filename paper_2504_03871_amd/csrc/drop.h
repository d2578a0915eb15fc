// Dropout whose mask is computed where it is needed and never stored: which elements of a matrix are kept follows from a seed, an
// offset and the element's row and column alone, so that a backward pass finds the forward's mask again.
//
// Eight adjacent columns of a row share one evaluation of Philox 4x32 with ten rounds (Salmon, Moraes, Dror and Shaw, "Parallel random
// numbers: as easy as 1, 2, 3", 2011): key = seed, counter = (column / 8, row, offset); column 8 c + j takes the low (j even) or
// high half of output word j / 2.  16 bits decide about an element: with 32 the generator, two 32 x 32 -> 64-bit products and four
// xors a round, would take half as long again as the memory traffic that it hides behind (six bytes an element).  The
// probability comes in steps of 2^-16, and the kept elements are scaled by the reciprocal of the one that is in force.
#pragma once
#include "common.h"

namespace moe {

struct DropArgs {
  const uint64_t* step;   // device, may be NULL
  uint64_t offset;
  uint32_t key0, key1;
  uint32_t cut;           // elements whose 16 bits are below it are dropped; 0: no dropout
  float scale;
};
inline DropArgs drop_args(const moe_drop* d) {
  DropArgs a = {nullptr, 0, 0, 0, 0, 1.f};
  if (d == nullptr) return a;
  const double cut = (double)d->p * 65536.0 + 0.5;   // p is in [0, 1)
  a.cut = cut >= 65535.0 ? 65535u : (uint32_t)cut;
  a.scale = (float)(65536.0 / (65536.0 - a.cut));
  a.step = d->step;
  a.offset = d->offset;
  a.key0 = (uint32_t)d->seed;
  a.key1 = (uint32_t)(d->seed >> 32);
  return a;
}

#ifdef __HIPCC__
__device__ __forceinline__ uint64_t drop_offset(const DropArgs& a) { return a.offset + (a.step != nullptr ? *a.step : 0); }

__device__ __forceinline__ uint4 philox(uint32_t c0, uint32_t c1, uint64_t offset, uint32_t k0, uint32_t k1) {
  uint32_t c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32);
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
    const uint32_t n0 = (uint32_t)(b >> 32) ^ c1 ^ k0, n2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
    c0 = n0;
    c1 = (uint32_t)b;
    c2 = n2;
    c3 = (uint32_t)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return make_uint4(c0, c1, c2, c3);
}

// Eight values of columns 8 group .. 8 group + 7 of a row: scaled, or zero whatever they were.
__device__ __forceinline__ void drop8(const DropArgs& a, uint64_t offset, uint32_t row, uint32_t group, float (&v)[8]) {
  const uint4 r = philox(group, row, offset, a.key0, a.key1);
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = (w[i] & 0xffffu) >= a.cut ? v[2 * i] * a.scale : 0.f;
    v[2 * i + 1] = (w[i] >> 16) >= a.cut ? v[2 * i + 1] * a.scale : 0.f;
  }
}
#endif

}  // namespace moe
