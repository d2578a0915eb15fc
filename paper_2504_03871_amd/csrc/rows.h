// Kernels that hold a whole row of a matrix in the registers of one or several waves: accesses of eight adjacent values, sums and
// maxima over a row, and its quantisation to 8-bit integers with one scale.
#pragma once
#include "common.h"

namespace moe {

// A row is dealt out in groups of eight values, neighbours to neighbours, `nch` to a thread: to one wave, four rows to a block of 256
// threads and no barrier, or to `waves` waves of a block of their own, as few as hold the row so that no thread is idle.
struct RowGeom { int waves, nch; };
inline int row_threads(const RowGeom& g) { return g.waves == 1 ? 256 : g.waves * WAVE; }
inline int rows_per_block(const RowGeom& g) { return g.waves == 1 ? 4 : 1; }
inline int row_waves(int groups, int nch) { return (groups + WAVE * nch - 1) / (WAVE * nch); }

#ifdef __HIPCC__
// Vectors that may start at any element: rows of any width are read and written 16 bytes at a time.
typedef unsigned any_u32x4 __attribute__((ext_vector_type(4), aligned(2)));
typedef unsigned any_u32x2 __attribute__((ext_vector_type(2), aligned(1)));

// Eight adjacent values of storage type T as they lie in memory.
template <typename T>
struct Raw8 {
  static constexpr int N = sizeof(T) / 2;   // 16-byte pieces
  any_u32x4 q[N];
};
template <typename T>
__device__ __forceinline__ void unpack8(const Raw8<T>& r, float (&v)[8]) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r.q[i / 4][i % 4]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const unsigned u = r.q[0][i];
      if constexpr (__is_same(T, bf16)) { v[2 * i] = __uint_as_float(u << 16); v[2 * i + 1] = __uint_as_float(u & 0xffff0000u); }
      else { v[2 * i] = f16_bits_to_f32(u & 0xffffu); v[2 * i + 1] = f16_bits_to_f32(u >> 16); }
    }
  }
}
template <typename T>
__device__ __forceinline__ Raw8<T> pack_row8(const float (&v)[8]) {
  Raw8<T> r;
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < 8; ++i) r.q[i / 4][i % 4] = __float_as_uint(v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) r.q[0][i] = __is_same(T, bf16) ? pack_bf16x2(v[2 * i], v[2 * i + 1]) : pack_f16x2(v[2 * i], v[2 * i + 1]);
  }
  return r;
}
// Values c .. c + 7 of a row of `width`; those past its end are zero, and are not written.  ODD: a row may end inside a group of eight.
// Its last group is then read as the row's last eight values, so that every lane makes the same vector load, and moved into place
// behind it (place8).  (Value by value, which makes a wave wait for up to seven loads in turn: rows of 516 fp32, 300 of them, 5.2
// instead of 4.2 us, 3001 of 1091 fp16 18 instead of 9.)
template <typename T, bool ODD, bool NT = true>
__device__ __forceinline__ Raw8<T> load_row8(const T* row, int c, int width) {
  Raw8<T> r = {};
  if (ODD && width < 8) {
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = c + i < width ? to_f32(row[c + i]) : 0.f;
    return pack_row8<T>(v);   // exact: they come from this type
  }
  if (ODD ? c < width : c + 8 <= width) {
    const int at = ODD ? min(c, width - 8) : c;
#pragma unroll
    for (int i = 0; i < Raw8<T>::N; ++i) {
      const any_u32x4* p = reinterpret_cast<const any_u32x4*>(row + at) + i;
      r.q[i] = NT ? __builtin_nontemporal_load(p) : *p;
    }
  }
  return r;
}
template <bool ODD>
__device__ __forceinline__ void place8(float (&v)[8], int c, int width) {
  if (!ODD || c >= width || c + 8 <= width || width < 8) return;
  const int by = 8 - width % 8;   // the same for every row
#pragma unroll
  for (int s = 4; s > 0; s >>= 1)
    if ((by & s) != 0) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = i + s < 8 ? v[i + s] : 0.f;
    }
}
template <typename T, bool ODD>
__device__ __forceinline__ void unpack_row8(const Raw8<T>& r, int c, int width, float (&v)[8]) {
  unpack8<T>(r, v);
  place8<ODD>(v, c, width);
}
template <typename T, bool ODD>
__device__ __forceinline__ void store_row8(T* row, int c, int width, const Raw8<T>& r) {
  if (c + 8 <= width) {
#pragma unroll
    for (int i = 0; i < Raw8<T>::N; ++i) __builtin_nontemporal_store(r.q[i], reinterpret_cast<any_u32x4*>(row + c) + i);
  } else if (ODD && c < width) {
    float v[8];
    unpack8<T>(r, v);
#pragma unroll
    for (int i = 0; i < 7; ++i)
      if (c + i < width) row[c + i] = from_f32<T>(v[i]);
  }
}

template <typename V, typename F>
__device__ __forceinline__ V wave_reduce(V v, F f) {
#pragma unroll
  for (int s = 32; s > 0; s >>= 1) v = f(v, __shfl_xor(v, s, WAVE));
  return v;
}
// Over the waves of a row, at most MAXW (1: a wave has a row); every thread gets the result.  `lds`: MAXW values, zeros for waves that the
// block does not have (row_reduce_init), and none that a reduction since the last barrier but one has used: rows alternate
// between two sets.
template <int MAXW, typename V>
__device__ __forceinline__ void row_reduce_init(V* lds) {   // both sets
  if constexpr (MAXW > 1) {
    if (threadIdx.x < 2 * MAXW) lds[threadIdx.x] = V(0);
    __syncthreads();
  }
}
template <int MAXW, typename V, typename F>
__device__ __forceinline__ V row_reduce(V v, V* lds, F f) {
  v = wave_reduce(v, f);
  if constexpr (MAXW > 1) {
    if (threadIdx.x % WAVE == 0) lds[threadIdx.x / WAVE] = v;
    __syncthreads();
    v = lds[0];
#pragma unroll
    for (int i = 1; i < MAXW; ++i) v = f(v, lds[i]);
  }
  return v;
}
__device__ __forceinline__ float add_f(float a, float b) { return a + b; }
__device__ __forceinline__ unsigned max_u(unsigned a, unsigned b) { return max(a, b); }

// ---- a row in 8 bits: codes -127 .. 127 with one scale ----
// m = max(largest magnitude, 2^-100), scale = m / 127 (as m times the fp32 number 1 / 127), code = round(v * (127 / m)): two fp32
// roundings before the one to a whole number, which moves a code only where v lies within 2^-23 of a tie.  The lower limit keeps
// 127 / m finite.  A row with an infinity or NaN has codes of zero and the scale NaN, so that its products are NaN.
struct RowScale { float up, scale; };
__device__ __forceinline__ RowScale row_scale(unsigned top) {   // bit pattern of the largest magnitude
  if (top >= 0x7f800000u) return {0.f, __uint_as_float(0x7fc00000u)};
  const float m = fmaxf(__uint_as_float(top), 7.8886090522101181e-31f);
  return {127.f / m, m * (1.f / 127.f)};
}
__device__ __forceinline__ unsigned top_of(unsigned top, const float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
  return top;
}
__device__ __forceinline__ any_u32x2 codes8(const float (&v)[8], float up) {
  unsigned w[2] = {0u, 0u};
  if (up != 0.f) {   // (a row with an infinity or NaN has none: 0 times those is no number)
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i / 4] |= ((unsigned)(int)rintf(v[i] * up) & 0xffu) << (8 * (i % 4));
  }
  return any_u32x2{w[0], w[1]};
}
template <bool ODD>
__device__ __forceinline__ void store_codes8(int8_t* row, int c, int width, const any_u32x2& q) {
  if (c + 8 <= width) {
    *reinterpret_cast<any_u32x2*>(row + c) = q;
  } else if (ODD && c < width) {
#pragma unroll
    for (int i = 0; i < 7; ++i)
      if (c + i < width) row[c + i] = (int8_t)(q[i / 4] >> (8 * (i % 4)));
  }
}
#endif

}  // namespace moe
