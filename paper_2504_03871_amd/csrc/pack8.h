// Blocks of 32 values in 8 bits each with a shared power of two: the arithmetic of packing and unpacking, and which rows of the
// permuted buffers take part.  What is packed where: pack8.hip; the backward that reads packed pre-activations: linear.hip.
#pragma once
#include "common.h"

namespace moe {

constexpr int BLOCK8 = 32;
inline int blocks8(int width) { return (width + BLOCK8 - 1) / BLOCK8; }

// Rows of the permuted buffers that this GPU computes: the shares of the experts.  offsets == NULL: every row.
struct RowRange {
  const int32_t *offsets, *kept, *lo, *hi;
  int E;
};

int launch_saved_pack8(const moe_cfg* c, int fmt, const void* saved, const RowRange& range, void* codes, void* scales, hipStream_t s);
int launch_saved_restore8(const moe_cfg* c, int fmt, const void* codes, const void* scales, const RowRange& range, void* saved, hipStream_t s);
int launch_pack8(int dtype, int fmt, long long rows, int width, long long pitch, const void* src, void* codes, void* scales, hipStream_t s);
int launch_unpack8(int dtype, int fmt, long long rows, int width, long long pitch, const void* codes, const void* scales, void* dst, hipStream_t s);

#ifdef __HIPCC__
constexpr int NOT_FINITE = 128;   // scale exponent of a block that stands for NaN

// The exponent of a block whose largest magnitude has the bit pattern `top` (fp32).
template <int FMT>
__device__ __forceinline__ int scale_exponent(unsigned top) {
  if (top >= 0x7f800000u) return NOT_FINITE;
  // mantissa bound up to which the largest code takes it: 1.75 (448 = 1.75 * 2^8), or just below 127.5 / 64 = 1.9921875
  constexpr unsigned MOST = FMT == MOE_PACK_E4M3 ? 0x600000u : 0x7effffu;
  constexpr int HIGHEST = FMT == MOE_PACK_E4M3 ? 8 : 0;
  // magnitudes below 2^-126 all get the lowest exponent
  const int e = (int)(top >> 23) - 127 - HIGHEST + ((top & 0x7fffffu) > MOST ? 1 : 0);
  return top < 0x00800000u ? -127 : min(max(e, -127), 127);   // above 2^127 there is only NaN's: the largest codes saturate
}

// Eight values times 2^up as codes; none is beyond the largest code (but for the saturation above).
template <int FMT>
__device__ __forceinline__ uint2 encode8(const float (&v)[8], int up) {
  unsigned w[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float s[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) s[j] = __builtin_amdgcn_ldexpf(v[4 * h + j], FMT == MOE_PACK_E4M3 ? up : up + 6);
    if constexpr (FMT == MOE_PACK_E4M3) {
      int p = __builtin_amdgcn_cvt_pk_fp8_f32(s[0], s[1], 0, false);
      w[h] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(s[2], s[3], p, true);
    } else {
      w[h] = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) w[h] |= ((unsigned)(int)fminf(fmaxf(rintf(s[j]), -127.f), 127.f) & 0xffu) << (8 * j);
    }
  }
  return make_uint2(w[0], w[1]);
}

template <typename T> __device__ __forceinline__ float largest_finite();
template <> __device__ __forceinline__ float largest_finite<float>() { return 3.4028234663852886e38f; }
template <> __device__ __forceinline__ float largest_finite<bf16>() { return 3.3895313892515355e38f; }
template <> __device__ __forceinline__ float largest_finite<f16>() { return 65504.f; }

// What eight codes stand for, none beyond T's largest finite number (a value that was rounded up may be).  The NaN codes of e4m3,
// which encode8 does not write but another program may, stay NaN.
template <typename T, int FMT>
__device__ __forceinline__ void decode8(const uint2& code, unsigned scale, float (&v)[8]) {
  const unsigned w[2] = {code.x, code.y};
  const int e = (int)scale - 127 - (FMT == MOE_PACK_E4M3 ? 0 : 6);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float s[4];
    if constexpr (FMT == MOE_PACK_E4M3) {
      typedef float f32x2 __attribute__((ext_vector_type(2)));
      const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[h], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[h], true);
      s[0] = a.x; s[1] = a.y; s[2] = b.x; s[3] = b.y;
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) s[j] = (float)(int)(int8_t)(w[h] >> (8 * j));
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float x = __builtin_amdgcn_ldexpf(s[j], e), m = largest_finite<T>();
      const float y = FMT == MOE_PACK_E4M3 && x != x ? x : fminf(fmaxf(x, -m), m);
      v[4 * h + j] = scale == 255u ? __uint_as_float(0x7fc00000u) : y;
    }
  }
}

// Which rows take part, from LDS: with slices the experts' first rows and ends, without them the one end of all rows.
struct RangeTable {
  const int32_t* t;   // [E] first rows, [E] ends
  int E;
  bool all, sliced;
  long long end;
  __device__ __forceinline__ long long limit(long long rows) const { return all ? rows : end; }
  __device__ __forceinline__ bool live(long long row) const {
    if (!sliced) return all || row < end;
    int lo = 0, hi = E;   // the last range that starts at or before the row
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (t[mid] <= row) lo = mid + 1; else hi = mid;
    }
    return lo > 0 && row < t[E + lo - 1];
  }
};
__device__ __forceinline__ RangeTable load_range(const RowRange& r, int32_t* lds) {
  RangeTable t = {lds, r.E, r.offsets == nullptr, r.lo != nullptr, 0};
  if (t.all) return t;
  t.end = (long long)r.offsets[r.E - 1] + r.kept[r.E - 1];   // the experts' rows follow each other
  if (!t.sliced) return t;
  for (int e = threadIdx.x; e < r.E; e += blockDim.x) {
    int l, h;
    share_of(r.lo, r.hi, r.kept[e], e, l, h);
    lds[e] = r.offsets[e] + l;
    lds[r.E + e] = r.offsets[e] + h;
  }
  __syncthreads();
  return t;
}
#endif

}  // namespace moe
