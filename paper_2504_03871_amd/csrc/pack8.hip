// Activations kept in 8 bits: packing, unpacking, and the saved planes of the expert layer from packed pre-activations.
//
// A block of 32 values of a row shares a power of two 2^e, the smallest with which the block's largest magnitude m is not
// saturated (2^127 at most): e4m3 codes: m <= 448 * 2^e; whole numbers of 64ths in 8 bits: m < 127.5 / 64 * 2^e.  Multiplying by a power of two
// is exact, so a code is the value itself rounded once to its grid, ties to even, and unpacking is exact (in a 16-bit type: but
// for subnormals).  A block with an infinity or a NaN, which eight bits could only hide, is marked and stands for NaN.  The
// element and scale formats are those of the OCP microscaling specification (MXFP8 E4M3, MXINT8; scale E8M0).
//
// All of it is one pass over memory: per element s bytes one way and 33/32 the other, 16 bytes per lane where rows allow.
#include "pack8.h"

namespace moe {

// 8 adjacent values of a row from column c on: 16-byte loads where the row's start allows (VEC), else one by one
template <typename T, bool VEC>
__device__ __forceinline__ void load8(const T* __restrict__ row, int c, int width, float (&v)[8]) {
  if (VEC && c + 8 <= width) {
#pragma unroll
    for (int i = 0; i < 8; i += Vec16<T>::N) {
      Vec16<T> q;
      q.load_nt(row + c + i);
      q.unpack(v + i);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = c + i < width ? to_f32(row[c + i]) : 0.f;
  }
}
template <typename T, bool VEC>
__device__ __forceinline__ void store8(T* __restrict__ row, int c, int width, const float (&v)[8]) {
  if (VEC && c + 8 <= width) {
#pragma unroll
    for (int i = 0; i < 8; i += Vec16<T>::N) {
      Vec16<T> q;
      q.pack(v + i);
      q.store_nt(row + c + i);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < width) row[c + i] = from_f32<T>(v[i]);
  }
}

struct Pack8Args {
  const void* src;
  void* dst;
  uint8_t* codes;
  uint8_t* scales;
  long long rows, pitch;   // of one plane; elements between rows
  int width, blocks;       // blocks of 32 in a row
  int planes;              // stacked one behind the other
  RowRange range;          // which rows: all, or those of the shares
};

// Four lanes hold a block, eight values each.
template <typename T, int FMT, bool VEC>
__global__ __launch_bounds__(256) void pack8_kernel(Pack8Args a) {
  __shared__ int32_t s_range[2 * MOE_MAX_E + 1];
  const RangeTable rt = load_range(a.range, s_range);
  const long long per_plane = a.rows * a.blocks * 4, n = per_plane * a.planes;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256) {
    const long long g = i >> 2, row = g / a.blocks, in_plane = row % a.rows;
    if (!rt.live(in_plane)) continue;   // the four lanes of a block go together
    const int b = (int)(g - row * a.blocks), q = (int)(i & 3), c = b * BLOCK8 + q * 8;
    float v[8];
    load8<T, VEC>(reinterpret_cast<const T*>(a.src) + row * a.pitch, c, a.width, v);
    unsigned top = 0;   // the magnitudes' bit patterns are ordered as the magnitudes are, infinity and NaN above all numbers
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(v[j]) & 0x7fffffffu);
    top = max(top, (unsigned)__shfl_xor((int)top, 1, 4));
    top = max(top, (unsigned)__shfl_xor((int)top, 2, 4));
    const int e = scale_exponent<FMT>(top);
    uint2 code = make_uint2(0u, 0u);
    if (e != NOT_FINITE) code = encode8<FMT>(v, -e);
    *reinterpret_cast<uint2*>(a.codes + g * BLOCK8 + q * 8) = code;
    if (q == 0) a.scales[g] = (uint8_t)(e + 127);
  }
}

template <typename T, int FMT, bool VEC>
__global__ __launch_bounds__(256) void unpack8_kernel(Pack8Args a) {
  const long long n = a.rows * a.blocks * 4;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256) {
    const long long g = i >> 2, row = g / a.blocks;
    const int b = (int)(g - row * a.blocks), q = (int)(i & 3), c = b * BLOCK8 + q * 8;
    if (c >= a.width) continue;
    float v[8];
    decode8<T, FMT>(*reinterpret_cast<const uint2*>(a.codes + g * BLOCK8 + q * 8), a.scales[g], v);
    store8<T, VEC>(reinterpret_cast<T*>(a.dst) + row * a.pitch, c, a.width, v);
  }
}

// Packed pre-activations -> every saved plane: A | gelu(A), or G | U | silu(G) U.
template <typename T, int FMT, bool SWIGLU>
__global__ __launch_bounds__(256) void restore8_kernel(Pack8Args a) {
  __shared__ int32_t s_range[2 * MOE_MAX_E + 1];
  const RangeTable rt = load_range(a.range, s_range);
  const long long n = a.rows * a.blocks * 4, plane = a.rows * a.width, code_plane = a.rows * a.blocks;
  T* dst = reinterpret_cast<T*>(a.dst);
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256) {
    const long long g = i >> 2, row = g / a.blocks;
    const int b = (int)(g - row * a.blocks), q = (int)(i & 3), c = b * BLOCK8 + q * 8;
    if (c >= a.width || !rt.live(row)) continue;
    float v[8], u[8], h[8];
    decode8<T, FMT>(*reinterpret_cast<const uint2*>(a.codes + g * BLOCK8 + q * 8), a.scales[g], v);
    if constexpr (SWIGLU) decode8<T, FMT>(*reinterpret_cast<const uint2*>(a.codes + (code_plane + g) * BLOCK8 + q * 8), a.scales[code_plane + g], u);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if constexpr (SWIGLU) h[j] = v[j] * sigmoid_f(v[j]) * u[j];
      else h[j] = sizeof(T) == 4 ? gelu_f(v[j]) : v[j] * phi_fast(v[j]);
    }
    T* at = dst + row * a.width;
    store8<T, true>(at, c, a.width, v);
    if constexpr (SWIGLU) store8<T, true>(at + plane, c, a.width, u);
    store8<T, true>(at + plane * (SWIGLU ? 2 : 1), c, a.width, h);
  }
}

static unsigned pack_grid(long long items) {
  const long long blocks = (items + 255) / 256;
  return (unsigned)(blocks < 256 * 32 ? blocks : 256 * 32);
}

template <typename T, int FMT>
static int pack_for(const Pack8Args& a, bool unpack, hipStream_t s) {
  // 16-byte accesses where every row starts at one; a row of fewer columns ends element by element
  const bool vec = a.pitch * sizeof(T) % 16 == 0;
  const unsigned grid = pack_grid(a.rows * a.blocks * 4 * a.planes);
  if (unpack) {
    if (vec) unpack8_kernel<T, FMT, true><<<grid, 256, 0, s>>>(a); else unpack8_kernel<T, FMT, false><<<grid, 256, 0, s>>>(a);
  } else {
    if (vec) pack8_kernel<T, FMT, true><<<grid, 256, 0, s>>>(a); else pack8_kernel<T, FMT, false><<<grid, 256, 0, s>>>(a);
  }
  return launch_status();
}
template <typename T, int FMT>
static int restore_for(const Pack8Args& a, bool swiglu, hipStream_t s) {
  const unsigned grid = pack_grid(a.rows * a.blocks * 4);
  if (swiglu) restore8_kernel<T, FMT, true><<<grid, 256, 0, s>>>(a); else restore8_kernel<T, FMT, false><<<grid, 256, 0, s>>>(a);
  return launch_status();
}
#define MOE_BY_TYPE(fn, ...)                                                                              \
  (dtype == MOE_DTYPE_BF16  ? (fmt == MOE_PACK_E4M3 ? fn<bf16, MOE_PACK_E4M3>(__VA_ARGS__) : fn<bf16, MOE_PACK_I8>(__VA_ARGS__))   \
   : dtype == MOE_DTYPE_F16 ? (fmt == MOE_PACK_E4M3 ? fn<f16, MOE_PACK_E4M3>(__VA_ARGS__) : fn<f16, MOE_PACK_I8>(__VA_ARGS__))     \
                            : (fmt == MOE_PACK_E4M3 ? fn<float, MOE_PACK_E4M3>(__VA_ARGS__) : fn<float, MOE_PACK_I8>(__VA_ARGS__)))

int launch_pack8(int dtype, int fmt, long long rows, int width, long long pitch, const void* src, void* codes, void* scales, hipStream_t s) {
  const Pack8Args a = {src, nullptr, (uint8_t*)codes, (uint8_t*)scales, rows, pitch, width, blocks8(width), 1, {}};
  return MOE_BY_TYPE(pack_for, a, false, s);
}
int launch_unpack8(int dtype, int fmt, long long rows, int width, long long pitch, const void* codes, const void* scales, void* dst, hipStream_t s) {
  const Pack8Args a = {nullptr, dst, (uint8_t*)const_cast<void*>(codes), (uint8_t*)const_cast<void*>(scales), rows, pitch, width, blocks8(width), 1, {}};
  return MOE_BY_TYPE(pack_for, a, true, s);
}
int launch_saved_pack8(const moe_cfg* c, int fmt, const void* saved, const RowRange& range, void* codes, void* scales, hipStream_t s) {
  const int dtype = c->dtype;
  const Pack8Args a = {saved, nullptr, (uint8_t*)codes, (uint8_t*)scales, (long long)c->T * c->k, c->d_ff, c->d_ff, blocks8(c->d_ff),
                       c->act == MOE_ACT_SWIGLU ? 2 : 1, range};
  return MOE_BY_TYPE(pack_for, a, false, s);
}
int launch_saved_restore8(const moe_cfg* c, int fmt, const void* codes, const void* scales, const RowRange& range, void* saved, hipStream_t s) {
  const int dtype = c->dtype;
  const Pack8Args a = {nullptr, saved, (uint8_t*)const_cast<void*>(codes), (uint8_t*)const_cast<void*>(scales), (long long)c->T * c->k, c->d_ff, c->d_ff,
                       blocks8(c->d_ff), 1, range};
  return MOE_BY_TYPE(restore_for, a, c->act == MOE_ACT_SWIGLU, s);
}

}  // namespace moe
