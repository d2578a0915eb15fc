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
  RowRange range;          // which rows: all, or those of the shares
};

// Work items are eight adjacent values of a row, four to a block; item i's codes are bytes 8 i .. 8 i + 7 of the plane's, its scale
// byte i / 4.  DENSE: rows without gaps between them or between their blocks, so that item i is elements 8 i .. 8 i + 7 of the plane
// and no row has to be known.  A thread takes U items, 256 apart, and requests them all before it uses the first.
struct Item { long long g; long long row; int c, q; };   // block, row, first column, part of the block
template <bool DENSE>
__device__ __forceinline__ Item item_of(const Pack8Args& a, long long i) {
  Item t;
  t.g = i >> 2;
  t.q = (int)(i & 3);
  t.row = 0;
  t.c = 0;
  if constexpr (!DENSE) {
    t.row = (t.g >> 32) == 0 ? (long long)((unsigned)t.g / (unsigned)a.blocks) : t.g / a.blocks;
    t.c = (int)(t.g - t.row * a.blocks) * BLOCK8 + t.q * 8;
  }
  return t;
}

// Four lanes hold a block.  blockIdx.y: plane.  Bound by HBM: two planes of 32768 x 8192 bf16, 1.07 GB read and 0.55 GB written,
// 258 us = 6.3 TB/s; with the row of every item found by a division and one item per thread 407.  One plane, dense 127 us, 8168 wide
// 142, 8166 wide (VEC false: element by element) 355; two planes in slices 327.
template <typename T, int FMT, bool DENSE, bool VEC, int U>
__global__ __launch_bounds__(256) void pack8_kernel(Pack8Args a) {
  __shared__ int32_t s_range[2 * MOE_MAX_E];
  const RangeTable rt = load_range(a.range, s_range);
  const long long n = a.rows * a.blocks * 4, i0 = (long long)blockIdx.x * (256 * U) + threadIdx.x;
  const long long live_items = DENSE ? min(n, rt.limit(a.rows) * a.blocks * 4) : n;
  const T* src = reinterpret_cast<const T*>(a.src) + (long long)blockIdx.y * a.rows * a.pitch;
  const long long plane = (long long)blockIdx.y * a.rows * a.blocks;
  float v[U][8];
  Item t[U];
  bool live[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const long long i = i0 + u * 256;
    live[u] = i < live_items;
    if (!live[u]) continue;
    t[u] = item_of<DENSE>(a, i);
    if constexpr (DENSE) load8<T, true>(src + i * 8, 0, 8, v[u]);
    else {
      live[u] = rt.live(t[u].row);
      if (live[u]) load8<T, VEC>(src + t[u].row * a.pitch, t[u].c, a.width, v[u]);
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (!live[u]) continue;   // the four lanes of a block go together
    unsigned top = 0;   // the magnitudes' bit patterns are ordered as the magnitudes are, infinity and NaN above all numbers
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(v[u][j]) & 0x7fffffffu);
    top = max(top, (unsigned)__shfl_xor((int)top, 1, 4));
    top = max(top, (unsigned)__shfl_xor((int)top, 2, 4));
    const int e = scale_exponent<FMT>(top);
    uint2 code = make_uint2(0u, 0u);
    if (e != NOT_FINITE) code = encode8<FMT>(v[u], -e);
    const long long g = plane + t[u].g;
    *reinterpret_cast<uint2*>(a.codes + g * BLOCK8 + t[u].q * 8) = code;
    if (t[u].q == 0) a.scales[g] = (uint8_t)(e + 127);
  }
}

template <typename T, int FMT, bool DENSE, bool VEC, int U>
__global__ __launch_bounds__(256) void unpack8_kernel(Pack8Args a) {
  const long long n = a.rows * a.blocks * 4, i0 = (long long)blockIdx.x * (256 * U) + threadIdx.x;
  T* dst = reinterpret_cast<T*>(a.dst);
  uint2 code[U];
  unsigned scale[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const long long i = min(i0 + u * 256, n - 1);
    code[u] = *reinterpret_cast<const uint2*>(a.codes + i * 8);
    scale[u] = a.scales[i >> 2];
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const long long i = i0 + u * 256;
    if (i >= n) break;
    float v[8];
    decode8<T, FMT>(code[u], scale[u], v);
    if constexpr (DENSE) store8<T, true>(dst + i * 8, 0, 8, v);
    else {
      const Item t = item_of<DENSE>(a, i);
      if (t.c < a.width) store8<T, VEC>(dst + t.row * a.pitch, t.c, a.width, v);
    }
  }
}

// Packed pre-activations -> every saved plane: A | gelu(A), or G | U | silu(G) U.  Bound by HBM's writes: 0.55 GB read, 1.61 GB
// written, 413 us = 5.2 TB/s, the rate of a fill.
template <typename T, int FMT, bool SWIGLU, bool DENSE, int U>
__global__ __launch_bounds__(256) void restore8_kernel(Pack8Args a) {
  __shared__ int32_t s_range[2 * MOE_MAX_E];
  const RangeTable rt = load_range(a.range, s_range);
  const long long n = a.rows * a.blocks * 4, i0 = (long long)blockIdx.x * (256 * U) + threadIdx.x;
  const long long live_items = DENSE ? min(n, rt.limit(a.rows) * a.blocks * 4) : n;
  const long long plane = a.rows * a.width, code_plane = a.rows * a.blocks * BLOCK8, scale_plane = a.rows * a.blocks;
  T* dst = reinterpret_cast<T*>(a.dst);
  uint2 code[U], code2[U];
  unsigned scale[U], scale2[U];
  bool live[U];
  Item t[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const long long i = i0 + u * 256;
    live[u] = i < live_items;
    if (!live[u]) continue;
    if constexpr (!DENSE) {
      t[u] = item_of<DENSE>(a, i);
      live[u] = t[u].c < a.width && rt.live(t[u].row);
      if (!live[u]) continue;
    }
    code[u] = *reinterpret_cast<const uint2*>(a.codes + i * 8);
    scale[u] = a.scales[i >> 2];
    if constexpr (SWIGLU) {
      code2[u] = *reinterpret_cast<const uint2*>(a.codes + code_plane + i * 8);
      scale2[u] = a.scales[scale_plane + (i >> 2)];
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (!live[u]) continue;
    const long long i = i0 + u * 256;
    float v[8], w[8], h[8];
    decode8<T, FMT>(code[u], scale[u], v);
    if constexpr (SWIGLU) decode8<T, FMT>(code2[u], scale2[u], w);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if constexpr (SWIGLU) h[j] = v[j] * (sizeof(T) == 4 ? sigmoid_f(v[j]) : __builtin_amdgcn_rcpf(1.f + __expf(-v[j]))) * w[j];
      else h[j] = sizeof(T) == 4 ? gelu_f(v[j]) : v[j] * phi_fast(v[j]);
    }
    T* at = DENSE ? dst + i * 8 : dst + t[u].row * a.width;
    const int c = DENSE ? 0 : t[u].c, width = DENSE ? 8 : a.width;
    store8<T, true>(at, c, width, v);
    if constexpr (SWIGLU) store8<T, true>(at + plane, c, width, w);
    store8<T, true>(at + plane * (SWIGLU ? 2 : 1), c, width, h);
  }
}

// Items per thread: one where the chip has fewer than it can hold at a time.  (Then a launch is all there is: 300 x 516 fp32, pack 3.2,
// unpack 2.7 us.)
constexpr int PACK_U = 4;
static dim3 pack_grid(long long items, int u, int planes) { return dim3((unsigned)((items + 256 * u - 1) / (256 * u)), planes); }
constexpr long long PACK_FEW = 256 * 2048;

template <typename T, int FMT, int U>
static int pack_u(const Pack8Args& a, int planes, bool unpack, hipStream_t s) {
  // rows that follow each other without a gap, of whole blocks; else 16-byte accesses where every row starts at one
  const bool dense = a.pitch == a.width && a.width % BLOCK8 == 0 && a.range.lo == nullptr, vec = a.pitch * sizeof(T) % 16 == 0;
  const dim3 grid = pack_grid(a.rows * a.blocks * 4, U, planes);
  if (unpack) {
    if (dense) unpack8_kernel<T, FMT, true, true, U><<<grid, 256, 0, s>>>(a);
    else if (vec) unpack8_kernel<T, FMT, false, true, U><<<grid, 256, 0, s>>>(a);
    else unpack8_kernel<T, FMT, false, false, U><<<grid, 256, 0, s>>>(a);
  } else {
    if (dense) pack8_kernel<T, FMT, true, true, U><<<grid, 256, 0, s>>>(a);
    else if (vec) pack8_kernel<T, FMT, false, true, U><<<grid, 256, 0, s>>>(a);
    else pack8_kernel<T, FMT, false, false, U><<<grid, 256, 0, s>>>(a);
  }
  return launch_status();
}
template <typename T, int FMT>
static int pack_for(const Pack8Args& a, int planes, bool unpack, hipStream_t s) {
  return a.rows * a.blocks * 4 * planes <= PACK_FEW ? pack_u<T, FMT, 1>(a, planes, unpack, s) : pack_u<T, FMT, PACK_U>(a, planes, unpack, s);
}
template <typename T, int FMT, bool SWIGLU>
static int restore_act(const Pack8Args& a, hipStream_t s) {
  constexpr int U = 2;
  const dim3 grid = pack_grid(a.rows * a.blocks * 4, U, 1);
  if (a.width % BLOCK8 == 0 && a.range.lo == nullptr) restore8_kernel<T, FMT, SWIGLU, true, U><<<grid, 256, 0, s>>>(a);
  else restore8_kernel<T, FMT, SWIGLU, false, U><<<grid, 256, 0, s>>>(a);
  return launch_status();
}
template <typename T, int FMT>
static int restore_for(const Pack8Args& a, bool swiglu, hipStream_t s) {
  return swiglu ? restore_act<T, FMT, true>(a, s) : restore_act<T, FMT, false>(a, s);
}
#define MOE_BY_TYPE(fn, ...)                                                                              \
  (dtype == MOE_DTYPE_BF16  ? (fmt == MOE_PACK_E4M3 ? fn<bf16, MOE_PACK_E4M3>(__VA_ARGS__) : fn<bf16, MOE_PACK_I8>(__VA_ARGS__))   \
   : dtype == MOE_DTYPE_F16 ? (fmt == MOE_PACK_E4M3 ? fn<f16, MOE_PACK_E4M3>(__VA_ARGS__) : fn<f16, MOE_PACK_I8>(__VA_ARGS__))     \
                            : (fmt == MOE_PACK_E4M3 ? fn<float, MOE_PACK_E4M3>(__VA_ARGS__) : fn<float, MOE_PACK_I8>(__VA_ARGS__)))

int launch_pack8(int dtype, int fmt, long long rows, int width, long long pitch, const void* src, void* codes, void* scales, hipStream_t s) {
  const Pack8Args a = {src, nullptr, (uint8_t*)codes, (uint8_t*)scales, rows, pitch, width, blocks8(width), {}};
  return MOE_BY_TYPE(pack_for, a, 1, false, s);
}
int launch_unpack8(int dtype, int fmt, long long rows, int width, long long pitch, const void* codes, const void* scales, void* dst, hipStream_t s) {
  const Pack8Args a = {nullptr, dst, (uint8_t*)const_cast<void*>(codes), (uint8_t*)const_cast<void*>(scales), rows, pitch, width, blocks8(width), {}};
  return MOE_BY_TYPE(pack_for, a, 1, true, s);
}
int launch_saved_pack8(const moe_cfg* c, int fmt, const void* saved, const RowRange& range, void* codes, void* scales, hipStream_t s) {
  const int dtype = c->dtype;
  const Pack8Args a = {saved, nullptr, (uint8_t*)codes, (uint8_t*)scales, (long long)c->T * c->k, c->d_ff, c->d_ff, blocks8(c->d_ff), range};
  return MOE_BY_TYPE(pack_for, a, c->act == MOE_ACT_SWIGLU ? 2 : 1, false, s);
}
int launch_saved_restore8(const moe_cfg* c, int fmt, const void* codes, const void* scales, const RowRange& range, void* saved, hipStream_t s) {
  const int dtype = c->dtype;
  const Pack8Args a = {nullptr, saved, (uint8_t*)const_cast<void*>(codes), (uint8_t*)const_cast<void*>(scales), (long long)c->T * c->k, c->d_ff, c->d_ff,
                       blocks8(c->d_ff), range};
  return MOE_BY_TYPE(restore_for, a, c->act == MOE_ACT_SWIGLU, s);
}

}  // namespace moe
