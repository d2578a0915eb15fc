// Rows and weights to 8-bit integers with one scale per row or per column: m = max(largest magnitude, 2^-100), codes round(v * (127 / m)),
// scale m / 127 (rows.h).
#include "quant8.h"

namespace moe {

// One pass: a row stays in registers between its maximum and its codes.  32768 rows of 4096 bf16 403 MB in 61 us, 6.6 TB/s; 65536 of 1024
// 36 us, 5.6 TB/s.
template <typename T, bool ODD, int MAXW, int NCH>
__global__ __launch_bounds__(MAXW == 1 ? 256 : MAXW * WAVE) void quant_rows_kernel(const T* src, long long rows, int width, long long pitch, RowRange range,
                                                                             int8_t* codes, float* scales) {
  constexpr int R = MAXW == 1 ? 4 : 1;
  __shared__ int32_t s_range[2 * MOE_MAX_E];
  __shared__ unsigned s_top[2][MAXW];
  const RangeTable rt = load_range(range, s_range);
  const long long end = rt.limit(rows);
  const int TPR = MAXW == 1 ? WAVE : (int)blockDim.x, tid = MAXW == 1 ? threadIdx.x % WAVE : threadIdx.x;
  row_reduce_init<MAXW>(s_top[0]);
  int turn = 0;
  for (long long row = (long long)blockIdx.x * R + (MAXW == 1 ? threadIdx.x / WAVE : 0); row < end; row += (long long)gridDim.x * R) {
    if (!rt.live(row)) continue;   // (the same for every thread of a row, and of a block where several waves share one)
    float v[NCH][8];
    unsigned top = 0;
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      unpack_row8<T, ODD>(load_row8<T, ODD>(src + row * pitch, (i * TPR + tid) * 8, width), (i * TPR + tid) * 8, width, v[i]);
      top = top_of(top, v[i]);
    }
    const RowScale q = row_scale(row_reduce<MAXW>(top, s_top[turn], max_u));
    turn ^= 1;
    if (tid == 0) scales[row] = q.scale;
#pragma unroll
    for (int i = 0; i < NCH; ++i) store_codes8<ODD>(codes + row * width, (i * TPR + tid) * 8, width, codes8(v[i], q.up));
  }
}

// A block takes 64 columns of a matrix and reads them twice: for the columns' maxima, then for the codes, whose 64 x 64 patches turn
// in LDS.  Work done once, when weights are loaded, and bound by how few blocks a single matrix has: bf16, 4096 x 14336 136 us, 14336 x 4096
// (64 blocks) 449 us, 0.4 TB/s of 176 MB read once and written; 8 of 4096 x 14336 521 us, 64 of 2048 x 1024 140 us, 2.7 and 2.9 TB/s.
template <typename T>
__global__ __launch_bounds__(256) void quant_weight_kernel(const T* W, int d_in, int d_out, int8_t* codes, float* scales) {
  constexpr int PITCH = 64 + 16;   // bytes between the columns of a patch
  __shared__ __align__(16) int8_t s_patch[64 * PITCH];
  __shared__ unsigned s_top[32][64];
  __shared__ float s_up[64];
  const int cg = threadIdx.x & 7, rl = threadIdx.x >> 3, c0 = blockIdx.x * 64;   // eight columns; row of 32
  const T* src = W + (size_t)blockIdx.y * d_in * d_out + c0;
  unsigned top[8] = {};
  for (int r = rl; r < d_in; r += 32) {
    float v[8];
    unpack8<T>(load_row8<T, false, false>(src + (size_t)r * d_out, cg * 8, 64), v);
#pragma unroll
    for (int j = 0; j < 8; ++j) top[j] = max(top[j], __float_as_uint(v[j]) & 0x7fffffffu);
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) s_top[rl][cg * 8 + j] = top[j];
  __syncthreads();
  if (threadIdx.x < 64) {
    unsigned t = 0;
    for (int r = 0; r < 32; ++r) t = max(t, s_top[r][threadIdx.x]);
    const RowScale q = row_scale(t);
    s_up[threadIdx.x] = q.up;
    scales[(size_t)blockIdx.y * d_out + c0 + threadIdx.x] = q.scale;
  }
  __syncthreads();
  float up[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) up[j] = s_up[cg * 8 + j];
  const int lane = threadIdx.x & 63, ct = threadIdx.x >> 6;   // a wave writes the tile of 16 columns
  int8_t* out = codes + (size_t)blockIdx.y * d_in * d_out + (size_t)(c0 / TILE8_N + ct) * (d_in / TILE8_K) * TILE8_BYTES + lane * 16;
  for (int k0 = 0; k0 < d_in; k0 += TILE8_K) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int r = rl + 32 * h;
      float v[8];
      unpack8<T>(load_row8<T, false, false>(src + (size_t)(k0 + r) * d_out, cg * 8, 64), v);
#pragma unroll
      for (int j = 0; j < 8; ++j) s_patch[(cg * 8 + j) * PITCH + r] = (int8_t)(up[j] != 0.f ? (int)rintf(v[j] * up[j]) : 0);
    }
    __syncthreads();
    *reinterpret_cast<uint4*>(out) = *reinterpret_cast<const uint4*>(s_patch + (ct * 16 + (lane & 15)) * PITCH + (lane >> 4) * 16);
    out += TILE8_BYTES;
    __syncthreads();
  }
}

constexpr int QUANT_MOST_BLOCKS = 1 << 16;   // further rows in further turns
// Two to four groups of eight per thread: a row is short work, and threads with several requests in flight make more of it than more
// threads.  (32768 rows of 4096 bf16, us: one group in eight waves 81, two in four waves 63; 16384 of 2048: 22.7, 19.1, four in one
// wave 18.4; 3001 of 2880 8.2, 6.4.)
static RowGeom quant_geom(int width) {
  const int g = (width + 7) / 8;
  if (g <= 128) return {1, 2};
  if (g <= 256) return {1, 4};
  const int nch = g <= 512 ? 2 : g <= 4096 ? 4 : 8;
  return {row_waves(g, nch), nch};
}
static_assert(MOE_MAX_ROW == 16 * WAVE * 8 * 8, "sixteen waves hold the widest row");
template <typename T>
static int quant_rows_for(long long rows, int width, long long pitch, const void* src, const RowRange& range, int8_t* codes, float* scales, hipStream_t s) {
  const RowGeom g = quant_geom(width);
  const long long per = rows_per_block(g), want = (rows + per - 1) / per;
  const unsigned grid = (unsigned)(want < QUANT_MOST_BLOCKS ? want : QUANT_MOST_BLOCKS);
#define MOE_QUANT_ROWS(O_, W_, C_) quant_rows_kernel<T, O_, W_, C_><<<grid, row_threads(g), 0, s>>>((const T*)src, rows, width, pitch, range, codes, scales)
#define MOE_QUANT_GEOM(O_)                        \
  do {                                            \
    if (g.waves == 1) { if (g.nch == 2) MOE_QUANT_ROWS(O_, 1, 2); else MOE_QUANT_ROWS(O_, 1, 4); } \
    else if (g.nch == 2) MOE_QUANT_ROWS(O_, 4, 2); \
    else if (g.nch == 4 && g.waves <= 8) MOE_QUANT_ROWS(O_, 8, 4); \
    else if (g.nch == 4) MOE_QUANT_ROWS(O_, 16, 4); \
    else MOE_QUANT_ROWS(O_, 16, 8);               \
  } while (0)
  if (width % 8 != 0) MOE_QUANT_GEOM(true);
  else MOE_QUANT_GEOM(false);
#undef MOE_QUANT_ROWS
  return launch_status();
}
int launch_quant_rows(int dtype, long long rows, int width, long long pitch, const void* src, const RowRange& range, int8_t* codes, float* scales, hipStream_t s) {
  if (dtype == MOE_DTYPE_F32) return quant_rows_for<float>(rows, width, pitch, src, range, codes, scales, s);
  if (dtype == MOE_DTYPE_BF16) return quant_rows_for<bf16>(rows, width, pitch, src, range, codes, scales, s);
  return quant_rows_for<f16>(rows, width, pitch, src, range, codes, scales, s);
}
int launch_quant_weight(int dtype, int n, int d_in, int d_out, const void* W, int8_t* codes, float* scales, hipStream_t s) {
  const dim3 grid(d_out / 64, n);
  if (dtype == MOE_DTYPE_F32) quant_weight_kernel<float><<<grid, 256, 0, s>>>((const float*)W, d_in, d_out, codes, scales);
  else if (dtype == MOE_DTYPE_BF16) quant_weight_kernel<bf16><<<grid, 256, 0, s>>>((const bf16*)W, d_in, d_out, codes, scales);
  else quant_weight_kernel<f16><<<grid, 256, 0, s>>>((const f16*)W, d_in, d_out, codes, scales);
  return launch_status();
}

}  // namespace moe
