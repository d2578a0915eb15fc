// Root-mean-square norm of a residual stream that takes in a branch, with dropout on the branch: forward and backward; and dropout
// by itself.
//   forward    h = residual + drop(x), rounded to the stream's type; r = 1 / sqrt(mean(h^2) + eps); y = gamma h r, written in the
//              storage type, in 8-bit integers with a scale for the row, or both
//   backward   u = h r, a = gamma dy; dh = r (a - u mean(a u)) + dh_add; dx = drop(dh) with the same mask; dgamma = sum over rows of dy u
// The norm is that of h as it is stored: the backward, which reads it, differentiates exactly what the forward computed, and a
// forward from a kept h gives the same bits.  Sums are fp32; every result is rounded once.
//
// One pass over memory each: a row stays in the registers of one or several waves (rows.h) between its sums and its results.  Bound by HBM:
// 16384 rows of 4096, bf16 in an fp32 stream, dropout 0.1: forward 805 MB in 148 us, 5.4 TB/s, backward 1074 MB in 216 us, 5.0 TB/s, and 5 us
// for adding gamma's partial sums (a copy of 2 GiB runs at 5.6 TB/s).  Small ones by latency: 300 rows of 516 fp32 4.5 and 5.3 us.
#include "gemm.h"
#include "norm.h"

namespace moe {

template <typename T, typename S, bool ODD, int MAXW, int NCH>
__global__ __launch_bounds__(MAXW == 1 ? 256 : MAXW * WAVE) void norm_fwd_kernel(NormFwdArgs a) {
  constexpr int R = MAXW == 1 ? 4 : 1;
  __shared__ __align__(16) float s_sum[2][MAXW];
  __shared__ __align__(16) unsigned s_top[2][MAXW];
  const int TPR = MAXW == 1 ? WAVE : (int)blockDim.x, tid = MAXW == 1 ? threadIdx.x % WAVE : threadIdx.x, d = a.d;
  row_reduce_init<MAXW>(s_sum[0]);
  row_reduce_init<MAXW>(s_top[0]);
  const T* gamma = reinterpret_cast<const T*>(a.gamma);
  const uint64_t offset = a.drop.cut != 0 ? drop_offset(a.drop) : 0;
  int turn = 0;
  for (int row = blockIdx.x * R + (MAXW == 1 ? threadIdx.x / WAVE : 0); row < a.T; row += gridDim.x * R, turn ^= 1) {
    const size_t at = (size_t)row * d;
    const T* x = reinterpret_cast<const T*>(a.x) + at;
    Raw8<T> xr[NCH];
    Raw8<S> rr[NCH];
#pragma unroll
    for (int i = 0; i < NCH; ++i) xr[i] = load_row8<T, ODD>(x, (i * TPR + tid) * 8, d);
    if (a.residual != nullptr) {
#pragma unroll
      for (int i = 0; i < NCH; ++i) rr[i] = load_row8<S, ODD>(reinterpret_cast<const S*>(a.residual) + at, (i * TPR + tid) * 8, d);
    }
    float v[NCH][8], sum = 0.f;
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      unpack_row8<T, ODD>(xr[i], (i * TPR + tid) * 8, d, v[i]);
      if (a.drop.cut != 0) drop8(a.drop, offset, (uint32_t)row, (uint32_t)(i * TPR + tid), v[i]);
      if (a.residual != nullptr) {
        float q[8];
        unpack_row8<S, ODD>(rr[i], (i * TPR + tid) * 8, d, q);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] += q[j];
      }
      const Raw8<S> h = pack_row8<S>(v[i]);
      if (a.h != nullptr) store_row8<S, ODD>(reinterpret_cast<S*>(a.h) + at, (i * TPR + tid) * 8, d, h);
      unpack8<S>(h, v[i]);
#pragma unroll
      for (int j = 0; j < 8; ++j) sum = fmaf(v[i][j], v[i][j], sum);
    }
    sum = row_reduce<MAXW>(sum, s_sum[turn], add_f);
    const float r = 1.f / sqrtf(sum / (float)d + a.eps);
    if (a.rstd != nullptr && tid == 0) a.rstd[row] = r;
    unsigned top = 0;
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int c = (i * TPR + tid) * 8;
      float g[8];
      if (gamma != nullptr) unpack_row8<T, ODD>(load_row8<T, ODD, false>(gamma, c, d), c, d, g);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        v[i][j] *= r;
        if (gamma != nullptr) v[i][j] *= g[j];
      }
      if (a.y != nullptr) store_row8<T, ODD>(reinterpret_cast<T*>(a.y) + at, c, d, pack_row8<T>(v[i]));
      top = top_of(top, v[i]);
    }
    if (a.codes != nullptr) {
      const RowScale q = row_scale(row_reduce<MAXW>(top, s_top[turn], max_u));
      if (tid == 0) a.scales[row] = q.scale;
#pragma unroll
      for (int i = 0; i < NCH; ++i) store_codes8<ODD>(a.codes + at, (i * TPR + tid) * 8, d, codes8(v[i], q.up));
    }
  }
}

// Gamma's gradient for a few columns from all rows: 128 threads for every eight columns, by rows, whose sums are added in order, in sixteen
// runs of eight first.
template <typename T, typename S, bool ODD, int THREADS>
__device__ __forceinline__ void dgamma_few(const NormBwdArgs& a, int block) {
  constexpr int LANES = FEW_LANES, MOST = THREADS / LANES * 8;   // columns of a block, at most
  __shared__ float part[LANES][MOST + 1], run[16][MOST + 1];
  const int groups = blockDim.x / LANES, cols = groups * 8, cg = threadIdx.x % groups, rl = threadIdx.x / groups, c0 = block * cols, c = c0 + cg * 8, d = a.d;
  const bool live = (int)threadIdx.x < groups * LANES;   // (a block need not be whole groups of 128 threads)
  float s[8] = {};
#pragma unroll 4
  for (int r = live ? rl : a.T; r < a.T; r += LANES) {
    const size_t at = (size_t)r * d;
    float w[8], u[8];
    unpack_row8<T, ODD>(load_row8<T, ODD, false>(reinterpret_cast<const T*>(a.dy) + at, c, d), c, d, w);
    unpack_row8<S, ODD>(load_row8<S, ODD, false>(reinterpret_cast<const S*>(a.h) + at, c, d), c, d, u);
    const float q = a.rstd[r];
#pragma unroll
    for (int j = 0; j < 8; ++j) s[j] = fmaf(w[j], u[j] * q, s[j]);
  }
  if (live) {
#pragma unroll
    for (int j = 0; j < 8; ++j) part[rl][cg * 8 + j] = s[j];
  }
  __syncthreads();
  const int col = threadIdx.x % cols, seg = threadIdx.x / cols;   // 16 segments of the live threads
  float sum = 0.f;
  if (live) {
#pragma unroll
    for (int r = 0; r < 8; ++r) sum += part[seg * 8 + r][col];
    run[seg][col] = sum;
  }
  __syncthreads();
  if ((int)threadIdx.x >= cols || c0 + col >= d) return;
#pragma unroll
  for (int r = 1; r < 16; ++r) sum += run[r][col];
  if (a.grad == MOE_DTYPE_F32) {
    float* out = reinterpret_cast<float*>(a.dgamma) + c0 + col;
    *out = sum + (a.accumulate ? *out : 0.f);
  } else {   // T: gamma's own type
    reinterpret_cast<T*>(a.dgamma)[c0 + col] = from_f32<T>(sum);
  }
}

template <typename T, typename S, bool ODD, int MAXW, int NCH>
__global__ __launch_bounds__(MAXW == 1 ? 256 : MAXW * WAVE) void norm_bwd_kernel(NormBwdArgs a) {
  // the columns' blocks first, they take longest; the blocks of an XCD next to each other, so that they share the lines that they cut
  const int block = (int)blockIdx.x - a.col_blocks;
  if (block < 0) return dgamma_few<T, S, ODD, MAXW == 1 ? 256 : MAXW * WAVE>(a, chunk_position(blockIdx.x, a.col_blocks, a.col_blocks / NUM_XCD + 1));
  constexpr int R = MAXW == 1 ? 4 : 1;
  __shared__ __align__(16) float s_sum[2][MAXW];
  const int TPR = MAXW == 1 ? WAVE : (int)blockDim.x, tid = MAXW == 1 ? threadIdx.x % WAVE : threadIdx.x, d = a.d;
  row_reduce_init<MAXW>(s_sum[0]);
  const T* gamma = reinterpret_cast<const T*>(a.gamma);
  const uint64_t offset = a.drop.cut != 0 ? drop_offset(a.drop) : 0;
  float dg[NCH][8] = {};
  int turn = 0;
  // The next row is requested before this one is used, where registers hold both.
  constexpr bool AHEAD = NCH < 4, ADD_EARLY = AHEAD || (sizeof(S) == 2 && !ODD);
  struct Row { Raw8<T> dy[NCH]; Raw8<S> h[NCH], add[NCH]; float r; };
  auto fetch = [&](int row, Row& f) {
    if (row >= a.T) return;
    const size_t at = (size_t)row * d;
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      f.dy[i] = load_row8<T, ODD>(reinterpret_cast<const T*>(a.dy) + at, (i * TPR + tid) * 8, d);
      f.h[i] = load_row8<S, ODD>(reinterpret_cast<const S*>(a.h) + at, (i * TPR + tid) * 8, d);
      if (ADD_EARLY && a.dh_add != nullptr) f.add[i] = load_row8<S, ODD>(reinterpret_cast<const S*>(a.dh_add) + at, (i * TPR + tid) * 8, d);
    }
    f.r = a.rstd[row];
  };
  Row now = {}, next = {};
  const int first = block * R + (MAXW == 1 ? threadIdx.x / WAVE : 0), stride = a.row_blocks * R;
  if constexpr (AHEAD) fetch(first, now);
  for (int row = first; row < a.T; row += stride, turn ^= 1) {
    if constexpr (AHEAD) fetch(row + stride, next);
    else fetch(row, now);
    const size_t at = (size_t)row * d;
    const float r = now.r;
    float w[NCH][8], u[NCH][8], dot = 0.f;
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      unpack_row8<T, ODD>(now.dy[i], (i * TPR + tid) * 8, d, w[i]);
      unpack_row8<S, ODD>(now.h[i], (i * TPR + tid) * 8, d, u[i]);
      float g[8];
      if (gamma != nullptr) unpack_row8<T, ODD>(load_row8<T, ODD, false>(gamma, (i * TPR + tid) * 8, d), (i * TPR + tid) * 8, d, g);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        u[i][j] *= r;
        dg[i][j] = fmaf(w[i][j], u[i][j], dg[i][j]);
        if (gamma != nullptr) w[i][j] *= g[j];
        dot = fmaf(w[i][j], u[i][j], dot);
      }
    }
    dot = row_reduce<MAXW>(dot, s_sum[turn], add_f) / (float)d;
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int c = (i * TPR + tid) * 8;
      float q[8];
      if (a.dh_add != nullptr) {
        if constexpr (!ADD_EARLY) now.add[i] = load_row8<S, ODD>(reinterpret_cast<const S*>(a.dh_add) + at, c, d);
        unpack_row8<S, ODD>(now.add[i], c, d, q);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        w[i][j] = r * (w[i][j] - u[i][j] * dot);
        if (a.dh_add != nullptr) w[i][j] += q[j];
      }
      if (a.dh != nullptr) store_row8<S, ODD>(reinterpret_cast<S*>(a.dh) + at, c, d, pack_row8<S>(w[i]));
      if (a.dx != nullptr) {
        if (a.drop.cut != 0) drop8(a.drop, offset, (uint32_t)row, (uint32_t)(i * TPR + tid), w[i]);
        store_row8<T, ODD>(reinterpret_cast<T*>(a.dx) + at, c, d, pack_row8<T>(w[i]));
      }
    }
    if constexpr (AHEAD) now = next;
  }
  if (a.partials == nullptr || a.col_blocks > 0) return;
  float* out = a.partials + (size_t)block * d;
  if constexpr (R > 1) {   // the block's waves one after the other: the same order every time
    __shared__ float s_dg[NCH * WAVE * 8];
    for (int w = 1; w < R; ++w) {
      if ((int)threadIdx.x / WAVE == w) {
#pragma unroll
        for (int i = 0; i < NCH; ++i)
#pragma unroll
          for (int j = 0; j < 8; ++j) s_dg[(i * 8 + j) * WAVE + tid] = dg[i][j];
      }
      __syncthreads();
      if (threadIdx.x < WAVE) {
#pragma unroll
        for (int i = 0; i < NCH; ++i)
#pragma unroll
          for (int j = 0; j < 8; ++j) dg[i][j] += s_dg[(i * 8 + j) * WAVE + tid];
      }
      __syncthreads();
    }
    if (threadIdx.x >= WAVE) return;
  }
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    const int c = (i * TPR + tid) * 8;
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (c + j < d) out[c + j] = dg[i][j];
  }
}

// Column sums of the partial sums: 16 columns by 64 rows at a time, whose sums are added in order.  (16 rows at a time: 6.6 us for 1024
// rows of 4096, every thread 64 loads long.)
constexpr int DGAMMA_ROWS = 64;
template <typename OT>
__global__ __launch_bounds__(16 * DGAMMA_ROWS) void norm_dgamma_kernel(const float* partials, int rows, int d, OT* out, int accumulate) {
  __shared__ float part[DGAMMA_ROWS][17];
  const int cl = threadIdx.x & 15, rl = threadIdx.x >> 4, c = blockIdx.x * 16 + cl;
  float sum = 0.f;
  if (c < d) {
#pragma unroll 8
    for (int r = rl; r < rows; r += DGAMMA_ROWS) sum += partials[(size_t)r * d + c];
  }
  part[rl][cl] = sum;
  __syncthreads();
  if (rl >= 4) return;
#pragma unroll
  for (int r = 4; r < DGAMMA_ROWS; r += 4) sum += part[rl + r][cl];
  sum += __shfl_down(sum, 32, WAVE);   // rows 0 and 2, 1 and 3; then those two
  sum += __shfl_down(sum, 16, WAVE);
  if (rl == 0 && c < d) out[c] = from_f32<OT>(sum + (accumulate ? to_f32(out[c]) : 0.f));
}

// A thread takes U groups of eight adjacent values, 256 apart, and requests them all before it uses the first.  Rows are found by a
// division of a block's own 32-bit numbers.  32768 rows of 4096 bf16 with a residual 805 MB in 136 us, 5.9 TB/s, without 537 MB in 88, 6.1 TB/s:
// HBM, with the vector ALUs at 0.77 of their cycles for the generator.
template <typename T, int U>
__global__ __launch_bounds__(256) void dropout_kernel(DropArgs drop, const T* x, const T* residual, T* y, long long rows, int width, unsigned groups) {
  const uint64_t offset = drop_offset(drop);
  const long long first = (long long)blockIdx.x * (256 * U), row0 = first / groups;
  const unsigned in0 = (unsigned)(first - row0 * groups);
  Raw8<T> xr[U], rr[U];
  long long row[U];
  unsigned g[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const unsigned i = in0 + u * 256 + threadIdx.x, q = i / groups;
    row[u] = row0 + q;
    g[u] = i - q * groups;
    if (row[u] >= rows) continue;
    xr[u] = load_row8<T, true>(x + row[u] * width, (int)g[u] * 8, width);
    if (residual != nullptr) rr[u] = load_row8<T, true>(residual + row[u] * width, (int)g[u] * 8, width);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (row[u] >= rows) break;
    float v[8];
    unpack_row8<T, true>(xr[u], (int)g[u] * 8, width, v);
    if (drop.cut != 0) drop8(drop, offset, (uint32_t)row[u], g[u], v);
    if (residual != nullptr) {
      float q[8];
      unpack_row8<T, true>(rr[u], (int)g[u] * 8, width, q);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] += q[j];
    }
    store_row8<T, true>(y + row[u] * width, (int)g[u] * 8, width, pack_row8<T>(v));
  }
}

// ---- launches ------------------------------------------------------------------------------------------------------
constexpr int NORM_MOST_BLOCKS = 1 << 16;   // further rows in further turns

// F(odd, most waves of a row, groups per thread) by the geometry of a row.
#define MOE_NORM_GEOM_(O_, G_, F_)                                          \
  do {                                                                      \
    if (G_.waves == 1) { if (G_.nch == 1) F_(O_, 1, 1); else F_(O_, 1, 2); } \
    else if (G_.nch == 1) F_(O_, 8, 1);                                     \
    else if (G_.nch == 2) F_(O_, 8, 2);                                     \
    else F_(O_, 8, 4);                                                      \
  } while (0)
#define MOE_NORM_GEOM(D_, G_, F_) do { if ((D_) % 8 != 0) MOE_NORM_GEOM_(true, G_, F_); else MOE_NORM_GEOM_(false, G_, F_); } while (0)

template <typename T, typename S>
static int norm_fwd_for(const NormFwdArgs& a, hipStream_t s) {
  const RowGeom geom = norm_geom(a.T, a.d);
  const int rows = rows_per_block(geom);
  const long long want = ((long long)a.T + rows - 1) / rows;
  const unsigned grid = (unsigned)(want < NORM_MOST_BLOCKS ? want : NORM_MOST_BLOCKS);
#define MOE_NORM_FWD(O_, W_, C_) norm_fwd_kernel<T, S, O_, W_, C_><<<grid, row_threads(geom), 0, s>>>(a)
  MOE_NORM_GEOM(a.d, geom, MOE_NORM_FWD);
#undef MOE_NORM_FWD
  return launch_status();
}
int launch_norm_fwd(const moe_norm* n, const NormFwdArgs& a, hipStream_t s) {
  if (n->dtype == MOE_DTYPE_F32) return norm_fwd_for<float, float>(a, s);
  if (n->dtype == MOE_DTYPE_BF16) return n->stream == MOE_DTYPE_F32 ? norm_fwd_for<bf16, float>(a, s) : norm_fwd_for<bf16, bf16>(a, s);
  return n->stream == MOE_DTYPE_F32 ? norm_fwd_for<f16, float>(a, s) : norm_fwd_for<f16, f16>(a, s);
}

template <typename T, typename S>
static int norm_bwd_for(const NormBwdArgs& a, hipStream_t s) {
  const RowGeom geom = norm_geom(a.T, a.d);
  const unsigned grid = (unsigned)(a.row_blocks + a.col_blocks);
#define MOE_NORM_BWD(O_, W_, C_) norm_bwd_kernel<T, S, O_, W_, C_><<<grid, row_threads(geom), 0, s>>>(a)
  MOE_NORM_GEOM(a.d, geom, MOE_NORM_BWD);
#undef MOE_NORM_BWD
  return launch_status();
}
template <typename OT>
static int dgamma_for(const float* partials, int rows, int d, void* out, int accumulate, hipStream_t s) {
  norm_dgamma_kernel<OT><<<(d + 15) / 16, 16 * DGAMMA_ROWS, 0, s>>>(partials, rows, d, (OT*)out, accumulate);
  return launch_status();
}
int launch_norm_bwd(const moe_norm* n, const NormBwdArgs& args, void* dgamma, int accumulate, hipStream_t s) {
  NormBwdArgs a = args;
  a.row_blocks = n->T > 0 ? norm_bwd_blocks(n->T, n->d) : 0;
  a.grad = n->grad;
  a.accumulate = accumulate;
  a.dgamma = dgamma;
  const int cols = few_cols(norm_geom(n->T, n->d));
  // (not where a result takes the place of what the columns' blocks read)
  const bool in_place = a.dx == a.dy || a.dh == a.dy || a.dx == a.h || a.dh == a.h;
  if (n->T > 0 && n->T <= NORM_FEW && dgamma != nullptr && !in_place) a.col_blocks = (n->d + cols - 1) / cols;
  if (n->T > 0) {
    int rc;
    if (n->dtype == MOE_DTYPE_F32) rc = norm_bwd_for<float, float>(a, s);
    else if (n->dtype == MOE_DTYPE_BF16) rc = n->stream == MOE_DTYPE_F32 ? norm_bwd_for<bf16, float>(a, s) : norm_bwd_for<bf16, bf16>(a, s);
    else rc = n->stream == MOE_DTYPE_F32 ? norm_bwd_for<f16, float>(a, s) : norm_bwd_for<f16, f16>(a, s);
    if (rc != MOE_OK || a.col_blocks > 0) return rc;
  }
  if (dgamma == nullptr || (n->T == 0 && accumulate)) return MOE_OK;
  return n->grad == MOE_DTYPE_F32    ? dgamma_for<float>(a.partials, a.row_blocks, n->d, dgamma, accumulate, s)
         : n->grad == MOE_DTYPE_BF16 ? dgamma_for<bf16>(a.partials, a.row_blocks, n->d, dgamma, accumulate, s)
                                     : dgamma_for<f16>(a.partials, a.row_blocks, n->d, dgamma, accumulate, s);
}

template <typename T>
static int dropout_for(long long rows, int width, const DropArgs& drop, const void* x, const void* residual, void* y, hipStream_t s) {
  const unsigned groups = (unsigned)((width + 7) / 8);
  const long long items = rows * groups;
  if (items >= 256 * 2048) {
    dropout_kernel<T, 2><<<(unsigned)((items + 511) / 512), 256, 0, s>>>(drop, (const T*)x, (const T*)residual, (T*)y, rows, width, groups);
  } else {
    dropout_kernel<T, 1><<<(unsigned)((items + 255) / 256), 256, 0, s>>>(drop, (const T*)x, (const T*)residual, (T*)y, rows, width, groups);
  }
  return launch_status();
}
int launch_dropout(int dtype, long long rows, int width, const DropArgs& drop, const void* x, const void* residual, void* y, hipStream_t s) {
  if (dtype == MOE_DTYPE_F32) return dropout_for<float>(rows, width, drop, x, residual, y, s);
  if (dtype == MOE_DTYPE_BF16) return dropout_for<bf16>(rows, width, drop, x, residual, y, s);
  return dropout_for<f16>(rows, width, drop, x, residual, y, s);
}

}  // namespace moe
