// Dense products with a fused epilogue, y = act(x W + bias) + residual, and their backward (the shared expert of an MoE block).
//
// The products run on the tiles of the grouped GEMMs (gemm_bf16_kernel.h, gemm_f32.hip) with one matrix and no tile map; bias,
// activation, residual and the rounding to the storage type sit in their epilogues, on the fp32 sums.  Where the sums of a
// tile are cut along K, so that few tiles fill the chip, the kernel that adds the parts has the epilogue.
//   forward   tiles of 64 x 128 to 256 x 256 by a cost model fitted to measurements, the last round cut along K; up to 64 rows the
//             weights are streamed (HBM), beyond that the matrix cores bound it
//   backward  dz = dy act'(pre) and its column sums in one pass (HBM); dx = dz W^T as the forward; dW = x^T dz on tiles of 256 x 256 or
//             128 x 128, the tokens cut into segments where the gradient has few tiles, whose sums a last pass adds up
#include "gemm.h"
#include "linear.h"
#include "pack8.h"
#include <algorithm>

namespace moe {

int linear_forward_f32(int act, const GemmArgs& g, hipStream_t s);   // gemm_f32.hip
int linear_backward_f32(bool two, const GemmArgs& g1, const GemmArgs& g2, hipStream_t s);
int linear_forward_bf16(int act, const GemmArgs& g, const LinearPlan& p, float* ws, hipStream_t s);   // linear_bf16.hip
int linear_input_grad_bf16(bool two, const GemmArgs& g, const LinearPlan& p, float* ws, hipStream_t s);
int linear_weight_grad_bf16(bool in_type, const GemmArgs& g, const LinearPlan& p, hipStream_t s);
int linear_both_grads_bf16(bool two, bool in_type, const GemmArgs& g1, const GemmArgs& g2, const LinearPlan& p, float* ws, hipStream_t s);
int linear_forward_f16(int act, const GemmArgs& g, const LinearPlan& p, float* ws, hipStream_t s);    // linear_f16.hip
int linear_input_grad_f16(bool two, const GemmArgs& g, const LinearPlan& p, float* ws, hipStream_t s);
int linear_weight_grad_f16(bool in_type, const GemmArgs& g, const LinearPlan& p, hipStream_t s);
int linear_both_grads_f16(bool two, bool in_type, const GemmArgs& g1, const GemmArgs& g2, const LinearPlan& p, float* ws, hipStream_t s);

constexpr int K_STAGE = 64;   // K values per stage of the 16-bit kernels

// ---- how a product is cut ------------------------------------------------------------------------------------------
// A tile shape of the 16-bit products: rows and columns (two matrices: of both together), how many tiles run at a time, and what a
// round of them takes, us: `fixed` in front of and behind the K loop, and per 64 K values `alone` where few tiles run and `full` where
// all do (tiles of 64 x 128: `alone` up to one on every compute unit, `full` with two).  Launch: 2 us.  Fitted to T x d x n:
//   one matrix    1024 x 1024 x 1024: 24.5 | 17.6 | 15.6 | 9.2 us in the order below;   300 x 4096 x 4096: 73 | 49 | 43 | 22;
//                 8192 x 4096 x 1024: 78 | 56 | 55 | 74;   8192 x 1024 x 4096: 58 | 73 | 64 | 91;   8192 x 2048 x 8192: 200 | 229 | 239 | 312
//   two           1024 x 1024 x 2048: 25.7 | 17.8 | 15.6 | 13.7;   4096 x 2048 x 4096: 101 | 125 | 111 | 157;   8192 x 2048 x 8192: 409 | 440 | 451 | 607
//   x^T dz        2048 x 1024 x 1024: 43 | 17;   8192 x 1024 x 4096: 143 | 63;   4096 x 2048 x 4096: 76 | 65;   4096 x 2048 x 8192: 96 | 128
// Few rows, weights that come from memory, parts as chosen: 1 x 4096 x 14336 (two) 41.5 us, 16 x 14336 x 4096 24.5: 5.7 and 4.8 TB/s.
struct Shape {
  int rows, cols, slots;
  double fixed, alone, full;
  double tiles_us(long long tiles, int stages) const {   // whole rounds of them, and the rest
    const long long r = tiles % slots, rounds = tiles / slots;
    double us = rounds * (fixed + stages * full);
    if (r > 0) us += fixed + stages * (slots > 256 ? (r <= 256 ? alone : full) : alone + (full - alone) * r / slots);
    return us;
  }
};
constexpr Shape SHAPES[] = {{256, 256, 256, 6.5, 1.0, 1.37}, {160, 256, 256, 5.0, 0.65, 0.91}, {128, 256, 256, 4.2, 0.58, 0.79}, {64, 128, 512, 2.5, 0.28, 0.54}};
constexpr Shape SHAPES_DUAL[] = {{256, 256, 256, 6.5, 1.07, 1.37}, {160, 256, 256, 5.5, 0.62, 0.86}, {128, 256, 256, 4.2, 0.6, 0.73}, {64, 256, 256, 3.3, 0.38, 0.5}};
constexpr Shape SHAPES_DW[] = {{256, 256, 256, 6.5, 1.05, 1.42}, {128, 128, 256, 3.5, 0.34, 0.44}};
constexpr double LAUNCH_US = 2.0, JOIN_US = 3.0, JOIN_US_PER_MB = 0.28;   // the adding launch; fp32 sums written and read again
constexpr int PART_STAGES = 4, MAX_PARTS = 16;   // K stages of 64 that a part has at least; parts at most

// How `stages` K stages of T x N sums are cut: the shape, and the K parts of its last round, that take the least time.
static RowCut cut_rows(long long T, int N, bool dual, int stages, double* us_of = nullptr) {
  RowCut best{};
  double least = 1e30;
  for (const Shape& s : dual ? SHAPES_DUAL : SHAPES) {
    RowCut c;
    c.rows = s.rows;
    c.cols = dual ? s.cols / 2 : s.cols;
    c.tiles = (T + c.rows - 1) / c.rows * ((N + c.cols - 1) / c.cols);
    const long long r = c.tiles % s.slots;
    for (int p = 1; p <= MAX_PARTS; ++p) {
      if (p > 1 && (r == 0 || p * r > s.slots || stages < p * PART_STAGES)) break;
      double us = s.tiles_us(c.tiles - r, stages) + s.tiles_us(r * p, (stages + p - 1) / p);
      if (p > 1) us += JOIN_US + JOIN_US_PER_MB * (double)r * p * s.rows * s.cols * 4 / 1e6;
      c.parts = p;
      c.first = p > 1 ? c.tiles - r : c.tiles;
      if (us < least) { least = us; best = c; }
    }
  }
  if (us_of != nullptr) *us_of = least;
  return best;
}
// fp32: tiles of 64 or 32 rows (f32_tile_rows) and 64 columns in K stages of 32, every tile cut into `parts`.  A stage takes the matrix
// cores 0.43 | 0.21 us of a compute unit per tile and at least 0.4 us, the way of its loads.  300 rows, K 1540, 516 columns: 90
// tiles in one part 23.4 us.
static RowCut cut_rows_f32(long long T, int N, int mats, int stages) {
  RowCut best{};
  double least = 1e30;
  for (int p = 1; p <= MAX_PARTS && (p == 1 || stages >= 4 * p); ++p) {
    RowCut c;
    c.rows = f32_tile_rows(T * p, 0, N);
    c.cols = F32_TILE_COLS;
    c.parts = p;
    c.first = 0;
    c.tiles = (T + c.rows - 1) / c.rows * ((N + c.cols - 1) / c.cols);
    const double stage = std::max(0.4, (c.rows == 64 ? 0.43 : 0.21) * mats * c.tiles * p / 256);
    double us = (stages + p - 1) / p * stage;
    if (p > 1) us += JOIN_US + JOIN_US_PER_MB * (double)T * N * 4 * p * mats / 1e6;
    if (us < least) { least = us; best = c; }
  }
  return best;
}
static size_t cut_bytes_f32(const RowCut& c, long long T, int N, int mats) { return c.parts > 1 ? (size_t)T * N * 4 * c.parts * mats : 0; }
constexpr int K_STAGE_F32 = 32;

static size_t cut_bytes(const RowCut& c, int mats) { return (size_t)(c.tiles - c.first) * c.parts * c.rows * c.cols * mats * 4; }

// Tiles of the weight gradient and segments of the tokens: the least time, the segments' sums counted as above.  A segment stays
// below 4 GiB of either operand (32-bit offsets).  fp32: 64 x 64 tiles, three on a compute unit, 2 us per 32 tokens.
static double cut_weight_grad(const moe_linear* c, int mats, LinearPlan& p) {
  const long long T = c->T;
  const bool half = c->dtype != MOE_DTYPE_F32;
  const double out_mb = (double)c->d_in * c->d_out * mats * 4 / 1e6;
  const long long row_bytes = (long long)std::max(c->d_in, c->d_out) * (half ? 2 : 4);
  const int first = (int)((T * row_bytes) / 0xf0000000ll) + 1;
  double least = 1e30;
  auto tiles_of = [&](int rows) { return (long long)((c->d_in + rows - 1) / rows) * ((c->d_out + rows - 1) / rows) * mats; };
  auto consider = [&](int rows, int segs, double us) {
    if (segs > 1) us += JOIN_US + JOIN_US_PER_MB * out_mb * segs;
    if (us < least) { least = us; p.dw_rows = rows; p.segs = segs; }
  };
  for (int segs = first; segs <= std::max(first, 16) && (segs == first || T / segs >= 256); ++segs) {
    const long long rows = (T + segs - 1) / segs;
    if (half) for (const Shape& s : SHAPES_DW) consider(s.rows, segs, s.tiles_us(tiles_of(s.rows) * segs, (int)((rows + K_STAGE - 1) / K_STAGE)));
    else consider(64, segs, (double)((tiles_of(64) * segs + F32_LOW_TILES - 1) / F32_LOW_TILES) * 0.06 * rows);
  }
  return least;
}
// Both gradients in one launch (16-bit; tiles of 64 x 128 and 128 x 128, one on a compute unit): where that takes less time than
// `apart`.  (So few tiles keep a segment's offsets far below 32 bits.)  One round of blocks: the longer of the two; two rounds: one after the other.  Two launches -> one, us: T x d x n
// 64 x 256 x 256 11.3 -> 7.8, 300 x 1024 x 1024 14.1 -> 9.2, 1024 x 1024 x 1024 19.1 -> 12.7, SwiGLU (dz included) 33.6 -> 22.7;
// 512 x 2048 x 1024 SwiGLU, 384 tiles, 26.4 -> 21.3; beyond two rounds 3000 x 1024 x 1024 28.3 -> 31.8.
constexpr int PAIR_TILES = 512;
static void try_pair(const moe_linear* c, int mats, double apart, LinearPlan& p) {
  const int dx_stages = mats * (c->d_out / K_STAGE);
  const long long dx_tiles = (long long)((c->T + 63) / 64) * ((c->d_in + 127) / 128);
  const long long dw_tiles = (long long)((c->d_in + 127) / 128) * ((c->d_out + 127) / 128) * mats;
  const double out_mb = (double)c->d_in * c->d_out * mats * 4 / 1e6;
  for (int segs = 1; segs <= 4 && (segs == 1 || c->T / segs >= 256); ++segs)
    for (int parts = 1; parts <= 8 && (parts == 1 || dx_stages >= parts * PART_STAGES); ++parts) {
      const long long n = dx_tiles * parts + dw_tiles * segs;
      if (n > PAIR_TILES) break;
      const double dx = 2.5 + 0.3 * ((dx_stages + parts - 1) / parts), dw = 3.5 + 0.45 * ((c->T + segs * K_STAGE - 1) / (segs * K_STAGE));
      double us = n <= 256 ? std::max(dx, dw) : dx + dw;
      if (parts > 1) us += JOIN_US + JOIN_US_PER_MB * (double)dx_tiles * parts * 64 * 128 * 4 / 1e6;
      if (segs > 1) us += JOIN_US + JOIN_US_PER_MB * out_mb * segs;
      if (us < apart) {
        apart = us;
        p.pair = true;
        p.dx = RowCut{dx_tiles, parts > 1 ? 0 : dx_tiles, 64, 128, parts};
        p.dw_rows = 128;
        p.segs = segs;
      }
    }
}
// the format of the pre-activations that the backward reads
static int pre_format(const moe_linear* c) { return c->act == MOE_ACT_NONE ? MOE_PACK_NONE : c->pre_pack; }
static int seg_rows(long long T, int segs) { return (int)(((T + segs - 1) / segs + 63) / 64 * 64); }

LinearPlan linear_plan(const moe_linear* c) {
  LinearPlan p{};
  const bool half = c->dtype != MOE_DTYPE_F32;
  const int mats = c->act == MOE_ACT_SWIGLU ? 2 : 1;
  const size_t es = half ? 2 : 4, T = c->T, N = c->d_out;
  size_t fwd = 0, off = 0;
  if (half) {
    p.fwd = cut_rows(c->T, c->d_out, mats == 2, c->d_in / K_STAGE);
    fwd = cut_bytes(p.fwd, mats);
  } else {
    p.fwd = cut_rows_f32(c->T, c->d_out, mats, (c->d_in + K_STAGE_F32 - 1) / K_STAGE_F32);
    fwd = cut_bytes_f32(p.fwd, c->T, c->d_out, mats);
  }
  // backward
  p.dz = off;
  if (c->act != MOE_ACT_NONE) off += align_up(mats * T * N * es, 256);
  p.bias_geom = bias_geom(c->T, c->d_out, act_bwd_cols(!half, pre_format(c)));
  p.db = off;
  off += align_up((size_t)mats * p.bias_geom.row_blocks * N * 4, 256);
  double dx_us = 0;
  if (half) p.dx = cut_rows(c->T, c->d_in, false, mats * (c->d_out / K_STAGE), &dx_us);
  else p.dx = cut_rows_f32(c->T, c->d_in, 1, mats * ((c->d_out + K_STAGE_F32 - 1) / K_STAGE_F32));
  p.segs = 1;
  if (c->T > 0) {
    const double dw_us = cut_weight_grad(c, mats, p);
    if (half) try_pair(c, mats, dx_us + dw_us + LAUNCH_US, p);
    else p.dw_rows = f32_tile_rows((long long)c->d_in * p.segs, 0, c->d_out);
    p.seg = seg_rows(c->T, p.segs);
    p.segs = (c->T + p.seg - 1) / p.seg;
  }
  p.dw_direct = p.segs == 1;   // the product writes the gradient itself
  p.split = off;
  off += align_up(half ? cut_bytes(p.dx, 1) : cut_bytes_f32(p.dx, c->T, c->d_in, 1), 256);
  p.dw = off;
  if (!p.dw_direct) off += align_up((size_t)mats * p.segs * c->d_in * N * 4, 256);
  p.fwd_total = c->T > 0 ? std::max(align_up(fwd, 256), (size_t)256) : 0;   // whole products need none; a call without one is a mistake still
  p.total = std::max(p.fwd_total, off);
  return p;
}

// ---- kernels -------------------------------------------------------------------------------------------------------
// dz = dy act'(pre), rounded to the storage type, and the column sums of the unrounded dz, one row of partial sums per block.
// A thread owns act_bwd_cols adjacent columns and walks down the rows of its block; cg threads span a block's columns.
// dz is kept in the storage type, which the matrix cores take: one rounding of the products' operand, as dy and the pre-activations
// have had theirs.  (With those of pre, a SwiGLU step's gradients are 3.1e-3 from those in 64 bits in bf16; rounded once, 1.7e-3.)
// Bound by HBM where there is much: SwiGLU 32768 x 14336 bf16, 4.7 GB, 0.78-0.92 ms = 5.1-6 TB/s, GELU 8192 x 4096, 201 MB,
// 40-44 us = 4.6-5; SwiGLU 4096 x 8192 from 8 bits, 270 MB, 70 us, by latency of two loads per row; few rows: 300 x 1540 fp32 9 us.
struct ActBwdArgs {
  const void* dy;
  const void *pre, *pre2;           // storage type, or codes
  const uint8_t *scales, *scales2;
  void *dz, *dz2;
  float *sums, *sums2;              // [row blocks][N] or NULL
  void *out, *out2;                 // one row block: the sums themselves, of type `grad`, or NULL
  int grad, accumulate;
  long long T;
  int N;
  BiasGeom gm;
};
template <typename ST, int ACT, int FMT>
__global__ __launch_bounds__(256) void act_bwd_kernel(ActBwdArgs a) {
  constexpr bool DUAL = ACT == MOE_ACT_SWIGLU;
  constexpr int VN = Vec16<ST>::N, CPT = act_bwd_cols(sizeof(ST) == 4, FMT);
  __shared__ float s_sum[4][64][(DUAL ? 2 : 1) * CPT + 1];
  const int cl = threadIdx.x & (a.gm.cg - 1), rl = threadIdx.x / a.gm.cg, rp = 256 / a.gm.cg;
  const int c = (blockIdx.x * a.gm.cg + cl) * CPT;
  const long long r0 = (long long)blockIdx.y * a.gm.rows, r1 = min(r0 + a.gm.rows, a.T);
  const int n = min(CPT, a.N - c);                     // columns of this thread: CPT, 4 (fp32) or none
  const int blocks = (a.N + BLOCK8 - 1) / BLOCK8;
  float sum[CPT] = {}, sum2[CPT] = {};
  auto load = [&](const void* p, long long r, float (&v)[CPT]) {
    const ST* at = reinterpret_cast<const ST*>(p) + r * a.N + c;
#pragma unroll
    for (int i = 0; i < CPT; i += VN)
      if (i < n) {
        Vec16<ST> q;
        q.load_nt(at + i);
        q.unpack(v + i);
      }
  };
  auto store = [&](void* p, long long r, const float (&v)[CPT]) {
    ST* at = reinterpret_cast<ST*>(p) + r * a.N + c;
#pragma unroll
    for (int i = 0; i < CPT; i += VN)
      if (i < n) {
        Vec16<ST> q;
        q.pack(v + i);
        q.store_nt(at + i);
      }
  };
  auto load_pre = [&](const void* p, const uint8_t* sc, long long r, float (&v)[CPT]) {
    if constexpr (FMT == MOE_PACK_NONE) load(p, r, v);
    else decode8<ST, FMT>(*reinterpret_cast<const uint2*>(reinterpret_cast<const uint8_t*>(p) + r * blocks * BLOCK8 + c), sc[r * blocks + c / BLOCK8], v);
  };
  // U rows of a thread are requested together; a row past the end repeats the last one and counts for nothing
  constexpr int U = CPT > VN ? 1 : 2;
  if (n > 0)
    for (long long ra = r0 + rl; ra < r1; ra += (long long)rp * U) {
      float dy[U][CPT] = {}, z[U][CPT] = {}, z2[U][CPT] = {};
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const long long r = min(ra + (long long)u * rp, r1 - 1);
        load(a.dy, r, dy[u]);
        if constexpr (ACT != MOE_ACT_NONE) load_pre(a.pre, a.scales, r, z[u]);
        if constexpr (DUAL) load_pre(a.pre2, a.scales2, r, z2[u]);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const long long r = ra + (long long)u * rp;
        if (r >= r1) break;
        float g[CPT], g2[CPT];
#pragma unroll
        for (int i = 0; i < CPT; ++i) {
          if constexpr (DUAL) {
            const float sg = sizeof(ST) == 4 ? sigmoid_f(z[u][i]) : __builtin_amdgcn_rcpf(1.f + __expf(-z[u][i]));
            g[i] = dy[u][i] * z2[u][i] * sg * fmaf(z[u][i], 1.f - sg, 1.f);
            g2[i] = dy[u][i] * z[u][i] * sg;
            sum2[i] += g2[i];
          } else if constexpr (ACT == MOE_ACT_GELU) {
            g[i] = dy[u][i] * (sizeof(ST) == 4 ? gelu_grad_f(z[u][i]) : gelu_grad_fast(z[u][i]));
          } else {
            g[i] = dy[u][i];
          }
          sum[i] += g[i];
        }
        if constexpr (ACT != MOE_ACT_NONE) store(a.dz, r, g);
        if constexpr (DUAL) store(a.dz2, r, g2);
      }
    }
  if (a.sums == nullptr && a.out == nullptr) return;
  // a wave's rows by exchanges between lanes, then the four waves in order
  for (int s = a.gm.cg; s < WAVE; s <<= 1)
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
      sum[i] += __shfl_xor(sum[i], s, WAVE);
      if constexpr (DUAL) sum2[i] += __shfl_xor(sum2[i], s, WAVE);
    }
  const int wave = threadIdx.x / WAVE;
  if ((threadIdx.x & (WAVE - 1)) < a.gm.cg) {
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
      s_sum[wave][cl][i] = sum[i];
      if constexpr (DUAL) s_sum[wave][cl][CPT + i] = sum2[i];
    }
  }
  __syncthreads();
  if (rl != 0 || n <= 0) return;
  for (int q = 1; q < 4; ++q)
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
      sum[i] += s_sum[q][cl][i];
      if constexpr (DUAL) sum2[i] += s_sum[q][cl][CPT + i];
    }
  if (a.out != nullptr) {
    auto put = [&](void* p, const float (&v)[CPT]) {
#pragma unroll
      for (int i = 0; i < CPT; ++i)
        if (i < n) {
          if (a.grad == MOE_DTYPE_F32) {
            float* o = reinterpret_cast<float*>(p) + c + i;
            *o = a.accumulate ? *o + v[i] : v[i];
          } else reinterpret_cast<ST*>(p)[c + i] = from_f32<ST>(v[i]);   // the storage type
        }
    };
    put(a.out, sum);
    if constexpr (DUAL) put(a.out2, sum2);
    return;
  }
#pragma unroll
  for (int i = 0; i < CPT; ++i)
    if (i < n) {
      a.sums[(size_t)blockIdx.y * a.N + c + i] = sum[i];
      if constexpr (DUAL) a.sums2[(size_t)blockIdx.y * a.N + c + i] = sum2[i];
    }
}

// out [n] (+)= the sum of `rows` rows of n floats, in row order; two of them (blockIdx.y) where the second is given.  Bound by HBM.
struct JoinArgs {
  const float* parts[2];
  void* out[2];
  size_t n;
  int rows, accumulate;
};
template <typename OT>
__global__ __launch_bounds__(256) void sum_rows_kernel(JoinArgs a) {
  const size_t i = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (i >= a.n) return;
  const float* src = a.parts[blockIdx.y] + i;
  OT* out = reinterpret_cast<OT*>(a.out[blockIdx.y]) + i;
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
  for (int r = 0; r < a.rows; ++r) s += *reinterpret_cast<const f32x4*>(src + (size_t)r * a.n);
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const float v = s[q] + (a.accumulate ? to_f32(out[q]) : 0.f);
    out[q] = from_f32<OT>(v);
  }
}

// The same for short rows, many of them: 16 threads of four columns by 16 rows at a time, whose sums are added in order.  Column sums
// of 4096: 2.1 MB of partial ones, 5 us, of which 2 are the launch.
template <typename OT>
__global__ __launch_bounds__(256) void sum_many_rows_kernel(JoinArgs a) {
  __shared__ f32x4 part[16][17];
  const int cl = threadIdx.x & 15, rl = threadIdx.x >> 4;
  const size_t i = ((size_t)blockIdx.x * 16 + cl) * 4;
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
  if (i < a.n) {
    const float* src = a.parts[blockIdx.y] + i;
#pragma unroll 8
    for (int r = rl; r < a.rows; r += 16) s += *reinterpret_cast<const f32x4*>(src + (size_t)r * a.n);
  }
  part[rl][cl] = s;
  __syncthreads();
  if (rl != 0 || i >= a.n) return;
#pragma unroll
  for (int r = 1; r < 16; ++r) s += part[r][cl];
  OT* out = reinterpret_cast<OT*>(a.out[blockIdx.y]) + i;
#pragma unroll
  for (int q = 0; q < 4; ++q) out[q] = from_f32<OT>(s[q] + (a.accumulate ? to_f32(out[q]) : 0.f));
}

__global__ void linear_zero_kernel(uint32_t* p, size_t n) {
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (i < n) p[i] = 0u;
}

// ---- launches ------------------------------------------------------------------------------------------------------
int launch_linear_fwd(const moe_linear* c, const void* x, const void* W, const void* Wb, const void* bias, const void* bias_b,
                      const void* residual, void* pre, void* pre_b, void* y, void* ws, hipStream_t s) {
  const LinearPlan p = linear_plan(c);
  GemmArgs g = {};
  g.A = x; g.B = W; g.B2 = Wb; g.C = pre; g.C2 = pre_b; g.C3 = y; g.S1 = residual; g.bias = bias; g.bias2 = bias_b;
  g.M = c->T; g.N = c->d_out; g.K = c->d_in; g.E = 1;
  g.chunked = row_tiles_chunked(c->T, c->d_in, c->d_out, 1, Wb != nullptr ? 2 : 1, c->dtype == MOE_DTYPE_F32 ? 4 : 2);
  if (c->dtype == MOE_DTYPE_F32) {
    g.tile_rows = p.fwd.rows;
    g.split_parts = p.fwd.parts;
    g.split_ws = (float*)ws;
    return linear_forward_f32(c->act, g, s);
  }
  return c->dtype == MOE_DTYPE_F16 ? linear_forward_f16(c->act, g, p, (float*)ws, s) : linear_forward_bf16(c->act, g, p, (float*)ws, s);
}

template <typename ST, int ACT>
static int launch_act_bwd(const ActBwdArgs& a, int fmt, hipStream_t s) {
  const dim3 grid(a.gm.col_blocks, a.gm.row_blocks);
  if (fmt == MOE_PACK_NONE) act_bwd_kernel<ST, ACT, MOE_PACK_NONE><<<grid, 256, 0, s>>>(a);
  else if (fmt == MOE_PACK_E4M3) act_bwd_kernel<ST, ACT, ACT == MOE_ACT_NONE ? MOE_PACK_NONE : MOE_PACK_E4M3><<<grid, 256, 0, s>>>(a);
  else act_bwd_kernel<ST, ACT, ACT == MOE_ACT_NONE ? MOE_PACK_NONE : MOE_PACK_I8><<<grid, 256, 0, s>>>(a);
  return launch_status();
}
template <typename ST>
static int act_bwd_for(int act, const ActBwdArgs& a, int fmt, hipStream_t s) {
  return act == MOE_ACT_SWIGLU ? launch_act_bwd<ST, MOE_ACT_SWIGLU>(a, fmt, s)
         : act == MOE_ACT_GELU ? launch_act_bwd<ST, MOE_ACT_GELU>(a, fmt, s)
                               : launch_act_bwd<ST, MOE_ACT_NONE>(a, fmt, s);
}
template <typename OT>
static int sum_rows_for(const JoinArgs& a, int mats, bool many, hipStream_t s) {
  if (many) sum_many_rows_kernel<OT><<<dim3((unsigned)((a.n / 4 + 15) / 16), mats), 256, 0, s>>>(a);
  else sum_rows_kernel<OT><<<dim3((unsigned)((a.n / 4 + 255) / 256), mats), 256, 0, s>>>(a);
  return launch_status();
}
static int launch_sum_rows(const JoinArgs& a, int mats, int type, bool many, hipStream_t s) {
  return type == MOE_DTYPE_BF16 ? sum_rows_for<bf16>(a, mats, many, s)
         : type == MOE_DTYPE_F16 ? sum_rows_for<f16>(a, mats, many, s)
                                 : sum_rows_for<float>(a, mats, many, s);
}
static int zero(void* p, size_t bytes, hipStream_t s) {
  if (p == nullptr) return MOE_OK;
  const size_t n = bytes / 4;
  linear_zero_kernel<<<dim3((unsigned)((n + 255) / 256)), 256, 0, s>>>((uint32_t*)p, n);
  return launch_status();
}

#define TRY(expr) do { const int rc_ = (expr); if (rc_ != MOE_OK) return rc_; } while (0)

int launch_linear_bwd(const moe_linear* c, const void* dy, const void* x, const void* W, const void* Wb, const void* pre, const void* pre_b,
                      const void* scales, const void* scales_b, const void* dx_add, void* dx, void* dW, void* dWb, void* dbias, void* dbias_b,
                      int accumulate, void* ws, hipStream_t s) {
  const int mats = c->act == MOE_ACT_SWIGLU ? 2 : 1, N = c->d_out, d = c->d_in;
  const size_t es = c->dtype == MOE_DTYPE_F32 ? 4 : 2, gs = c->grad == MOE_DTYPE_F32 ? 4 : 2;
  if (c->T == 0) {
    if (accumulate) return MOE_OK;
    TRY(zero(dW, (size_t)d * N * gs, s));
    TRY(zero(dWb, (size_t)d * N * gs, s));
    TRY(zero(dbias, (size_t)N * gs, s));
    return zero(dbias_b, (size_t)N * gs, s);
  }
  const LinearPlan p = linear_plan(c);
  char* w = static_cast<char*>(ws);
  const size_t plane = (size_t)c->T * N * es;
  const void *dz = dy, *dz2 = nullptr;
  if (c->act != MOE_ACT_NONE || dbias != nullptr) {
    ActBwdArgs a = {};
    a.dy = dy; a.pre = pre; a.pre2 = pre_b;
    a.scales = static_cast<const uint8_t*>(scales); a.scales2 = static_cast<const uint8_t*>(scales_b);
    if (c->act != MOE_ACT_NONE) { a.dz = w + p.dz; dz = a.dz; }
    if (mats == 2) { a.dz2 = w + p.dz + plane; dz2 = a.dz2; }
    const bool few = dbias != nullptr && bias_few(c->T, N);
    if (few) { a.out = dbias; a.out2 = dbias_b; a.grad = c->grad; a.accumulate = accumulate; }
    else if (dbias != nullptr) {
      a.sums = reinterpret_cast<float*>(w + p.db);
      a.sums2 = a.sums + (size_t)p.bias_geom.row_blocks * N;
    }
    a.T = c->T; a.N = N; a.gm = few ? bias_geom_few(c->T, N, act_bwd_cols(es == 4, pre_format(c))) : p.bias_geom;
    TRY(c->dtype == MOE_DTYPE_F32   ? act_bwd_for<float>(c->act, a, pre_format(c), s)
        : c->dtype == MOE_DTYPE_F16 ? act_bwd_for<f16>(c->act, a, pre_format(c), s)
                                    : act_bwd_for<bf16>(c->act, a, pre_format(c), s));
    if (dbias != nullptr && !few) {
      const JoinArgs j = {{a.sums, a.sums2}, {dbias, dbias_b}, (size_t)N, p.bias_geom.row_blocks, accumulate};
      TRY(launch_sum_rows(j, mats, c->grad, true, s));
    }
  }
  // dx = dz W^T (+ dz2 Wb^T) + dx_add
  GemmArgs g1 = {}, g2 = {};
  g1.A = dz; g1.A2 = dz2; g1.B = W; g1.B2 = Wb; g1.C3 = dx; g1.S1 = dx_add;
  g1.M = c->T; g1.N = d; g1.K = N; g1.E = 1;
  g1.chunked = row_tiles_chunked(c->T, N, d, 1, mats, (int)es);
  float* split = reinterpret_cast<float*>(w + p.split);
  // dW = x^T dz, dWb = x^T dz2: both in one launch
  const size_t out = (size_t)d * N;
  float* sums = reinterpret_cast<float*>(w + p.dw);
  if (dW != nullptr) {
    g2.A = x; g2.B = dz; g2.B2 = dz2;
    g2.C = p.dw_direct ? dW : sums;
    if (mats == 2) g2.C2 = p.dw_direct ? dWb : static_cast<void*>(sums + out * p.segs);
    g2.M = d; g2.N = N; g2.K = c->T; g2.E = p.segs; g2.seg = p.seg;
    g2.accumulate = p.dw_direct && accumulate;
  }
  if (es == 4) {
    g1.tile_rows = p.dx.rows; g1.split_parts = p.dx.parts; g1.split_ws = split;
    g2.tile_rows = p.dw_rows;
    if (dx != nullptr || dW != nullptr) TRY(linear_backward_f32(mats == 2, g1, g2, s));
  } else {
    const bool f16 = c->dtype == MOE_DTYPE_F16, in_type = p.dw_direct && c->grad != MOE_DTYPE_F32;
    if (p.pair && dx != nullptr && dW != nullptr) TRY(f16 ? linear_both_grads_f16(mats == 2, in_type, g1, g2, p, split, s) : linear_both_grads_bf16(mats == 2, in_type, g1, g2, p, split, s));
    else {
      if (dx != nullptr) TRY(f16 ? linear_input_grad_f16(mats == 2, g1, p, split, s) : linear_input_grad_bf16(mats == 2, g1, p, split, s));
      if (dW != nullptr) TRY(f16 ? linear_weight_grad_f16(in_type, g2, p, s) : linear_weight_grad_bf16(in_type, g2, p, s));
    }
  }
  if (dW == nullptr) return MOE_OK;
  if (p.dw_direct) return MOE_OK;
  const JoinArgs j = {{sums, sums + out * p.segs}, {dW, dWb}, out, p.segs, accumulate};
  return launch_sum_rows(j, mats, c->grad, false, s);
}

}  // namespace moe
