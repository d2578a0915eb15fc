// Dense products with a fused epilogue, y = act(x W + bias) + residual, and their backward (the shared expert of an MoE block).
//
// The products run on the tiles of the grouped GEMMs (gemm_bf16_kernel.h, gemm_skinny_kernel.h, gemm_f32.hip) with one matrix and
// no tile map; bias, activation, residual and the rounding to the storage type sit in their epilogues, on the fp32 sums.  Where the
// sums of a tile are cut along K, so that few tiles fill the chip, the kernel that adds the parts has the epilogue.
//   forward   up to SKINNY_ROWS rows: 64 x 128 tiles, every one cut along K (a read of the weights: HBM);
//             more: 160- or 256-row tiles (matrix cores), the last round cut along K
//   backward  dz = dy act'(pre) and its column sums in one pass (HBM); dx = dz W^T on row tiles; dW = x^T dz on 256 x 256 tiles, the
//             tokens cut into segments where the gradient has few tiles, whose sums a last pass adds up
#include "gemm_bf16_kernel.h"
#include "gemm_skinny_kernel.h"
#include "linear.h"
#include "pack8.h"
#include <algorithm>

namespace moe {

int launch_linear_f32(int mode, int epi, bool chain, const GemmArgs& g, hipStream_t s);   // gemm_f32.hip

// ---- how a product is cut ------------------------------------------------------------------------------------------
// Tiles of the last round of 256 are cut along K as tail_split does, by the same model (tenths of a microsecond: a round takes
// K / 4, a slot 1, the adding launch 20), but of any K: here the host knows the number of tiles.
constexpr int PART_STAGES = 4;   // K stages of 64 that a part has at least
static RowCut cut_rows(long long T, int N, int K, bool dual, int stages_of) {
  RowCut c;
  c.tile_rows = T <= MID_AVERAGE_FEW ? MID_ROWS : 256;   // the line of mid_applies for one expert
  const int bn = dual ? 128 : 256;
  c.tiles = (T + c.tile_rows - 1) / c.tile_rows * ((N + bn - 1) / bn);
  c.first = c.tiles;
  c.parts = 1;
  const int r = (int)(c.tiles % TAIL_SLOTS), round = stages_of * 16;
  int best = round - 20;
  for (int p = 2; r > 0 && p <= TAIL_MAX_PARTS && p * r <= TAIL_SLOTS && stages_of >= p * PART_STAGES; ++p)
    if (round / p + p * r < best) { best = round / p + p * r; c.parts = p; }
  if (c.parts > 1) c.first = c.tiles - r;
  (void)K;
  return c;
}
static size_t cut_bytes(const RowCut& c) { return (size_t)(c.tiles - c.first) * c.parts * c.tile_rows * 256 * 4; }

// Few rows: K parts per 128-column tile so that two blocks per compute unit are on their way
static int skinny_parts(int N, int K) {
  const int tiles = (N + SKINNY_BN - 1) / SKINNY_BN, stages = K / BKT;
  return std::max(1, std::min({512 / tiles, stages / 2, 16}));
}

// Segments of the tokens for the weight gradient.  16-bit: rounds of 256 tiles of 26 us per 1024 tokens against writing and
// reading the segments' sums at about 4 TB/s.  A segment stays below 4 GiB of either operand (32-bit offsets).
static int dw_segments(const moe_linear* c, int mats) {
  const long long T = c->T;
  const bool half = c->dtype != MOE_DTYPE_F32;
  const long long out = (long long)c->d_in * c->d_out * mats;
  const long long row_bytes = (long long)std::max(c->d_in, c->d_out) * (half ? 2 : 4);
  const int least = (int)((T * row_bytes) / 0xf0000000ll) + 1;
  long long tiles, slots;
  double per_row;   // us of a round per token
  if (half) {
    tiles = (long long)((c->d_in + 255) / 256) * ((c->d_out + 255) / 256) * mats;
    slots = 256;
    per_row = 26.0 / 1024;
  } else {
    tiles = (long long)((c->d_in + 63) / 64) * ((c->d_out + 63) / 64) * mats;
    slots = F32_LOW_TILES;
    per_row = 0.06;
  }
  int best = least;
  double cost = 1e30;
  for (int s = least; s <= std::max(least, 16) && (s == least || T / s >= 256); ++s) {
    const double rounds = (double)((tiles * s + slots - 1) / slots);
    double us = rounds * per_row * (double)((T + s - 1) / s);
    if (s > 1) us += 3.0 + (double)out * 4 * s * 2 / 4e6;
    if (us < cost * 0.97) { cost = us; best = s; }
  }
  return best;
}
static int seg_rows(long long T, int segs) { return (int)(((T + segs - 1) / segs + 63) / 64 * 64); }

LinearPlan linear_plan(const moe_linear* c) {
  LinearPlan p{};
  const bool half = c->dtype != MOE_DTYPE_F32;
  const int mats = c->act == MOE_ACT_SWIGLU ? 2 : 1;
  const size_t es = half ? 2 : 4, T = c->T, N = c->d_out;
  size_t fwd = 0, off = 0;
  p.skinny = half && c->T <= SKINNY_ROWS;
  if (p.skinny) {
    p.parts = skinny_parts(c->d_out, c->d_in);
    fwd = (size_t)mats * p.parts * T * N * 4;
  } else if (half) {
    p.fwd = cut_rows(c->T, c->d_out, c->d_in, mats == 2, c->d_in / BKT);
    fwd = cut_bytes(p.fwd);
  }
  // backward
  p.dz = off;
  if (c->act != MOE_ACT_NONE) off += align_up(mats * T * N * es, 256);
  p.bias_geom = bias_geom(c->T, c->d_out);
  p.db = off;
  off += align_up((size_t)mats * p.bias_geom.row_blocks * N * 4, 256);
  p.split = off;
  if (half) {
    p.dx = cut_rows(c->T, c->d_in, c->d_out, false, mats * (c->d_out / BKT));
    off += align_up(cut_bytes(p.dx), 256);
  }
  p.dw = off;
  p.segs = c->T > 0 ? dw_segments(c, mats) : 1;
  p.seg = seg_rows(c->T, p.segs);
  p.segs = c->T > 0 ? (c->T + p.seg - 1) / p.seg : 1;
  p.dw_direct = p.segs == 1;   // the product writes the gradient itself
  if (!p.dw_direct) off += align_up((size_t)mats * p.segs * c->d_in * N * 4, 256);
  p.total = std::max(align_up(fwd, 256), off);
  return p;
}

// ---- kernels -------------------------------------------------------------------------------------------------------
template <typename ST, int MODE, int EPI, bool DUAL, bool CHAIN, int BM, int BN, int WGM, int WGN>
__global__ __launch_bounds__(WGM* WGN * 64, 1) void linear_rows_kernel(GemmArgs g) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  gemm_bf16_tile<ST, MODE, EPI, DUAL, CHAIN, BM, BN, WGM, WGN, false, false, true>(g, blockIdx.x, smem);
}
template <typename ST, bool DUAL>
__global__ __launch_bounds__(256, 2) void linear_few_kernel(GemmArgs g) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  gemm_skinny_tile<ST, EPI_STORE, DUAL, true>(g, smem);
}

// Adds the parts of split tiles in part order and applies the epilogue; a thread owns eight adjacent columns of a row.
// few: the layout of linear_few_kernel, every row and column; else that of the split row tiles.
template <typename ST, int EPI>
__global__ __launch_bounds__(256) void linear_join_kernel(GemmArgs g, int few) {
  constexpr bool DUAL = EPI == EPI_LIN_SWIGLU;
  const float *src, *src2;
  size_t pitch;      // floats between the parts
  long long row;
  int col;
  const int parts = g.split_parts;
  if (few) {
    const int per_row = g.N / 8;
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i >= g.M * per_row) return;
    row = i / per_row;
    col = (i % per_row) * 8;
    pitch = (size_t)g.M * g.N;
    src = g.split_ws + (size_t)row * g.N + col;
    src2 = src + pitch * parts;
  } else {
    constexpr int BN = DUAL ? 128 : 256, TPR = BN / 8, RPB = 256 / TPR;   // threads per row, rows per block
    const int per_tile = g.tile_rows / RPB;
    const int q = blockIdx.x / per_tile, m = (blockIdx.x % per_tile) * RPB + threadIdx.x / TPR, n = (threadIdx.x % TPR) * 8;
    int rt, nt;
    if (!block_to_tile(g.split_first + q, (g.M + g.tile_rows - 1) / g.tile_rows, g.M / g.tile_rows, (g.N + BN - 1) / BN, g.chunked != 0, rt, nt)) return;
    row = (long long)rt * g.tile_rows + m;
    col = nt * BN + n;
    if (row >= g.M || col >= g.N) return;
    pitch = (size_t)g.tile_rows * 256;
    src = g.split_ws + (size_t)q * parts * pitch + m * BN + n;
    src2 = src + (size_t)g.tile_rows * BN;
  }
  float z[8] = {}, z2[8] = {};
  for (int p = 0; p < parts; ++p) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const f32x4 v = *reinterpret_cast<const f32x4*>(src + p * pitch + 4 * h);
#pragma unroll
      for (int i = 0; i < 4; ++i) z[4 * h + i] += v[i];
      if constexpr (DUAL) {
        const f32x4 w = *reinterpret_cast<const f32x4*>(src2 + p * pitch + 4 * h);
#pragma unroll
        for (int i = 0; i < 4; ++i) z2[4 * h + i] += w[i];
      }
    }
  }
  const size_t at = (size_t)row * g.N + col;
  Vec16<ST> q;
  float f[8];
  auto add = [&](const void* p, size_t off, float (&to)[8]) {
    if (p == nullptr) return;
    q.load(reinterpret_cast<const ST*>(p) + off);
    q.unpack(f);
#pragma unroll
    for (int i = 0; i < 8; ++i) to[i] += f[i];
  };
  auto put = [&](void* p, const float (&v)[8]) {
    q.pack(v);
    q.store(reinterpret_cast<ST*>(p) + at);
  };
  add(g.bias, col, z);
  if (EPI != EPI_LIN_NONE && g.C != nullptr) put(g.C, z);
  if constexpr (DUAL) {
    add(g.bias2, col, z2);
    if (g.C != nullptr) put(g.C2, z2);
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] = z[i] * sigmoid_fast(z[i]) * z2[i];
  } else if constexpr (EPI == EPI_LIN_GELU) {
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] = z[i] * phi_fast(z[i]);
  }
  add(g.S1, at, z);
  put(g.C3, z);
}

// dz = dy act'(pre), rounded to the storage type, and the column sums of the unrounded dz, one row of partial sums per block.
// A thread owns eight adjacent columns and walks down the rows of its block; cg threads span a block's columns.
struct ActBwdArgs {
  const void* dy;
  const void *pre, *pre2;           // storage type, or codes
  const uint8_t *scales, *scales2;
  void *dz, *dz2;
  float *sums, *sums2;              // [row blocks][N] or NULL
  long long T;
  int N;
  BiasGeom gm;
};
template <typename ST, int ACT, int FMT>
__global__ __launch_bounds__(256) void act_bwd_kernel(ActBwdArgs a) {
  constexpr bool DUAL = ACT == MOE_ACT_SWIGLU;
  constexpr int VN = Vec16<ST>::N;
  __shared__ float s_sum[256][DUAL ? 17 : 9];
  const int cl = threadIdx.x & (a.gm.cg - 1), rl = threadIdx.x / a.gm.cg, rp = 256 / a.gm.cg;
  const int c = (blockIdx.x * a.gm.cg + cl) * 8;
  const long long r0 = (long long)blockIdx.y * a.gm.rows, r1 = min(r0 + a.gm.rows, a.T);
  const int n = min(8, a.N - c);                       // columns of this thread: 8, 4 (fp32) or none
  const int blocks = (a.N + BLOCK8 - 1) / BLOCK8;
  float sum[8] = {}, sum2[8] = {};
  auto load = [&](const void* p, long long r, float (&v)[8]) {
    const ST* at = reinterpret_cast<const ST*>(p) + r * a.N + c;
#pragma unroll
    for (int i = 0; i < 8; i += VN)
      if (i < n) {
        Vec16<ST> q;
        q.load_nt(at + i);
        q.unpack(v + i);
      }
  };
  auto store = [&](void* p, long long r, const float (&v)[8]) {
    ST* at = reinterpret_cast<ST*>(p) + r * a.N + c;
#pragma unroll
    for (int i = 0; i < 8; i += VN)
      if (i < n) {
        Vec16<ST> q;
        q.pack(v + i);
        q.store_nt(at + i);
      }
  };
  auto load_pre = [&](const void* p, const uint8_t* sc, long long r, float (&v)[8]) {
    if constexpr (FMT == MOE_PACK_NONE) load(p, r, v);
    else decode8<ST, FMT>(*reinterpret_cast<const uint2*>(reinterpret_cast<const uint8_t*>(p) + r * blocks * BLOCK8 + c), sc[r * blocks + c / BLOCK8], v);
  };
  // U rows of a thread are requested together; a row past the end repeats the last one and counts for nothing
  constexpr int U = sizeof(ST) == 4 ? 1 : 2;
  if (n > 0)
    for (long long ra = r0 + rl; ra < r1; ra += (long long)rp * U) {
      float dy[U][8] = {}, z[U][8] = {}, z2[U][8] = {};
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
        float g[8], g2[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if constexpr (DUAL) {
            const float sg = sizeof(ST) == 4 ? sigmoid_f(z[u][i]) : sigmoid_fast(z[u][i]);
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
  if (a.sums == nullptr) return;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    s_sum[threadIdx.x][i] = sum[i];
    if constexpr (DUAL) s_sum[threadIdx.x][8 + i] = sum2[i];
  }
  __syncthreads();
  if (rl != 0 || n <= 0) return;
  for (int q = 1; q < rp; ++q)   // in row order: deterministic
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      sum[i] += s_sum[q * a.gm.cg + cl][i];
      if constexpr (DUAL) sum2[i] += s_sum[q * a.gm.cg + cl][8 + i];
    }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < n) {
      a.sums[(size_t)blockIdx.y * a.N + c + i] = sum[i];
      if constexpr (DUAL) a.sums2[(size_t)blockIdx.y * a.N + c + i] = sum2[i];
    }
}

// out [n] (+)= the sum of `parts` rows of n floats, in row order; two of them (blockIdx.y) where the second is given.
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

// The same for short rows, many of them: 16 threads of four columns by 16 rows at a time, whose sums are added in order.
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
template <typename K>
static int more_lds(K kern, int lds) {   // above 64 KB, on every launch: nothing is remembered
  const hipError_t err = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  return err == hipSuccess ? MOE_OK : set_hip_error(err);
}

template <typename ST, int MODE, int EPI, bool DUAL, bool CHAIN, int BM>
static int launch_rows_bm(const GemmArgs& g, long long tiles, hipStream_t s) {
  constexpr int BN = DUAL ? 128 : 256, WGM = DUAL && BM == 256 ? 4 : 2;
  constexpr int lds = gemm_bf16_lds_bytes<BM, BN, DUAL>();
  auto kern = linear_rows_kernel<ST, MODE, EPI, DUAL, CHAIN, BM, BN, WGM, 8 / WGM>;
  const int rc = more_lds(kern, lds);
  if (rc != MOE_OK) return rc;
  const long long blocks = MODE == MODE_TN ? dw_blocks(g, BM, BN) : g.split_first + (tiles - g.split_first) * g.split_parts;
  if (blocks > 0x7fffffffll) return MOE_ERR_BAD_SHAPE;
  kern<<<dim3((unsigned)blocks), 512, lds, s>>>(g);
  return launch_status();
}
template <typename ST, int EPI>
static int launch_join(const GemmArgs& g, long long blocks, int few, hipStream_t s) {
  linear_join_kernel<ST, EPI><<<dim3((unsigned)blocks), 256, 0, s>>>(g, few);
  return launch_status();
}
template <typename ST, int MODE, int EPI, bool CHAIN>
static int launch_rows(GemmArgs g, const RowCut& cut, float* split_ws, hipStream_t s) {
  constexpr bool DUAL = EPI == EPI_LIN_SWIGLU;
  constexpr int BN = DUAL ? 128 : 256;
  if (cut.tiles > 0x7fffffffll) return MOE_ERR_BAD_SHAPE;
  g.tile_rows = cut.tile_rows;
  g.split_first = (int)cut.first;
  g.split_parts = cut.parts;
  g.split_ws = split_ws;
  int rc = cut.tile_rows == MID_ROWS ? launch_rows_bm<ST, MODE, EPI, DUAL, CHAIN, MID_ROWS>(g, cut.tiles, s)
                                     : launch_rows_bm<ST, MODE, EPI, DUAL, CHAIN, 256>(g, cut.tiles, s);
  if (rc != MOE_OK || cut.parts == 1) return rc;
  return launch_join<ST, EPI>(g, (cut.tiles - cut.first) * (cut.tile_rows * BN / 8 / 256), 0, s);
}
template <typename ST, int EPI>
static int launch_few(GemmArgs g, int parts, float* split_ws, hipStream_t s) {
  constexpr bool DUAL = EPI == EPI_LIN_SWIGLU;
  constexpr int lds = skinny_stages<DUAL>() * skinny_stage_bytes<DUAL>();
  auto kern = linear_few_kernel<ST, DUAL>;
  const int rc = more_lds(kern, lds);
  if (rc != MOE_OK) return rc;
  g.split_parts = parts;
  g.split_ws = split_ws;
  kern<<<dim3((unsigned)((g.N + SKINNY_BN - 1) / SKINNY_BN * parts)), 256, lds, s>>>(g);
  const int rc2 = launch_status();
  if (rc2 != MOE_OK) return rc2;
  return launch_join<ST, EPI>(g, ((long long)g.M * (g.N / 8) + 255) / 256, 1, s);
}
template <typename ST, int EPI>
static int fwd_half(const GemmArgs& g, const LinearPlan& p, float* ws, hipStream_t s) {
  return p.skinny ? launch_few<ST, EPI>(g, p.parts, ws, s) : launch_rows<ST, MODE_NN, EPI, false>(g, p.fwd, ws, s);
}
template <typename ST>
static int fwd_half_act(int act, const GemmArgs& g, const LinearPlan& p, float* ws, hipStream_t s) {
  return act == MOE_ACT_SWIGLU ? fwd_half<ST, EPI_LIN_SWIGLU>(g, p, ws, s)
         : act == MOE_ACT_GELU ? fwd_half<ST, EPI_LIN_GELU>(g, p, ws, s)
                               : fwd_half<ST, EPI_LIN_NONE>(g, p, ws, s);
}

int launch_linear_fwd(const moe_linear* c, const void* x, const void* W, const void* Wb, const void* bias, const void* bias_b,
                      const void* residual, void* pre, void* pre_b, void* y, void* ws, hipStream_t s) {
  const LinearPlan p = linear_plan(c);
  GemmArgs g = {};
  g.A = x; g.B = W; g.B2 = Wb; g.C = pre; g.C2 = pre_b; g.C3 = y; g.S1 = residual; g.bias = bias; g.bias2 = bias_b;
  g.M = c->T; g.N = c->d_out; g.K = c->d_in; g.E = 1;
  g.chunked = row_tiles_chunked(c->T, c->d_in, c->d_out, 1, Wb != nullptr ? 2 : 1, c->dtype == MOE_DTYPE_F32 ? 4 : 2);
  if (c->dtype == MOE_DTYPE_F32)
    return launch_linear_f32(MODE_NN, c->act == MOE_ACT_SWIGLU ? EPI_LIN_SWIGLU : c->act == MOE_ACT_GELU ? EPI_LIN_GELU : EPI_LIN_NONE, false, g, s);
  return c->dtype == MOE_DTYPE_F16 ? fwd_half_act<f16>(c->act, g, p, (float*)ws, s) : fwd_half_act<bf16>(c->act, g, p, (float*)ws, s);
}

template <typename ST, int ACT>
static int launch_act_bwd(const ActBwdArgs& a, int fmt, hipStream_t s) {
  const dim3 grid(a.gm.col_blocks, a.gm.row_blocks);
  if (ACT == MOE_ACT_NONE || fmt == MOE_PACK_NONE) act_bwd_kernel<ST, ACT, MOE_PACK_NONE><<<grid, 256, 0, s>>>(a);
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
    if (dbias != nullptr) {
      a.sums = reinterpret_cast<float*>(w + p.db);
      a.sums2 = a.sums + (size_t)p.bias_geom.row_blocks * N;
    }
    a.T = c->T; a.N = N; a.gm = p.bias_geom;
    TRY(c->dtype == MOE_DTYPE_F32   ? act_bwd_for<float>(c->act, a, c->pre_pack, s)
        : c->dtype == MOE_DTYPE_F16 ? act_bwd_for<f16>(c->act, a, c->pre_pack, s)
                                    : act_bwd_for<bf16>(c->act, a, c->pre_pack, s));
    if (dbias != nullptr) {
      const JoinArgs j = {{a.sums, a.sums2}, {dbias, dbias_b}, (size_t)N, p.bias_geom.row_blocks, accumulate};
      TRY(launch_sum_rows(j, mats, c->grad, true, s));
    }
  }
  GemmArgs g = {};
  g.E = 1;
  if (dx != nullptr) {   // dx = dz W^T (+ dz2 Wb^T) + dx_add
    g.A = dz; g.A2 = dz2; g.B = W; g.B2 = Wb; g.C3 = dx; g.S1 = dx_add;
    g.M = c->T; g.N = d; g.K = N;
    g.chunked = row_tiles_chunked(c->T, N, d, 1, mats, (int)es);
    float* split = reinterpret_cast<float*>(w + p.split);
    if (es == 4) TRY(launch_linear_f32(MODE_NT, EPI_LIN_NONE, mats == 2, g, s));
    else if (c->dtype == MOE_DTYPE_F16)
      TRY(mats == 2 ? (launch_rows<f16, MODE_NT, EPI_LIN_NONE, true>(g, p.dx, split, s)) : (launch_rows<f16, MODE_NT, EPI_LIN_NONE, false>(g, p.dx, split, s)));
    else
      TRY(mats == 2 ? (launch_rows<bf16, MODE_NT, EPI_LIN_NONE, true>(g, p.dx, split, s)) : (launch_rows<bf16, MODE_NT, EPI_LIN_NONE, false>(g, p.dx, split, s)));
  }
  if (dW == nullptr) return MOE_OK;
  // dW = x^T dz, dWb = x^T dz2: both in one launch
  const size_t out = (size_t)d * N;
  float* sums = reinterpret_cast<float*>(w + p.dw);
  g = GemmArgs{};
  g.A = x; g.B = dz; g.B2 = dz2;
  g.C = p.dw_direct ? dW : sums;
  if (mats == 2) g.C2 = p.dw_direct ? dWb : static_cast<void*>(sums + out * p.segs);
  g.M = d; g.N = N; g.K = c->T; g.E = p.segs; g.seg = p.seg;
  g.accumulate = p.dw_direct && accumulate;
  if (es == 4) TRY(launch_linear_f32(MODE_TN, EPI_DW, false, g, s));
  else if (p.dw_direct && c->grad != MOE_DTYPE_F32)
    TRY(c->dtype == MOE_DTYPE_F16 ? (launch_rows_bm<f16, MODE_TN, EPI_LIN_NONE, false, false, 256>(g, 0, s))
                                  : (launch_rows_bm<bf16, MODE_TN, EPI_LIN_NONE, false, false, 256>(g, 0, s)));
  else if (c->dtype == MOE_DTYPE_F16) TRY((launch_rows_bm<f16, MODE_TN, EPI_DW, false, false, 256>(g, 0, s)));
  else TRY((launch_rows_bm<bf16, MODE_TN, EPI_DW, false, false, 256>(g, 0, s)));
  if (p.dw_direct) return MOE_OK;
  const JoinArgs j = {{sums, sums + out * p.segs}, {dW, dWb}, out, p.segs, accumulate};
  return launch_sum_rows(j, mats, c->grad, false, s);
}

}  // namespace moe
