// Products of 8-bit integers with a scale for each token and channel: how they are cut, and their launches.  Kernels: gemm_i8_kernel.h.
#include "gemm_i8.h"
#include <algorithm>

namespace moe {

// A tile shape, rows and columns (two matrices: of both together), how many a compute unit holds, and what a round of them takes, us: `fixed`
// in front of and behind the K loop, and per 128 K values `alone` where up to half of the 256 compute units have a tile, `one` where all have
// one, `two` where all have two; with a second tile on some, these take nine tenths of that; `second`: what a second matrix adds to `fixed`.
// Fitted to (us, bf16, in the order of the shapes)
//   T x K x N             256 x 256   256 x 128   128 x 128: 1 | 2 to a unit   64 x 128
//   1024 x 1024 x 2048       16.2        10.6             8.4 | 8.0               6.7
//   300 x 4096 x 4096        39.5        23.4            17.3 | 19.5             13.5
//   1500 x 2880 x 2048       32.6        21.2            15.2 | 16.2             17.9
//   3001 x 2880 x 1152       31.3        20.7            16.1 | 17.0             18.1
//   4096 x 4096 x 1024       40.1        23.9            20.6 | 20.6             23.5
//   4096 x 4096 x 2048       42.0        33.2            40.4 | 34.3             44.7
//   3000 x 8192 x 4096       85.2       102             104   | 95.6            116
//   8192 x 8192 x 2048      100         114             140   | 121             155
// and alike for two matrices (1500 x 1024 x 1024: 17.0, 10.8, 7.9 | 8.7, 7.8).  What bounds the smaller ones is the caches' traffic: 64 x 128 tiles take 24 KB a stage, 18 TB/s together.
// Tiles of 64 in one | two | four | eight K parts: 64 x 14336 x 4096 32.5 | 22.4 | 16.7 | 17.2 (strips: 29), 100 x 8192 x 1024 19.1 | 14.0 | 11.2 | 10.9,
// 128 x 4096 x 4096 11.8 | 12.5 | 13.4 | 19.0.  Strips against the best tiles: 16 x 14336 x 4096 12.1 | 14.9, 32 x 4096 x 4096 7.0 | 9.2, 32 x 14336 x
// 4096 17.2 | 15.3, 64 x 4096 x 4096 10.7 | 10.8, 24 x 4096 x 14336 of two matrices 20.7 | 22.2, 64 of them - | 20.7 (5.8 TB/s).
// Up to 32 rows always strips, also where tiles in K parts are faster (17 to 32 rows of long K): those calls need no workspace, which the
// interface promises and a program that generates relies on.
struct Shape8 {
  int rows, cols, per_cu;
  double fixed, second, alone, one, two;
  double us(long long tiles, int stages, int mats) const {
    const long long slots = 256 * per_cu, r = tiles % slots, rounds = tiles / slots;
    const double around = fixed + (mats - 1) * second;
    double t = rounds * (around + stages * (per_cu > 1 ? two : one));
    if (r > 256) t += around + stages * two * (0.9 + 0.1 * (r - 256) / 256);
    else if (r > 0) t += around + stages * (alone + (one - alone) * std::max(0ll, r - 128) / 128);
    return t;
  }
};
constexpr Shape8 SHAPES8[] = {{256, 256, 1, 8.3, 0, 0.98, 1.43, 0}, {256, 128, 1, 6.0, 0, 0.54, 0.81, 0}, {128, 128, 1, 5.3, -0.5, 0.35, 0.485, 0},
                              {128, 128, 2, 4.4, 0.8, 0.42, 0.52, 0.89}, {64, 128, 2, 4.2, -0.2, 0.27, 0.285, 0.59}};
constexpr double JOIN8_US = 2.5, JOIN8_US_PER_MB = 0.6;   // the adding launch; sums written and read again
constexpr int PART8_STAGES = 4;    // stages that a part has at least

// Waves that share a strip's K range of `tiles` tiles of 64 values: all eight where the strips are few, else as many as leave each
// sixteen tiles, so that a wave has requests enough in flight and a block enough to do.  (us, eight | four | two waves: 4 x 2048 x 2048, two
// matrices, 3.7 | 4.6 | 6.1; 16 x 4096 x 14336, two, 20.3 | 19.4 | 19.8; 4 tokens x 8 of 256 experts, d 2048, f 1024, both products
// 46.7 | 38.7 | 36.5.  Sixteen waves: 16 x 14336 x 4096 12.9 instead of 12.1.)
static int few_nk(long long strips, int tiles) {
  if (strips <= 512) return 8;
  return tiles >= 128 ? 8 : tiles >= 64 ? 4 : tiles >= 32 ? 2 : 1;
}

Cut8 cut_linear8(long long T, int N, int K, int mats) {
  if (T <= FEW_ROWS8) return Cut8{true, T <= 16 ? 16 : 32, TILE8_N, 0, 1};
  Cut8 best = {};
  double least = 1e30;
  const int stages = (K + 127) / 128;
  for (const Shape8& s : SHAPES8) {
    const int cols = s.cols / mats;
    const long long tiles = (T + s.rows - 1) / s.rows * ((N + cols - 1) / cols);
    for (int p = 1; p <= MAX_PARTS8; ++p) {
      if (p > 1 && (s.rows == 256 || p * tiles > 256 * s.per_cu || stages < p * PART8_STAGES)) break;
      double us = s.us(tiles * p, (stages + p - 1) / p, mats);
      if (p > 1) us += JOIN8_US + JOIN8_US_PER_MB * (double)p * T * N * mats * 4 / 1e6;
      if (us < least) { least = us; best = Cut8{false, s.rows, cols, s.per_cu, p}; }
    }
  }
  return best;
}

// Few rows per expert: strips of 16 columns and groups of 16 rows, for each of which the expert's weights are read again.  Both products
// with their map, us, strips | tiles of 64 | 128 | 256 rows: d 2048, f 1024, SwiGLU, 64 experts, rows per expert (uneven loads)
//   4: 68 | 71 | 75 | 85     8: 79 | 80 | 84 | 94     16: 99 | 90 | 91 | 98     32: 135 | 92 | 98 | 103     64: 214 | 104 | 112 | 133
//   128: 398 | 157 | 136 | 159     1024: - | 744 | 575 | 525;     128 experts, 512: - | 828 | 653 | 565
// d 4096, f 14336, 8 experts
//   2: 213 | 223 | 258 | 321     4: 239 | 251 | 271 | 335     16: 337 | 253 | 275 | 340     64: 930 | 384 | 299 | 350     256: - | 784 | 633 | 498
// Fitted to eight experts or more.  With fewer the line comes early: from eight rows per expert to nine, d 4096, f 14336, 1 expert 36 -> 57,
// 2 66 -> 99, 4 115 -> 144, 8 221 -> 238; d 2048, f 1024, 10.4 -> 17.5, 10.6 -> 17.6, 12.2 -> 19.0, 15.7 -> 20.4: tiles of 64 rows without K parts
// leave compute units idle.  And it goes by the mean: where one expert has nearly all rows, strips read its weights once for every sixteen.
int expert8_tile_rows(long long rows, int E) { return rows <= 8ll * E ? 0 : rows <= 40ll * E ? 64 : rows <= 200ll * E ? 128 : 256; }

static int gemm8(int dtype, int act, const Gemm8Args& g, const Cut8& c, int max_tiles, hipStream_t s) {
  if (dtype == MOE_DTYPE_F32) return gemm8_f32(act, g, c, max_tiles, s);
  return dtype == MOE_DTYPE_BF16 ? gemm8_bf16(act, g, c, max_tiles, s) : gemm8_f16(act, g, c, max_tiles, s);
}

int launch_linear8(const moe_linear8* c, const void* x, const float* xs, const void* W, const float* w_scales, const void* Wb, const float* wb_scales,
                   const void* bias, const void* bias_b, const void* residual, void* y, void* ws, hipStream_t s) {
  const int mats = c->act == MOE_ACT_SWIGLU ? 2 : 1;
  const Cut8 cut = cut_linear8(c->T, c->d_out, c->d_in, mats);
  Gemm8Args g = {};
  g.A = (const int8_t*)x; g.a_scale = xs;
  g.B = (const int8_t*)W; g.B2 = (const int8_t*)Wb; g.b_scale = w_scales; g.b2_scale = wb_scales;
  g.bias = bias; g.bias2 = bias_b; g.residual = residual; g.C = y;
  g.M = c->T; g.N = c->d_out; g.K = c->d_in;
  g.chunked = row_tiles_chunked(c->T, c->d_in, c->d_out, 1, mats, 1);
  g.few_nk = few_nk(c->d_out / TILE8_N, c->d_in / TILE8_K);
  g.stream = streams8((long long)mats * c->d_in * c->d_out);
  g.parts = (int32_t*)ws;
  g.n_parts = cut.parts;
  return gemm8(c->dtype, c->act, g, cut, 0, s);
}

int launch_expert8(int dtype, int act, const Gemm8Args& args, int tile_rows, int max_tiles, int rows, hipStream_t s) {
  Gemm8Args g = args;
  const int mats = act == MOE_ACT_SWIGLU ? 2 : 1;
  g.chunked = row_tiles_chunked(rows, g.K, g.N, g.E, mats, 1);
  g.n_parts = 1;
  // Tiles of 256 x 128 where those of 256 x 256 leave half of the compute units without one (us, both products, 256 -> 128 columns: 2000 tokens x 2 of
  // 8 experts, d 1024, f 2048, 68.0 -> 59.8; 1700 x 2 of 4, f 4096, 91 -> 76; 2000 x 1 of 2, f 2048, 51 -> 42; up to 200 tiles the same
  // within 3 %, all of them: 8000 x 2 of 8, d 512, f 2048, 105 -> 117).
  const long long tiles = (rows / 256 + g.E / 2) * ((g.N * mats + 255) / 256);
  const Cut8 cut = {tile_rows == 0, tile_rows, (tile_rows == 256 && tiles >= 128 ? 256 : 128) / mats, tile_rows == 256 ? 1 : 2, 1};
  if (cut.few) {
    max_tiles = std::min(g.E, rows) + rows / 16;   // every expert's last group may be a part of one
    g.few_nk = few_nk((long long)(g.N / TILE8_N) * std::min(g.E, rows), g.K / TILE8_K);
  }
  return gemm8(dtype, act, g, cut, max_tiles, s);
}

}  // namespace moe
