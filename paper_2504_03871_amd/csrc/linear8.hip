// Products of 8-bit integers with a scale for each token and channel: how they are cut, and their launches.  Kernels: gemm_i8_kernel.h.
#include "gemm_i8.h"
#include <algorithm>

namespace moe {

// A tile shape, rows and columns (two matrices: of both together), how many run at a time, and what a round of them takes, us: `fixed` in
// front of and behind the K loop, and per 128 K values `alone` where few tiles run and `full` where all do.
struct Shape8 {
  int rows, cols, slots;
  double fixed, alone, full;
  double us(long long tiles, int stages) const {
    const long long r = tiles % slots, rounds = tiles / slots;
    double t = rounds * (fixed + stages * full);
    if (r > 0) t += fixed + stages * (alone + (full - alone) * r / slots);
    return t;
  }
};
constexpr Shape8 SHAPES8[] = {{256, 256, 256, 6.5, 1.05, 1.37}, {128, 128, 512, 4.0, 0.5, 0.8}, {64, 128, 512, 3.0, 0.35, 0.54}};
constexpr int FEW_ROWS = 64;       // up to here the weights are streamed
constexpr int FEW_STRIPS = 256;    // strips of 16 columns that fill the chip; fewer are cut along K
constexpr int FEW_PART = 16;       // tiles of 64 K values that a part has at least
static int few_rows(long long rows) { return rows <= 16 ? 16 : rows <= 32 ? 32 : 64; }

Cut8 cut_linear8(long long T, int N, int K, int mats) {
  if (T <= FEW_ROWS) {
    const int strips = N / TILE8_N, parts = std::min({(FEW_STRIPS + strips - 1) / strips, K / TILE8_K / FEW_PART, 16});
    return Cut8{true, few_rows(T), TILE8_N, std::max(parts, 1)};
  }
  Cut8 best = {};
  double least = 1e30;
  for (const Shape8& s : SHAPES8) {
    const int cols = s.cols / mats;
    const double us = s.us((T + s.rows - 1) / s.rows * ((N + cols - 1) / cols), (K + 127) / 128);
    if (us < least) { least = us; best = Cut8{false, s.rows, cols, 1}; }
  }
  return best;
}

int expert8_tile_rows(long long rows, int E) { return rows <= (long long)FEW_ROWS * E ? 0 : rows <= 256ll * E ? 128 : 256; }

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
  g.parts = (int32_t*)ws;
  g.n_parts = cut.parts;
  return gemm8(c->dtype, c->act, g, cut, 0, s);
}

int launch_expert8(int dtype, int act, const Gemm8Args& args, int tile_rows, int max_tiles, int rows, hipStream_t s) {
  Gemm8Args g = args;
  const int mats = act == MOE_ACT_SWIGLU ? 2 : 1;
  g.n_parts = 1;
  g.chunked = row_tiles_chunked(rows, g.K, g.N, g.E, mats, 1);
  Cut8 cut = {tile_rows == 0, tile_rows, 0, 1};
  if (cut.few) {
    cut.rows = few_rows((rows + g.E - 1) / g.E);
    max_tiles = std::min(g.E, rows) + rows / cut.rows;   // every expert's last group may be a part of one
  }
  return gemm8(dtype, act, g, cut, max_tiles, s);
}

}  // namespace moe
