// The norm in front of a block: what its forward and backward take, and how its rows are dealt out.
#pragma once
#include "drop.h"
#include "rows.h"

namespace moe {

struct NormFwdArgs {
  const void *x, *residual, *gamma;
  void* h;
  float* rstd;
  void* y;
  int8_t* codes;
  float* scales;
  DropArgs drop;
  int T, d;
  float eps;
};
struct NormBwdArgs {
  const void *dy, *h, *gamma;
  const float* rstd;
  const void* dh_add;
  void *dh, *dx;
  float* partials;   // [row_blocks][d], or NULL: no gradient of gamma
  void* dgamma;
  DropArgs drop;
  int T, d;
  int grad, accumulate;
  int row_blocks, col_blocks;   // col_blocks: of few rows' gradient of gamma (NORM_FEW), else 0
};
// A wave holds a row of up to 1024 values by itself, or, so that few rows fill the chip, two waves share one of more than 512.  (Forward |
// backward, us, one wave -> two: 300 rows of 516 fp32 4.8 | 8.5 -> 3.9 | 7.5; 4096 of 700 bf16 7.7 | 12.3 -> 8.3 | 16.8; 8192 of 1024
// 13.1 | 18.2 -> 13.4 | 24.7.)  Wider rows: one group of eight per thread up to 4096 values, and no more threads than groups (16384
// rows of 4096 bf16 in an fp32 stream, forward: one group 141, two 146, eight groups in one wave 168; 3001 of 1091 fp16: three waves
// 8.9, two groups in four waves 14.8).
inline RowGeom norm_geom(int T, int d) {
  const int g = (d + 7) / 8;
  if (g <= 64) return {1, 1};
  if (g <= 128 && T > 1024) return {1, 2};
  const int nch = g <= 512 ? 1 : g <= 1024 ? 2 : 4;
  return {row_waves(g, nch), nch};
}
static_assert(MOE_MAX_NORM == 8 * WAVE * 4 * 8, "eight waves hold the widest row");
// Blocks of the backward, each with a row of partial sums of gamma's gradient: whole numbers of blocks per compute unit, few enough for
// the sums to be small beside the rows.  (us at 256 | 512 | 768 | 1024 blocks: 16384 x 2048 bf16 95 | 59 | 54 | 57; 16384 x 4096 in an fp32
// stream 217 | 213 | 214 | 218, 384 blocks 257; 8192 x 8192 110 | 117 | 123 | 130; 8192 x 1024 22.5 | 18.6 | 19.6 | 22.4.)
inline int norm_bwd_blocks(int T, int d) {
  const RowGeom g = norm_geom(T, d);
  const int rows = rows_per_block(g), per_cu = g.waves == 1 ? 2 : g.nch > 1 ? 1 : g.waves <= 2 ? 4 : g.waves <= 4 ? 3 : 2;
  const long long want = ((long long)T + rows - 1) / rows, most = 256 * per_cu;
  return (int)(want < most ? want : most);
}
// Few rows: gamma's gradient in blocks of the same launch, which read them again, FEW_LANES rows at a time, instead of partial sums and a
// launch that adds them.  (Partial sums -> this, us: 300 x 516 fp32 7.7 -> 4.3; 512 x 4096 bf16 16.5 -> 5.7; 1024 x 1024 11.6 -> 4.4; 1024 x 4096
// 20.5 -> 9.7, in blocks of no order 14; 2048 x 1024 9.8 -> 6.2; 2048 x 4096 25.6 -> 24.6; 1024 x 16384 48.6 -> 41.7; 4096 x 1024 11.9 ->
// 14.8; 8192 x 1024 18 -> 52, and no better in segments of the rows.)
constexpr int NORM_FEW = 2048;
constexpr int FEW_LANES = 128;   // threads to every eight columns
inline int few_cols(const RowGeom& g) { return row_threads(g) / FEW_LANES * 8; }
// (enough for any smaller T too)
inline size_t norm_bwd_ws_bytes(const moe_norm* n) { return align_up((size_t)(n->T < 1024 ? n->T : 1024) * n->d * 4, 256); }

int launch_norm_fwd(const moe_norm* n, const NormFwdArgs& a, hipStream_t s);
int launch_norm_bwd(const moe_norm* n, const NormBwdArgs& a, void* dgamma, int accumulate, hipStream_t s);
int launch_dropout(int dtype, long long rows, int width, const DropArgs& drop, const void* x, const void* residual, void* y, hipStream_t s);

}  // namespace moe
