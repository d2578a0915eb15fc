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
  float* partials;   // [blocks][d], or NULL: no gradient of gamma
  DropArgs drop;
  int T, d;
};
inline RowGeom norm_geom(int d) {
  const int g = (d + 7) / 8;
  if (d % 8 != 0) return g <= 128 ? RowGeom{1, 2} : g <= 512 ? RowGeom{4, 2} : RowGeom{8, 4};
  return g <= 64 ? RowGeom{1, 1} : g <= 128 ? RowGeom{1, 2} : g <= 256 ? RowGeom{1, 4} : g <= 512 ? RowGeom{4, 2} : g <= 1024 ? RowGeom{4, 4} : RowGeom{8, 4};
}
static_assert(MOE_MAX_NORM == 8 * WAVE * 4 * 8, "the widest variant");
// Blocks of the backward, each with a row of partial sums of gamma's gradient: enough to fill the chip, and few enough for the
// sums to be small beside the rows.
inline int norm_bwd_blocks(int T, int d) {
  const RowGeom g = norm_geom(d);
  const int rows = rows_per_block(g.wpr), most = g.wpr == 8 ? 512 : 1024;
  const long long want = ((long long)T + rows - 1) / rows;
  return (int)(want < most ? want : most);
}
inline size_t norm_bwd_ws_bytes(const moe_norm* n) { return align_up((size_t)norm_bwd_blocks(n->T, n->d) * n->d * 4, 256); }

int launch_norm_fwd(const moe_norm* n, const NormFwdArgs& a, hipStream_t s);
int launch_norm_bwd(const moe_norm* n, const NormBwdArgs& a, void* dgamma, int accumulate, hipStream_t s);
int launch_dropout(int dtype, long long rows, int width, const DropArgs& drop, const void* x, const void* residual, void* y, hipStream_t s);

}  // namespace moe
