// How a dense product and its backward are cut and where their intermediate results lie (linear.hip).
#pragma once
#include "common.h"

namespace moe {

// Tiles of a 16-bit product, rows x cols (of either matrix, where there are two): those from `first` on are cut along K into `parts`.
struct RowCut { long long tiles, first; int rows, cols, parts; };

// Blocks of the pass over dy: cg threads (a power of two) of eight columns each span a block's columns, `rows` rows per block.
struct BiasGeom { int cg, rows, col_blocks, row_blocks; };
inline BiasGeom bias_geom(long long T, int N) {
  BiasGeom g;
  const int groups = (N + 7) / 8;
  g.cg = 1;
  while (g.cg < groups && g.cg < 64) g.cg <<= 1;
  g.col_blocks = (groups + g.cg - 1) / g.cg;
  const int rp = 256 / g.cg;   // rows at a time
  const long long want = 2048 / g.col_blocks > 0 ? 2048 / g.col_blocks : 1;
  long long rows = (T + want - 1) / want;
  rows = (rows + rp - 1) / rp * rp;
  if (rows < rp) rows = rp;
  while ((T + rows - 1) / rows > 65535) rows *= 2;
  g.rows = (int)rows;
  g.row_blocks = (int)((T + rows - 1) / rows);
  return g;
}

// Few rows whose column sums are wanted: a block takes all rows of 8 to 32 columns, in at most four steps, and writes the sums
// itself, without a launch that adds up partial ones.  Up to a million values: its pieces of a row are short.
inline bool bias_few(long long T, int N) { return T <= 1024 && T * N <= 1 << 20; }
inline BiasGeom bias_geom_few(long long T, int N) {
  const int cg = T <= 128 ? 4 : T <= 256 ? 2 : 1;
  return BiasGeom{cg, (int)T, ((N + 7) / 8 + cg - 1) / cg, 1};
}

struct LinearPlan {
  RowCut fwd, dx;
  BiasGeom bias_geom;
  int dw_rows;        // weight gradient: edge of its tiles
  int segs, seg;      // ... segments of the tokens, rows of one
  bool dw_direct;     // ... written by the product itself
  bool pair;          // both gradients in one launch
  size_t dz, db, split, dw, total;   // workspace: byte offsets of the backward's regions; the forward has it to itself
};
LinearPlan linear_plan(const moe_linear* c);
int launch_linear_fwd(const moe_linear* c, const void* x, const void* W, const void* Wb, const void* bias, const void* bias_b,
                      const void* residual, void* pre, void* pre_b, void* y, void* ws, hipStream_t s);
int launch_linear_bwd(const moe_linear* c, const void* dy, const void* x, const void* W, const void* Wb, const void* pre, const void* pre_b,
                      const void* scales, const void* scales_b, const void* dx_add, void* dx, void* dW, void* dWb, void* dbias, void* dbias_b,
                      int accumulate, void* ws, hipStream_t s);

}  // namespace moe
