// How a dense product and its backward are cut and where their intermediate results lie (linear.hip).
#pragma once
#include "common.h"

namespace moe {

// Tiles of a 16-bit product, rows x cols (of either matrix, where there are two): those from `first` on are cut along K into `parts`.
struct RowCut { long long tiles, first; int rows, cols, parts; };

// Columns per thread of the pass over dy: 16 bytes of it, eight where a pre-activation is packed.  (fp32 with eight: few rows
// have half the blocks.  Backward, us, eight -> four: GELU 64 x 256 x 256 11.4 -> 10.6, SwiGLU 13.5 -> 11.7, 1024 x 512 x 512 68 -> 58.)
constexpr int act_bwd_cols(bool f32, int fmt) { return f32 && fmt == MOE_PACK_NONE ? 4 : 8; }
// Blocks of that pass: cg threads (a power of two) of `cols` columns each span a block's columns, `rows` rows per block.
struct BiasGeom { int cg, rows, col_blocks, row_blocks; };
inline BiasGeom bias_geom(long long T, int N, int cols) {
  BiasGeom g;
  const int groups = (N + cols - 1) / cols;
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

// Few rows whose column sums are wanted: a block takes all rows of 4 to 32 columns, in at most four steps (eight where the columns
// make more blocks than compute units), and writes the sums itself, without a launch that adds up partial ones.  Up to a million
// values: its pieces of a row are short.  (fp32, 300 x 516 x 1540, a step: a block per four columns 48.0 us, per eight 45.2.)
inline bool bias_few(long long T, int N) { return T <= 1024 && T * N <= 1 << 20; }
inline BiasGeom bias_geom_few(long long T, int N, int cols) {
  const int groups = (N + cols - 1) / cols;
  int cg = T <= 128 ? 4 : T <= 256 ? 2 : 1;
  if (groups > 256 * cg) cg *= 2;
  return BiasGeom{cg, (int)T, (groups + cg - 1) / cg, 1};
}

struct LinearPlan {
  RowCut fwd, dx;
  BiasGeom bias_geom;
  int dw_rows;        // weight gradient: edge of its tiles
  int segs, seg;      // ... segments of the tokens, rows of one
  bool dw_direct;     // ... written by the product itself
  bool pair;          // both gradients in one launch
  size_t dz, db, split, dw, total;   // the backward's workspace: byte offsets of its regions, all of it
  size_t fwd_total;                  // the forward's, which it has to itself
};
LinearPlan linear_plan(const moe_linear* c);
int launch_linear_fwd(const moe_linear* c, const void* x, const void* W, const void* Wb, const void* bias, const void* bias_b,
                      const void* residual, void* pre, void* pre_b, void* y, void* ws, hipStream_t s);
int launch_linear_bwd(const moe_linear* c, const void* dy, const void* x, const void* W, const void* Wb, const void* pre, const void* pre_b,
                      const void* scales, const void* scales_b, const void* dx_add, void* dx, void* dW, void* dWb, void* dbias, void* dbias_b,
                      int accumulate, void* ws, hipStream_t s);

}  // namespace moe
