// Products of 8-bit integers with a scale for each row and column (linear8.hip, gemm_i8_kernel.h).
#pragma once
#include "gemm.h"
#include "quant8.h"

namespace moe {

struct Gemm8Args {
  const int8_t* A;          // [rows][K]
  const float* a_scale;     // [rows]
  const int32_t* src_of;    // experts' first product: row r of the permuted order is row src_of[r] / per_row of A; NULL: r itself
  int per_row, src_rows;    // assignments per row of A, and how many rows it has
  const int8_t *B, *B2;     // tiles of quant8.h, a matrix (or two) or one for each expert
  const float *b_scale, *b2_scale;
  const void *bias, *bias2, *residual;   // storage type, may be NULL
  void* C;
  int M, N, K;
  // experts: row tiles from a map (large tiles), or found from these by every block (few rows); E == 0: M dense rows
  const RowTile* tiles;
  const int32_t* ntiles;
  const int32_t *offsets, *kept, *lo, *hi;
  int E;
  int chunked;              // order of the tiles (block_to_tile)
  int32_t* parts;           // few rows, dense: sums of K parts, [part][matrix][row][N]
  int n_parts;
};

// How a product is cut: few rows (row groups of `rows` = 16, 32 or 64, strips of 16 columns, K parts), or tiles of rows x cols.
struct Cut8 { bool few; int rows, cols, parts; };
Cut8 cut_linear8(long long T, int N, int K, int mats);
inline size_t linear8_ws_bytes(const Cut8& c, long long T, int N, int mats) {
  return c.few && c.parts > 1 ? align_up((size_t)c.parts * mats * T * N * 4, 256) : 256;   // (a call without one is a mistake still)
}
// Row tiles of the experts' products: 0 for the few-row kernel
int expert8_tile_rows(long long rows, int E);

int launch_linear8(const moe_linear8* c, const void* x, const float* xs, const void* W, const float* ws8, const void* Wb, const float* wbs, const void* bias,
                   const void* bias_b, const void* residual, void* y, void* ws, hipStream_t s);
// an experts' product: g without its shape-dependent fields; max_tiles of tile_rows rows (0: the few-row kernel)
int launch_expert8(int dtype, int act, const Gemm8Args& g, int tile_rows, int max_tiles, int rows, hipStream_t s);
int gemm8_bf16(int act, const Gemm8Args& g, const Cut8& c, int max_tiles, hipStream_t s);   // linear8_bf16.hip and its like
int gemm8_f16(int act, const Gemm8Args& g, const Cut8& c, int max_tiles, hipStream_t s);
int gemm8_f32(int act, const Gemm8Args& g, const Cut8& c, int max_tiles, hipStream_t s);

}  // namespace moe
