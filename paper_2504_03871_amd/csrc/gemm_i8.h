// Products of 8-bit integers with a scale for each row and column (linear8.hip, gemm_i8_kernel.h).
#pragma once
#include "gemm.h"
#include "quant8.h"

namespace moe {

struct Gemm8Args {
  const int8_t* A;          // [rows][K]
  const float* a_scale;     // [rows]
  const int32_t* src_of;    // experts' first product: row r of the permuted order is row src_of[r] / per_row of A; NULL: r itself
  int src_rows;             // rows of A
  uint64_t per_row;         // assignments per row of A, as a factor (quotient_factor)
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
  int stream;               // weights read once are requested as streaming data (streams8)
  int quantise;             // few rows, no activation: A is rows of the storage type, quantised in the product (few8_quantises)
  int few_nk;               // few rows: waves that share a strip's K range (1, 2, 4 or 8)
  int32_t* parts;           // dense tiles: sums of K parts, [part][matrix][row][N]
  int n_parts;
};

// a / k for 0 <= a < 2^30 and 1 <= k <= 8 as a * factor >> 33: the factor is above 2^33 / k by at most one, so the quotient by at most
// 2^30 / 2^33 = 1 / 8, which carries no fraction (r / k, r < k) up to the next whole number.  (k = 8: a < 2^30, so by less than 1 / 8.)
inline uint64_t quotient_factor(int k) { return (1ull << 33) / k + 1; }
static_assert(MOE_MAX_K <= 8, "quotient_factor");

// How a product is cut: up to 32 rows (rows = 16 or 32) in strips of 16 columns, else tiles of rows x cols, `per_cu` of them to a compute unit, their
// K range in `parts`.
constexpr int FEW_ROWS8 = 32, MAX_PARTS8 = 8;
struct Cut8 { bool few; int rows, cols, per_cu, parts; };
Cut8 cut_linear8(long long T, int N, int K, int mats);
// Room for the parts' sums: enough for any smaller T too.  Tiles that are cut make one round of blocks, 512 of 128 x 128 sums at most.
inline size_t linear8_ws_bytes(long long T, int N, int mats) {
  const size_t all = (size_t)MAX_PARTS8 * mats * T * N * 4, most = (size_t)512 * 128 * 128 * 4;
  return T <= FEW_ROWS8 ? 0 : align_up(all < most ? all : most, 256);
}
// Whether weights that are read once are requested as streaming data: where they are more than the memory-side cache keeps for the next
// time.  Strips and tiles below 256 rows, us, plain -> streaming, both products: 4 tokens x 2 of 8 experts, d 4096, f 14336, 183 -> 160, 32
// tokens 249 -> 226, 64 tokens 247 -> 228, 256 tokens 297 -> 288; 32 x 8 of 128, d 2048, f 1024 (805 MB at most) 104 -> 95; 512 x 4 of 64 (403
// MB) 95 -> 88.  Dense weights of 59 to 117 MB that come from memory gain 4 to 8 %, but lose up to 30 % where the cache still has them (16 x
// 14336 x 4096 12.0 -> 15.9), so they stay plain.
inline bool streams8(long long weights) { return weights >= MEMORY_SIDE_CACHE / 4 * 5; }
// Row tiles of the experts' products: 0 for the few-row kernel
int expert8_tile_rows(long long rows, int E);
// Few rows per expert: whether the second product quantises its rows itself, in every block that reads them, instead of a launch in front of
// it.  (Both products, us, launch -> this: 4 tokens x 8 of 256 experts, d 2048, f 1024, 40.2 -> 36.3; 64 x 4 of 64, d 1024, f 512, 25.2 -> 22.0;
// 8 x 2 of 8, d 1024, f 2048, 17.6 -> 15.5; where the weights take long the same within 1 %: 32 x 8 of 128 93.3 -> 92.3, 16 x 8 76.8 -> 77.8,
// 64 x 8 of 128, d 7168, f 2048, 667 -> 673.)
constexpr int FEW_QUANT_MAX = 2048;   // values of a row: four groups of eight in a lane, two rows to a wave
inline bool few8_quantises(int tile_rows, int K) { return tile_rows == 0 && K <= FEW_QUANT_MAX; }

int launch_linear8(const moe_linear8* c, const void* x, const float* xs, const void* W, const float* ws8, const void* Wb, const float* wbs, const void* bias,
                   const void* bias_b, const void* residual, void* y, void* ws, hipStream_t s);
// an experts' product: g without its shape-dependent fields; max_tiles of tile_rows rows (0: the few-row kernel)
int launch_expert8(int dtype, int act, const Gemm8Args& g, int tile_rows, int max_tiles, int rows, hipStream_t s);
int gemm8_bf16(int act, const Gemm8Args& g, const Cut8& c, int max_tiles, hipStream_t s);   // linear8_bf16.hip and its like
int gemm8_f16(int act, const Gemm8Args& g, const Cut8& c, int max_tiles, hipStream_t s);
int gemm8_f32(int act, const Gemm8Args& g, const Cut8& c, int max_tiles, hipStream_t s);

}  // namespace moe
