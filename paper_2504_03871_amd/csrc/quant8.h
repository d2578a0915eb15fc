// 8-bit integers with one scale per row (activations) or column (weights), and the order in which the matrix cores take weights.
#pragma once
#include "pack8.h"
#include "rows.h"

namespace moe {

// A weight matrix [d_in][d_out] in 8 bits lies in tiles of 64 rows x 16 columns, 1 KB each: for 16 columns all their rows first.  In a
// tile sixteen rows of a column are 16 adjacent bytes, the 16 columns of those follow each other, and the four runs of 16 rows:
// byte 16 l + j of a tile is row 16 (l / 16) + j, column l % 16, which is what lane l gives the 16 x 16 x 64 instruction.  So a
// wave's operand is one contiguous 1 KB load, from memory or from LDS, without swizzle or bank conflict.
constexpr int TILE8_K = 64, TILE8_N = 16, TILE8_BYTES = TILE8_K * TILE8_N;

// `range`: rows of the permuted buffers that take part (offsets == NULL: all)
int launch_quant_rows(int dtype, long long rows, int width, long long pitch, const void* src, const RowRange& range, int8_t* codes, float* scales, hipStream_t s);
int launch_quant_weight(int dtype, int n, int d_in, int d_out, const void* W, int8_t* codes, float* scales, hipStream_t s);

}  // namespace moe
