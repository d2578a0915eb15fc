// The 16-bit kernels of the dense products (linear.hip) for one storage type: row tiles, the adding of K parts.
#pragma once
#include "gemm_bf16_kernel.h"
#include "linear.h"

namespace moe {

// One product.  Large ones are bound by the matrix cores (T x d x n, bf16: 32768 x 4096 x 14336, SwiGLU forward 5.8 ms = 1325 TFLOP/s,
// dx 5.2 = 1488, dW 5.6 = 1374); ordinary ones by what all blocks do at the same time before and after K: 8192 x 1024 x 4096 with
// GELU, residual and pre-activations 94-110 us, of which K is 45, the 200 MB of the epilogue 36 at the rate of a copy and GELU 10
// (two blocks of 128 x 128 on a compute unit, whose epilogues overlap the other's K, 115; 160 and 128 rows 103 and 99).  Few rows
// are a read of the weights: 1 x 4096 x 14336 SwiGLU 235 MB, 37 us; 16 x 14336 x 4096 117 MB, 21 us.
template <typename ST, int MODE, int EPI, bool DUAL, bool CHAIN, int BM, int BN, int WGM, int WGN, bool STREAM = false>
__global__ __launch_bounds__(WGM* WGN * 64, WGM * WGN == 4 ? 2 : 1) void linear_rows_kernel(GemmArgs g) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  gemm_bf16_tile<ST, MODE, EPI, DUAL, CHAIN, BM, BN, WGM, WGN, false, STREAM, true>(g, blockIdx.x, smem);
}
// The input's gradient (g1, tiles of 64 x 128) and the weights' (g2, 128 x 128) in one launch, where together they do not fill the chip:
// they need nothing of each other.
template <typename ST, bool CHAIN, int EPI2>
__global__ __launch_bounds__(256, 1) void linear_pair_kernel(GemmArgs g1, GemmArgs g2, int first_blocks) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  if ((int)blockIdx.x < first_blocks) gemm_bf16_tile<ST, MODE_NT, EPI_LIN_NONE, false, CHAIN, 64, 128, 2, 2, false, false, true>(g1, blockIdx.x, smem);
  else gemm_bf16_tile<ST, MODE_TN, EPI2, false, false, 128, 128, 2, 2, false, false, true>(g2, blockIdx.x - first_blocks, smem);
}

// Adds the parts of split tiles in part order and applies the epilogue; a thread owns eight adjacent columns of a row.  4-5 us for
// up to a few MB of parts, as for any small launch; 4096 x 2048 in two parts, 84 MB, 16 us = 5.2 TB/s.
template <typename ST, int EPI>
__global__ __launch_bounds__(256) void linear_join_kernel(GemmArgs g) {
  constexpr bool DUAL = EPI == EPI_LIN_SWIGLU;
  const int parts = g.split_parts, BN = g.tile_cols, TPR = BN / 8, RPB = 256 / TPR;   // threads per row, rows per block
  const int per_tile = g.tile_rows / RPB;
  const int q = blockIdx.x / per_tile, m = (blockIdx.x % per_tile) * RPB + threadIdx.x / TPR, n = (threadIdx.x % TPR) * 8;
  int rt, nt;
  if (!block_to_tile(g.split_first + q, (g.M + g.tile_rows - 1) / g.tile_rows, g.M / g.tile_rows, (g.N + BN - 1) / BN, g.chunked != 0, rt, nt)) return;
  const long long row = (long long)rt * g.tile_rows + m;
  const int col = nt * BN + n;
  if (row >= g.M || col >= g.N) return;
  const size_t pitch = (size_t)g.tile_rows * BN * (DUAL ? 2 : 1);      // floats between the parts
  const float* src = g.split_ws + (size_t)q * parts * pitch + m * BN + n;
  const float* src2 = src + (size_t)g.tile_rows * BN;
  float z[8] = {}, z2[8] = {};
#pragma unroll 4
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
  Vec16<ST> vec;
  float f[8];
  auto add = [&](const void* p, size_t off, float (&to)[8]) {
    if (p == nullptr) return;
    vec.load(reinterpret_cast<const ST*>(p) + off);
    vec.unpack(f);
#pragma unroll
    for (int i = 0; i < 8; ++i) to[i] += f[i];
  };
  auto put = [&](void* p, const float (&v)[8]) {
    vec.pack(v);
    vec.store(reinterpret_cast<ST*>(p) + at);
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

template <typename K>
static int more_lds(K kern, int lds) {   // above 64 KB, on every launch: nothing is remembered
  const hipError_t err = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  return err == hipSuccess ? MOE_OK : set_hip_error(err);
}

template <typename ST, int MODE, int EPI, bool DUAL, bool CHAIN, int BM, int BN, int WGM, int WGN, bool STREAM = false>
static int launch_tiles(const GemmArgs& g, long long blocks, hipStream_t s) {
  constexpr int lds = gemm_bf16_lds_bytes<BM, BN, DUAL>();
  auto kern = linear_rows_kernel<ST, MODE, EPI, DUAL, CHAIN, BM, BN, WGM, WGN, STREAM>;
  const int rc = more_lds(kern, lds);
  if (rc != MOE_OK) return rc;
  if (blocks > 0x7fffffffll) return MOE_ERR_BAD_SHAPE;
  kern<<<dim3((unsigned)blocks), WGM * WGN * 64, lds, s>>>(g);
  return launch_status();
}
template <typename ST, int EPI>
static int launch_join(const GemmArgs& g, long long blocks, hipStream_t s) {
  linear_join_kernel<ST, EPI><<<dim3((unsigned)blocks), 256, 0, s>>>(g);
  return launch_status();
}
template <typename ST, int MODE, int EPI, bool CHAIN>
static int launch_rows(GemmArgs g, const RowCut& cut, float* split_ws, hipStream_t s) {
  constexpr bool DUAL = EPI == EPI_LIN_SWIGLU;
  if (cut.tiles > 0x7fffffffll) return MOE_ERR_BAD_SHAPE;
  g.tile_rows = cut.rows;
  g.tile_cols = cut.cols;
  g.split_first = (int)cut.first;
  g.split_parts = cut.parts;
  g.split_ws = split_ws;
  const long long blocks = cut.first + (cut.tiles - cut.first) * cut.parts;
  int rc;
  switch (cut.rows) {
    case 256: rc = launch_tiles<ST, MODE, EPI, DUAL, CHAIN, 256, DUAL ? 128 : 256, DUAL ? 4 : 2, DUAL ? 2 : 4>(g, blocks, s); break;
    case 160: rc = launch_tiles<ST, MODE, EPI, DUAL, CHAIN, 160, DUAL ? 128 : 256, 2, 4>(g, blocks, s); break;
    case 128: rc = launch_tiles<ST, MODE, EPI, DUAL, CHAIN, 128, DUAL ? 128 : 256, 2, 4>(g, blocks, s); break;
    default:
      // one row tile: every weight is read once, and requested as streaming data
      if (MODE == MODE_NN && g.M <= 64) rc = launch_tiles<ST, MODE, EPI, DUAL, CHAIN, 64, 128, 2, DUAL ? 4 : 2, MODE == MODE_NN>(g, blocks, s);
      else rc = launch_tiles<ST, MODE, EPI, DUAL, CHAIN, 64, 128, 2, DUAL ? 4 : 2>(g, blocks, s);
  }
  if (rc != MOE_OK || cut.parts == 1) return rc;
  return launch_join<ST, EPI>(g, (cut.tiles - cut.first) * (cut.rows * cut.cols / 8 / 256), s);
}
template <typename ST, int EPI>
static int launch_dw(const GemmArgs& g, int rows, hipStream_t s) {
  switch (rows) {
    case 256: return launch_tiles<ST, MODE_TN, EPI, false, false, 256, 256, 2, 4>(g, dw_blocks(g, 256, 256), s);
    default: return launch_tiles<ST, MODE_TN, EPI, false, false, 128, 128, 4, 2>(g, dw_blocks(g, 128, 128), s);
  }
}
template <typename ST>
static int fwd_half_act(int act, const GemmArgs& g, const LinearPlan& p, float* ws, hipStream_t s) {
  return act == MOE_ACT_SWIGLU ? launch_rows<ST, MODE_NN, EPI_LIN_SWIGLU, false>(g, p.fwd, ws, s)
         : act == MOE_ACT_GELU ? launch_rows<ST, MODE_NN, EPI_LIN_GELU, false>(g, p.fwd, ws, s)
                               : launch_rows<ST, MODE_NN, EPI_LIN_NONE, false>(g, p.fwd, ws, s);
}

template <typename ST, bool CHAIN, int EPI2>
static int launch_pair(GemmArgs g1, const GemmArgs& g2, const LinearPlan& p, float* ws, hipStream_t s) {
  constexpr int lds1 = gemm_bf16_lds_bytes<64, 128, false>(), lds2 = gemm_bf16_lds_bytes<128, 128, false>(), lds = lds1 > lds2 ? lds1 : lds2;
  auto kern = linear_pair_kernel<ST, CHAIN, EPI2>;
  const int rc = more_lds(kern, lds);
  if (rc != MOE_OK) return rc;
  g1.tile_rows = p.dx.rows;
  g1.tile_cols = p.dx.cols;
  g1.split_first = (int)p.dx.first;
  g1.split_parts = p.dx.parts;
  g1.split_ws = ws;
  // a multiple of the XCD count: a tile number still tells the XCD for the second product
  const long long n1 = (p.dx.tiles * p.dx.parts + NUM_XCD - 1) / NUM_XCD * NUM_XCD, n2 = dw_blocks(g2, 128, 128);
  kern<<<dim3((unsigned)(n1 + n2)), 256, lds, s>>>(g1, g2, (int)n1);
  const int rc2 = launch_status();
  if (rc2 != MOE_OK || p.dx.parts == 1) return rc2;
  return launch_join<ST, EPI_LIN_NONE>(g1, p.dx.tiles * (p.dx.rows * p.dx.cols / 8 / 256), s);
}

// What linear.hip calls for a storage type
template <typename ST>
struct LinearHalf {
  static int forward(int act, const GemmArgs& g, const LinearPlan& p, float* ws, hipStream_t s) { return fwd_half_act<ST>(act, g, p, ws, s); }
  static int input_grad(bool two, const GemmArgs& g, const LinearPlan& p, float* ws, hipStream_t s) {
    return two ? launch_rows<ST, MODE_NT, EPI_LIN_NONE, true>(g, p.dx, ws, s) : launch_rows<ST, MODE_NT, EPI_LIN_NONE, false>(g, p.dx, ws, s);
  }
  // in_type: in the storage type instead of fp32
  static int weight_grad(bool in_type, const GemmArgs& g, const LinearPlan& p, hipStream_t s) {
    return in_type ? launch_dw<ST, EPI_LIN_NONE>(g, p.dw_rows, s) : launch_dw<ST, EPI_DW>(g, p.dw_rows, s);
  }
  static int both_grads(bool two, bool in_type, const GemmArgs& g1, const GemmArgs& g2, const LinearPlan& p, float* ws, hipStream_t s) {
    if (two) return in_type ? launch_pair<ST, true, EPI_LIN_NONE>(g1, g2, p, ws, s) : launch_pair<ST, true, EPI_DW>(g1, g2, p, ws, s);
    return in_type ? launch_pair<ST, false, EPI_LIN_NONE>(g1, g2, p, ws, s) : launch_pair<ST, false, EPI_DW>(g1, g2, p, ws, s);
  }
};

}  // namespace moe
