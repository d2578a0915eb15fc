// Products of 8-bit integers on the gfx950 matrix cores: y = act(z) + residual, z = a_scale b_scale (A B) + bias, with 32-bit integer sums, which
// are exact.  Two kernels: tiles of up to 256 x 256 for many rows, and strips of 16 columns, streamed, for few.
//
// Tiles.  v_mfma_i32_16x16x64_i8 has the operand registers of the 16-bit 16 x 16 x 32 instruction and twice its products, so a stage of
// 128 K values is as many bytes as one of 64 there, and the pipeline is the one of gemm_bf16_kernel.h: LDS stages filled by loads that
// write LDS directly, three of A and two of B, two K steps to an iteration with one block barrier, in regions of one row tile's
// instructions each, behind which the reads of the next step's fragments and this step's share of the loads are issued.  A comes in rows and
// is swizzled in LDS (kc_off); B comes in the order of the instruction (quant8.h) and is read lane by lane.  Sums of 64 K values past
// the end (an odd number of them) are those of a B of zeros, which the descriptor's byte count gives.
// The weights are the instruction's first operand: a lane has four adjacent columns of one row of every 16 x 16 tile.
#pragma once
#include "gemm_bf16_kernel.h"
#include "gemm_i8.h"

namespace moe {

// Nothing from here on is fused that is not written so, whatever stands around it: a row's result is the same bits in every kernel,
// beside however many other rows.
#pragma clang fp contract(off)

typedef int i32x4 __attribute__((ext_vector_type(4)));
template <int V> struct Const { static constexpr int value = V; };   // a number that a lambda takes as a type
constexpr int BK8 = 128;   // K values (bytes) per LDS stage

// what depends on the type of the results
template <typename ST> __device__ __forceinline__ float gelu8(float z) { return __is_same(ST, float) ? gelu_f(z) : z * phi_fast(z); }
template <typename ST> __device__ __forceinline__ float silu8(float z) { return __is_same(ST, float) ? z * sigmoid_f(z) : z * sigmoid_fast(z); }

// Four adjacent columns of one row: sums to act(z), in fp32.
template <typename ST, int ACT>
__device__ __forceinline__ f32x4 finish8(const i32x4& a, const i32x4& a2, float row, const f32x4& col, const f32x4& col2, const f32x4& bias, const f32x4& bias2) {
  f32x4 y;
#pragma unroll
  for (int v = 0; v < 4; ++v) {
    const float z = fmaf((float)a[v], row * col[v], bias[v]);
    if constexpr (ACT == MOE_ACT_SWIGLU) y[v] = silu8<ST>(z) * fmaf((float)a2[v], row * col2[v], bias2[v]);
    else if constexpr (ACT == MOE_ACT_GELU) y[v] = gelu8<ST>(z);
    else y[v] = z;
  }
  return y;
}
template <typename ST>
__device__ __forceinline__ f32x4 load4(const void* base, size_t i) {   // four values of a vector of the storage type, or zeros
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  if (base == nullptr) return v;
  const ST* p = reinterpret_cast<const ST*>(base) + i;
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = to_f32(p[j]);
  return v;
}
__device__ __forceinline__ i32x4 mfma8(const i32x4& a, const i32x4& b, const i32x4& c) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0); }

// Row of A behind row r of the product: the token of an assignment (held inside A whatever the index says), or the row itself.
__device__ __forceinline__ int row_of_a(const Gemm8Args& g, int r) {
  return g.src_of == nullptr ? r : min(max(g.src_of[r] / g.per_row, 0), g.src_rows - 1);
}

template <int BM, int BN, bool DUAL>
constexpr int gemm8_lds_bytes() { return 3 * BM * BK8 + 2 * BN * BK8 * (DUAL ? 2 : 1); }

template <typename ST, int ACT, int BM, int BN, int WGM, int WGN, int PER_CU, bool GROUPED>
__global__ __launch_bounds__(WGM* WGN * 64, PER_CU* WGM* WGN / 4) void gemm8_kernel(Gemm8Args g) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  constexpr bool DUAL = ACT == MOE_ACT_SWIGLU;
  constexpr int NT = WGM * WGN * 64;
  constexpr int WTM = BM / 32 / WGM, TM = 2 * WTM, TNN = BN / WGN / 16;   // row tiles, column tiles (of either matrix) of a wave
  constexpr int A_BYTES = BM * BK8, B_BYTES = BN * BK8, B_STAGE = B_BYTES * (DUAL ? 2 : 1), B_AT = 3 * A_BYTES;
  constexpr int LA = BM * 8 / NT, LB1 = BN * 8 / NT, LB = LB1 * (DUAL ? 2 : 1);   // 16-byte loads per thread and stage
  static_assert(BM * 8 % NT == 0 && BN * 8 % NT == 0 && WTM * 32 * WGM == BM && TNN % 2 == 0, "whole loads, whole waves");
  static_assert((WGM * WGN) % 2 == 0, "a wave's loads of B are all of the same half of a stage");

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / WGN, wn = wave % WGN;
  const int ntn = (g.N + BN - 1) / BN, n_rt = GROUPED ? g.ntiles[0] : (g.M + BM - 1) / BM, n_full = GROUPED ? g.ntiles[1] : g.M / BM;
  int rt, nt;
  if (!block_to_tile(blockIdx.x, n_rt, n_full, ntn, g.chunked != 0, rt, nt)) return;
  rt = __builtin_amdgcn_readfirstlane(rt);
  nt = __builtin_amdgcn_readfirstlane(nt);
  RowTile t;
  if constexpr (GROUPED) t = g.tiles[rt];
  else t = RowTile{0, rt * BM, min(BM, g.M - rt * BM), 0};
  const int e = __builtin_amdgcn_readfirstlane(t.e), row0 = __builtin_amdgcn_readfirstlane(t.row0), mvalid = __builtin_amdgcn_readfirstlane(t.nrows);
  const int n0 = nt * BN, K = g.K;
  const int ni = min(max(((mvalid + 31) / 32 - wm + WGM - 1) / WGM, 0), WTM);   // this wave's 32-row bands with valid rows

  i32x4 acc[TM][TNN] = {}, acc2[DUAL ? TM : 1][DUAL ? TNN : 1] = {};

  // operands: of A the rows of this tile (by token: all of it), of B this expert's matrix
  const bool gather = GROUPED && g.src_of != nullptr;
  const rsrc_t ra = gather ? make_rsrc(g.A, (size_t)g.src_rows * K) : make_rsrc(g.A + (size_t)row0 * K, (size_t)mvalid * K);
  const size_t mat = (size_t)g.N * K;
  const rsrc_t rb = make_rsrc(g.B + e * mat, mat), rb2 = make_rsrc((DUAL ? g.B2 : g.B) + e * mat, mat);
  const int KT = K / TILE8_K, KS = (KT + 1) / 2;   // tiles of 64 K values, stages
  unsigned a_vo[LA], b_vo[LB1];
#pragma unroll
  for (int i = 0; i < LA; ++i) {
    const int id = tid + NT * i, r = id / 8, pc = id % 8;
    const int rr = min(r, mvalid - 1);   // rows past the tile repeat its last one; what they give is not stored
    a_vo[i] = (unsigned)(gather ? row_of_a(g, row0 + rr) : rr) * (unsigned)K + (unsigned)(pc ^ ((r / 2) & 7)) * 16u;
  }
#pragma unroll
  for (int i = 0; i < LB1; ++i) {
    const int id = wave + NT / 64 * i;   // 1 KB tile of the stage: column tile id / 2, half id % 2 = wave % 2
    b_vo[i] = ((unsigned)(n0 / TILE8_N + id / 2) * (unsigned)KT + (unsigned)(id & 1)) * TILE8_BYTES + (unsigned)lane * 16u;
  }
  const int half = wave & 1;
  const unsigned smem_base = lds_addr(smem);
  const int wbase = wave * 1024;
  int a_fr[2];
#pragma unroll
  for (int ks = 0; ks < 2; ++ks) a_fr[ks] = kc_off(wm * 32 + (lane & 15), ks * 4 + (lane >> 4));
  const int b_fr = B_AT + wn * TNN * 2 * TILE8_BYTES + lane * 16;

  auto load_a = [&](int q, int stage, int buf) { load_to_lds16(ra, smem_base + buf + wbase + NT * 16 * q, a_vo[q] + (unsigned)stage * BK8); };
  auto load_b = [&](int q, int stage, int buf) {
    const int c = DUAL ? q / 2 : q;
    const bool first = !DUAL || q % 2 == 0;
    const unsigned off = 2 * stage + half < KT ? b_vo[c] + (unsigned)stage * (2 * TILE8_BYTES) : OUT_OF_RANGE;
    load_to_lds16(first ? rb : rb2, smem_base + B_AT + buf + (first ? 0 : B_BYTES) + wbase + NT * 16 * c, off);
  };
  i32x4 af[TM], bf[2][TNN], bf2[2][DUAL ? TNN : 1];
  auto frag_a = [&](int i, int buf, int ks) {
    af[i] = *reinterpret_cast<const i32x4*>(smem + buf + a_fr[ks] + ((i >> 1) * WGM * 32 + (i & 1) * 16) * BK8);
  };
  auto frag_b = [&](int set, int j, int buf, int ks) {
    const char* p = smem + b_fr + buf + (j * 2 + ks) * TILE8_BYTES;
    bf[set][j] = *reinterpret_cast<const i32x4*>(p);
    if constexpr (DUAL) bf2[set][j] = *reinterpret_cast<const i32x4*>(p + B_BYTES);
  };
  constexpr int WAIT_P = ((LA + LB) & 15) | (((LA + LB) >> 4) << 14) | 0x70 | (15 << 8);   // s_waitcnt vmcnt(LA + LB) only
  constexpr int WAIT_A = LA | 0x70;                                                        // s_waitcnt vmcnt(LA) lgkmcnt(0)
  static_assert(LA + LB < 64 && LA < 16, "the wait counter");
  auto barrier = [&]() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  // One K step on fragment set `set`: behind row tile r's instructions, its fragment of the next step (ks of the stages at abuf, bbuf),
  // the next step's fragments of B in the first TNN regions, and this region's loads.
  auto step = [&](auto set_, bool next, int abuf, int bbuf, int ks, auto do_load, int bands) {
    constexpr int set = decltype(set_)::value;
#pragma unroll
    for (int r = 0; r < TM; ++r) {
      if ((r >> 1) < bands) {
#pragma unroll
        for (int j = 0; j < TNN; ++j) {
          acc[r][j] = mfma8(bf[set][j], af[r], acc[r][j]);
          if constexpr (DUAL) acc2[r][j] = mfma8(bf2[set][j], af[r], acc2[r][j]);
        }
      }
      if (next) {
        frag_a(r, abuf, ks);
#pragma unroll
        for (int j = 0; j < TNN; ++j)
          if (j % TM == r) frag_b(set ^ 1, j, bbuf, ks);
      }
      do_load(r);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  int a0 = 0, a1 = A_BYTES, a2 = 2 * A_BYTES, b0 = 0, b1 = B_STAGE;
  auto prologue = [&](int stage, int abuf, int bbuf) {
#pragma unroll
    for (int q = 0; q < LB; ++q) load_b(q, stage, bbuf);
#pragma unroll
    for (int q = 0; q < LA; ++q) load_a(q, stage, abuf);
  };
  prologue(0, a0, b0);
  if (KS > 1) {
    prologue(1, a1, b1);
    __builtin_amdgcn_s_waitcnt(WAIT_P);
  } else {
    __builtin_amdgcn_s_waitcnt(0x70 | (15 << 8));
  }
  barrier();
  auto mainloop = [&](int bands) {
#pragma unroll
    for (int i = 0; i < TM; ++i) frag_a(i, a0, 0);
#pragma unroll
    for (int j = 0; j < TNN; ++j) frag_b(0, j, b0, 0);
    __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0)
    // Iteration S: K step 0 reads the fragments of K step 1 and requests A of stage S + 2, whose LDS has been free since the last barrier;
    // then every wave waits for stage S + 1 (B of it, and A, are older than those loads) and for its reads, and joins the barrier;
    // K step 1 reads the first fragments of stage S + 1 and requests B of stage S + 2 into what stage S has left.
    auto iteration = [&](int S, bool more, auto load) {
      constexpr bool LOAD = decltype(load)::value != 0;
      step(Const<0>{}, true, a0, b0, 1, [&](int r) {
        if constexpr (LOAD) {
#pragma unroll
          for (int q = 0; q < LA; ++q)
            if (q * TM / LA == r) load_a(q, S + 2, a2);
        }
      }, bands);
      if (more) {
        if constexpr (LOAD) __builtin_amdgcn_s_waitcnt(WAIT_A);
        else __builtin_amdgcn_s_waitcnt(0);
        barrier();
      }
      step(Const<1>{}, more, a1, b1, 0, [&](int r) {
        if constexpr (LOAD) {
#pragma unroll
          for (int q = 0; q < LB; ++q)
            if (q * TM / (2 * LB) == r) load_b(q, S + 2, b0);
        }
      }, bands);
      const int a = a0; a0 = a1; a1 = a2; a2 = a;
      const int b = b0; b0 = b1; b1 = b;
    };
    int S = 0;
#pragma unroll 1
    for (; S + 2 < KS; ++S) iteration(S, true, Const<1>{});
#pragma unroll 1
    for (; S < KS; ++S) iteration(S, S + 1 < KS, Const<0>{});
  };
  if (ni == WTM) mainloop(WTM);
  else mainloop(ni);

  // Epilogue.  act(z) in the accumulators' layout, then exchanges between lanes to whole lines (gemm_bf16_kernel.h), the residual there.
  constexpr int C = TNN * 16;
  const int col_w = n0 + wn * C;
  if (col_w >= g.N) return;
  const int grp = lane >> 4, r8 = lane & 7, right = (lane >> 3) & 1;
  const float* bs = g.b_scale + (size_t)e * g.N;
  const float* bs2 = DUAL ? g.b2_scale + (size_t)e * g.N : bs;
  const size_t first = (size_t)row0 * g.N + n0, bytes = ((size_t)mvalid * g.N - n0) * sizeof(ST);
  const __amdgpu_buffer_rsrc_t oy = out_rsrc(reinterpret_cast<ST*>(g.C) + first, bytes);
  const __amdgpu_buffer_rsrc_t res = out_rsrc(reinterpret_cast<const ST*>(g.residual) + (g.residual != nullptr ? first : 0), g.residual != nullptr ? bytes : 0);
  const unsigned pitch = (unsigned)g.N * sizeof(ST);
  auto band_row = [&](int i) { return ((i >> 1) * WGM + wm) * 32 + (i & 1) * 16; };
  f32x4 sw[TNN], sw2[DUAL ? TNN : 1], bias[TNN], bias2[DUAL ? TNN : 1];
#pragma unroll
  for (int j = 0; j < TNN; ++j) {
    const int c = col_w + j * 16 + grp * 4;
    sw[j] = *reinterpret_cast<const f32x4*>(bs + c);
    bias[j] = load4<ST>(g.bias, c);
    if constexpr (DUAL) { sw2[j] = *reinterpret_cast<const f32x4*>(bs2 + c); bias2[j] = load4<ST>(g.bias2, c); }
  }
  float sx[TM];
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int m = min(band_row(i) + (lane & 15), mvalid - 1);
    sx[i] = g.a_scale[row_of_a(g, row0 + m)];
  }
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    if (band_row(i) >= mvalid) continue;
    f32x4 y[TNN];
#pragma unroll
    for (int j = 0; j < TNN; ++j)
      y[j] = finish8<ST, ACT>(acc[i][j], acc2[DUAL ? i : 0][DUAL ? j : 0], sx[i], sw[j], sw2[DUAL ? j : 0], bias[j], bias2[DUAL ? j : 0]);
    if constexpr (__is_same(ST, float)) {
#pragma unroll
      for (int j = 0; j < TNN; j += 2) {
        swap8(y[j], y[j + 1]);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int m = band_row(i) + h * 8 + r8;
          const unsigned off = m < mvalid ? (unsigned)m * pitch + (unsigned)(wn * C + j * 16 + right * 16 + grp * 4) * 4u : OUT_OF_RANGE;
          const f32x4 r = __builtin_bit_cast(f32x4, buf_load16_nt(res, off));
          buf_store16<AUX_NT>(oy, off, __builtin_bit_cast(u32x4, y[j + h] + r));
        }
      }
    } else {
      typedef Half16<ST> H;
#pragma unroll
      for (int j = 0; j < TNN; j += 2) join_tiles(y[j], y[j + 1]);   // a lane: eight adjacent columns of 32
      if constexpr (TNN == 4) { swap8(y[0], y[2]); swap8(y[1], y[3]); }
#pragma unroll
      for (int h = 0; h < TNN / 2; ++h) {
        const int m = band_row(i) + (TNN == 4 ? h * 8 + r8 : (lane & 15));
        const unsigned off = m < mvalid ? (unsigned)m * pitch + (unsigned)(wn * C + (TNN == 4 ? right * 32 : h * 32) + lane_col8(grp)) * 2u : OUT_OF_RANGE;
        const u32x4 r = buf_load16_nt(res, off);
        u32x4 o;
#pragma unroll
        for (int q = 0; q < 4; ++q)
          o[q] = H::pack2(y[2 * h + q / 2][q % 2 * 2] + H::lo(r[q]), y[2 * h + q / 2][q % 2 * 2 + 1] + H::hi(r[q]));
        buf_store16<AUX_NT>(oy, off, o);
      }
    }
  }
}

// ---- few rows ----
// A block takes a strip of 16 columns and a group of 16 MT rows; its waves share out the K range, 64 values at a time in turn, and add their
// sums in LDS, in any order the same: they are integers.  An operand of B is one contiguous 1 KB load of a wave, of A 16 rows x 64
// bytes that all strips read from the caches.  Bound by the read of the weights.
// Experts: blockIdx.y is the n-th group of 16 MT rows of some expert, which every block finds for itself from the experts' row counts.
constexpr int FEW_WAVES = 8;

template <typename ST, int ACT, int MT, bool GROUPED>
__global__ __launch_bounds__(FEW_WAVES * 64) void few8_kernel(Gemm8Args g) {
  constexpr bool DUAL = ACT == MOE_ACT_SWIGLU;
  constexpr int MATS = DUAL ? 2 : 1, ROWS = 16 * MT, U = MT == 1 ? 4 : 2;
  __shared__ __align__(16) i32x4 s_sum[FEW_WAVES][MATS * MT][64];
  __shared__ int s_tile[3], s_scan[FEW_WAVES];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int e = 0, row0 = blockIdx.y * ROWS, rows = min(ROWS, g.M - row0);
  if constexpr (GROUPED) {
    static_assert(MOE_MAX_E <= FEW_WAVES * 64, "a thread per expert");
    int l = 0, h = 0;
    if (tid < g.E) share_of(g.lo, g.hi, g.kept[tid], tid, l, h);
    const int mine = (h - l + ROWS - 1) / ROWS;
    if (tid == 0) s_tile[0] = -1;
    const int scan = wave_scan_i(mine);
    if (lane == 63) s_scan[wave] = scan;
    __syncthreads();
    int before = scan - mine;
    for (int w = 0; w < wave; ++w) before += s_scan[w];
    const int q = (int)blockIdx.y - before;
    if (q >= 0 && q < mine) {
      s_tile[0] = tid;
      s_tile[1] = g.offsets[tid] + l + q * ROWS;
      s_tile[2] = min(ROWS, h - l - q * ROWS);
    }
    __syncthreads();
    e = __builtin_amdgcn_readfirstlane(s_tile[0]);
    if (e < 0) return;
    row0 = __builtin_amdgcn_readfirstlane(s_tile[1]);
    rows = __builtin_amdgcn_readfirstlane(s_tile[2]);
  }
  const int K = g.K, KT = K / TILE8_K, n0 = blockIdx.x * TILE8_N;
  const int k0 = GROUPED ? 0 : (int)((long long)blockIdx.z * KT / g.n_parts), k1 = GROUPED ? KT : (int)((long long)(blockIdx.z + 1) * KT / g.n_parts);
  const size_t strip = (size_t)e * g.N * K + (size_t)n0 * K + lane * 16;
  const int8_t *pb = g.B + strip, *pb2 = DUAL ? g.B2 + strip : pb;
  const int8_t* pa[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
    pa[i] = g.A + (size_t)row_of_a(g, row0 + min(i * 16 + (lane & 15), rows - 1)) * K + (lane >> 4) * 16;   // (rows past the group repeat its last)
  i32x4 acc[MATS][MT] = {};
  auto run = [&](int k, auto n_) {
    constexpr int N_ = decltype(n_)::value;
    i32x4 b[N_][MATS], a[N_][MT];
#pragma unroll
    for (int u = 0; u < N_; ++u) {
      const size_t at = (size_t)(k + u * FEW_WAVES);
      b[u][0] = *reinterpret_cast<const i32x4*>(pb + at * TILE8_BYTES);
      if constexpr (DUAL) b[u][1] = *reinterpret_cast<const i32x4*>(pb2 + at * TILE8_BYTES);
#pragma unroll
      for (int i = 0; i < MT; ++i) a[u][i] = *reinterpret_cast<const i32x4*>(pa[i] + at * TILE8_K);
    }
#pragma unroll
    for (int u = 0; u < N_; ++u)
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int q = 0; q < MATS; ++q) acc[q][i] = mfma8(b[u][q], a[u][i], acc[q][i]);
  };
  int k = k0 + wave;
  for (; k + (U - 1) * FEW_WAVES < k1; k += U * FEW_WAVES) run(k, Const<U>{});
  for (; k < k1; k += FEW_WAVES) run(k, Const<1>{});
#pragma unroll
  for (int q = 0; q < MATS; ++q)
#pragma unroll
    for (int i = 0; i < MT; ++i) s_sum[wave][q * MT + i][lane] = acc[q][i];
  __syncthreads();
  if (wave >= MT) return;
  const int m = wave * 16 + (lane & 15), c = n0 + (lane >> 4) * 4;
  if (m >= rows) return;
  i32x4 sum[MATS];
#pragma unroll
  for (int q = 0; q < MATS; ++q) {
    sum[q] = s_sum[0][q * MT + wave][lane];
#pragma unroll
    for (int w = 1; w < FEW_WAVES; ++w) sum[q] += s_sum[w][q * MT + wave][lane];
  }
  const size_t row = row0 + m;
  if (!GROUPED && g.n_parts > 1) {
#pragma unroll
    for (int q = 0; q < MATS; ++q)
      *reinterpret_cast<i32x4*>(g.parts + ((size_t)(blockIdx.z * MATS + q) * g.M + row) * g.N + c) = sum[q];
    return;
  }
  const size_t cs = (size_t)e * g.N + c;
  const f32x4 sw = *reinterpret_cast<const f32x4*>(g.b_scale + cs), sw2 = DUAL ? *reinterpret_cast<const f32x4*>(g.b2_scale + cs) : sw;
  f32x4 y = finish8<ST, ACT>(sum[0], sum[MATS - 1], g.a_scale[row_of_a(g, (int)row)], sw, sw2, load4<ST>(g.bias, c), load4<ST>(DUAL ? g.bias2 : nullptr, c));
  y += load4<ST>(g.residual, row * g.N + c);
  ST* out = reinterpret_cast<ST*>(g.C) + row * g.N + c;
  if constexpr (__is_same(ST, float)) *reinterpret_cast<f32x4*>(out) = y;
  else *reinterpret_cast<u32x2*>(out) = u32x2{Half16<ST>::pack2(y[0], y[1]), Half16<ST>::pack2(y[2], y[3])};
}

// Adds the K parts; a thread has four adjacent columns of a row.
template <typename ST, int ACT>
__global__ __launch_bounds__(256) void few8_join_kernel(Gemm8Args g) {
  constexpr int MATS = ACT == MOE_ACT_SWIGLU ? 2 : 1;
  const size_t per_row = g.N / 4, i = (size_t)blockIdx.x * 256 + threadIdx.x, row = i / per_row;
  const int c = (int)(i - row * per_row) * 4;
  if (row >= (size_t)g.M) return;
  i32x4 sum[MATS] = {};
  for (int p = 0; p < g.n_parts; ++p)
#pragma unroll
    for (int q = 0; q < MATS; ++q) sum[q] += *reinterpret_cast<const i32x4*>(g.parts + ((size_t)(p * MATS + q) * g.M + row) * g.N + c);
  const f32x4 sw = *reinterpret_cast<const f32x4*>(g.b_scale + c), sw2 = MATS > 1 ? *reinterpret_cast<const f32x4*>(g.b2_scale + c) : sw;
  f32x4 y = finish8<ST, ACT>(sum[0], sum[MATS - 1], g.a_scale[row], sw, sw2, load4<ST>(g.bias, c), load4<ST>(MATS > 1 ? g.bias2 : nullptr, c));
  y += load4<ST>(g.residual, row * g.N + c);
  ST* out = reinterpret_cast<ST*>(g.C) + row * g.N + c;
  if constexpr (__is_same(ST, float)) *reinterpret_cast<f32x4*>(out) = y;
  else *reinterpret_cast<u32x2*>(out) = u32x2{Half16<ST>::pack2(y[0], y[1]), Half16<ST>::pack2(y[2], y[3])};
}

// ---- launches ----
template <typename ST, int ACT, int BM, int BN, int WGM, int WGN, int PER_CU, bool GROUPED>
static int gemm8_launch(const Gemm8Args& g, long long row_tiles, hipStream_t s) {
  constexpr int LDS = gemm8_lds_bytes<BM, BN, ACT == MOE_ACT_SWIGLU>();
  static_assert(LDS * PER_CU <= LDS_BYTES, "blocks that a compute unit holds");
  const void* fn = reinterpret_cast<const void*>(gemm8_kernel<ST, ACT, BM, BN, WGM, WGN, PER_CU, GROUPED>);
  if (LDS > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
    if (e != hipSuccess) return set_hip_error(e);
  }
  const long long grid = row_tiles * ((g.N + BN - 1) / BN);
  gemm8_kernel<ST, ACT, BM, BN, WGM, WGN, PER_CU, GROUPED><<<(unsigned)grid, WGM * WGN * 64, LDS, s>>>(g);
  return launch_status();
}
template <typename ST, int ACT, bool GROUPED>
static int few8_launch(const Gemm8Args& g, int rows, int groups, hipStream_t s) {
  const dim3 grid(g.N / TILE8_N, groups, GROUPED ? 1 : g.n_parts);
  if (rows == 16) few8_kernel<ST, ACT, 1, GROUPED><<<grid, FEW_WAVES * 64, 0, s>>>(g);
  else if (rows == 32) few8_kernel<ST, ACT, 2, GROUPED><<<grid, FEW_WAVES * 64, 0, s>>>(g);
  else few8_kernel<ST, ACT, 4, GROUPED><<<grid, FEW_WAVES * 64, 0, s>>>(g);
  if (!GROUPED && g.n_parts > 1) few8_join_kernel<ST, ACT><<<(unsigned)(((size_t)g.M * (g.N / 4) + 255) / 256), 256, 0, s>>>(g);
  return launch_status();
}
template <typename ST, int ACT, bool GROUPED>
static int gemm8_act(const Gemm8Args& g, const Cut8& c, int max_tiles, hipStream_t s) {
  constexpr int D = ACT == MOE_ACT_SWIGLU ? 2 : 1;   // columns are of both matrices together
  if (c.few) return few8_launch<ST, ACT, GROUPED>(g, c.rows, GROUPED ? max_tiles : (g.M + c.rows - 1) / c.rows, s);
  const long long rt = GROUPED ? max_tiles : (g.M + c.rows - 1) / c.rows;
  if (c.rows == 256) return gemm8_launch<ST, ACT, 256, 256 / D, 2, 4, 1, GROUPED>(g, rt, s);
  if (c.rows == 128) return gemm8_launch<ST, ACT, 128, 128 / D, 2, 2, 2, GROUPED>(g, rt, s);
  return gemm8_launch<ST, ACT, 64, 128 / D, 2, 2, 2, GROUPED>(g, rt, s);
}
template <typename ST>
static int gemm8_for(int act, const Gemm8Args& g, const Cut8& c, int max_tiles, hipStream_t s) {
  if (g.E > 0) {
    if constexpr (!__is_same(ST, float)) {
      if (act == MOE_ACT_SWIGLU) return gemm8_act<ST, MOE_ACT_SWIGLU, true>(g, c, max_tiles, s);
      if (act == MOE_ACT_GELU) return gemm8_act<ST, MOE_ACT_GELU, true>(g, c, max_tiles, s);
      return gemm8_act<ST, MOE_ACT_NONE, true>(g, c, max_tiles, s);
    }
    return MOE_ERR_BAD_DTYPE;
  }
  if (act == MOE_ACT_SWIGLU) return gemm8_act<ST, MOE_ACT_SWIGLU, false>(g, c, max_tiles, s);
  if (act == MOE_ACT_GELU) return gemm8_act<ST, MOE_ACT_GELU, false>(g, c, max_tiles, s);
  return gemm8_act<ST, MOE_ACT_NONE, false>(g, c, max_tiles, s);
}

}  // namespace moe
