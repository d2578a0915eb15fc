// Products of 8-bit integers on the gfx950 matrix cores: y = act(z) + residual, z = a_scale b_scale (A B) + bias, with 32-bit integer sums, which
// are exact.  Two kernels: tiles of up to 256 x 256 for many rows, and strips of 16 columns, streamed, for few.
//
// Tiles.  v_mfma_i32_16x16x64_i8 has the operand registers of the 16-bit 16 x 16 x 32 instruction and twice its products, so a stage of
// 128 K values is as many bytes as one of 64 there, and the pipeline is the one of gemm_bf16_kernel.h: LDS stages filled by loads that
// write LDS directly, three of A and two of B (64 rows, or 128 that have a compute unit alone: three of both), two K steps to an iteration with one block barrier, in regions of one row tile's
// instructions each, behind which the reads of the next step's fragments and this step's share of the loads are issued.  A comes in rows and
// is swizzled in LDS (kc_off); B comes in the order of the instruction (quant8.h) and is read lane by lane.  Sums of 64 K values past
// the end (an odd number of them) are those of a B of zeros, which the descriptor's byte count gives.
// The weights are the instruction's first operand: a lane has four adjacent columns of one row of every 16 x 16 tile.
// Measured: 8192 x 8192 x 8192 415 us, 2650 TOP/s; 32768 x 4096 x 14336, two matrices and SwiGLU, 2.85 ms, 2700 TOP/s, matrix cores busy 0.70 of the
// cycles at a clock that their power holds at 1.6 to 1.8 GHz; 8192 x 2048 x 8192 131 us, 2100 TOP/s, where the 7 us in front of and behind K
// of every round of tiles, mostly the results' way to memory, count for more.
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

// Phi(v) for results of 16 bits: erfc(x) = exp(-x^2) t (a0 + a1 t + ... + a5 t^5), t = 1 / (1 + p x), x = |v| / sqrt(2): one exponential and one
// reciprocal like phi_fast (common.h), whose coefficients keep the absolute error of erfc small.  These, and p, were fitted (least squares
// with weights moved towards the largest errors) to the smallest error relative to erfc for x up to 10: 4e-6, and 1.5e-5 with the rounding of
// the exponential's argument at v = -12.6.  So GELU's tail, next to zero, is as good as its type; phi_fast is 4.7e-4 off at -4, half a step of
// fp16 there, and 6.5e-3 at -7, where bf16's is at most 3.9e-3.  The halves of a0 ... stand below.  (3001 x 2880 x 1088 with GELU: 26.1 us with either.)
__device__ __forceinline__ float phi_tail(float v) {
  const float x = fabsf(v) * 0.70710678118654752440f;
  const float t = __builtin_amdgcn_rcpf(fmaf(0.436f, x, 1.0f));
  const float poly = fmaf(t, fmaf(t, fmaf(t, fmaf(t, fmaf(t, -0.0752838403f, 0.188452139f), 0.0083345063f), 0.136168554f), 0.11909198f), 0.123234712f);
  const float half = t * poly * __builtin_amdgcn_exp2f(-(x * x) * 1.44269504088896340736f);
  return v >= 0.f ? 1.0f - half : half;
}
// what depends on the type of the results
template <typename ST> __device__ __forceinline__ float gelu8(float z) { return __is_same(ST, float) ? gelu_f(z) : z * phi_tail(z); }
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
    // A number in fp32, also for the compiler, which else rounds a product to fp16 without rounding it to fp32 first, in some kernels.
    if constexpr (__is_same(ST, f16)) asm("" : "+v"(y[v]));
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
  if (g.src_of == nullptr) return r;
  const int a = max(g.src_of[r], 0);
  return min((int)((uint64_t)(unsigned)a * g.per_row >> 33), g.src_rows - 1);
}

// DEPTH 2: two stages of B and three of A; 3: three of both.
template <int BM, int BN, bool DUAL, int DEPTH>
constexpr int gemm8_lds_bytes() { return DEPTH == 2 ? 3 * BM * BK8 + 2 * BN * BK8 * (DUAL ? 2 : 1) : DEPTH * BK8 * (BM + BN * (DUAL ? 2 : 1)); }

template <typename ST, int ACT, int BM, int BN, int WGM, int WGN, int PER_CU, int DEPTH, bool STREAM, bool GROUPED>
__global__ __launch_bounds__(WGM* WGN * 64, PER_CU* WGM* WGN / 4) void gemm8_kernel(Gemm8Args g) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  constexpr bool DUAL = ACT == MOE_ACT_SWIGLU;
  constexpr int NT = WGM * WGN * 64;
  constexpr int WTM = BM / 32 / WGM, TM = 2 * WTM, TNN = BN / WGN / 16;   // row tiles, column tiles (of either matrix) of a wave
  constexpr int A_BYTES = BM * BK8, B_BYTES = BN * BK8, B_STAGE = B_BYTES * (DUAL ? 2 : 1), B_AT = (DEPTH == 2 ? 3 : DEPTH) * A_BYTES;
  constexpr int LA = BM * 8 / NT, LB1 = BN * 8 / NT, LB = LB1 * (DUAL ? 2 : 1);   // 16-byte loads per thread and stage
  static_assert(BM * 8 % NT == 0 && BN * 8 % NT == 0 && WTM * 32 * WGM == BM && TNN % 2 == 0, "whole loads, whole waves");
  static_assert((WGM * WGN) % 2 == 0, "a wave's loads of B are all of the same half of a stage");

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / WGN, wn = wave % WGN;
  const int ntn = (g.N + BN - 1) / BN, n_rt = GROUPED ? g.ntiles[0] : (g.M + BM - 1) / BM, n_full = GROUPED ? g.ntiles[1] : g.M / BM;
  const int n_parts = GROUPED ? 1 : g.n_parts, part = n_parts > 1 ? blockIdx.x % n_parts : 0;
  int rt, nt;
  if (!block_to_tile(n_parts > 1 ? blockIdx.x / n_parts : blockIdx.x, n_rt, n_full, ntn, g.chunked != 0, rt, nt)) return;
  rt = __builtin_amdgcn_readfirstlane(rt);
  nt = __builtin_amdgcn_readfirstlane(nt);
  RowTile t;
  if constexpr (GROUPED) t = g.tiles[rt];
  else t = RowTile{0, rt * BM, min(BM, g.M - rt * BM), 0};
  const int e = __builtin_amdgcn_readfirstlane(t.e), row0 = __builtin_amdgcn_readfirstlane(t.row0), mvalid = __builtin_amdgcn_readfirstlane(t.nrows);
  const int n0 = nt * BN, K = g.K;
  const int ni = min(max(((mvalid + 31) / 32 - wm + WGM - 1) / WGM, 0), WTM);   // this wave's 32-row bands with valid rows

  // The tile's scales and bias, one per thread: BM of rows, BN (twice) of columns.  Requested here and passed round in LDS when that is free, so that
  // no wave waits for memory between the last product and the first result.  (Bias loaded behind the K loop: 1000 x 1024 x 1024 with GELU 7.6 us instead
  // of 7.2, 8192 x 1024 x 4096 SwiGLU 87 instead of 84.  The residual of small tiles, requested in front of K, was no gain and costs registers.)
  static_assert(BM + BN * (DUAL ? 2 : 1) <= NT * 2 && BM <= NT, "two values per thread at most");
  const float* b_scale = g.b_scale + (size_t)e * g.N;
  const float* b2_scale = DUAL ? g.b2_scale + (size_t)e * g.N : b_scale;
  const float my_row = tid < BM ? g.a_scale[row_of_a(g, row0 + min(tid, mvalid - 1))] : 0.f;
  const float my_col = tid < BN ? b_scale[min(n0 + tid, g.N - 1)] : 0.f;
  const float my_col2 = DUAL && tid < BN ? b2_scale[min(n0 + tid, g.N - 1)] : 0.f;
  const ST *bias_p = reinterpret_cast<const ST*>(g.bias), *bias2_p = reinterpret_cast<const ST*>(g.bias2);
  const float my_bias = bias_p != nullptr && tid < BN ? to_f32(bias_p[min(n0 + tid, g.N - 1)]) : 0.f;
  const float my_bias2 = DUAL && bias2_p != nullptr && tid < BN ? to_f32(bias2_p[min(n0 + tid, g.N - 1)]) : 0.f;

  i32x4 acc[TM][TNN] = {}, acc2[DUAL ? TM : 1][DUAL ? TNN : 1] = {};

  // operands: of A the rows of this tile (by token: all of it), of B this expert's matrix
  const bool gather = GROUPED && g.src_of != nullptr;
  const rsrc_t ra = gather ? make_rsrc(g.A, (size_t)g.src_rows * K) : make_rsrc(g.A + (size_t)row0 * K, (size_t)mvalid * K);
  const size_t mat = (size_t)g.N * K;
  const rsrc_t rb = make_rsrc(g.B + e * mat, mat), rb2 = make_rsrc((DUAL ? g.B2 : g.B) + e * mat, mat);
  const int KT = K / TILE8_K, stages = (KT + 1) / 2;   // tiles of 64 K values, stages
  const int S0 = part * stages / n_parts, KS = (part + 1) * stages / n_parts;   // this block's
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
  auto load_b = [&](auto once, int q, int stage, int buf) {
    const int c = DUAL ? q / 2 : q;
    const bool first = !DUAL || q % 2 == 0;
    const unsigned off = 2 * stage + half < KT ? b_vo[c] + (unsigned)stage * (2 * TILE8_BYTES) : OUT_OF_RANGE;
    const unsigned to = smem_base + B_AT + buf + (first ? 0 : B_BYTES) + wbase + NT * 16 * c;
    if constexpr (decltype(once)::value != 0) load_to_lds16_nt(first ? rb : rb2, to, off);
    else load_to_lds16(first ? rb : rb2, to, off);
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
  static_assert(LA + LB < 64, "the wait counter");
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

  auto request = [&](auto once, int stage, int abuf, int bbuf) {
#pragma unroll
    for (int q = 0; q < LB; ++q) load_b(once, q, stage, bbuf);
#pragma unroll
    for (int q = 0; q < LA; ++q) load_a(q, stage, abuf);
  };
  constexpr int L = LA + LB;
  // s_waitcnt vmcnt(n) lgkmcnt(0): the n newest loads may be in flight, every read of LDS is done
#define MOE_WAIT8(n_) __builtin_amdgcn_s_waitcnt(((n_) & 15) | (((n_) >> 4) << 14) | 0x70)
  auto mainloop = [&](auto once, int bands) {
    if constexpr (DEPTH == 2) {
      int a0 = 0, a1 = A_BYTES, a2 = 2 * A_BYTES, b0 = 0, b1 = B_STAGE;
      request(once, S0, a0, b0);
      if (KS - S0 > 1) {
        request(once, S0 + 1, a1, b1);
        MOE_WAIT8(L);
      } else {
        MOE_WAIT8(0);
      }
      barrier();
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
          if constexpr (LOAD) MOE_WAIT8(LA);
          else MOE_WAIT8(0);
          barrier();
        }
        step(Const<1>{}, more, a1, b1, 0, [&](int r) {
          if constexpr (LOAD) {
#pragma unroll
            for (int q = 0; q < LB; ++q)
              if (q * TM / LB == r) load_b(once, q, S + 2, b0);   // (in the first half of the regions: 0.6 % slower)
          }
        }, bands);
        const int a = a0; a0 = a1; a1 = a2; a2 = a;
        const int b = b0; b0 = b1; b1 = b;
      };
      int S = S0;
#pragma unroll 1
      for (; S + 2 < KS; ++S) iteration(S, true, Const<1>{});
#pragma unroll 1
      for (; S < KS; ++S) iteration(S, S + 1 < KS, Const<0>{});
    } else {
      // Three stages of both, all requested ahead: where a compute unit has one or two small blocks, a stage's products are over long before
      // a load requested an iteration ago has landed.  Stage S + 3 goes where stage S was, in K step 1 of iteration S.  (Tiles of 64 x 128,
      // us, the pipeline above -> this one: 300 x 4096 x 4096 17.8 -> 13.1, 64 x 14336 x 4096 52 -> 33, 8192 x 2048 x 8192 188 -> 179.  Four and six
      // stages leave room for one block: 300 x 4096 x 4096 15.1 and 15.7, 8192 x 2048 x 8192 266 and 293.  128 x 128, three stages and
      // one block per compute unit: 300 x 4096 x 4096 19.1 -> 17.2, but 8192 x 2048 x 8192 146 -> 177.)
      static_assert(DEPTH == 3 && 2 * L < 64, "the wait counter");
#pragma unroll
      for (int q = 0; q < DEPTH; ++q)
        if (S0 + q < KS) request(once, S0 + q, q * A_BYTES, q * B_STAGE);
      auto wait_for = [&](int left) {   // all but `left` stages
        if (left >= 2) MOE_WAIT8(2 * L);
        else if (left == 1) MOE_WAIT8(L);
        else MOE_WAIT8(0);
      };
      wait_for(min(KS - S0, DEPTH) - 1);
      barrier();
#pragma unroll
      for (int i = 0; i < TM; ++i) frag_a(i, 0, 0);
#pragma unroll
      for (int j = 0; j < TNN; ++j) frag_b(0, j, 0, 0);
      __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0)
      int at = 0;   // which stage of LDS is multiplied
      auto iteration = [&](int S, bool more, auto load) {
        constexpr bool LOAD = decltype(load)::value != 0;
        const int next = at + 1 == DEPTH ? 0 : at + 1;
        step(Const<0>{}, true, at * A_BYTES, at * B_STAGE, 1, [&](int) {}, bands);
        if (more) {
          if constexpr (LOAD) MOE_WAIT8((DEPTH - 2) * L);
          else wait_for(KS - 2 - S);
          barrier();
        }
        step(Const<1>{}, more, next * A_BYTES, next * B_STAGE, 0, [&](int r) {
          if constexpr (LOAD) {
#pragma unroll
            for (int q = 0; q < L; ++q)
              if (q * TM / L == r) {
                if (q < LB) load_b(once, q, S + DEPTH, at * B_STAGE);
                else load_a(q - LB, S + DEPTH, at * A_BYTES);
              }
          }
        }, bands);
        at = next;
      };
      int S = S0;
#pragma unroll 1
      for (; S + DEPTH < KS; ++S) iteration(S, true, Const<1>{});
#pragma unroll 1
      for (; S < KS; ++S) iteration(S, S + 1 < KS, Const<0>{});
    }
  };
#undef MOE_WAIT8
  if constexpr (STREAM) {
    // weights that one row tile takes, of more than the caches hold (Gemm8Args.stream).  (Chosen at each load, the wave's branches cost the K
    // loop a quarter: 128 x 4096 x 4096 11.9 -> 15.6 us.)
    if (GROUPED ? __builtin_amdgcn_readfirstlane(t.mates) == 0 : n_rt == 1) mainloop(Const<1>{}, ni);
    else mainloop(Const<0>{}, ni);
  } else {
    if (ni == WTM) mainloop(Const<0>{}, WTM);
    else mainloop(Const<0>{}, ni);
  }

  if (!GROUPED && n_parts > 1) {   // 32-bit sums of this K part, whole lines
    constexpr int CW = TNN * 16;
    if (n0 + wn * CW >= g.N) return;
    auto put = [&](i32x4 (&s)[TM][TNN], int matrix) {
      int32_t* out = g.parts + ((size_t)(part * (DUAL ? 2 : 1) + matrix) * g.M + row0) * g.N + n0 + wn * CW;
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TNN; j += 2) {
          u32x4 v[2] = {__builtin_bit_cast(u32x4, s[i][j]), __builtin_bit_cast(u32x4, s[i][j + 1])};
          swap8(v[0], v[1]);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int m = ((i >> 1) * WGM + wm) * 32 + (i & 1) * 16 + h * 8 + (lane & 7);
            if (m < mvalid) *reinterpret_cast<u32x4*>(out + (size_t)m * g.N + j * 16 + ((lane >> 3) & 1) * 16 + (lane >> 4) * 4) = v[h];
          }
        }
    };
    put(acc, 0);
    if constexpr (DUAL) put(acc2, 1);
    return;
  }

  // Epilogue.  The scales round LDS, act(z) in the accumulators' layout, then exchanges between lanes to whole lines (gemm_bf16_kernel.h).
  float* s_row = reinterpret_cast<float*>(smem);
  float *s_col = s_row + BM, *s_bias = s_col + BN * (DUAL ? 2 : 1);
  barrier();   // every wave has read its last fragments
  if (tid < BM) s_row[tid] = my_row;
  if (tid < BN) {
    s_col[tid] = my_col;
    s_bias[tid] = my_bias;
    if constexpr (DUAL) { s_col[BN + tid] = my_col2; s_bias[BN + tid] = my_bias2; }
  }
  __syncthreads();
  constexpr int C = TNN * 16;
  const int col_w = n0 + wn * C;
  if (col_w >= g.N) return;
  const int grp = lane >> 4, r8 = lane & 7, right = (lane >> 3) & 1;
  const size_t first = (size_t)row0 * g.N + n0, bytes = ((size_t)mvalid * g.N - n0) * sizeof(ST);
  const __amdgpu_buffer_rsrc_t oy = out_rsrc(reinterpret_cast<ST*>(g.C) + first, bytes);
  const unsigned pitch = (unsigned)g.N * sizeof(ST);
  auto band_row = [&](int i) { return ((i >> 1) * WGM + wm) * 32 + (i & 1) * 16; };
  f32x4 sw[TNN], sw2[DUAL ? TNN : 1], bias[TNN], bias2[DUAL ? TNN : 1];
#pragma unroll
  for (int j = 0; j < TNN; ++j) {
    const int c = wn * C + j * 16 + grp * 4;
    sw[j] = *reinterpret_cast<const f32x4*>(s_col + c);
    bias[j] = *reinterpret_cast<const f32x4*>(s_bias + c);
    if constexpr (DUAL) { sw2[j] = *reinterpret_cast<const f32x4*>(s_col + BN + c); bias2[j] = *reinterpret_cast<const f32x4*>(s_bias + BN + c); }
  }
  auto finish = [&](int i, f32x4 (&y)[TNN]) {
    const float sx = s_row[band_row(i) + (lane & 15)];
#pragma unroll
    for (int j = 0; j < TNN; ++j)
      y[j] = finish8<ST, ACT>(acc[i][j], acc2[DUAL ? i : 0][DUAL ? j : 0], sx, sw[j], sw2[DUAL ? j : 0], bias[j], bias2[DUAL ? j : 0]);
  };
  // where the lane's piece h of row tile i lies: eight columns (16 bits) or four (fp32) of a row
  constexpr int PIECES = __is_same(ST, float) ? TNN : TNN / 2;
  auto at = [&](int i, int h) {
    int m, c;
    if constexpr (__is_same(ST, float)) { m = (h & 1) * 8 + r8; c = (h >> 1) * 32 + right * 16 + grp * 4; }
    else if constexpr (TNN == 4) { m = h * 8 + r8; c = right * 32 + lane_col8(grp); }
    else { m = lane & 15; c = h * 32 + lane_col8(grp); }
    m += band_row(i);
    return m < mvalid ? (unsigned)m * pitch + (unsigned)(wn * C + c) * (unsigned)sizeof(ST) : OUT_OF_RANGE;
  };
  // half lines are written through: the neighbouring wave has the other half
  constexpr int AUX = !__is_same(ST, float) && TNN == 2 ? AUX_WT : AUX_NT;
  if (g.residual == nullptr) {
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      if (band_row(i) >= mvalid) continue;
      f32x4 y[TNN];
      finish(i, y);
      if constexpr (__is_same(ST, float)) {
#pragma unroll
        for (int j = 0; j < TNN; j += 2) {
          swap8(y[j], y[j + 1]);
#pragma unroll
          for (int h = 0; h < 2; ++h) buf_store16<AUX>(oy, at(i, j + h), __builtin_bit_cast(u32x4, y[j + h]));
        }
      } else {
        typedef Half16<ST> H;
        u32x4 v[TNN / 2];
#pragma unroll
        for (int h = 0; h < TNN / 2; ++h) {
          u32x2 c[2];
#pragma unroll
          for (int q = 0; q < 2; ++q) c[q] = u32x2{H::pack2(y[2 * h + q][0], y[2 * h + q][1]), H::pack2(y[2 * h + q][2], y[2 * h + q][3])};
          v[h] = join_tiles(c[0], c[1]);
        }
        if constexpr (TNN == 4) swap8(v[0], v[1]);
#pragma unroll
        for (int h = 0; h < TNN / 2; ++h) buf_store16<AUX>(oy, at(i, h), v[h]);
      }
    }
    return;
  }
  // With a residual the exchanges are made in fp32, and it is requested AHEAD row tiles ahead.
  constexpr int AHEAD = TM < 3 ? TM : 3;
  const __amdgpu_buffer_rsrc_t res = out_rsrc(reinterpret_cast<const ST*>(g.residual) + first, bytes);
  u32x4 rv[AHEAD][PIECES];
  auto load_res = [&](int i) {
#pragma unroll
    for (int h = 0; h < PIECES; ++h) rv[i % AHEAD][h] = buf_load16_nt(res, at(i, h));
  };
#pragma unroll
  for (int i = 0; i < AHEAD - 1; ++i) load_res(i);
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    if (i + AHEAD - 1 < TM) load_res(i + AHEAD - 1);
    if (band_row(i) >= mvalid) continue;
    f32x4 y[TNN];
    finish(i, y);
    if constexpr (__is_same(ST, float)) {
#pragma unroll
      for (int j = 0; j < TNN; j += 2) {
        swap8(y[j], y[j + 1]);
#pragma unroll
        for (int h = 0; h < 2; ++h) buf_store16<AUX>(oy, at(i, j + h), __builtin_bit_cast(u32x4, y[j + h] + __builtin_bit_cast(f32x4, rv[i % AHEAD][j + h])));
      }
    } else {
      typedef Half16<ST> H;
#pragma unroll
      for (int j = 0; j < TNN; j += 2) join_tiles(y[j], y[j + 1]);   // a lane: eight adjacent columns of 32
      if constexpr (TNN == 4) { swap8(y[0], y[2]); swap8(y[1], y[3]); }
#pragma unroll
      for (int h = 0; h < PIECES; ++h) {
        const u32x4 r = rv[i % AHEAD][h];
        u32x4 o;
#pragma unroll
        for (int q = 0; q < 4; ++q)
          o[q] = H::pack2(y[2 * h + q / 2][q % 2 * 2] + H::lo(r[q]), y[2 * h + q / 2][q % 2 * 2 + 1] + H::hi(r[q]));
        buf_store16<AUX>(oy, at(i, h), o);
      }
    }
  }
}

// ---- few rows ----
// A block of eight waves takes strips of 16 columns (NS = 2: pairs of them) and a group of 16 MT rows: 8 / nk strips, the K range of each shared
// out among nk waves, 128 values at a time in turn, whose sums are added in LDS, in any order the same: they are integers.  An operand of B is
// one contiguous 1 KB load of a wave, of A 16 rows x 64 bytes that all strips read from the caches, the other half of whose lines is the next one;
// the next U of either are requested before the last are used.  (64 values at a time: 16 x 14336 x 4096 16.1 us from memory instead of 14.9,
// 32 of them 22.1 instead of 19.7, 32 tokens x 2 of 8 experts, d 4096, f 14336, 224 instead of 218.  Two in flight instead of four: 1 x 14336 x
// 4096 12.1 -> 13.1 and 32 tokens x 8 of 128 experts 93 -> 95; eight: worse.)
// Bound by the read of the weights, with more than eight rows also by that of A, which takes a lookup for every row: 1 x 4096 x 14336 of two
// matrices 18.4 us, 6.4 TB/s with a part in the caches, 22.8 (5.1) from memory, 16 rows 19.2 and 25.2; 4 tokens x 2 of 8 experts 160 us, 6.6 TB/s.
// A pair of strips shares what is read of A, but leaves half as many blocks: worth it with two tiles of rows from 8192 columns on (from memory, one
// strip | two: 17 x 8192 x 8192 18.8 | 15.3, 32 24.2 | 18.2, 32 x 4096 x 14336 of two matrices 33.1 | 27.5, 32 x 8192 x 28672 77.8 | 61.5,
// 32 x 2048 x 8192 of two 10.8 | 10.7; 32 x 4096 x 4096 7.9 | 10.0; one tile of rows: 16 x 8192 x 8192 16.8 | 15.4, but 8 14.5 | 15.0).
// QUANT: A is rows of the storage type, which every block quantises into LDS for itself while its first weights are on their way (rows.h:
// the codes and scales that moe_quant_rows gives).
// Experts: blockIdx.y is the n-th group of 16 MT rows of some expert, which every block finds for itself from the experts' row counts.
constexpr int FEW_WAVES = 8;
constexpr int FEW_PAIRS = 512;   // strips from which a wave takes two
static_assert(16 * (FEW_QUANT_MAX + 16) + FEW_WAVES * 1024 < 64 * 1024, "LDS of a launch without an attribute");

template <typename ST, int ACT, int MT, int NS, bool STREAM, bool GROUPED, bool QUANT>
__global__ __launch_bounds__(FEW_WAVES * 64) void few8_kernel(Gemm8Args g) {
  constexpr bool DUAL = ACT == MOE_ACT_SWIGLU;
  constexpr int MATS = DUAL ? 2 : 1, ROWS = 16 * MT, U = MT == 1 ? 4 : 2;
  __shared__ __align__(16) i32x4 s_sum[FEW_WAVES][MATS * MT][64];
  __shared__ int s_tile[3], s_scan[FEW_WAVES];
  extern __shared__ __attribute__((aligned(16))) char smem[];   // QUANT: the rows' codes
  __shared__ float s_scale[ROWS];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int e = 0, row0 = blockIdx.y * ROWS, rows = min(ROWS, g.M - row0);
  if constexpr (GROUPED) {
    static_assert(MOE_MAX_E <= FEW_WAVES * 64, "a thread per expert");
    int l = 0, h = 0, at = 0;
    if (tid < g.E) {
      at = g.offsets[tid];
      share_of(g.lo, g.hi, g.kept[tid], tid, l, h);
    }
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
      s_tile[1] = at + l + q * ROWS;
      s_tile[2] = min(ROWS, h - l - q * ROWS);
    }
    __syncthreads();
    e = __builtin_amdgcn_readfirstlane(s_tile[0]);
    if (e < 0) return;
    row0 = __builtin_amdgcn_readfirstlane(s_tile[1]);
    rows = __builtin_amdgcn_readfirstlane(s_tile[2]);
  }
  const int nk = g.few_nk, strips = FEW_WAVES / nk, kw = wave % nk;   // this wave's part of K
  const int K = g.K, KT = K / TILE8_K, n0 = (blockIdx.x * strips + wave / nk) * NS * TILE8_N;
  const bool has = n0 < g.N;   // (the last block may have fewer strips)
  const int k1 = has ? KT : 0;
  const size_t strip = ((size_t)e * g.N + n0) * K + lane * 16;
  const int8_t *pb = g.B + strip, *pb2 = DUAL ? g.B2 + strip : pb;
  const int8_t* pa[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
    pa[i] = g.A + (size_t)row_of_a(g, row0 + min(i * 16 + (lane & 15), rows - 1)) * K + (lane >> 4) * 16;   // (rows past the group repeat its last)
  i32x4 acc[NS][MATS][MT] = {};
  const char* la = smem + (QUANT ? min(lane & 15, rows - 1) * (K + 16) + (lane >> 4) * 16 : 0);
  struct Operands { i32x4 b[U][NS][MATS], a[U][QUANT ? 1 : MT]; };
  auto weights = [](const int8_t* p) {
    if constexpr (STREAM) return __builtin_nontemporal_load(reinterpret_cast<const i32x4*>(p));
    else return *reinterpret_cast<const i32x4*>(p);
  };
  // tiles k, k + nk, ... of this wave, U of them; past the end the last one again, which is then not used
  auto fetch = [&](int k, Operands& o) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const size_t at = (size_t)min(k + (u >> 1) * 2 * nk + (u & 1), k1 - 1);
#pragma unroll
      for (int n = 0; n < NS; ++n) {
        o.b[u][n][0] = weights(pb + ((size_t)n * KT + at) * TILE8_BYTES);
        if constexpr (DUAL) o.b[u][n][1] = weights(pb2 + ((size_t)n * KT + at) * TILE8_BYTES);
      }
      if constexpr (!QUANT) {
#pragma unroll
        for (int i = 0; i < MT; ++i) o.a[u][i] = *reinterpret_cast<const i32x4*>(pa[i] + at * TILE8_K);
      }
    }
  };
  auto use = [&](int k, const Operands& o) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int kt = k + (u >> 1) * 2 * nk + (u & 1);
      if (kt >= k1) break;
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        i32x4 a;
        if constexpr (QUANT) a = *reinterpret_cast<const i32x4*>(la + kt * TILE8_K);
        else a = o.a[u][i];
#pragma unroll
        for (int n = 0; n < NS; ++n)
#pragma unroll
          for (int q = 0; q < MATS; ++q) acc[n][q][i] = mfma8(o.b[u][n][q], a, acc[n][q][i]);
      }
    }
  };
  int k = 2 * kw;
  Operands x, y;
  if constexpr (QUANT) {
    // a wave takes two rows; they are requested before the first weights, whose latency their codes hide in
    constexpr int RPW = ROWS / FEW_WAVES, NCH = FEW_QUANT_MAX / (8 * WAVE);
    Raw8<ST> raw[RPW][NCH];
#pragma unroll
    for (int r = 0; r < RPW; ++r)
#pragma unroll
      for (int i = 0; i < NCH; ++i)
        raw[r][i] = load_row8<ST, false, false>(reinterpret_cast<const ST*>(g.A) + (size_t)(row0 + min(wave + r * FEW_WAVES, rows - 1)) * K, (i * WAVE + lane) * 8, K);
    if (k < k1) fetch(k, x);
#pragma unroll
    for (int r = 0; r < RPW; ++r) {
      const int m = wave + r * FEW_WAVES;
      float v[NCH][8];
      unsigned top = 0;
#pragma unroll
      for (int i = 0; i < NCH; ++i) {
        unpack8<ST>(raw[r][i], v[i]);
        top = top_of(top, v[i]);
      }
      if (m >= rows) break;
      const RowScale q = row_scale(wave_reduce(top, max_u));
      if (lane == 0) s_scale[m] = q.scale;
#pragma unroll
      for (int i = 0; i < NCH; ++i)
        if ((i * WAVE + lane) * 8 < K) *reinterpret_cast<any_u32x2*>(smem + m * (K + 16) + (i * WAVE + lane) * 8) = codes8(v[i], q.up);
    }
    __syncthreads();
  }
  if (k < k1) {
    if constexpr (!QUANT) fetch(k, x);
    for (;;) {
      const int k2 = k + U * nk;
      if (k2 < k1) fetch(k2, y);
      use(k, x);
      if (k2 >= k1) break;
      k = k2 + U * nk;
      if (k < k1) fetch(k, x);
      use(k2, y);
      if (k >= k1) break;
    }
  }
#pragma unroll
  for (int n = 0; n < NS; ++n) {
    if (n > 0) __syncthreads();
#pragma unroll
    for (int q = 0; q < MATS; ++q)
#pragma unroll
      for (int i = 0; i < MT; ++i) s_sum[wave][q * MT + i][lane] = acc[n][q][i];
    __syncthreads();
    // the strips' MT row tiles of 16 go round the waves
    for (int j = wave; j < strips * MT; j += FEW_WAVES) {
      const int st = j / MT, i = j % MT, m = i * 16 + (lane & 15), c = ((blockIdx.x * strips + st) * NS + n) * TILE8_N + (lane >> 4) * 4;
      if (m >= rows || c >= g.N) continue;
      i32x4 sum[MATS];
#pragma unroll
      for (int q = 0; q < MATS; ++q) {
        sum[q] = s_sum[st * nk][q * MT + i][lane];
        for (int w = 1; w < nk; ++w) sum[q] += s_sum[st * nk + w][q * MT + i][lane];
      }
      const size_t row = row0 + m;
      const size_t cs = (size_t)e * g.N + c;
      const f32x4 sw = *reinterpret_cast<const f32x4*>(g.b_scale + cs), sw2 = DUAL ? *reinterpret_cast<const f32x4*>(g.b2_scale + cs) : sw;
      const float sx = QUANT ? s_scale[m] : g.a_scale[row_of_a(g, (int)row)];
      f32x4 y = finish8<ST, ACT>(sum[0], sum[MATS - 1], sx, sw, sw2, load4<ST>(g.bias, c), load4<ST>(DUAL ? g.bias2 : nullptr, c));
      if (g.residual != nullptr) y += load4<ST>(g.residual, row * g.N + c);   // (not zeros: -0 would lose its sign)
      ST* out = reinterpret_cast<ST*>(g.C) + row * g.N + c;
      if constexpr (__is_same(ST, float)) *reinterpret_cast<f32x4*>(out) = y;
      else *reinterpret_cast<u32x2*>(out) = u32x2{Half16<ST>::pack2(y[0], y[1]), Half16<ST>::pack2(y[2], y[3])};
    }
  }
}

// Adds the K parts of a product cut so; a thread has four adjacent columns of a row.
template <typename ST, int ACT>
__global__ __launch_bounds__(256) void join8_kernel(Gemm8Args g) {
  constexpr int MATS = ACT == MOE_ACT_SWIGLU ? 2 : 1;
  const unsigned per_row = g.N / 4, i = blockIdx.x * 256 + threadIdx.x, row = i / per_row;
  const int c = (int)(i - row * per_row) * 4;
  if (row >= (unsigned)g.M) return;
  i32x4 sum[MATS] = {};
#pragma unroll
  for (int p = 0; p < MAX_PARTS8; ++p)
    if (p < g.n_parts)
#pragma unroll
      for (int q = 0; q < MATS; ++q) sum[q] += *reinterpret_cast<const i32x4*>(g.parts + ((size_t)(p * MATS + q) * g.M + row) * g.N + c);
  const f32x4 sw = *reinterpret_cast<const f32x4*>(g.b_scale + c), sw2 = MATS > 1 ? *reinterpret_cast<const f32x4*>(g.b2_scale + c) : sw;
  f32x4 y = finish8<ST, ACT>(sum[0], sum[MATS - 1], g.a_scale[row], sw, sw2, load4<ST>(g.bias, c), load4<ST>(MATS > 1 ? g.bias2 : nullptr, c));
  const size_t at = (size_t)row * g.N + c;
  if (g.residual != nullptr) y += load4<ST>(g.residual, at);
  ST* out = reinterpret_cast<ST*>(g.C) + at;
  if constexpr (__is_same(ST, float)) *reinterpret_cast<f32x4*>(out) = y;
  else *reinterpret_cast<u32x2*>(out) = u32x2{Half16<ST>::pack2(y[0], y[1]), Half16<ST>::pack2(y[2], y[3])};
}

// ---- launches ----
template <typename ST, int ACT, int BM, int BN, int WGM, int WGN, int PER_CU, int DEPTH, bool STREAM, bool GROUPED>
static int gemm8_run(const Gemm8Args& g, long long row_tiles, hipStream_t s) {
  constexpr int LDS = gemm8_lds_bytes<BM, BN, ACT == MOE_ACT_SWIGLU, DEPTH>();
  static_assert(LDS * PER_CU <= LDS_BYTES, "blocks that a compute unit holds");
  const void* fn = reinterpret_cast<const void*>(gemm8_kernel<ST, ACT, BM, BN, WGM, WGN, PER_CU, DEPTH, STREAM, GROUPED>);
  if (LDS > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
    if (e != hipSuccess) return set_hip_error(e);
  }
  const long long grid = row_tiles * ((g.N + BN - 1) / BN) * (GROUPED ? 1 : g.n_parts);
  gemm8_kernel<ST, ACT, BM, BN, WGM, WGN, PER_CU, DEPTH, STREAM, GROUPED><<<(unsigned)grid, WGM * WGN * 64, LDS, s>>>(g);
  if (!GROUPED && g.n_parts > 1) join8_kernel<ST, ACT><<<(unsigned)(((size_t)g.M * (g.N / 4) + 255) / 256), 256, 0, s>>>(g);
  return launch_status();
}
template <typename ST, int ACT, int BM, int BN, int WGM, int WGN, int PER_CU, int DEPTH, bool GROUPED>
static int gemm8_launch(const Gemm8Args& g, long long row_tiles, hipStream_t s) {
  if constexpr (BM < 256)
    if (g.stream) return gemm8_run<ST, ACT, BM, BN, WGM, WGN, PER_CU, DEPTH, true, GROUPED>(g, row_tiles, s);
  return gemm8_run<ST, ACT, BM, BN, WGM, WGN, PER_CU, DEPTH, false, GROUPED>(g, row_tiles, s);
}
template <typename ST, int ACT, int MT, int NS, bool STREAM, bool GROUPED, bool QUANT>
static int few8_run(const Gemm8Args& g, int groups, hipStream_t s) {
  const int strips = FEW_WAVES / g.few_nk * NS;
  few8_kernel<ST, ACT, MT, NS, STREAM, GROUPED, QUANT>
      <<<dim3((g.N / TILE8_N + strips - 1) / strips, groups), FEW_WAVES * 64, QUANT ? 16 * MT * (g.K + 16) : 0, s>>>(g);
  return launch_status();
}
template <typename ST, int ACT, int MT, int NS, bool GROUPED, bool QUANT = false>
static int few8_launch(const Gemm8Args& g, int groups, hipStream_t s) {
  return g.stream ? few8_run<ST, ACT, MT, NS, true, GROUPED, QUANT>(g, groups, s) : few8_run<ST, ACT, MT, NS, false, GROUPED, QUANT>(g, groups, s);
}
template <typename ST, int ACT, bool GROUPED>
static int gemm8_act(const Gemm8Args& g, const Cut8& c, int max_tiles, hipStream_t s) {
  constexpr int D = ACT == MOE_ACT_SWIGLU ? 2 : 1;   // columns are of both matrices together
  if (c.few) {
    if constexpr (GROUPED && ACT == MOE_ACT_NONE)
      if (g.quantise) return few8_launch<ST, ACT, 1, 1, true, true>(g, max_tiles, s);
    if constexpr (GROUPED) return few8_launch<ST, ACT, 1, 1, true>(g, max_tiles, s);
    else if (c.rows == 16) return few8_launch<ST, ACT, 1, 1, false>(g, 1, s);
    else return g.N / TILE8_N >= FEW_PAIRS ? few8_launch<ST, ACT, 2, 2, false>(g, 1, s) : few8_launch<ST, ACT, 2, 1, false>(g, 1, s);
  }
  const long long rt = GROUPED ? max_tiles : (g.M + c.rows - 1) / c.rows;
  // two matrices: four waves down, so that a wave has 64 columns of either and writes whole lines (fp32 has them with 32)
  if (c.rows == 256 && c.cols * D == 256) {
    constexpr int DOWN = __is_same(ST, float) ? 2 : 2 * D;
    return gemm8_launch<ST, ACT, 256, 256 / D, DOWN, 8 / DOWN, 1, 2, GROUPED>(g, rt, s);
  }
  if (c.rows == 256) return gemm8_launch<ST, ACT, 256, 128 / D, 4, 2, 1, 2, GROUPED>(g, rt, s);
  if constexpr (!GROUPED) {
    if (c.rows == 128 && c.per_cu == 1) return gemm8_launch<ST, ACT, 128, 128 / D, 2 * D, 4 / D, 1, 3, GROUPED>(g, rt, s);
  }
  if (c.rows == 128) return gemm8_launch<ST, ACT, 128, 128 / D, 2, 2, 2, 2, GROUPED>(g, rt, s);
  return gemm8_launch<ST, ACT, 64, 128 / D, 2, 2, 2, 3, GROUPED>(g, rt, s);
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
