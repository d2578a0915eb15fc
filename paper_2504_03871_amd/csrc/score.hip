// Scored routing: from gate logits to experts and weights by softmax or sigmoid scores, with a bias that takes part in the
// choice only, groups of experts, and weights renormalised and scaled; and the gradient of the logits.
//
//   s = softmax(l) or sigmoid(l);  c = s + b;  a group's score = its best c, or the sum of its two best;  the top_groups best
//   groups (equal scores: lower group), in them the k best c (equal: lower expert);  w_j = scale s_j / (renorm ? sum_i s_i : 1)
//   p_j = w_j / scale, D = sum_i p_i dw_i:
//     renorm, softmax  dl_j = scale p_j (dw_j - D)               renorm, sigmoid  dl_j = scale p_j (1 - s_j) (dw_j - D)
//     sigmoid          dl_j = scale s_j (1 - s_j) dw_j           softmax          dl_e = scale s_e ([e chosen] dw_e - D), every e
//
// Sixteen lanes own a token (four tokens per wave): lane i holds the V = 2^n experts from i V on, so that the lowest lane and
// the lowest slot of equal keys is the lowest expert, and a maximum over the token is four steps within a row of 16 lanes.
#include "common.h"
#include <type_traits>

namespace moe {

typedef float f32x4 __attribute__((ext_vector_type(4)));
constexpr int SC_LANES = 16, SC_ROWS = 256 / SC_LANES;   // lanes per token, tokens per block

struct ScoreArgs {
  const float* logits;
  const float* balance;    // may be NULL
  int32_t* topk_idx;
  float* topk_w;
  int T, E, k;
  int softmax, groups, top_groups, rank, renorm;
  int group_lanes;         // lanes that hold a group, where that is a power of two and no lane holds two groups; else 0
  float scale;
};

// ---- reductions over the 16 lanes of a token; every lane gets the result ----
template <int N> __device__ __forceinline__ float row_ror(float v) {
  return __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), 0x120 + N, 0xf, 0xf, true));
}
__device__ __forceinline__ float row_max(float v) {
  v = fmaxf(v, row_ror<1>(v));
  v = fmaxf(v, row_ror<2>(v));
  v = fmaxf(v, row_ror<4>(v));
  return fmaxf(v, row_ror<8>(v));
}
__device__ __forceinline__ float row_sum(float v) {
  v += row_ror<1>(v);
  v += row_ror<2>(v);
  v += row_ror<4>(v);
  return v + row_ror<8>(v);
}
// the token's 16 bits of a wave-wide vote
__device__ __forceinline__ unsigned row_vote(bool b) {
  return (unsigned)(__ballot(b) >> (threadIdx.x & (WAVE - SC_LANES))) & 0xffffu;
}

// LDS that one wave writes and reads: in order, once the compiler keeps the order
__device__ __forceinline__ void wave_lds_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// A logit or a bias that takes part: minus infinity and NaN do not, plus infinity counts as the largest number (so that sums of two
// keys are numbers or minus infinity).
__device__ __forceinline__ float usable(float l) { return l > -INFINITY ? fminf(l, 3.4028234663852886e38f) : -INFINITY; }

// lane i's V values of a row of E, `rest` past its end
template <int V>
__device__ __forceinline__ void load_row(const float* __restrict__ row, int E, int lane, float rest, float (&l)[V]) {
  const int e0 = lane * V;
  if (V >= 4 && (E & 3) == 0) {
    float4 q[V < 4 ? 1 : V / 4];
#pragma unroll
    for (int v = 0; v < V; v += 4) q[v / 4] = *reinterpret_cast<const float4*>(row + min(e0 + v, E - 4));
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const float4 p = q[v / 4];
      l[v] = e0 + v < E ? (v % 4 == 0 ? p.x : v % 4 == 1 ? p.y : v % 4 == 2 ? p.z : p.w) : rest;
    }
  } else {
#pragma unroll
    for (int v = 0; v < V; ++v) l[v] = row[min(e0 + v, E - 1)];
#pragma unroll
    for (int v = 0; v < V; ++v) l[v] = e0 + v < E ? l[v] : rest;
  }
}

// ---- the choice, in single precision ----
// Keys c (-inf: cannot be chosen) and what they are made of: the largest score plus the largest bias.  BY_LOGIT: the scores
// grow with the logits and nothing is added to them, so the logits themselves are the keys, exact ones (0 is returned); minus
// zero, which equals zero, becomes it.
template <int V, bool BY_LOGIT>
__device__ __forceinline__ float make_keys(const ScoreArgs& a, const float (&l)[V], float row_top, int lane, float (&key)[V]) {
  if constexpr (BY_LOGIT) {
#pragma unroll
    for (int v = 0; v < V; ++v) key[v] = l[v] + 0.f;
    return 0.f;
  } else {
    float b[V], top_s = 0.f, top_b = 0.f;
    if (a.balance != nullptr) load_row<V>(a.balance, a.E, lane, 0.f, b);
    if (a.softmax) {
      float z = 0.f;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        key[v] = l[v] > -INFINITY ? __expf(l[v] - row_top) : 0.f;
        z += key[v];
      }
      z = row_sum(z);
      const float inv = z > 0.f ? __builtin_amdgcn_rcpf(z) : 0.f;
#pragma unroll
      for (int v = 0; v < V; ++v) key[v] *= inv;
    } else {
#pragma unroll
      for (int v = 0; v < V; ++v) key[v] = __builtin_amdgcn_rcpf(1.f + __expf(-l[v]));   // 0 for minus infinity
    }
#pragma unroll
    for (int v = 0; v < V; ++v) top_s = fmaxf(top_s, key[v]);
    if (a.balance != nullptr) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const bool open = b[v] > -INFINITY;   // usable(), with one selection for both
        const float u = fminf(b[v], 3.4028234663852886e38f);
        top_b = fmaxf(top_b, open ? fabsf(u) : 0.f);
        key[v] = l[v] > -INFINITY && open ? key[v] + u : -INFINITY;
      }
    } else {
#pragma unroll
      for (int v = 0; v < V; ++v) key[v] = l[v] > -INFINITY ? key[v] : -INFINITY;
    }
    return row_max(top_s) + row_max(top_b);
  }
}

// the best two of (b >= n) and (ob >= on)
template <typename F>
__device__ __forceinline__ void merge_two(F& b, F& n, F ob, F on) {
  const F lo = b < ob ? b : ob, hi = b < ob ? ob : b, m = n < on ? on : n;
  n = lo < m ? m : lo;
  b = hi;
}
template <int CTRL> __device__ __forceinline__ float dpp_of(float v) {
  return __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xf, 0xf, true));
}
// merges over runs of 2^steps adjacent lanes; each step pairs runs whose lanes already agree, so that mirrors serve as well
__device__ __forceinline__ void merge_lanes(float& b, float& n, int lanes) {
  if (lanes > 1) merge_two(b, n, dpp_of<0xB1>(b), dpp_of<0xB1>(n));      // lane ^ 1
  if (lanes > 2) merge_two(b, n, dpp_of<0x4E>(b), dpp_of<0x4E>(n));      // lane ^ 2
  if (lanes > 4) merge_two(b, n, dpp_of<0x141>(b), dpp_of<0x141>(n));    // halves of eight mirrored
  if (lanes > 8) merge_two(b, n, dpp_of<0x140>(b), dpp_of<0x140>(n));    // the row mirrored
}

// the larger of two numbers that are none of them NaN, in one instruction (fmaxf first makes sure of that)
__device__ __forceinline__ float larger(float a, float b) { return __builtin_amdgcn_fmed3f(a, b, INFINITY); }
// how many of the 15 other lanes hold a larger value
template <int R> __device__ __forceinline__ int lanes_above(float g) {
  if constexpr (R < SC_LANES) return (row_ror<R>(g) > g ? 1 : 0) + lanes_above<R + 1>(g);
  else return 0;
}

// Groups: closes the keys outside the top_groups best.  Returns whether it is not certain which these are: the scores of the last
// group that is in and the first that is out lie within `unit` of each other.
// Where a group is a run of 2^n whole lanes (a.group_lanes), its lanes find its best two together; else lane g reads group g's keys
// from LDS.
template <int V>
__device__ __forceinline__ bool restrict_groups(const ScoreArgs& a, float (&key)[V], int lane, float* keys_lds, float unit) {
  const int size = a.E / a.groups, e0 = lane * V;
  const int lanes = a.group_lanes > 0 ? a.group_lanes : 1;
  float g = -INFINITY, best = -INFINITY, next = -INFINITY;
  if (a.group_lanes > 0) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      next = __builtin_amdgcn_fmed3f(best, next, key[v]);   // best >= next: the middle one is the new second
      best = larger(best, key[v]);
    }
    merge_lanes(best, next, a.group_lanes);
  } else {
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (e0 + v < a.E) keys_lds[e0 + v] = key[v];
    wave_lds_sync();
    if (lane < a.groups)
      for (int i = 0; i < size; ++i) {
        const float c = keys_lds[lane * size + i];
        next = __builtin_amdgcn_fmed3f(best, next, c);
        best = larger(best, c);
      }
    wave_lds_sync();
  }
  const bool holds = lane < a.groups * lanes;   // the lane holds a group's score, with the other lanes of the group
  if (holds) g = a.rank == 2 ? best + next : best;
  const bool in = holds && lanes_above<1>(g) < a.top_groups * lanes;
  const unsigned who = row_vote(in);
  const float worst_in = -row_max(in ? -g : -INFINITY), best_out = row_max(in || !holds ? -INFINITY : g);
  if (a.group_lanes > 0) {
#pragma unroll
    for (int v = 0; v < V; ++v) key[v] = in ? key[v] : -INFINITY;
  } else {
    int grp = e0 / size, left = size - e0 % size;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if (!((who >> (grp & 31)) & 1u)) key[v] = -INFINITY;
      if (--left == 0) { ++grp; left = size; }
    }
  }
  // equal scores at the border let too many in
  return __builtin_popcount(who) != a.top_groups * lanes || (best_out > -INFINITY && !(worst_in - best_out > unit));
}

// The k + 1 largest keys, best first, to pick_e in LDS (-1: none left), and what is not certain about them: ORDER, keys within `unit`
// of each other among them; ALL, more than them.  Exact keys (BY_LOGIT) have an order that is certain unless they agree but for the
// bits that the slot takes: what lies far from the choice, a mask of -1e9 say, does not widen a bound.  (32768 tokens, 8 of 256, a
// twentieth masked so: 11 us; by a bound from the largest logit, under which every token was uncertain, 43.  All logits equal: 42.)
// Every lane keeps the best DEPTH of its keys in order, with the slot in place of the lowest bits, so that taking the
// token's best is a step within its 16 lanes and a shift in one of them.  (Going through all V keys per choice: 32768
// tokens, 8 of 256 experts in 8 groups, 77 us, with every uncertain token in double precision 43; as it is 24.)  A lane whose list runs out while
// it had more keys than the list holds also leaves ALL open.
enum { CERTAIN = 0, ORDER = 1, ALL = 2 };
// numbers in order as integers, and back
__device__ __forceinline__ int ordered(float f) { const int i = (int)__float_as_uint(f); return i ^ ((i >> 31) & 0x7fffffff); }
__device__ __forceinline__ float from_ordered(int i) { return __uint_as_float((unsigned)(i ^ ((i >> 31) & 0x7fffffff))); }
__device__ __forceinline__ int middle(int a, int b, int c) {
  int m;
  asm("v_med3_i32 %0, %1, %2, %3" : "=v"(m) : "v"(a), "v"(b), "v"(c));
  return m;
}
template <int N> __device__ __forceinline__ int row_ror(int v) { return __builtin_amdgcn_update_dpp(0, v, 0x120 + N, 0xf, 0xf, true); }
__device__ __forceinline__ int row_max(int v) {
  v = max(v, row_ror<1>(v));
  v = max(v, row_ror<2>(v));
  v = max(v, row_ror<4>(v));
  return max(v, row_ror<8>(v));
}
template <int V, bool BY_LOGIT>
__device__ __forceinline__ int pick_fast(const ScoreArgs& a, const float (&key)[V], int lane, float unit, int* pick_e) {
  constexpr int DEPTH = V < 8 ? V : 8;   // (six: 34.9 us with the gradient instead of 33.1; four: 51.6)
  constexpr int SLOT = V - 1, CLOSED = (int)0x80000000u;   // below any key
  int best[DEPTH];
#pragma unroll
  for (int q = 0; q < DEPTH; ++q) best[q] = CLOSED;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int i = (ordered(__builtin_amdgcn_fmed3f(key[v], -3.0e38f, 3.0e38f)) & ~SLOT) | v;
    const int x = key[v] > -INFINITY ? i : CLOSED;
#pragma unroll
    for (int q = DEPTH - 1; q > 0; --q) best[q] = middle(x, best[q - 1], best[q]);   // best[q - 1] >= best[q]
    best[0] = max(best[0], x);
  }
  bool order = false, edge = false;   // edge: of the last key that is chosen and the first that is not
  int last = CLOSED, taken = 0;
  float last_f = INFINITY;
  // whether the order of the last key and a key `top` that can be chosen is open (no key has the upper bits of CLOSED)
  auto near_last = [&](int top) { return BY_LOGIT ? (unsigned)(last ^ top) <= (unsigned)SLOT : !(last_f - from_ordered(top) > unit); };
  for (int j = 0; j <= a.k; ++j) {
    const int top = row_max(best[0]);
    edge = top != CLOSED && near_last(top);
    order |= edge;
    last = top;
    last_f = from_ordered(top);
    if (lane == __builtin_ctz(row_vote(best[0] == top))) {
      pick_e[j] = top != CLOSED ? lane * V + (top & SLOT) : -1;
      if (top != CLOSED) {
#pragma unroll
        for (int q = 0; q + 1 < DEPTH; ++q) best[q] = best[q + 1];
        best[DEPTH - 1] = CLOSED;
        ++taken;
      }
    }
  }
  const int top = row_max(best[0]);
  const bool beyond = edge && top != CLOSED && near_last(top);
  if (row_vote(beyond || (V > DEPTH && taken == DEPTH))) return ALL;
  return order ? ORDER : CERTAIN;
}

// Puts the k + 1 candidates in their exact order: lane j compares candidate j's key (logit, or sigmoid score plus bias in double
// precision) with the others'.
template <bool BY_LOGIT>
__device__ __forceinline__ void settle(const ScoreArgs& a, int lane, const float* logits, int* pick_e) {
  const int e = lane <= a.k ? pick_e[lane] : -1;
  double c = e >= 0 ? (double)logits[e] : (double)-INFINITY;
  if (!BY_LOGIT && e >= 0) c = 1.0 / (1.0 + exp(-c)) + (a.balance != nullptr ? (double)usable(a.balance[e]) : 0.0);
  int rank = 0;
  for (int i = 0; i <= a.k; ++i) {
    const double o = __shfl(c, i, SC_LANES);
    const int oe = __shfl(e, i, SC_LANES);
    rank += (oe >= 0 && (o > c || (o == c && oe < e))) ? 1 : 0;
  }
  wave_lds_sync();
  if (e >= 0) pick_e[rank] = e;
}

// ---- the choice, exactly ----
// One token by the whole wave, in double precision, whose scores decide; by the logits as they are where they order the experts.
template <int CTRL> __device__ __forceinline__ double dpp_of(double v) {
  const unsigned long long b = (unsigned long long)__double_as_longlong(v);
  const unsigned lo = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(unsigned)b, CTRL, 0xf, 0xf, true);
  const unsigned hi = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(unsigned)(b >> 32), CTRL, 0xf, 0xf, true);
  return __longlong_as_double((long long)(lo | (unsigned long long)hi << 32));
}
__device__ __forceinline__ double wave_max(double v) {   // (no NaN)
  auto up = [](double a, double b) { return a < b ? b : a; };
  v = up(v, dpp_of<0x121>(v));   // within rows of 16: rotations by 1, 2, 4, 8
  v = up(v, dpp_of<0x122>(v));
  v = up(v, dpp_of<0x124>(v));
  v = up(v, dpp_of<0x128>(v));
  v = up(v, __shfl_xor(v, 16, WAVE));
  return up(v, __shfl_xor(v, 32, WAVE));
}
template <int V, bool BY_LOGIT>
__device__ __forceinline__ void choose_exact(const ScoreArgs& a, int t, int* pick_e) {
  constexpr int VW = V < 4 ? 1 : V / 4;   // lane i holds the experts from i VW on
  const int lane = threadIdx.x & (WAVE - 1), e0 = lane * VW;
  const float* row = a.logits + (size_t)t * a.E;
  double key[VW];
  float l[VW];
#pragma unroll
  for (int v = 0; v < VW; ++v) {
    l[v] = e0 + v < a.E ? usable(row[e0 + v]) : -INFINITY;
    key[v] = l[v];
  }
  if constexpr (!BY_LOGIT) {
    if (a.softmax) {
      double top = -INFINITY, z = 0;
#pragma unroll
      for (int v = 0; v < VW; ++v) top = fmax(top, key[v]);
      top = wave_max(top);
#pragma unroll
      for (int v = 0; v < VW; ++v) {
        key[v] = l[v] > -INFINITY ? exp(key[v] - top) : 0.0;
        z += key[v];
        __builtin_amdgcn_sched_barrier(0);   // one after the other: together they take registers that the tokens' common path pays for
      }
#pragma unroll
      for (int s = 1; s < WAVE; s <<= 1) z += __shfl_xor(z, s, WAVE);
#pragma unroll
      for (int v = 0; v < VW; ++v) key[v] = z > 0 ? key[v] / z : 0.0;
    } else {
#pragma unroll
      for (int v = 0; v < VW; ++v) {
        key[v] = l[v] > -INFINITY ? 1.0 / (1.0 + exp(-key[v])) : 0.0;
        __builtin_amdgcn_sched_barrier(0);
      }
    }
#pragma unroll
    for (int v = 0; v < VW; ++v) {
      if (a.balance != nullptr && e0 + v < a.E) key[v] += (double)usable(a.balance[e0 + v]);
      key[v] = l[v] > -INFINITY ? key[v] : (double)-INFINITY;
    }
  }
  if (a.groups > 1) {
    const int size = a.E / a.groups;
    double g = -INFINITY;   // lane q: of group q
    const int run = size / VW;
    if (size % VW == 0 && (run & (run - 1)) == 0) {   // groups of 2^n whole lanes: all at once
      double best = -INFINITY, next = -INFINITY;
#pragma unroll
      for (int v = 0; v < VW; ++v) merge_two(best, next, key[v], (double)-INFINITY);
      for (int s = 1; s < run; s <<= 1) merge_two(best, next, __shfl_xor(best, s, WAVE), __shfl_xor(next, s, WAVE));
      const double sum = a.rank == 2 ? best + next : best;
      const double mine = __shfl(sum, min(lane * run, WAVE - 1), WAVE);
      if (lane < a.groups) g = mine;
    } else for (int q = 0; q < a.groups; ++q) {
      double best = -INFINITY, next = -INFINITY;
#pragma unroll
      for (int v = 0; v < VW; ++v)
        if (e0 + v >= q * size && e0 + v < (q + 1) * size) merge_two(best, next, key[v], (double)-INFINITY);
#pragma unroll
      for (int s = 1; s < WAVE; s <<= 1) merge_two(best, next, __shfl_xor(best, s, WAVE), __shfl_xor(next, s, WAVE));
      if (lane == q) g = a.rank == 2 ? best + next : best;
    }
    int ahead = 0;
    for (int j = 0; j < a.groups; ++j) {
      const double o = __shfl(g, j, WAVE);
      ahead += (o > g || (o == g && j < lane)) ? 1 : 0;
    }
    const unsigned long long in = __ballot(lane < a.groups && ahead < a.top_groups);
#pragma unroll
    for (int v = 0; v < VW; ++v)
      if (!((in >> ((e0 + v) / size & 63)) & 1)) key[v] = -INFINITY;
  }
  for (int j = 0; j < a.k; ++j) {
    double mine = key[0];
#pragma unroll
    for (int v = 1; v < VW; ++v) mine = fmax(mine, key[v]);
    const double top = wave_max(mine);
    const unsigned long long have = __ballot(mine == top);
    if (lane == __builtin_ctzll(have)) {
      int e = -1;
#pragma unroll
      for (int v = VW - 1; v >= 0; --v)
        if (key[v] == top) e = e0 + v;
      if (top > (double)-INFINITY) {
#pragma unroll
        for (int v = 0; v < VW; ++v)
          if (e == e0 + v) key[v] = -INFINITY;
      } else e = -1;
      pick_e[j] = e;
    }
  }
}

// Weight (without the scale) of the slot that lane j < k of a token holds; e < 0: an empty one.  z: the softmax's sum over all
// experts, of exp(l - row_top).  one_minus_s: 1 - sigmoid(l), for the gradient.
__device__ __forceinline__ float slot_weight(const ScoreArgs& a, bool live, float l, float row_top, float z, float& one_minus_s) {
  one_minus_s = 1.f;
  const float top = row_max(live ? l : -INFINITY);
  float s = 0.f;
  if (live) {
    if (a.softmax) s = a.renorm ? expf(l - top) : expf(l - row_top) / z;
    else {
      const float t = expf(-fabsf(l)), r = 1.f / (1.f + t);
      s = l >= 0.f ? r : t * r;
      one_minus_s = l >= 0.f ? t * r : r;
      if (a.renorm && top < -60.f) s = expf(l - top);   // all of them tiny: sigmoid(l) = exp(l) to 2^-86, and their ratios remain
    }
  }
  if (a.renorm) {
    const float sum = row_sum(s);
    if (live) s /= sum;
  }
  return s;
}

template <int V>
__device__ __forceinline__ float top_of(const float (&l)[V]) {
  float m = l[0];
#pragma unroll
  for (int v = 1; v < V; ++v) m = fmaxf(m, l[v]);
  return row_max(m);
}
// sum of exp(l - top) over the token's experts
template <int V>
__device__ __forceinline__ float softmax_sum(const float (&l)[V], float top) {
  float z = 0.f;
#pragma unroll
  for (int v = 0; v < V; ++v) z += l[v] > -INFINITY ? expf(l[v] - top) : 0.f;
  return row_sum(z);
}

// The choice.  Bound by its instructions (vector ALUs busy 95 % of the cycles), not by the one pass over the logits: 32768 tokens, 8 of 256 experts, four of eight groups,
// 23.8 us for 36 MB; 8191 tokens, 6 of 64, 4.3 us, and a call of four tokens 5.3, both the length of one wave's work.
template <int V, bool BY_LOGIT>
__global__ __launch_bounds__(256) void score_kernel(ScoreArgs a) {
  __shared__ float keys[SC_ROWS][SC_LANES * V];
  __shared__ int pick_e[SC_ROWS][MOE_MAX_K + 1];
  const int lane = threadIdx.x & (SC_LANES - 1), r = threadIdx.x / SC_LANES;
  const int t = blockIdx.x * SC_ROWS + r, tc = min(t, a.T - 1);   // tokens past the batch repeat the last one and write nothing
  float l[V];
  load_row<V>(a.logits + (size_t)tc * a.E, a.E, lane, -INFINITY, l);
#pragma unroll
  for (int v = 0; v < V; ++v) l[v] = usable(l[v]);
  const float top = top_of<V>(l);
  int open;
  {
    // What two keys must differ by for their order to be certain.  A score in single precision: the exponential's argument is
    // good to 2^-24 of itself, which x e^-x <= 0.37 turns into less than 2^-25 of the largest score; the exponential, the
    // sum and the reciprocal add 2^-22 at most, the bias 2^-24 of the key; twice, for two keys: 2^-20.8, 5.6e-7, of the largest
    // score and bias; for two sums of two, with their own roundings, three times that.  The slot's four bits change
    // a key by up to 15 steps of at most 2^-23 of it, two keys by 30: 4.2e-6 in all.  Next to zero steps stay as they are: a
    // sigmoid below 2^-126 may come out as zero, the slot's bits are 15 steps of 2^-149, which is below 2^-124 for two keys and
    // below 2^-122 for two sums of two.
    float key[V];
    const float most = make_keys<V, BY_LOGIT>(a, l, top, lane, key);
    const bool groups_open = a.groups > 1 && restrict_groups<V>(a, key, lane, keys[r], BY_LOGIT ? 0.f : fmaxf(1.7e-6f * most, 0x1p-122f));
    open = pick_fast<V, BY_LOGIT>(a, key, lane, fmaxf(4.2e-6f * most, 0x1p-124f), pick_e[r]);
    if (groups_open) open = ALL;
    if (!BY_LOGIT && open == ORDER && a.softmax) open = ALL;   // a softmax score takes the sum over all experts
  }
  // what the weights need of the logits, before the rare path below wants the registers
  const float z = a.softmax && !a.renorm ? softmax_sum<V>(l, top) : 1.f;
#pragma unroll
  for (int v = 0; v < V; ++v) keys[r][lane * V + v] = l[v];
  wave_lds_sync();
  if (__ballot(open == ORDER)) {
    if (open == ORDER) settle<BY_LOGIT>(a, lane, keys[r], pick_e[r]);
  }
  for (unsigned long long rows = __ballot(open == ALL && t < a.T); rows != 0;) {   // the rest, seldom, one token after the other
    const int of = __builtin_ctzll(rows) / SC_LANES;
    rows &= ~(0xffffull << (of * SC_LANES));
    const int first = (threadIdx.x / WAVE) * (WAVE / SC_LANES) + of;          // the token's place in the block
    wave_lds_sync();
    choose_exact<V, BY_LOGIT>(a, blockIdx.x * SC_ROWS + first, pick_e[first]);
  }
  wave_lds_sync();
  const int e = lane < a.k ? pick_e[r][lane] : -1;
  const float le = e >= 0 ? keys[r][e] : -INFINITY;
  float unused;
  const float w = slot_weight(a, e >= 0, le, top, z, unused);
  if (t < a.T && lane < a.k) {
    a.topk_idx[(size_t)t * a.k + lane] = e;
    a.topk_w[(size_t)t * a.k + lane] = w * a.scale;
  }
}

// Gradient of the logits.  The slots' gradients meet their experts in an LDS row, which leaves in pieces of 256 bytes.
// Bound by HBM: 32768 tokens, 8 of 256 experts, 33.6 MB written and 19 MB read (the chosen logits' lines), 8.3 us = 6.3 TB/s; over
// all experts, 8191 tokens of 64, 3.8 us.
template <int V>
__global__ __launch_bounds__(256) void score_bwd_kernel(ScoreArgs a, const float* __restrict__ d_topk_w, float* __restrict__ d_logits) {
  constexpr int P = V < 4 ? V : 4, N = V / P;   // lane i has N pieces of P experts, piece j from (16 j + i) P on
  __shared__ float grad[SC_ROWS][SC_LANES * V];
  const int lane = threadIdx.x & (SC_LANES - 1), r = threadIdx.x / SC_LANES;
  const int t = blockIdx.x * SC_ROWS + r, tc = min(t, a.T - 1);
  const bool dense = a.softmax && !a.renorm;   // the sum over all experts has a gradient too
  const bool whole = P == 4 && (a.E & 3) == 0;
  const float* row = a.logits + (size_t)tc * a.E;
  int e = lane < a.k ? a.topk_idx[(size_t)tc * a.k + lane] : -1;
  if (e >= a.E) e = -1;
  const float dw0 = lane < a.k ? d_topk_w[(size_t)tc * a.k + lane] : 0.f;
  float l[V], top = 0.f, z = 1.f;
  if (dense) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int c = (j * SC_LANES + lane) * P;
      if (whole) {
        float4 q = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
        if (c < a.E) q = *reinterpret_cast<const float4*>(row + c);
        if constexpr (P == 4) { l[j * P] = q.x; l[j * P + 1] = q.y; l[j * P + 2] = q.z; l[j * P + 3] = q.w; }
      } else {
#pragma unroll
        for (int p = 0; p < P; ++p) l[j * P + p] = c + p < a.E ? row[c + p] : -INFINITY;
      }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) l[v] = usable(l[v]);
    top = top_of<V>(l);
  }
#pragma unroll
  for (int j = 0; j < N; ++j)
#pragma unroll
    for (int p = 0; p < P; ++p) grad[r][(j * SC_LANES + lane) * P + p] = 0.f;
  const float le = e >= 0 ? usable(row[e]) : -INFINITY;
  if (dense) {
    z = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      l[v] = l[v] > -INFINITY ? expf(l[v] - top) : 0.f;   // from here on the exponentials
      z += l[v];
    }
    z = row_sum(z);
  }
  const bool live = le > -INFINITY;
  const float dw = live ? dw0 : 0.f;
  float one_minus_s;
  const float p = slot_weight(a, live, le, top, z, one_minus_s);
  const float D = row_sum(p * dw);
  wave_lds_sync();
  if (live) grad[r][e] = dense ? dw : a.scale * p * one_minus_s * (a.renorm ? dw - D : dw);
  wave_lds_sync();
  if (t >= a.T) return;
  float* out = d_logits + (size_t)t * a.E;
  const float f = dense ? (z > 0.f ? a.scale / z : 0.f) : 1.f;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int c = (j * SC_LANES + lane) * P;
    float o[P];
#pragma unroll
    for (int q = 0; q < P; ++q) {
      o[q] = grad[r][c + q];
      if (dense) o[q] = f * l[j * P + q] * (o[q] - D);
    }
    if (whole) {
      if constexpr (P == 4)
        if (c < a.E) *reinterpret_cast<float4*>(out + c) = make_float4(o[0], o[1], o[2], o[3]);
    } else {
#pragma unroll
      for (int q = 0; q < P; ++q)
        if (c + q < a.E) out[c + q] = o[q];
    }
  }
}

// dx += d_logits Wr^T, over the chosen experts: a wave per token adds up their rows of the weight's transpose [E][d].
// For gradients that only the chosen experts have; bound by those rows, which come from the L2s: 32768 tokens x 4096, 8 of
// 256 experts, 259 us: 4.3 GB of rows, 16.6 TB/s, and 0.5 GB of dx.
template <typename T>
__global__ __launch_bounds__(256) void score_dx_chosen_kernel(const float* __restrict__ d_logits, const int32_t* __restrict__ topk_idx,
                                                              const float* __restrict__ WrT, T* __restrict__ dx, int Tn, int d, int E, int k) {
  constexpr int VN = Vec16<T>::N, U = 4;   // 16-byte pieces of a row of dx per lane in flight
  const int lane = threadIdx.x & (WAVE - 1), t = (int)((blockIdx.x * blockDim.x + threadIdx.x) / WAVE);
  if (t >= Tn) return;
  float g[MOE_MAX_K];
  int at[MOE_MAX_K];
#pragma unroll
  for (int j = 0; j < MOE_MAX_K; ++j)
    if (j < k) {
      const int e = topk_idx[(size_t)t * k + j];
      const bool live = e >= 0 && e < E;
      at[j] = live ? e : 0;
      g[j] = live ? d_logits[(size_t)t * E + e] : 0.f;
    }
  T* row = dx + (size_t)t * d;
  for (int c0 = lane * VN; c0 < d; c0 += WAVE * VN * U) {
    Vec16<T> v[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (c0 + u * WAVE * VN < d) v[u].load_nt(row + c0 + u * WAVE * VN);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int c = c0 + u * WAVE * VN;
      if (c >= d) break;
      float sum[VN];
      v[u].unpack(sum);
#pragma unroll
      for (int j = 0; j < MOE_MAX_K; ++j)
        if (j < k) {
#pragma unroll
          for (int i = 0; i < VN; i += 4) {
            const f32x4 w = *reinterpret_cast<const f32x4*>(WrT + (size_t)at[j] * d + c + i);
#pragma unroll
            for (int q = 0; q < 4; ++q) sum[i + q] = fmaf(g[j], w[q], sum[i + q]);
          }
        }
      v[u].pack(sum);
      v[u].store_nt(row + c);
    }
  }
}

// The same over all experts, on the matrix cores in fp32: tokens as M, columns as N, experts as K.  A block: 32 tokens x 256 columns,
// a wave 32 x 64.  Of every 16 experts lane group g = lane / 16 supplies 4 g + s in step s, and lane c = lane % 16 holds columns
// 4 c .. 4 c + 3 as column tiles 0 .. 3: one 16-byte read of the gradients serves four steps, one of the weights four tiles, and the
// sums leave as four adjacent columns.  8192 tokens, 64 experts, d 1024 | 4096: 20 | 61 us with the transpose, of which dx itself is
// 6 | 24 at the rate of a copy; by multiply-adds, eight tokens x four columns per thread, 37 | 128.  Tokens past the batch and experts past E count with a gradient of zero.
constexpr int SDX_TOK = 32, SDX_COLS = 256;
template <typename T>
__global__ __launch_bounds__(256) void score_dx_all_kernel(const float* __restrict__ d_logits, const float* __restrict__ WrT, T* __restrict__ dx,
                                                           int Tn, int d, int E) {
  extern __shared__ __attribute__((aligned(16))) float dl[];   // [32][pitch]: sixteen rows' 16 bytes in different banks
  const int steps = (E + 15) / 16, pitch = steps * 16 + 4;
  const int t0 = blockIdx.x * SDX_TOK, lane = threadIdx.x & (WAVE - 1), c = lane & 15, grp = lane >> 4;
  for (int i = threadIdx.x; i < SDX_TOK * steps * 16; i += 256) {
    const int q = i / (steps * 16), e = i - q * (steps * 16);
    dl[q * pitch + e] = t0 + q < Tn && e < E ? d_logits[(size_t)(t0 + q) * E + e] : 0.f;
  }
  __syncthreads();
  const int col = blockIdx.y * SDX_COLS + threadIdx.x / WAVE * 64 + c * 4;
  const float* w = WrT + min(col, d - 4);   // columns past the row repeat its last four and are not stored
  f32x4 acc[2][4] = {};
  for (int q = 0; q < steps; ++q) {
    const f32x4 a0 = *reinterpret_cast<const f32x4*>(dl + c * pitch + q * 16 + grp * 4);
    const f32x4 a1 = *reinterpret_cast<const f32x4*>(dl + (16 + c) * pitch + q * 16 + grp * 4);
    f32x4 b[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) b[s] = *reinterpret_cast<const f32x4*>(w + (size_t)min(q * 16 + grp * 4 + s, E - 1) * d);
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        acc[0][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(a0[s], b[s][j], acc[0][j], 0, 0, 0);
        acc[1][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(a1[s], b[s][j], acc[1][j], 0, 0, 0);
      }
  }
  if (col >= d) return;
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int v = 0; v < 4; ++v) {   // register v of a lane: token 4 grp + v
      const int t = t0 + h * 16 + grp * 4 + v;
      if (t >= Tn) break;
      T* o = dx + (size_t)t * d + col;
      T was[4];
      __builtin_memcpy(was, o, sizeof was);
#pragma unroll
      for (int j = 0; j < 4; ++j) was[j] = from_f32<T>(to_f32(was[j]) + acc[h][j][v]);
      __builtin_memcpy(o, was, sizeof was);
    }
}

// logits = x Wr + bias for few tokens: a block takes all of d for 16 experts and up to TT tokens.  A thread has four adjacent experts
// and every 256th run of four rows of Wr, so that d is walked in d / 1024 steps; its sums meet in the wave, then in LDS, in order.
// Bound by the latency of those steps: one token, d 4096, 256 experts, 4.2 MB of weights, the call with the choice 10 us.
constexpr int SL_COLS = 16, SL_THREADS = 1024;
template <typename T, int TT>
__global__ __launch_bounds__(SL_THREADS) void score_logits_kernel(const T* __restrict__ x, const float* __restrict__ Wr,
                                                                  const float* __restrict__ bias, float* __restrict__ logits, int Tn, int d, int E) {
  constexpr int WAVES = SL_THREADS / WAVE;
  __shared__ float part[WAVES][4][TT * 4 + 1];
  const int g = threadIdx.x & 3, q = threadIdx.x >> 2, e = blockIdx.x * SL_COLS + g * 4, t0 = blockIdx.y * TT;
  f32x4 acc[TT] = {};
  if (e < E)
#pragma unroll 2
    for (int c = q * 4; c < d; c += SL_THREADS) {
      f32x4 w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = *reinterpret_cast<const f32x4*>(Wr + (size_t)(c + i) * E + e);
#pragma unroll
      for (int s = 0; s < TT; ++s) {
        T v[4];
        __builtin_memcpy(v, x + (size_t)min(t0 + s, Tn - 1) * d + c, sizeof v);   // tokens past the batch repeat the last one
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float f = to_f32(v[i]);
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[s][j] = fmaf(f, w[i][j], acc[s][j]);
        }
      }
    }
#pragma unroll
  for (int s = 0; s < TT; ++s)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float v = acc[s][j];
      for (int lanes = 4; lanes < WAVE; lanes <<= 1) v += __shfl_xor(v, lanes, WAVE);
      if ((threadIdx.x & (WAVE - 1)) < 4) part[threadIdx.x / WAVE][g][s * 4 + j] = v;
    }
  __syncthreads();
  const int s = threadIdx.x / SL_COLS, col = threadIdx.x % SL_COLS, to = blockIdx.x * SL_COLS + col;
  if (s >= TT || t0 + s >= Tn || to >= E) return;
  float sum = bias != nullptr ? bias[to] : 0.f;
  for (int w = 0; w < WAVES; ++w) sum += part[w][col >> 2][s * 4 + (col & 3)];
  logits[(size_t)(t0 + s) * E + to] = sum;
}

static int per_lane(int E) { return E <= 16 ? 1 : E <= 32 ? 2 : E <= 64 ? 4 : E <= 128 ? 8 : 16; }
static int group_lanes(int E, int groups) {
  const int size = E / groups, n = size / per_lane(E);
  return size % per_lane(E) == 0 && (n & (n - 1)) == 0 ? n : 0;
}
static ScoreArgs score_args(const moe_cfg* c, const moe_score* sc, const float* logits, const float* balance, int32_t* idx, float* w) {
  return ScoreArgs{logits, balance, idx, w, c->T, c->E, c->k, sc->score == MOE_SCORE_SOFTMAX, sc->groups, sc->top_groups, sc->group_rank,
                   sc->renorm != 0, group_lanes(c->E, sc->groups), sc->scale};
}

template <int V>
static int launch_score_v(const ScoreArgs& a, bool by_logit, hipStream_t s) {
  const unsigned grid = (unsigned)((a.T + SC_ROWS - 1) / SC_ROWS);
  if (by_logit) score_kernel<V, true><<<grid, 256, 0, s>>>(a);
  else score_kernel<V, false><<<grid, 256, 0, s>>>(a);
  return launch_status();
}
int launch_score(const moe_cfg* c, const moe_score* sc, const float* logits, const float* balance, int32_t* idx, float* w, hipStream_t s) {
  const ScoreArgs a = score_args(c, sc, logits, balance, idx, w);
  // Both scores grow with their logit: without a bias, and where no scores are added up, the logits decide
  const bool by_logit = balance == nullptr && (sc->groups == 1 || sc->group_rank == 1);
  switch (per_lane(c->E)) {
    case 1: return launch_score_v<1>(a, by_logit, s);
    case 2: return launch_score_v<2>(a, by_logit, s);
    case 4: return launch_score_v<4>(a, by_logit, s);
    case 8: return launch_score_v<8>(a, by_logit, s);
    default: return launch_score_v<16>(a, by_logit, s);
  }
}

int launch_score_bwd(const moe_cfg* c, const moe_score* sc, const float* logits, const int32_t* idx, const float* dw, float* d_logits, hipStream_t s) {
  const ScoreArgs a = score_args(c, sc, logits, nullptr, const_cast<int32_t*>(idx), nullptr);
  const unsigned grid = (unsigned)((a.T + SC_ROWS - 1) / SC_ROWS);
  switch (per_lane(c->E)) {
    case 1: score_bwd_kernel<1><<<grid, 256, 0, s>>>(a, dw, d_logits); break;
    case 2: score_bwd_kernel<2><<<grid, 256, 0, s>>>(a, dw, d_logits); break;
    case 4: score_bwd_kernel<4><<<grid, 256, 0, s>>>(a, dw, d_logits); break;
    case 8: score_bwd_kernel<8><<<grid, 256, 0, s>>>(a, dw, d_logits); break;
    default: score_bwd_kernel<16><<<grid, 256, 0, s>>>(a, dw, d_logits);
  }
  return launch_status();
}

template <typename T>
static int launch_score_dx_for(const moe_cfg* c, bool all, const int32_t* idx, const float* d_logits, const float* WrT, T* dx, hipStream_t s) {
  if (all) {
    const size_t lds = SDX_TOK * ((c->E + 15) / 16 * 16 + 4) * sizeof(float);   // 33 KB at most
    const dim3 grid((c->T + SDX_TOK - 1) / SDX_TOK, (c->d_model + SDX_COLS - 1) / SDX_COLS);
    score_dx_all_kernel<T><<<grid, 256, lds, s>>>(d_logits, WrT, dx, c->T, c->d_model, c->E);
  } else {
    score_dx_chosen_kernel<T><<<dim3((c->T + 3) / 4), 256, 0, s>>>(d_logits, idx, WrT, dx, c->T, c->d_model, c->E, c->k);
  }
  return launch_status();
}
int launch_score_dx(const moe_cfg* c, const moe_score* sc, const int32_t* idx, const float* d_logits, const float* WrT, void* dx, hipStream_t s) {
  // where only the chosen have one, their rows alone are faster at every ratio of E to k (T x d x E, k, us, chosen | all):
  // 8192 x 1024 x 8, 2 7 | 7; 8192 x 1024 x 64, 6 13 | 20; 8192 x 4096 x 128, 8 67 | 108; 32768 x 4096 x 256, 8 259 | 849
  const bool all = sc->score == MOE_SCORE_SOFTMAX && !sc->renorm;
  if (c->dtype == MOE_DTYPE_BF16) return launch_score_dx_for(c, all, idx, d_logits, WrT, (bf16*)dx, s);
  if (c->dtype == MOE_DTYPE_F16) return launch_score_dx_for(c, all, idx, d_logits, WrT, (f16*)dx, s);
  return launch_score_dx_for(c, all, idx, d_logits, WrT, (float*)dx, s);
}

template <typename T>
static int launch_score_logits_for(const moe_cfg* c, const T* x, const float* Wr, const float* bias, float* logits, hipStream_t s) {
  const int tt = c->T == 1 ? 1 : c->T <= 4 ? 4 : 8;
  const dim3 grid((c->E + SL_COLS - 1) / SL_COLS, (c->T + tt - 1) / tt);
  if (tt == 1) score_logits_kernel<T, 1><<<grid, SL_THREADS, 0, s>>>(x, Wr, bias, logits, c->T, c->d_model, c->E);
  else if (tt == 4) score_logits_kernel<T, 4><<<grid, SL_THREADS, 0, s>>>(x, Wr, bias, logits, c->T, c->d_model, c->E);
  else score_logits_kernel<T, 8><<<grid, SL_THREADS, 0, s>>>(x, Wr, bias, logits, c->T, c->d_model, c->E);
  return launch_status();
}
// Against moe_route's product (E > 32: a block per 16 or more tokens that walks all of d), the whole call, T x d x E, us, this | that:
// bf16 1 x 4096 x 256 10 | 73, 256 x 4096 x 256 35 | 82, 512 x 1024 x 64 14 | 19, 1024 x 1024 x 64 24 | 19, 512 x 1024 x 256 43 | 45;
// fp32 4 x 4096 x 64 12 | 149, 1024 x 1024 x 256 76 | 95, 2048 x 1024 x 256 144 | 98; up to 32 experts (another kernel there)
// 4 x 4096 x 32 12 | 15, 16 x 4096 x 32 17 | 16, 64 x 1024 x 8 13 | 11.
bool score_logits_few(const moe_cfg* c) {
  const bool f32 = c->dtype == MOE_DTYPE_F32;
  return c->E % 4 == 0 && (c->T <= 4 || (c->E > 32 && (long long)c->T * c->E <= (f32 ? 1 << 18 : 1 << 16) && (f32 || c->T <= 512)));
}
int launch_score_logits(const moe_cfg* c, const void* x, const float* Wr, const float* bias, float* logits, hipStream_t s) {
  if (c->dtype == MOE_DTYPE_BF16) return launch_score_logits_for(c, (const bf16*)x, Wr, bias, logits, s);
  if (c->dtype == MOE_DTYPE_F16) return launch_score_logits_for(c, (const f16*)x, Wr, bias, logits, s);
  return launch_score_logits_for(c, (const float*)x, Wr, bias, logits, s);
}

}  // namespace moe
