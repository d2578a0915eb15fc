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

namespace moe {

constexpr int SC_LANES = 16, SC_ROWS = 256 / SC_LANES;   // lanes per token, tokens per block

struct ScoreArgs {
  const float* logits;
  const float* balance;    // may be NULL
  int32_t* topk_idx;
  float* topk_w;
  int T, E, k;
  int softmax, groups, top_groups, rank, renorm;
  float scale;
};

// ---- reductions over the 16 lanes of a token; every lane gets the result ----
template <int N> __device__ __forceinline__ float row_ror(float v) {
  return __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), 0x120 + N, 0xf, 0xf, false));
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
__device__ __forceinline__ double row_max(double v) {
#pragma unroll
  for (int s = 1; s < SC_LANES; s <<= 1) v = fmax(v, __shfl_xor(v, s, SC_LANES));
  return v;
}
__device__ __forceinline__ double row_sum(double v) {
#pragma unroll
  for (int s = 1; s < SC_LANES; s <<= 1) v += __shfl_xor(v, s, SC_LANES);
  return v;
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

// A logit that takes part: minus infinity and NaN do not, plus infinity counts as the largest number.
__device__ __forceinline__ float usable(float l) { return l > -INFINITY ? fminf(l, 3.4028234663852886e38f) : -INFINITY; }

__device__ __forceinline__ float score_exp(float v) { return __expf(v); }
__device__ __forceinline__ double score_exp(double v) { return exp(v); }
__device__ __forceinline__ float score_sigmoid(float l) { return __builtin_amdgcn_rcpf(1.f + __expf(-l)); }
__device__ __forceinline__ double score_sigmoid(double l) { return 1.0 / (1.0 + exp(-l)); }

// The token's choice in arithmetic F: chosen experts and their logits to pick_e, pick_l [k] in LDS (-1: none left).  BY_LOGIT:
// the scores grow with the logits and nothing is added to them, so the logits themselves are the keys.
// Returns whether two keys (or the scores of two groups) that decide lie closer together than F resolves.
template <typename F, int V, bool BY_LOGIT>
__device__ __forceinline__ bool choose(const ScoreArgs& a, const float (&l)[V], float row_top, int lane, F* keys_lds, int* pick_e, float* pick_l) {
  F key[V], top_s = 0, top_b = 0;
  const int e0 = lane * V;
  if constexpr (BY_LOGIT) {
#pragma unroll
    for (int v = 0; v < V; ++v) key[v] = (F)l[v];
  } else {
    F inv = 1;
    if (a.softmax) {
      F z = 0;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        key[v] = l[v] > -INFINITY ? score_exp((F)l[v] - (F)row_top) : (F)0;
        z += key[v];
      }
      z = row_sum(z);
      inv = z > 0 ? 1 / z : (F)0;
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const F s = a.softmax ? key[v] * inv : l[v] > -INFINITY ? score_sigmoid((F)l[v]) : (F)0;
      const F b = a.balance != nullptr && e0 + v < a.E ? (F)a.balance[e0 + v] : (F)0;
      const F c = s + b;
      top_s = s > top_s ? s : top_s;
      const F mag = b < 0 ? -b : b;
      if (mag < (F)INFINITY && mag > top_b) top_b = mag;
      key[v] = (l[v] > -INFINITY && c > (F)-INFINITY) ? c : (F)-INFINITY;
    }
    top_s = row_max(top_s);
    top_b = row_max(top_b);
  }
  // What two keys must differ by for their order to be certain.  Single precision: the exponential's argument is good to
  // 2^-24 of itself, which x e^-x <= 0.37 turns into less than 2^-24 of the largest score, exponential, reciprocal and sum add a
  // few units in the last place, the bias one: 2^-21 of the largest magnitudes together, for either key, with room.
  const F unit = sizeof(F) == 4 ? (F)1.9073486328125e-6 * (top_s + top_b) : (F)0;   // 2^-19
  bool close = false;

  if (a.groups > 1) {
    const int size = a.E / a.groups;
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (e0 + v < a.E) keys_lds[e0 + v] = key[v];
    wave_lds_sync();
    F best = (F)-INFINITY, next = (F)-INFINITY;
    if (lane < a.groups)
      for (int i = 0; i < size; ++i) {
        const F c = keys_lds[lane * size + i];
        if (c > best) { next = best; best = c; } else if (c > next) next = c;
      }
    wave_lds_sync();
    const F g = lane >= a.groups ? (F)-INFINITY : a.rank == 2 ? best + next : best;
    int ahead = 0;
#pragma unroll
    for (int j = 0; j < SC_LANES; ++j) {
      const F o = __shfl(g, j, SC_LANES);
      ahead += (o > g || (o == g && j < lane)) ? 1 : 0;
    }
    const bool in = lane < a.groups && ahead < a.top_groups;
    const unsigned allowed = row_vote(in);
    if constexpr (!BY_LOGIT) {
      const F worst_in = -row_max(in ? -g : (F)-INFINITY), best_out = row_max(in ? (F)-INFINITY : g);
      if (best_out > (F)-INFINITY && !(worst_in - best_out > 2 * unit)) close = true;
    }
    int grp = e0 / size, left = size - e0 % size;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if (!((allowed >> (grp & 31)) & 1u)) key[v] = (F)-INFINITY;
      if (--left == 0) { ++grp; left = size; }
    }
  }

  F last = (F)INFINITY;
  for (int j = 0; j <= a.k; ++j) {   // one more than is chosen: the first that is not
    F mine = key[0];
#pragma unroll
    for (int v = 1; v < V; ++v) mine = key[v] > mine ? key[v] : mine;
    const F top = row_max(mine);
    if constexpr (!BY_LOGIT) { if (j > 0 && top > (F)-INFINITY && !(last - top > unit)) close = true; }
    last = top;
    if (j == a.k) break;
    const unsigned have = row_vote(mine == top);
    if (top > (F)-INFINITY) {
      if (lane == __builtin_ctz(have)) {
        bool done = false;
#pragma unroll
        for (int v = 0; v < V; ++v)
          if (!done && key[v] == top) {
            done = true;
            key[v] = (F)-INFINITY;
            pick_e[j] = e0 + v;
            pick_l[j] = l[v];
          }
      }
    } else if (lane == 0) {
      pick_e[j] = -1;
      pick_l[j] = -INFINITY;
    }
  }
  wave_lds_sync();
  return close;
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

// lane i's V logits of token t
template <int V>
__device__ __forceinline__ void load_logits(const ScoreArgs& a, int t, int lane, float (&l)[V]) {
  const float* row = a.logits + (size_t)t * a.E;
  const int e0 = lane * V;
  if (V >= 4 && (a.E & 3) == 0) {
#pragma unroll
    for (int v = 0; v < V; v += 4) {
      float4 q = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
      if (e0 + v < a.E) q = *reinterpret_cast<const float4*>(row + e0 + v);
      l[v] = q.x;
      if constexpr (V >= 4) { l[v + 1] = q.y; l[v + 2] = q.z; l[v + 3] = q.w; }
    }
  } else {
#pragma unroll
    for (int v = 0; v < V; ++v) l[v] = e0 + v < a.E ? row[e0 + v] : -INFINITY;
  }
#pragma unroll
  for (int v = 0; v < V; ++v) l[v] = usable(l[v]);
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

template <int V, bool BY_LOGIT>
__global__ __launch_bounds__(256) void score_kernel(ScoreArgs a) {
  __shared__ double keys[SC_ROWS][SC_LANES * V];   // by the pass in single precision as floats
  __shared__ int pick_e[SC_ROWS][MOE_MAX_K];
  __shared__ float pick_l[SC_ROWS][MOE_MAX_K];
  const int lane = threadIdx.x & (SC_LANES - 1), r = threadIdx.x / SC_LANES;
  const int t = blockIdx.x * SC_ROWS + r;
  const bool row = t < a.T;
  float l[V];
  load_logits<V>(a, min(t, a.T - 1), lane, l);   // tokens past the batch repeat the last one and write nothing
  const float top = top_of<V>(l);
  const bool close = choose<float, V, BY_LOGIT>(a, l, top, lane, reinterpret_cast<float*>(keys[r]), pick_e[r], pick_l[r]);
  if constexpr (!BY_LOGIT) {
    // Keys that lie closer together than single precision tells apart are ordered in double precision.
    if (__ballot(close)) choose<double, V, BY_LOGIT>(a, l, top, lane, keys[r], pick_e[r], pick_l[r]);
  }
  const int e = lane < a.k ? pick_e[r][lane] : -1;
  const float le = lane < a.k ? pick_l[r][lane] : -INFINITY;
  const float z = a.softmax && !a.renorm ? softmax_sum<V>(l, top) : 1.f;
  float unused;
  const float w = slot_weight(a, e >= 0, le, top, z, unused);
  if (row && lane < a.k) {
    a.topk_idx[(size_t)t * a.k + lane] = e;
    a.topk_w[(size_t)t * a.k + lane] = w * a.scale;
  }
}

// Gradient of the logits.  The slots' gradients meet their experts in an LDS row, which leaves as whole lines.
template <int V>
__global__ __launch_bounds__(256) void score_bwd_kernel(ScoreArgs a, const float* __restrict__ d_topk_w, float* __restrict__ d_logits) {
  __shared__ float grad[SC_ROWS][SC_LANES * V];
  const int lane = threadIdx.x & (SC_LANES - 1), r = threadIdx.x / SC_LANES;
  const int t = blockIdx.x * SC_ROWS + r, tc = min(t, a.T - 1);
  const bool dense = a.softmax && !a.renorm;   // the sum over all experts has a gradient too
  float l[V], top = 0.f, z = 1.f;
  if (dense) {
    load_logits<V>(a, tc, lane, l);
    top = top_of<V>(l);
    z = softmax_sum<V>(l, top);
  }
#pragma unroll
  for (int v = 0; v < V; ++v) grad[r][lane * V + v] = 0.f;
  int e = lane < a.k ? a.topk_idx[(size_t)tc * a.k + lane] : -1;
  if (e >= a.E) e = -1;
  const float le = e >= 0 ? usable(a.logits[(size_t)tc * a.E + e]) : -INFINITY;
  const bool live = le > -INFINITY;
  const float dw = live ? d_topk_w[(size_t)tc * a.k + lane] : 0.f;
  float one_minus_s;
  const float p = slot_weight(a, live, le, top, z, one_minus_s);
  const float D = row_sum(p * dw);
  wave_lds_sync();
  if (live) grad[r][e] = dense ? dw : a.scale * p * one_minus_s * (a.renorm ? dw - D : dw);
  wave_lds_sync();
  if (t >= a.T) return;
  float* out = d_logits + (size_t)t * a.E;
  const int e0 = lane * V;
  float o[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    o[v] = grad[r][e0 + v];
    if (dense) o[v] = l[v] > -INFINITY ? a.scale * (expf(l[v] - top) / z) * (o[v] - D) : 0.f;
  }
  if (V >= 4 && (a.E & 3) == 0) {
#pragma unroll
    for (int v = 0; v < V; v += 4)
      if constexpr (V >= 4)
        if (e0 + v < a.E) *reinterpret_cast<float4*>(out + e0 + v) = make_float4(o[v], o[v + 1], o[v + 2], o[v + 3]);
  } else {
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (e0 + v < a.E) out[e0 + v] = o[v];
  }
}

// dx += d_logits Wr^T.  A block owns SDX_TOK tokens and 256 4-column groups; the weight's transpose [E][d] is read once per
// block, for the experts that any of the tokens has a gradient for.
constexpr int SDX_TOK = 8;
template <typename T>
__global__ __launch_bounds__(256) void score_dx_kernel(const float* __restrict__ d_logits, const float* __restrict__ WrT, T* __restrict__ dx,
                                                       int Tn, int d, int E) {
  __shared__ float dl[MOE_MAX_E][SDX_TOK];
  const int t0 = blockIdx.x * SDX_TOK;
  for (int i = threadIdx.x; i < E * SDX_TOK; i += 256) {
    const int e = i % E, q = i / E;
    dl[e][q] = t0 + q < Tn ? d_logits[(size_t)(t0 + q) * E + e] : 0.f;
  }
  __syncthreads();
  for (int c = threadIdx.x * 4; c < d; c += 1024) {
    float acc[SDX_TOK][4] = {};
    for (int e = 0; e < E; ++e) {
      float g[SDX_TOK];
      bool any = false;
#pragma unroll
      for (int q = 0; q < SDX_TOK; ++q) { g[q] = dl[e][q]; any |= g[q] != 0.f; }
      if (!any) continue;
      const float4 w = *reinterpret_cast<const float4*>(WrT + (size_t)e * d + c);
#pragma unroll
      for (int q = 0; q < SDX_TOK; ++q) {
        acc[q][0] = fmaf(g[q], w.x, acc[q][0]);
        acc[q][1] = fmaf(g[q], w.y, acc[q][1]);
        acc[q][2] = fmaf(g[q], w.z, acc[q][2]);
        acc[q][3] = fmaf(g[q], w.w, acc[q][3]);
      }
    }
#pragma unroll
    for (int q = 0; q < SDX_TOK; ++q)
      if (t0 + q < Tn) {
        T* o = dx + (size_t)(t0 + q) * d + c;
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = from_f32<T>(to_f32(o[i]) + acc[q][i]);
      }
  }
}

static ScoreArgs score_args(const moe_cfg* c, const moe_score* sc, const float* logits, const float* balance, int32_t* idx, float* w) {
  return ScoreArgs{logits, balance, idx, w, c->T, c->E, c->k, sc->score == MOE_SCORE_SOFTMAX, sc->groups, sc->top_groups, sc->group_rank,
                   sc->renorm != 0, sc->scale};
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
  if (c->E <= 16) return launch_score_v<1>(a, by_logit, s);
  if (c->E <= 32) return launch_score_v<2>(a, by_logit, s);
  if (c->E <= 64) return launch_score_v<4>(a, by_logit, s);
  if (c->E <= 128) return launch_score_v<8>(a, by_logit, s);
  return launch_score_v<16>(a, by_logit, s);
}

int launch_score_bwd(const moe_cfg* c, const moe_score* sc, const float* logits, const int32_t* idx, const float* dw, float* d_logits, hipStream_t s) {
  const ScoreArgs a = score_args(c, sc, logits, nullptr, const_cast<int32_t*>(idx), nullptr);
  const unsigned grid = (unsigned)((a.T + SC_ROWS - 1) / SC_ROWS);
  if (c->E <= 16) score_bwd_kernel<1><<<grid, 256, 0, s>>>(a, dw, d_logits);
  else if (c->E <= 32) score_bwd_kernel<2><<<grid, 256, 0, s>>>(a, dw, d_logits);
  else if (c->E <= 64) score_bwd_kernel<4><<<grid, 256, 0, s>>>(a, dw, d_logits);
  else if (c->E <= 128) score_bwd_kernel<8><<<grid, 256, 0, s>>>(a, dw, d_logits);
  else score_bwd_kernel<16><<<grid, 256, 0, s>>>(a, dw, d_logits);
  return launch_status();
}

int launch_score_dx(const moe_cfg* c, const float* d_logits, const float* WrT, void* dx, hipStream_t s) {
  const unsigned grid = (unsigned)((c->T + SDX_TOK - 1) / SDX_TOK);
  if (c->dtype == MOE_DTYPE_BF16) score_dx_kernel<bf16><<<grid, 256, 0, s>>>(d_logits, WrT, (bf16*)dx, c->T, c->d_model, c->E);
  else if (c->dtype == MOE_DTYPE_F16) score_dx_kernel<f16><<<grid, 256, 0, s>>>(d_logits, WrT, (f16*)dx, c->T, c->d_model, c->E);
  else score_dx_kernel<float><<<grid, 256, 0, s>>>(d_logits, WrT, (float*)dx, c->T, c->d_model, c->E);
  return launch_status();
}

}  // namespace moe
