// smoe_route_scores: top-k routing from softmax or sigmoid scores, with a bias that takes part in the choice only and a
// choice of groups before the choice of experts.
//
// Scores, sums and comparisons are binary64: a bias of 0.01 decides between scores that lie 1e-3 apart, and two scores
// that are equal in binary32 need not be equal.  One wave per token; lane l holds the experts l, l + 64, ...  Bound: the
// latency of the picks (k reductions over the wave, one after the other) and the binary64 exponentials, not the logits'
// bytes.
#include "route_device.hpp"

struct ScoreArgs {
  RouteArgs r;
  int score, n_group, topk_group, group_score, group_size;
};

#define SC_WAVES 4

// Monotone map double -> uint64; NaN below every number, 0 left for "not to be chosen".
__device__ __forceinline__ uint64_t orderable64(double v) {
  if (v != v) return 1u;
  if (v == 0.0) v = 0.0;
  const uint64_t u = (uint64_t)__double_as_longlong(v);
  return (u >> 63) ? ~u : (u | 0x8000000000000000ull);
}

__device__ __forceinline__ double readlane_f64(double v, int l) {
  const uint64_t u = (uint64_t)__double_as_longlong(v);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)u, l), hi = (uint32_t)__builtin_amdgcn_readlane((int)(u >> 32), l);
  return __longlong_as_double((long long)(((uint64_t)hi << 32) | lo));
}

template <int CTRL> __device__ __forceinline__ double dpp_f64(double v) {
  const uint64_t u = (uint64_t)__double_as_longlong(v);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, 0xF, 0xF, true);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(u >> 32), CTRL, 0xF, 0xF, true);
  return __longlong_as_double((long long)(((uint64_t)hi << 32) | lo));
}

__device__ __forceinline__ double wave_sum64(double v) {
  v += dpp_f64<0xB1>(v);
  v += dpp_f64<0x4E>(v);
  v += dpp_f64<0x124>(v);
  v += dpp_f64<0x128>(v);
  return (readlane_f64(v, 0) + readlane_f64(v, 16)) + (readlane_f64(v, 32) + readlane_f64(v, 48));
}

// One token by one wave.  z: its logits; lds: E doubles of this wave's own (used with more than one group).
template <int NJ>
__device__ __forceinline__ void select_scores_wave(const ScoreArgs& a, int t, const float* z, int lane, double* lds) {
  const int E = a.r.E;
  float zv[NJ];
  double s[NJ];
#pragma unroll
  for (int j = 0; j < NJ; j++) zv[j] = lane + 64 * j < E ? z[lane + 64 * j] : -INFINITY;
  if (a.score == SMOE_SCORE_SIGMOID) {
#pragma unroll
    for (int j = 0; j < NJ; j++) s[j] = 1.0 / (1.0 + exp(-(double)zv[j]));
  } else {
    uint32_t zmax = 0;
#pragma unroll
    for (int j = 0; j < NJ; j++) { const uint32_t o = zv[j] != zv[j] ? 0u : orderable(zv[j]); zmax = o > zmax ? o : zmax; }
    const float m = unorderable(wave_umax(zmax));
    double den = 0.0;
#pragma unroll
    for (int j = 0; j < NJ; j++) {
      // equal to the largest (also where that is infinite): 1; minus infinity: 0; NaN passes through exp
      s[j] = zv[j] == -INFINITY ? 0.0 : zv[j] == m ? 1.0 : exp((double)zv[j] - (double)m);
      den += s[j];
    }
    den = wave_sum64(den);
#pragma unroll
    for (int j = 0; j < NJ; j++) s[j] = den == 0.0 ? 0.0 : s[j] / den;
  }
  uint64_t ord[NJ];
#pragma unroll
  for (int j = 0; j < NJ; j++) {
    const int e = lane + 64 * j;
    const double sel = e < E && a.r.bias ? s[j] + (double)a.r.bias[e] : s[j];
    ord[j] = e < E ? orderable64(sel) : 0u;
    if (a.n_group > 1 && e < E) lds[e] = sel == sel ? sel : -INFINITY;
  }
  if (a.n_group > 1) {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    // lane g: score of group g; the lanes begin at different places of their groups, so that they read different banks
    double b0 = -INFINITY, b1 = -INFINITY;
    const int gs = a.group_size;
    if (lane < a.n_group) {
      int at = lane % gs;
      for (int i = 0; i < gs; i++) {
        const double v = lds[lane * gs + at];
        at = at + 1 == gs ? 0 : at + 1;
        if (v > b0) { b1 = b0; b0 = v; } else if (v > b1) b1 = v;
      }
    }
    const uint64_t mine = orderable64(a.group_score == SMOE_GROUP_TOP2 && gs > 1 ? b0 + b1 : b0);
    int rank = 0;
    for (int g = 0; g < a.n_group; g++) {
      const uint64_t o = ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(mine >> 32), g) << 32) | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)mine, g);
      rank += o > mine || (o == mine && g < lane);
    }
    const uint64_t in = __ballot(lane < a.n_group && rank < a.topk_group);
#pragma unroll
    for (int j = 0; j < NJ; j++) {
      const int e = lane + 64 * j;
      if (e < E && !((in >> (e / gs)) & 1u)) ord[j] = 0u;
    }
  }
  double wsum = 0.0, myw = 0.0;
  int mysel = 0;
  for (int r = 0; r < a.r.k; r++) {
    uint64_t best = ord[0];
    double sb = s[0];
    int jb = 0;
#pragma unroll
    for (int j = 1; j < NJ; j++) if (ord[j] > best) { best = ord[j]; sb = s[j]; jb = j; }
    const uint32_t hi = wave_umax((uint32_t)(best >> 32));
    uint64_t cand = __ballot((uint32_t)(best >> 32) == hi);
    if (cand & (cand - 1)) {                                  // several share the upper half
      const uint32_t lo = wave_umax((uint32_t)(best >> 32) == hi ? (uint32_t)best : 0u);
      cand = __ballot(best == (((uint64_t)hi << 32) | lo));
    }
    int ls = (int)__builtin_ctzll(cand);
    if (NJ > 1 && (cand & (cand - 1))) {                      // equal scores: the lowest index
      const uint32_t mine = (cand >> lane) & 1u ? (uint32_t)(lane + 64 * jb) : 0xFFFFFFFFu;
      ls = (int)(~wave_umax(~mine)) & 63;
    }
    const int js = __builtin_amdgcn_readlane(jb, ls);
    const double w = readlane_f64(sb, ls);
#pragma unroll
    for (int j = 0; j < NJ; j++) if (lane == ls && jb == j) ord[j] = 0u;
    wsum += w;
    if (lane == r) { mysel = ls + 64 * js; myw = w; }
  }
  if (lane < a.r.k) {
    const double w = a.r.norm_topk ? (wsum == 0.0 ? 0.0 : myw / wsum) : myw;
    a.r.idx[(size_t)t * a.r.k + lane] = mysel;
    a.r.w[(size_t)t * a.r.k + lane] = (float)(w * (double)a.r.routed_scale);
  }
}

// ---- short form, E = 64 NJ at most and groups that are whole lanes: lane l holds the NJ experts from NJ l on, everything is ordered by fp32 keys, and a
// token whose keys lie too close together to be sure of the binary64 order is left to select_scores_wave.
//   The key of an expert is its logit where the order of the scores is the logits' own (no bias; no sum of two scores), else the fp32 score
// plus bias.  A score is off by at most 5 half steps of 1 (of a sigmoid: argument of the exponential s (1 - s) |z| 1.5 < 0.4, exponential 0.5, sum 1, reciprocal 2;
// of a softmax: argument 1, exponential 2, divisor and product 2) and the sum with a bias below 4 by one of its own: two keys more than
// 2^-20 max(1, |key|) apart are in order.  Logits more than 2^-30 apart, and where they decide
// sigmoids at most 15, have binary64 scores that differ (slope of the sigmoid at 15: 3e-7).
__device__ __forceinline__ float wave_fmax(float v) { return unorderable(wave_umax(orderable(v))); }

template <int CTRL> __device__ __forceinline__ void merge_top2(float& b0, float& b1) {
  const float o0 = dpp_f32<CTRL>(b0), o1 = dpp_f32<CTRL>(b1);
  b1 = fmaxf(fminf(b0, o0), fmaxf(b1, o1));
  b0 = fmaxf(b0, o0);
}

// false: nothing is written, the token needs the long form
template <int NJ>
__device__ __forceinline__ bool select_scores_short(const ScoreArgs& a, int t, const float* z, int lane) {
  const int E = a.r.E, k = a.r.k;
  const bool in = lane * NJ < E, sigmoid = a.score == SMOE_SCORE_SIGMOID;
  float zv[NJ], v[NJ];
  if (NJ == 4) {
    const float4 q = in ? *(const float4*)(z + lane * 4) : make_float4(0, 0, 0, 0);
    zv[0] = q.x; zv[NJ > 1 ? 1 : 0] = q.y; zv[NJ > 2 ? 2 : 0] = q.z; zv[NJ > 3 ? 3 : 0] = q.w;
  } else if (NJ == 2) {
    const float2 q = in ? *(const float2*)(z + lane * 2) : make_float2(0, 0);
    zv[0] = q.x; zv[NJ > 1 ? 1 : 0] = q.y;
  } else {
    zv[0] = in ? z[lane] : 0.0f;
  }
  bool fine = true;
#pragma unroll
  for (int j = 0; j < NJ; j++) fine = fine && (fabsf(zv[j]) < 80.0f || zv[j] == -INFINITY);
  float bias[NJ];
#pragma unroll
  for (int j = 0; j < NJ; j++) {
    bias[j] = a.r.bias && in ? a.r.bias[lane * NJ + j] : 0.0f;
    fine = fine && fabsf(bias[j]) < 4.0f;
  }
  if (__ballot(!fine)) return false;                                    // (NaN, plus infinity, a bias as a mask)
  const bool by_score = a.r.bias || (a.n_group > 1 && a.group_score == SMOE_GROUP_TOP2);
  const bool need_den = !sigmoid && (by_score || !a.r.norm_topk);
  float m = 0.0f;
  double den = 1.0;
  if (!sigmoid) {
    float top = zv[0];
#pragma unroll
    for (int j = 1; j < NJ; j++) top = fmaxf(top, zv[j]);
    m = wave_fmax(in ? top : -INFINITY);
    if (m == -INFINITY) return false;
  }
  if (need_den) {
    den = 0.0;
#pragma unroll
    for (int j = 0; j < NJ; j++) den += in ? exp((double)zv[j] - (double)m) : 0.0;
    den = wave_sum64(den);
  }
  if (by_score) {
    const float r_den = (float)(1.0 / den);
#pragma unroll
    for (int j = 0; j < NJ; j++) {
      v[j] = sigmoid ? __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(zv[j] * -1.44269502f)) : __builtin_amdgcn_exp2f((zv[j] - m) * 1.44269502f) * r_den;
      v[j] += bias[j];
    }
  } else {
#pragma unroll
    for (int j = 0; j < NJ; j++) v[j] = zv[j];
  }
  const float unit = by_score ? 9.5367431640625e-7f : 9.313225746154785e-10f;      // 2^-20, 2^-30
  auto apart = [&](float hi, float lo) { return hi - lo > unit * (by_score ? fmaxf(1.0f, fabsf(hi)) : 1.0f); };
  uint32_t ord[NJ];
#pragma unroll
  for (int j = 0; j < NJ; j++) ord[j] = in ? orderable(v[j]) : 0u;
  if (a.n_group > 1) {
    const int lpg = a.group_size / NJ;                                  // lanes of a group: a power of two
    float b0 = v[0], b1 = -INFINITY;
#pragma unroll
    for (int j = 1; j < NJ; j++) { b1 = fmaxf(b1, fminf(b0, v[j])); b0 = fmaxf(b0, v[j]); }
    if (lpg > 1) merge_top2<0xB1>(b0, b1);
    if (lpg > 2) merge_top2<0x4E>(b0, b1);
    if (lpg > 4) merge_top2<0x141>(b0, b1);                             // row_half_mirror: the other four of eight
    if (lpg > 8) merge_top2<0x140>(b0, b1);                             // row_mirror: the other eight of sixteen
    if (lpg > 16) {
      const float o0 = __shfl_xor(b0, 16), o1 = __shfl_xor(b1, 16);
      b1 = fmaxf(fminf(b0, o0), fmaxf(b1, o1)); b0 = fmaxf(b0, o0);
    }
    const bool two = a.group_score == SMOE_GROUP_TOP2 && a.group_size > 1;
    const float score = two ? b0 + b1 : b0;
    int rank = 0;
    const int mine = lane / lpg;
    for (int g = 0; g < a.n_group; g++) {
      const float o = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(score), g * lpg));
      rank += o > score || (o == score && g < mine);
    }
    const bool chosen = rank < a.topk_group;
    if (a.topk_group < a.n_group) {
      const float worst = -wave_fmax(in && chosen ? -score : -INFINITY), best_out = wave_fmax(in && !chosen ? score : -INFINITY);
      // (two sums of two, each number off by up to 9 half steps of 1, each sum by 10 of its own; equal logits without a bias are equal scores)
      if (!apart(worst, best_out + (two ? 4.0f * unit : 0.0f)) && (by_score || worst != best_out)) return false;
      if (!by_score && sigmoid && worst > 15.0f) return false;
    }
    if (!chosen)
#pragma unroll
      for (int j = 0; j < NJ; j++) ord[j] = 0u;
  }
  // k picks and, where there is one, the best that is left
  int mysel = 0;
  float myz = 0.0f, last = 0.0f;
  const int avail = a.topk_group * a.group_size;
  for (int r = 0; r <= k && r < avail; r++) {
    uint32_t best = ord[0];
    int jb = 0;
    float zb = zv[0];
#pragma unroll
    for (int j = 1; j < NJ; j++) if (ord[j] > best) { best = ord[j]; jb = j; zb = zv[j]; }
    const uint32_t top = wave_umax(best);
    const float vt = unorderable(top);
    if (r > 0 && !apart(last, vt) && (by_score || last != vt)) return false;
    if (!by_score && sigmoid && vt > 15.0f) return false;
    last = vt;
    const int ls = (int)__builtin_ctzll(__ballot(best == top));         // the lowest index among equal keys
    if (r == k) break;
    const int js = __builtin_amdgcn_readlane(jb, ls);
    const float zs = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(zb), ls));
    if (lane == r) { mysel = ls * NJ + js; myz = zs; }
#pragma unroll
    for (int j = 0; j < NJ; j++) if (lane == ls && jb == j) ord[j] = 0u;
  }
  double w = 0.0;
  if (lane < k) w = sigmoid ? 1.0 / (1.0 + exp(-(double)myz)) : exp((double)myz - (double)m) / den;
  if (a.r.norm_topk) {                                                  // (den cancels)
    const double sum = wave_sum64(w);
    w = sum == 0.0 ? 0.0 : w / sum;
  }
  if (lane < k) {
    a.r.idx[(size_t)t * k + lane] = mysel;
    a.r.w[(size_t)t * k + lane] = (float)(w * (double)a.r.routed_scale);
  }
  return true;
}

// given logits: one wave per token
template <int NJ, int SHORT>
__global__ __launch_bounds__(64 * SC_WAVES) void route_scores_kernel(ScoreArgs a, int T) {
  extern __shared__ double sdyn[];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, t = (int)blockIdx.x * SC_WAVES + wave;
  if (t >= T) return;
  const float* z = a.r.logits + (size_t)t * a.r.E;
  if constexpr (SHORT > 0)
    if (select_scores_short<SHORT>(a, t, z, lane)) return;
  select_scores_wave<NJ>(a, t, z, lane, sdyn + wave * a.r.E);
}

// router mat-vec of NT tokens by a work-group, as in smoe_route, then one wave per token
template <int ACT, int NT, int NJ>
__global__ __launch_bounds__(RT_THREADS) void route_scores_x_kernel(ScoreArgs a, int T) {
  extern __shared__ __align__(16) uint8_t xdyn[];
  const int E = a.r.E, t0 = (int)blockIdx.x * NT, nt = min(NT, T - t0);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  double* sel = (double*)xdyn;                                        // [NT][E]
  float* zt = (float*)(xdyn + (size_t)NT * E * 8);                    // [NT][E], then the activations
  router_logits_block<ACT, NT>(a.r, t0, nt, zt, (uint8_t*)zt + ((NT * E * 4 + 15) & ~15));
  __syncthreads();
  for (int q = wave; q < nt; q += RT_NW) select_scores_wave<NJ>(a, t0 + q, zt + q * E, lane, sel + q * E);
}

template <int ACT, int NT> static size_t scores_x_lds(int E, int d) { return (size_t)NT * E * 8 + RouteLds<ACT, NT>::bytes(E, d, false); }

template <int ACT, int NT>
static int launch_scores_x(smoe_ctx* ctx, const ScoreArgs& a, int T) {
  const int E = a.r.E, grid = (T + NT - 1) / NT;
  const size_t lds = scores_x_lds<ACT, NT>(E, a.r.d_model);
  // half as many tokens per work-group where the activations of NT do not fit the LDS that a launch has without asking
  if constexpr (NT > 1) if (lds > 64u * 1024u) return launch_scores_x<ACT, NT / 2>(ctx, a, T);
  if (E <= 64) route_scores_x_kernel<ACT, NT, 1><<<grid, RT_THREADS, lds, ctx->stream>>>(a, T);
  else route_scores_x_kernel<ACT, NT, 4><<<grid, RT_THREADS, lds, ctx->stream>>>(a, T);
  HIPCHK(ctx, hipGetLastError());
  return SMOE_OK;
}

extern "C" int smoe_route_scores(smoe_ctx* ctx, int T, int E, int k, int d_model, const float* logits_dev, const void* x_dev, int act_dtype,
                                 const float* w_router_dev, int score, int n_group, int topk_group, int group_score, const float* bias_dev,
                                 int norm_topk, float routed_scale, int32_t* idx_dev, float* w_dev) {
  if (!ctx || (act_dtype != SMOE_F32 && act_dtype != SMOE_BF16)) return SMOE_EINVAL;
  if (score != SMOE_SCORE_SOFTMAX && score != SMOE_SCORE_SIGMOID) return SMOE_EINVAL;
  if (group_score != SMOE_GROUP_MAX && group_score != SMOE_GROUP_TOP2) return SMOE_EINVAL;
  if (T < 0 || T > (1 << 22) || E <= 0 || E > SMOE_MAX_EXPERTS || k <= 0 || k > SMOE_MAX_TOPK || n_group <= 0 || n_group > 64 || E % n_group ||
      topk_group <= 0 || topk_group > n_group || k > topk_group * (E / n_group))
    return SMOE_ESHAPE;
  if (T == 0) return SMOE_OK;
  if (!idx_dev || !w_dev || (!logits_dev && (!x_dev || !w_router_dev))) return SMOE_EINVAL;
  if (!logits_dev && d_model <= 0) return SMOE_ESHAPE;
  if (!aligned16(logits_dev) || !aligned16(x_dev) || !aligned16(w_router_dev) || !aligned16(bias_dev) || !aligned16(idx_dev) || !aligned16(w_dev))
    return SMOE_EALIGN;
  const bool bf16 = act_dtype == SMOE_BF16;
  if (!logits_dev && (bf16 ? scores_x_lds<SMOE_BF16, 1>(E, d_model) : scores_x_lds<SMOE_F32, 1>(E, d_model)) > 64u * 1024u) return SMOE_ESIZE;
  ON_DEVICE_OF(ctx);
  const ScoreArgs a{{E, k, d_model, logits_dev, x_dev, w_router_dev, bias_dev, norm_topk, routed_scale, nullptr, idx_dev, w_dev},
                    score, n_group, topk_group, group_score, E / n_group};
  if (!logits_dev) {
    // tokens per work-group as in smoe_route: the smallest number that needs no more work-groups than there are CUs
    const int cu = ctx->n_cu;
    if (T <= cu) return bf16 ? launch_scores_x<SMOE_BF16, 1>(ctx, a, T) : launch_scores_x<SMOE_F32, 1>(ctx, a, T);
    if (T <= 2 * cu) return bf16 ? launch_scores_x<SMOE_BF16, 2>(ctx, a, T) : launch_scores_x<SMOE_F32, 2>(ctx, a, T);
    if (!bf16 || T <= 4 * cu) return bf16 ? launch_scores_x<SMOE_BF16, 4>(ctx, a, T) : launch_scores_x<SMOE_F32, 4>(ctx, a, T);
    return launch_scores_x<SMOE_BF16, 8>(ctx, a, T);
  }
  const int grid = (T + SC_WAVES - 1) / SC_WAVES;
  const size_t lds = n_group > 1 ? (size_t)SC_WAVES * E * 8 : 0;
  // the short form needs whole lanes in a group, a power of two of them up to 32, and rows that are read 4 NJ bytes at a time
  const int nj = E <= 64 ? 1 : E <= 128 ? 2 : 4, lpg = E / n_group / nj;
  const bool brief = E % nj == 0 && (n_group == 1 || (E / n_group % nj == 0 && lpg <= 32 && (lpg & (lpg - 1)) == 0));
  if (brief && nj == 1) route_scores_kernel<1, 1><<<grid, 64 * SC_WAVES, lds, ctx->stream>>>(a, T);
  else if (brief && nj == 2) route_scores_kernel<4, 2><<<grid, 64 * SC_WAVES, lds, ctx->stream>>>(a, T);
  else if (brief) route_scores_kernel<4, 4><<<grid, 64 * SC_WAVES, lds, ctx->stream>>>(a, T);
  else if (E <= 64) route_scores_kernel<1, 0><<<grid, 64 * SC_WAVES, lds, ctx->stream>>>(a, T);
  else route_scores_kernel<4, 0><<<grid, 64 * SC_WAVES, lds, ctx->stream>>>(a, T);
  HIPCHK(ctx, hipGetLastError());
  return SMOE_OK;
}
