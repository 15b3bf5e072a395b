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
    // `lpg` lanes, a power of two, share a group's experts and join their two largest (one lane for each group in one sweep: 8.1 us for one
    // token, 256 experts in 8 groups, against 6.1)
    double b0 = -INFINITY, b1 = -INFINITY;
    const int gs = a.group_size, lpg_log = 31 - __builtin_clz(64u / (unsigned)a.n_group), lpg = 1 << lpg_log;
    const int group = lane >> lpg_log;
    if (group < a.n_group)
      for (int i = lane & (lpg - 1); i < gs; i += lpg) {
        const double v = lds[group * gs + i];
        b1 = fmax(b1, fmin(b0, v));
        b0 = fmax(b0, v);
      }
    for (int s = 1; s < lpg; s <<= 1) {
      const double o0 = __shfl_xor(b0, s), o1 = __shfl_xor(b1, s);
      b1 = fmax(fmin(b0, o0), fmax(b1, o1));
      b0 = fmax(b0, o0);
    }
    const uint64_t mine = orderable64(a.group_score == SMOE_GROUP_TOP2 && gs > 1 ? b0 + b1 : b0);
    int rank = 0;
    for (int g = 0; g < a.n_group; g++) {
      const int at = g << lpg_log;
      const uint64_t o = ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(mine >> 32), at) << 32) | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)mine, at);
      rank += o > mine || (o == mine && g < group);
    }
    const uint64_t in = __ballot(group < a.n_group && rank < a.topk_group);
#pragma unroll
    for (int j = 0; j < NJ; j++) {
      const int e = lane + 64 * j;
      if (e < E && !((in >> ((e / gs) << lpg_log)) & 1u)) ord[j] = 0u;
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

// ---- short form: sixteen lanes per token, lane r of them with the NJ experts from NJ r on, ordered by fp32 keys.  A
// token whose keys lie too close together to be sure of the binary64 order is left to select_scores_wave.
//   The key of an expert is its logit where the order of the scores is the logits' own (no bias; no sum of two scores), else the fp32 score
// plus bias.  A score is off by at most 5 half steps of 1 (of a sigmoid: argument of the exponential s (1 - s) |z| 1.5 < 0.4, exponential 0.5, sum 1, reciprocal 2;
// of a softmax: argument 1, exponential 2, divisor and product 2) and the sum with a bias below 4 by one of its own: two keys more than
// 2^-20 max(1, |key|) apart are in order.  Logits more than 2^-30 apart, and where they decide
// sigmoids at most 15, have binary64 scores that differ (slope of the sigmoid at 15: 3e-7).
//   Bound: vector issue.  16384 tokens, 256 experts in 8 groups, top-8: 28 us with a short form of one token per wave, 22 with the pick found by comparing and taken
// out by a mask (140 instructions a pick, now 50), 19.6 - 20.1 now, of which some 0.8 are the few tokens that need the long form (19.3 for logits far apart; 29.7 by the long
// form alone).
template <int CTRL> __device__ __forceinline__ uint32_t dpp_u32(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true); }
// the four steps of a reduction over a row of sixteen lanes: neighbour, neighbouring pair, other four of eight, other eight
#define ROW_REDUCE(v, OP)      \
  v = OP(v, dpp_u32<0xB1>(v)); \
  v = OP(v, dpp_u32<0x4E>(v)); \
  v = OP(v, dpp_u32<0x141>(v)); \
  v = OP(v, dpp_u32<0x140>(v));
__device__ __forceinline__ uint32_t row_umax(uint32_t v) { ROW_REDUCE(v, max) return v; }
__device__ __forceinline__ uint32_t row_umin(uint32_t v) { ROW_REDUCE(v, min) return v; }
__device__ __forceinline__ float row_fmax(float v) { return unorderable(row_umax(orderable(v))); }
__device__ __forceinline__ double row_sum64(double v) {
  v += dpp_f64<0xB1>(v);
  v += dpp_f64<0x4E>(v);
  v += dpp_f64<0x141>(v);
  v += dpp_f64<0x140>(v);
  return v;
}
template <int CTRL> __device__ __forceinline__ void merge_top2(float& b0, float& b1) {
  const float o0 = dpp_f32<CTRL>(b0), o1 = dpp_f32<CTRL>(b1);
  b1 = fmaxf(fminf(b0, o0), fmaxf(b1, o1));
  b0 = fmaxf(b0, o0);
}

// Token t by sixteen lanes (rl: the lane's number among them).  False in all of them: nothing was written, the token needs the long form.
template <int NJ>
__device__ __forceinline__ bool select_scores_row(const ScoreArgs& a, int t, bool write, int lane) {
  const int E = a.r.E, k = a.r.k, rl = lane & 15;
  const bool in = rl * NJ < E, sigmoid = a.score == SMOE_SCORE_SIGMOID;      // (E is a multiple of 4: experts of the last lane may be missing, by fours)
  const float* z = a.r.logits + (size_t)t * E;
  float zv[NJ], v[NJ], bias[NJ];
#pragma unroll
  for (int j = 0; j < NJ; j += 4) {
    const bool have = rl * NJ + j < E;
    const float4 q = have ? *(const float4*)(z + rl * NJ + j) : make_float4(0, 0, 0, 0);
    const float4 b = have && a.r.bias ? *(const float4*)(a.r.bias + rl * NJ + j) : make_float4(0, 0, 0, 0);
    zv[j] = q.x; zv[j + 1] = q.y; zv[j + 2] = q.z; zv[j + 3] = q.w;
    bias[j] = b.x; bias[j + 1] = b.y; bias[j + 2] = b.z; bias[j + 3] = b.w;
  }
  uint32_t zbig = 0, bbig = 0;                                          // largest magnitudes, as bit patterns (NaN above all)
#pragma unroll
  for (int j = 0; j < NJ; j++) {
    const uint32_t u = __float_as_uint(zv[j]);
    zbig = max(zbig, u == 0xFF800000u ? 0u : u & 0x7FFFFFFFu);
    bbig = max(bbig, __float_as_uint(bias[j]) & 0x7FFFFFFFu);
  }
  bool fine = zbig < __float_as_uint(80.0f) && bbig < __float_as_uint(4.0f);      // not: NaN, plus infinity, a bias as a mask
  const bool by_score = a.r.bias || (a.n_group > 1 && a.group_score == SMOE_GROUP_TOP2);
  const bool need_den = !sigmoid && (by_score || !a.r.norm_topk);
  float m = 0.0f;
  double den = 1.0;
  if (!sigmoid) {
    float top = -INFINITY;
#pragma unroll
    for (int j = 0; j < NJ; j++) top = fmaxf(top, rl * NJ + j < E ? zv[j] : -INFINITY);
    m = row_fmax(top);
    fine = fine && m > -INFINITY;
    if (need_den) {
      den = 0.0;
#pragma unroll
      for (int j = 0; j < NJ; j++) den += rl * NJ + j < E ? exp((double)zv[j] - (double)m) : 0.0;
      den = row_sum64(den);
    }
  }
  if (by_score) {
    const float r_den = (float)(1.0 / den);
#pragma unroll
    for (int j = 0; j < NJ; j++)
      v[j] = (sigmoid ? __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(zv[j] * -1.44269502f)) : __builtin_amdgcn_exp2f((zv[j] - m) * 1.44269502f) * r_den) + bias[j];
  } else {
#pragma unroll
    for (int j = 0; j < NJ; j++) v[j] = zv[j];
  }
  const float unit = by_score ? 9.5367431640625e-7f : 9.313225746154785e-10f;      // 2^-20, 2^-30
  auto apart = [&](float hi, float lo) { return hi - lo > unit * (by_score ? fmaxf(1.0f, fabsf(hi)) : 1.0f); };
  uint32_t ord[NJ];
#pragma unroll
  for (int j = 0; j < NJ; j++) ord[j] = rl * NJ + j < E ? (orderable(v[j]) & ~15u) | (15u - j) : 0u;
  if (a.n_group > 1) {
    const int lpg = a.group_size / NJ;                                  // lanes of a group: a power of two up to 8
    float b0 = v[0], b1 = -INFINITY;
#pragma unroll
    for (int j = 1; j < NJ; j++) { b1 = fmaxf(b1, fminf(b0, v[j])); b0 = fmaxf(b0, v[j]); }
    if (lpg > 1) merge_top2<0xB1>(b0, b1);
    if (lpg > 2) merge_top2<0x4E>(b0, b1);
    if (lpg > 4) merge_top2<0x141>(b0, b1);
    const bool two = a.group_score == SMOE_GROUP_TOP2;
    const float score = two ? b0 + b1 : b0;
    int rank = 0;
    const int mine = rl / lpg;
    for (int g = 0; g < a.n_group; g++) {
      const float o = __shfl(score, (lane & 48) + g * lpg);
      rank += o > score || (o == score && g < mine);
    }
    const bool chosen = rank < a.topk_group;
    if (a.topk_group < a.n_group) {
      const float worst = -row_fmax(in && chosen ? -score : -INFINITY), best_out = row_fmax(in && !chosen ? score : -INFINITY);
      // (two sums of two, each number off by up to 9 half steps of 1, each sum by 10 of its own; equal logits without a bias are equal scores)
      fine = fine && (apart(worst, best_out + (two ? 4.0f * unit : 0.0f)) || (!by_score && worst == best_out));
      fine = fine && (by_score || !sigmoid || worst <= 15.0f);
    }
#pragma unroll
    for (int j = 0; j < NJ; j++) ord[j] = chosen ? ord[j] : 0u;
  }
  // k picks and, where there is one, the best that is left.  The lowest four bits of a key are the expert's place in its lane, so that a pick is a
  // minimum of distances below the last one, without masks: keys not below it wrap round to more than any distance.
  int mysel = 0;
  uint32_t top = 0;
  const int avail = a.topk_group * a.group_size;
  for (int r = 0; r <= k && r < avail; r++) {
    uint32_t mine = 0xFFFFFFFFu;
#pragma unroll
    for (int j = 0; j < NJ; j++) mine = min(mine, top - 1u - ord[j]);
    const uint32_t step = row_umin(mine), next = top - 1u - step;
    // what the four bits hide is counted in: lower bound of the last key against upper bound of this one
    const float vt = unorderable(next | 15u);
    fine = fine && (r == 0 || apart(unorderable(top & ~15u), vt)) && (by_score || !sigmoid || vt <= 15.0f);
    top = next;
    if (r == k) break;
    const uint32_t who = (uint32_t)(__ballot(mine == step) >> (lane & 48)) & 0xFFFFu;      // (one lane: two with the same key are not apart, and show below)
    fine = fine && !(who & (who - 1u));
    if (rl == r) mysel = (int)(__builtin_ctz(who) * NJ + 15u - (top & 15u));
  }
  fine = !((__ballot(!fine) >> (lane & 48)) & 0xFFFFu);
  double w = 0.0;
  if (rl < k) {
    const double zs = (double)z[min(mysel, E - 1)];
    w = sigmoid ? 1.0 / (1.0 + exp(-zs)) : exp(zs - (double)m) / den;
  }
  if (a.r.norm_topk) {                                                  // (den cancels)
    const double sum = row_sum64(w);
    w = sum == 0.0 ? 0.0 : w / sum;
  }
  if (fine && write && rl < k) {
    a.r.idx[(size_t)t * k + rl] = mysel;
    a.r.w[(size_t)t * k + rl] = (float)(w * (double)a.r.routed_scale);
  }
  return fine;
}

// given logits: four tokens a wave by the short form, what that leaves by the whole wave
template <int NJ, int LONG>
__global__ __launch_bounds__(64 * SC_WAVES) void route_scores_kernel(ScoreArgs a, int T) {
  extern __shared__ double sdyn[];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, t0 = ((int)blockIdx.x * SC_WAVES + wave) * 4;
  if (t0 >= T) return;
  const int t = t0 + (lane >> 4);
  const bool done = select_scores_row<NJ>(a, min(t, T - 1), t < T, lane);
  const uint64_t left = __ballot(!done && t < T);
  for (int q = 0; q < 4; q++)
    if ((left >> (16 * q)) & 1u) select_scores_wave<LONG>(a, t0 + q, a.r.logits + (size_t)(t0 + q) * a.r.E, lane, sdyn + wave * a.r.E);
}
// the same by the long form alone, a wave per token
template <int LONG>
__global__ __launch_bounds__(64 * SC_WAVES) void route_scores_long_kernel(ScoreArgs a, int T) {
  extern __shared__ double sdyn[];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, t = (int)blockIdx.x * SC_WAVES + wave;
  if (t < T) select_scores_wave<LONG>(a, t, a.r.logits + (size_t)t * a.r.E, lane, sdyn + wave * a.r.E);
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
  if (T > ROWS_A_LAUNCH * NT) {
    const size_t n = (size_t)ROWS_A_LAUNCH * NT;
    ScoreArgs rest = a;
    rest.r.x = (const uint8_t*)a.r.x + n * a.r.d_model * (ACT == SMOE_F32 ? 4 : 2);
    rest.r.idx += n * a.r.k;
    rest.r.w += n * a.r.k;
    if (const int rc = launch_scores_x<ACT, NT>(ctx, a, (int)n)) return rc;
    return launch_scores_x<ACT, NT>(ctx, rest, T - (int)n);
  }
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
  ScoreArgs a{{E, k, d_model, logits_dev, x_dev, w_router_dev, bias_dev, norm_topk, routed_scale, nullptr, idx_dev, w_dev},
                    score, n_group, topk_group, group_score, E / n_group};
  if (!logits_dev && T == 1 && ctx->ws) {
    // One token: the mat-vec is spread over E / 4 work-groups, its logits stand in the context's workspace (the same sums, bit for bit).  d 2048, 64 /
    // 256 experts: 5.0 / 6.3 us instead of 7.8 / 23.8 by one work-group, which is what a context without a workspace gets.
    float* z = (float*)(ctx->ws + WS_IDX_OFF);
    if (const int rc = smoe_launch_router_logits(ctx, E, d_model, x_dev, act_dtype, w_router_dev, z)) return rc;
    a.r.logits = z;
  }
  if (!a.r.logits) {
    // tokens per work-group as in smoe_route: the smallest number that needs no more work-groups than there are CUs
    const int cu = ctx->n_cu;
    if (T <= cu) return bf16 ? launch_scores_x<SMOE_BF16, 1>(ctx, a, T) : launch_scores_x<SMOE_F32, 1>(ctx, a, T);
    if (T <= 2 * cu) return bf16 ? launch_scores_x<SMOE_BF16, 2>(ctx, a, T) : launch_scores_x<SMOE_F32, 2>(ctx, a, T);
    if (!bf16 || T <= 4 * cu) return bf16 ? launch_scores_x<SMOE_BF16, 4>(ctx, a, T) : launch_scores_x<SMOE_F32, 4>(ctx, a, T);
    return launch_scores_x<SMOE_BF16, 8>(ctx, a, T);
  }
  // The short form needs rows of 16-byte pieces and groups of whole lanes, a power of two of them up to 8.  With few tokens its longer chain of
  // instructions counts and not their number.  Microseconds a call in a captured graph, short / long form, by tokens:
  //                                             2048         2049         4096         8192          16384
  //   60 experts, softmax, top-4             4.3 / 2.9    4.3 / 2.9    4.4 / 3.7    5.0 / 5.0     6.7 / 7.8
  //   64 experts, sigmoid + bias, top-6      4.7 / 3.1    4.7 / 3.1    5.2 / 3.8    5.5 / 5.3     7.2 / 8.4
  //   128 experts, softmax, top-8            6.1 / 5.4    6.1 / 6.0    6.2 / 7.4    7.3 / 11.6    11.5 / 20.2
  //   256 experts, sigmoid + bias, top-8     9.0 / 5.6    9.0 / 6.1    9.2 / 7.6    10.8 / 12.3   17.1 / 21.9
  //   256 in 8 groups, the same              11.1 / 7.3   11.0 / 8.1   11.2 / 9.9   13.0 / 16.5   19.6 / 29.7
  // The switch at 2048 is right for 128 experts; with 64 and fewer the short form pays from some 8192 tokens on, with 256 from some 6000.
  const size_t lds = n_group > 1 ? (size_t)SC_WAVES * E * 8 : 0;
  const int nj = E <= 64 ? 4 : E <= 128 ? 8 : 16, lpg = E / n_group / nj;
  const bool brief = T > 2048 && E % 4 == 0 && (n_group == 1 || (E / n_group % nj == 0 && (lpg & (lpg - 1)) == 0));
  const int per = SC_WAVES * (brief ? 4 : 1), grid = (T + per - 1) / per;
  if (brief && nj == 4) route_scores_kernel<4, 1><<<grid, 64 * SC_WAVES, lds, ctx->stream>>>(a, T);
  else if (brief && nj == 8) route_scores_kernel<8, 4><<<grid, 64 * SC_WAVES, lds, ctx->stream>>>(a, T);
  else if (brief) route_scores_kernel<16, 4><<<grid, 64 * SC_WAVES, lds, ctx->stream>>>(a, T);
  else if (E <= 64) route_scores_long_kernel<1><<<grid, 64 * SC_WAVES, lds, ctx->stream>>>(a, T);
  else route_scores_long_kernel<4><<<grid, 64 * SC_WAVES, lds, ctx->stream>>>(a, T);
  HIPCHK(ctx, hipGetLastError());
  return SMOE_OK;
}
