// smoe_residual_norm: what stands between two blocks of a layer stack.
//   b  = sum_j w[t,j] y[t,j]                     the block's slots joined by their gate weights
//   b  = b / sqrt(mean(b^2) + eps) * post_w      norm after the block
//   h' = h + scale * gate * b                    residual stream
//   x  = h' / sqrt(mean(h'^2) + eps) * pre_w     norm before the next block
// One pass: a row stays in the registers of its work-group between the sums, so y and h are read once and h' and x
// written once.  Bound: HBM bytes with many rows, the launch and one memory round trip with few.  All arithmetic is
// fp32; h' enters the second norm as it is before it is rounded to the residual's type.
#include "common.hpp"
#include <type_traits>

struct NormArgs {
  const void* y; const float* slot_w; const void* post_w; const void* gate; const void* res; const void* pre_w;
  void* res_out; void* x_out;
  int T, d, k, gate_rows;
  float scale, eps;
};

// Sum over the NT threads of a work-group (or the wave alone, NT = 64), in every thread.
template <int NT> __device__ __forceinline__ float block_sum(float v, float* red, int row) {
  v = wave_sum(v);
  if (NT == 64) return v;
  if ((threadIdx.x & 63) == 0) red[row * (NT / 64) + (threadIdx.x >> 6)] = v;
  __syncthreads();
  float s = 0.0f;
#pragma unroll
  for (int i = 0; i < NT / 64; i++) s += red[row * (NT / 64) + i];
  return s;
}

// A row belongs to NT threads (64: four rows a work-group, else the whole work-group), NC pieces of 8 columns each.
template <int ACT, int RES, int NT, int NC>
__global__ __launch_bounds__(NT == 64 ? 256 : NT) void residual_norm_kernel(NormArgs a) {
  __shared__ float red[2 * (NT / 64)];
  const int t = NT == 64 ? (int)blockIdx.x * 4 + (threadIdx.x >> 6) : (int)blockIdx.x;
  const int tid = NT == 64 ? threadIdx.x & 63 : threadIdx.x;
  if (NT == 64 && t >= a.T) return;                     // (whole waves; no barrier in this form)
  const int d = a.d;
  const float inv_d = 1.0f / (float)d;
  const size_t row = (size_t)t * d;
  float b[NC][8];
#pragma unroll
  for (int c = 0; c < NC; c++)
#pragma unroll
    for (int i = 0; i < 8; i++) b[c][i] = 0.0f;
  for (int j = 0; j < a.k; j++) {
    const float w = a.slot_w ? a.slot_w[(size_t)t * a.k + j] : 1.0f;
#pragma unroll
    for (int c = 0; c < NC; c++) {
      const int at = (c * NT + tid) * 8;
      if (at < d) {
        float v[8];
        load8<ACT>(a.y, ((size_t)t * a.k + j) * d + at, v);
#pragma unroll
        for (int i = 0; i < 8; i++) b[c][i] = fmaf(w, v[i], b[c][i]);
      }
    }
  }
  if (a.post_w) {
    float s = 0.0f;
#pragma unroll
    for (int c = 0; c < NC; c++)
#pragma unroll
      for (int i = 0; i < 8; i++) s = fmaf(b[c][i], b[c][i], s);
    const float r = 1.0f / sqrtf(block_sum<NT>(s, red, 0) * inv_d + a.eps);
#pragma unroll
    for (int c = 0; c < NC; c++) {
      const int at = (c * NT + tid) * 8;
      if (at < d) {
        float v[8];
        load8<ACT>(a.post_w, at, v);
#pragma unroll
        for (int i = 0; i < 8; i++) b[c][i] = b[c][i] * r * v[i];
      }
    }
  }
  float s = 0.0f;
#pragma unroll
  for (int c = 0; c < NC; c++) {
    const int at = (c * NT + tid) * 8;
    if (at < d) {
      float h[8];
      if (a.k > 0) {
        if (a.gate) {
          float v[8];
          load8<ACT>(a.gate, (a.gate_rows ? row : 0) + at, v);
#pragma unroll
          for (int i = 0; i < 8; i++) b[c][i] *= v[i];
        }
#pragma unroll
        for (int i = 0; i < 8; i++) b[c][i] *= a.scale;
      }
      if (a.res) {
        load8<RES>(a.res, row + at, h);
#pragma unroll
        for (int i = 0; i < 8; i++) b[c][i] += h[i];
      }
      if (a.res_out) store8<RES>(a.res_out, row + at, b[c]);
#pragma unroll
      for (int i = 0; i < 8; i++) s = fmaf(b[c][i], b[c][i], s);
    }
  }
  if (!a.x_out) return;
  const float r = 1.0f / sqrtf(block_sum<NT>(s, red, 1) * inv_d + a.eps);
#pragma unroll
  for (int c = 0; c < NC; c++) {
    const int at = (c * NT + tid) * 8;
    if (at < d) {
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; i++) v[i] = 1.0f;
      if (a.pre_w) load8<ACT>(a.pre_w, at, v);
#pragma unroll
      for (int i = 0; i < 8; i++) v[i] = b[c][i] * r * v[i];
      store8<ACT>(a.x_out, row + at, v);
    }
  }
}

template <int ACT, int RES>
static int launch_norm(smoe_ctx* ctx, NormArgs a) {
  if (a.T > ROWS_A_LAUNCH) {
    const size_t n = ROWS_A_LAUNCH, act = ACT == SMOE_F32 ? 4 : 2, res = RES == SMOE_F32 ? 4 : 2;
    NormArgs rest = a;
    a.T = ROWS_A_LAUNCH;
    rest.T -= ROWS_A_LAUNCH;
    auto skip = [](auto& p, size_t bytes) { if (p) p = (std::remove_reference_t<decltype(p)>)((uintptr_t)p + bytes); };
    skip(rest.y, n * a.k * a.d * act); skip(rest.slot_w, n * a.k * 4); skip(rest.res, n * a.d * res); skip(rest.res_out, n * a.d * res); skip(rest.x_out, n * a.d * act);
    if (a.gate_rows) skip(rest.gate, n * a.d * act);
    if (const int rc = launch_norm<ACT, RES>(ctx, a)) return rc;
    return launch_norm<ACT, RES>(ctx, rest);
  }
  const int pieces = a.d / 8;
  hipStream_t st = ctx->stream;
  if (pieces <= 64) residual_norm_kernel<ACT, RES, 64, 1><<<(a.T + 3) / 4, 256, 0, st>>>(a);
  else if (pieces <= 256) residual_norm_kernel<ACT, RES, 256, 1><<<a.T, 256, 0, st>>>(a);
  else if (pieces <= 512) residual_norm_kernel<ACT, RES, 256, 2><<<a.T, 256, 0, st>>>(a);
  else if (pieces <= 1024) residual_norm_kernel<ACT, RES, 512, 2><<<a.T, 512, 0, st>>>(a);
  else residual_norm_kernel<ACT, RES, 1024, 2><<<a.T, 1024, 0, st>>>(a);
  HIPCHK(ctx, hipGetLastError());
  return SMOE_OK;
}

extern "C" int smoe_residual_norm(smoe_ctx* ctx, int T, int d, int k, const void* y_dev, const float* slot_w_dev, const void* post_w_dev,
                                  const void* gate_dev, int gate_rows, float scale, const void* res_dev, const void* pre_w_dev, float eps,
                                  int act_dtype, int res_dtype, void* res_out_dev, void* x_out_dev) {
  if (!ctx || (act_dtype != SMOE_F32 && act_dtype != SMOE_BF16) || (res_dtype != SMOE_F32 && res_dtype != SMOE_BF16)) return SMOE_EINVAL;
  if ((gate_rows != 0 && gate_rows != 1) || !(eps >= 0.0f)) return SMOE_EINVAL;
  if (T < 0 || T > (1 << 22) || d <= 0 || d % 8 || d > 16384 || k < 0 || k > SMOE_MAX_SLOTS) return SMOE_ESHAPE;
  if (T == 0) return SMOE_OK;
  if ((!res_out_dev && !x_out_dev) || (!y_dev && !res_dev)) return SMOE_EINVAL;
  if ((y_dev != nullptr) != (k > 0) || (!y_dev && (slot_w_dev || post_w_dev || gate_dev))) return SMOE_EINVAL;
  if (x_out_dev && (x_out_dev == res_out_dev || x_out_dev == y_dev || x_out_dev == res_dev)) return SMOE_EINVAL;
  if (res_out_dev && res_out_dev == y_dev) return SMOE_EINVAL;
  if (!aligned16(y_dev) || !aligned16(slot_w_dev) || !aligned16(post_w_dev) || !aligned16(gate_dev) || !aligned16(res_dev) || !aligned16(pre_w_dev) ||
      !aligned16(res_out_dev) || !aligned16(x_out_dev))
    return SMOE_EALIGN;
  ON_DEVICE_OF(ctx);
  const NormArgs a{y_dev, slot_w_dev, post_w_dev, gate_dev, res_dev, pre_w_dev, res_out_dev, x_out_dev, T, d, k, gate_rows, scale, eps};
  if (act_dtype == SMOE_F32) return res_dtype == SMOE_F32 ? launch_norm<SMOE_F32, SMOE_F32>(ctx, a) : launch_norm<SMOE_F32, SMOE_BF16>(ctx, a);
  return res_dtype == SMOE_F32 ? launch_norm<SMOE_BF16, SMOE_F32>(ctx, a) : launch_norm<SMOE_BF16, SMOE_BF16>(ctx, a);
}
