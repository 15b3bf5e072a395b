// smoe_mx_quantize, smoe_mx_dequantize and smoe_mx_matvec: microscaled 4-bit floats, and the product of a few unquantised
// rows with them.
#include "mx.hpp"

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// ------------------------------------------------------------------------------- there and back
template <int CTRL> __device__ __forceinline__ uint32_t dpp_max_u32(uint32_t v) {
  const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true);
  return o > v ? o : v;
}

// A thread takes 8 columns, the four lanes of a quad a block.  The largest magnitude is found on the bit patterns
// (ordered as the numbers are, NaN last); floor(log2) of it is its exponent field.  Bound: bytes moved.
template <int SRC>
__global__ __launch_bounds__(256) void mx_quantize_kernel(const void* src, size_t n8, uint32_t* codes, uint8_t* scales) {
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n8) return;                                        // (whole quads: K is a multiple of 32)
  float v[8];
  load8<SRC>(src, i * 8, v);
  uint32_t big = 0;
#pragma unroll
  for (int j = 0; j < 8; j++) { const uint32_t u = __float_as_uint(v[j]) & 0x7FFFFFFFu; big = u > big ? u : big; }
  big = dpp_max_u32<0xB1>(big);
  big = dpp_max_u32<0x4E>(big);
  const uint32_t ex = big >> 23, byte = ex == 255 ? 255u : ex > 2 ? ex - 2 : 0u;
  const float scale = mx_scale(byte);
  uint32_t c = 0;
  if (byte != 255) {                                          // the conversion divides by the scale, rounds to nearest even and saturates at 6
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], scale, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], scale, 3);
  }
  codes[i] = c;
  if ((i & 3) == 0) scales[i >> 2] = (uint8_t)byte;
}

template <int DST>
__global__ __launch_bounds__(256) void mx_dequantize_kernel(const uint32_t* codes, const uint8_t* scales, size_t n8, void* dst) {
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n8) return;
  const float scale = mx_scale(scales[i >> 2]);
  const uint32_t c = codes[i];
  float v[8];
  const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 1);
  const f32x2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 2), e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 3);
  v[0] = a[0] * scale; v[1] = a[1] * scale; v[2] = b[0] * scale; v[3] = b[1] * scale;
  v[4] = d[0] * scale; v[5] = d[1] * scale; v[6] = e[0] * scale; v[7] = e[1] * scale;
  store8<DST>(dst, i * 8, v);
}

static int check_rows(long long rows, int K) {
  if (rows < 0 || K <= 0 || K % 32 || rows > (1ll << 34) / K) return SMOE_ESHAPE;
  return SMOE_OK;
}

extern "C" int smoe_mx_quantize(smoe_ctx* ctx, long long rows, int K, const void* src_dev, int src_dtype, uint8_t* codes_dev, uint8_t* scales_dev) {
  if (!ctx || (src_dtype != SMOE_F32 && src_dtype != SMOE_BF16)) return SMOE_EINVAL;
  if (const int rc = check_rows(rows, K)) return rc;
  if (rows == 0) return SMOE_OK;
  if (!src_dev || !codes_dev || !scales_dev) return SMOE_EINVAL;
  if (!aligned16(src_dev) || !aligned16(codes_dev) || !aligned16(scales_dev)) return SMOE_EALIGN;
  ON_DEVICE_OF(ctx);
  const size_t n8 = (size_t)rows * K / 8;
  const unsigned grid = (unsigned)((n8 + 255) / 256);
  if (src_dtype == SMOE_F32) mx_quantize_kernel<SMOE_F32><<<grid, 256, 0, ctx->stream>>>(src_dev, n8, (uint32_t*)codes_dev, scales_dev);
  else mx_quantize_kernel<SMOE_BF16><<<grid, 256, 0, ctx->stream>>>(src_dev, n8, (uint32_t*)codes_dev, scales_dev);
  HIPCHK(ctx, hipGetLastError());
  return SMOE_OK;
}

extern "C" int smoe_mx_dequantize(smoe_ctx* ctx, long long rows, int K, const uint8_t* codes_dev, const uint8_t* scales_dev, void* dst_dev, int dst_dtype) {
  if (!ctx || (dst_dtype != SMOE_F32 && dst_dtype != SMOE_BF16)) return SMOE_EINVAL;
  if (const int rc = check_rows(rows, K)) return rc;
  if (rows == 0) return SMOE_OK;
  if (!dst_dev || !codes_dev || !scales_dev) return SMOE_EINVAL;
  if (!aligned16(dst_dev) || !aligned16(codes_dev) || !aligned16(scales_dev)) return SMOE_EALIGN;
  ON_DEVICE_OF(ctx);
  const size_t n8 = (size_t)rows * K / 8;
  const unsigned grid = (unsigned)((n8 + 255) / 256);
  if (dst_dtype == SMOE_F32) mx_dequantize_kernel<SMOE_F32><<<grid, 256, 0, ctx->stream>>>((const uint32_t*)codes_dev, scales_dev, n8, dst_dev);
  else mx_dequantize_kernel<SMOE_BF16><<<grid, 256, 0, ctx->stream>>>((const uint32_t*)codes_dev, scales_dev, n8, dst_dev);
  HIPCHK(ctx, hipGetLastError());
  return SMOE_OK;
}

// ------------------------------------------------------------------------------- a few rows
// y[slot] = W[idx[slot]] x, W microscaled, x as it is.  Bound: the bytes of the selected matrices.
//   A work-group takes 16 RT weight rows of one expert and up to 16 of the slots that chose this expert, so that every weight
// byte is read once however many tokens share it.  Work-groups go by slots (that of a slot that is not the first of its expert has
// nothing to do) or, with fewer experts than slots, by experts.  Its four or eight waves share the columns out, 128 at a time (32 columns of a row are one 16-byte load of a lane) and in turn,
// so that the two halves of a line of weights are asked for together
// (a wave with neighbouring columns of its own: 29.5 against 28.3 us in fp32, 23.3 against 21.5 in bf16; 16 tokens, top-6 of 64, N 2048, K 1408), and add their sums up through
// LDS.  The figures here and below are microseconds a call in a captured graph that goes round over several layers' weights, so that these come from HBM.
//   Codes are expanded to bf16, which holds e2m1 times a power of two exactly (below 2^128; infinite from there on), and multiplied by matrix instructions with
// fp32 sums.  fp32 activations go in as three bf16 numbers whose sum they are (8 + 8 + 8 bits, cut off, not rounded), so
// these products are exact too (bits below 2^-133, bf16's smallest, are cut off); the splitting is seven vector instructions a number, which is why it serves RT tiles of rows at once.
struct MatvecArgs {
  const uint8_t* codes; const uint8_t* scales; const void* x; const int32_t* idx; void* y;
  int E, N, K, T, k, x_slots, swiglu, by_expert;
};

template <int ACT> __device__ __forceinline__ void store1(void* p, size_t i, float v) {
  if (ACT == SMOE_F32) ((float*)p)[i] = v;
  else ((__bf16*)p)[i] = (__bf16)v;
}

// eight activations as they lie in memory, and as PARTS operands of a matrix instruction
template <int ACT> struct RawX { u32x4 v[ACT == SMOE_F32 ? 2 : 1]; };
template <int ACT, int PARTS>
__device__ __forceinline__ void operands(const RawX<ACT>& r, bool ok, bf16x8 (&p)[PARTS]) {
  if constexpr (ACT == SMOE_BF16) {
    p[0] = __builtin_bit_cast(bf16x8, ok ? r.v[0] : u32x4{0, 0, 0, 0});
  } else {
    union { uint32_t u[4]; bf16x8 v; } o[3];
#pragma unroll
    for (int i = 0; i < 4; i++) {
      uint32_t h[2][3];
#pragma unroll
      for (int j = 0; j < 2; j++) {
        const uint32_t u = ok ? r.v[i >> 1][2 * (i & 1) + j] : 0u;
        const float x = __uint_as_float(u);
        h[j][0] = u & 0xFFFF0000u;
        // (an infinity leaves nothing; a NaN whose bits were cut off leaves a NaN)
        const float rest = (u & 0x7FFFFFFFu) == 0x7F800000u ? 0.0f : x - __uint_as_float(h[j][0]);
        h[j][1] = __float_as_uint(rest) & 0xFFFF0000u;
        h[j][2] = __float_as_uint(rest - __uint_as_float(h[j][1]));
      }
#pragma unroll
      for (int m = 0; m < 3; m++) o[m].u[i] = __builtin_amdgcn_perm(h[1][m], h[0][m], 0x07060302u);
    }
#pragma unroll
    for (int m = 0; m < 3; m++) p[m] = o[m].v;
  }
}

template <int ACT, int RT, int MV_WAVES>
__global__ __launch_bounds__(64 * MV_WAVES) void mx_matvec_kernel(MatvecArgs a) {
  constexpr int PARTS = ACT == SMOE_F32 ? 3 : 1, ROWS = 16 * RT;
  __shared__ int slots[SMOE_MAX_MULTI * SMOE_MAX_TOPK];
  __shared__ int wave_n[MV_WAVES];
  __shared__ __align__(16) float part[MV_WAVES][ROWS][17];          // before it is that: fp32 activations as parts
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int c = lane & 15, g = lane >> 4;
  const int n = a.T * a.k, s0 = (int)blockIdx.y;
  int e = 0, n_mine = n;
  auto expert = [&](int i) { const int v = a.idx[i]; return v < 0 ? 0 : v >= a.E ? a.E - 1 : v; };
  if (a.T == 1) {                                             // every slot by itself
    if (a.idx) e = expert(s0);
    n_mine = 1;
  } else if (a.idx) {
    e = a.by_expert ? s0 : expert(s0);
    const bool is = tid < n && expert(tid) == e;
    const uint64_t b = __ballot(is);
    if (lane == 0) wave_n[wave] = (int)__builtin_popcountll(b);
    __syncthreads();
    int base = 0, total = 0;
#pragma unroll
    for (int w = 0; w < MV_WAVES; w++) { base += w < wave ? wave_n[w] : 0; total += wave_n[w]; }
    if (is) slots[base + (int)__builtin_popcountll(b & ((1ull << lane) - 1))] = tid;
    __syncthreads();
    if (total == 0 || (!a.by_expert && slots[0] != s0)) return;      // (uniform over the work-group)
    n_mine = total;
  } else {
    if (tid < n) slots[tid] = tid;
    __syncthreads();
  }
  const int r0 = (int)blockIdx.x * ROWS, nb = a.K >> 5;
  const uint8_t* wc[RT];
  const uint8_t* ws[RT];
#pragma unroll
  for (int t = 0; t < RT; t++) {
    const size_t row = (size_t)e * a.N + min(r0 + 16 * t + c, a.N - 1);
    wc[t] = a.codes + row * (size_t)(a.K >> 1);
    ws[t] = a.scales + row * (size_t)nb;
  }
  const int units = (nb + 3) >> 2;
  // fp32 activations of so few slots that they fit are taken apart once for the whole work-group, [slot][part][units * 128], zeros behind the last block, else by
  // every lane for itself.  Microseconds with / without (top-6 of 64, N 2048, K 1408): one token 7.2 / 7.5, 4 tokens 11.4 / 13.2, 8 tokens 19.6 / 20.7, 16 tokens
  // 28.3 / 29.2, where the work-groups of experts with three slots and more go on as long as before.  Dense, K 2048: N 2048, one token 5.6 / 5.4, 4 tokens 6.0 / 5.6; N 8192, one token
  // 9.1 / 10.2, 4 tokens 11.0 / 10.4; K and N 8192, one token 33.6 / 30.4.
  __bf16* split = (__bf16*)part;
  const int Kp = units * 128;
  const bool shared = PARTS > 1 && n_mine <= 16 && n_mine * Kp * PARTS * 2 <= (int)sizeof(part);
  u32x4 w[RT];
  uint32_t sb[RT];
  auto fetch = [&](int u) {
    const int bc = min(u * 4 + g, nb - 1);
#pragma unroll
    for (int t = 0; t < RT; t++) {
      w[t] = *(const u32x4*)(wc[t] + (size_t)bc * 16);
      sb[t] = ws[t][bc];
    }
  };
  fetch(wave);
  if (shared) {
    for (int i = tid; i < n_mine * (Kp / 8); i += 64 * MV_WAVES) {
      const int m = i / (Kp / 8), at = (i - m * (Kp / 8)) * 8, slot = a.T == 1 ? s0 : slots[m];
      const float* x = (const float*)a.x + (size_t)(a.x_slots ? slot : slot / a.k) * a.K;
      RawX<ACT> r;
#pragma unroll
      for (int v = 0; v < (ACT == SMOE_F32 ? 2 : 1); v++) r.v[v] = *(const u32x4*)(x + min(at, a.K - 8) + v * 4);
      bf16x8 p[PARTS];
      operands<ACT>(r, at < a.K, p);
#pragma unroll
      for (int q = 0; q < PARTS; q++) *(bf16x8*)(split + (m * PARTS + q) * Kp + at) = p[q];
    }
    __syncthreads();
  }
  for (int m0 = 0; m0 < n_mine; m0 += 16) {
    const int slot = a.T == 1 ? s0 : slots[min(m0 + c, n_mine - 1)];
    const size_t xrow = (size_t)(a.x_slots ? slot : slot / a.k) * a.K;
    f32x4 acc[RT];
#pragma unroll
    for (int t = 0; t < RT; t++) acc[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    for (int u = wave; u < units; u += MV_WAVES) {
      const int bc = min(u * 4 + g, nb - 1);
      RawX<ACT> x[4];
      if (!shared) {
#pragma unroll
        for (int s = 0; s < 4; s++)
#pragma unroll
          for (int v = 0; v < (ACT == SMOE_F32 ? 2 : 1); v++)
            x[s].v[v] = *(const u32x4*)((const uint8_t*)a.x + (xrow + (size_t)bc * 32 + s * 8) * (ACT == SMOE_F32 ? 4 : 2) + v * 16);
      }
      const bool ok = u * 4 + g < nb;                         // a block that does not exist: activations 0, scale 1
      float sc[RT];
#pragma unroll
      for (int t = 0; t < RT; t++) sc[t] = ok ? mx_scale(sb[t]) : 1.0f;
#pragma unroll
      for (int s = 0; s < 4; s++) {
        bf16x8 p[PARTS];
        if (shared) {
#pragma unroll
          for (int m = 0; m < PARTS; m++) p[m] = *(const bf16x8*)(split + (min(c, n_mine - 1) * PARTS + m) * Kp + (u * 4 + g) * 32 + s * 8);
        } else {
          operands<ACT>(x[s], ok, p);
        }
#pragma unroll
        for (int t = 0; t < RT; t++) {
          const uint32_t q = w[t][s];
          union { bf16x2 h[4]; bf16x8 v; } wf;
          wf.h[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q, sc[t], 0);
          wf.h[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q, sc[t], 1);
          wf.h[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q, sc[t], 2);
          wf.h[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q, sc[t], 3);
#pragma unroll
          for (int m = PARTS - 1; m >= 0; m--) acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf.v, p[m], acc[t], 0, 0, 0);
        }
      }
      if (u + MV_WAVES < units || m0 + 16 < n_mine) fetch(u + MV_WAVES < units ? u + MV_WAVES : wave);
    }
    if (shared) __syncthreads();
#pragma unroll
    for (int t = 0; t < RT; t++)
#pragma unroll
      for (int i = 0; i < 4; i++) part[wave][16 * t + 4 * g + i][c] = acc[t][i];
    __syncthreads();
    const int rows = a.swiglu ? ROWS / 2 : ROWS, cols = min(16, n_mine - m0);
    for (int i = tid; i < rows * cols; i += 64 * MV_WAVES) {
      const int rr = i % rows, cc = i / rows;
      auto sum = [&](int r) {
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < MV_WAVES; w++) s += part[w][r][cc];
        return s;
      };
      const size_t yrow = (size_t)(a.T == 1 ? s0 : slots[m0 + cc]);
      if (a.swiglu) {
        if (r0 + 2 * rr < a.N) store1<ACT>(a.y, yrow * (a.N >> 1) + (r0 >> 1) + rr, swiglu(sum(2 * rr), sum(2 * rr + 1)));
      } else {
        if (r0 + rr < a.N) store1<ACT>(a.y, yrow * a.N + r0 + rr, sum(rr));
      }
    }
    __syncthreads();
  }
}

template <int ACT, int RT, int MV_WAVES> static void launch_matvec(smoe_ctx* ctx, const MatvecArgs& a) {
  const dim3 grid((a.N + 16 * RT - 1) / (16 * RT), !a.idx ? 1 : a.by_expert ? a.E : a.T * a.k);
  mx_matvec_kernel<ACT, RT, MV_WAVES><<<grid, 64 * MV_WAVES, 0, ctx->stream>>>(a);
}

extern "C" int smoe_mx_matvec(smoe_ctx* ctx, int E, int N, int K, const uint8_t* w_codes_dev, const uint8_t* w_scales_dev, int T, int k,
                              const void* x_dev, int act_dtype, int x_slots, const int32_t* idx_dev, int swiglu, void* y_dev) {
  if (!ctx || (act_dtype != SMOE_F32 && act_dtype != SMOE_BF16) || (x_slots != 0 && x_slots != 1) || (swiglu != 0 && swiglu != 1)) return SMOE_EINVAL;
  if (E <= 0 || E > SMOE_MAX_EXPERTS || T < 0 || T > SMOE_MAX_MULTI || k <= 0 || k > SMOE_MAX_TOPK) return SMOE_ESHAPE;
  if (const int rc = check_mx_matrix(N, K)) return rc;
  if (T == 0) return SMOE_OK;
  if (!idx_dev && (E != 1 || k != 1)) return SMOE_ESHAPE;
  if (!w_codes_dev || !w_scales_dev || !x_dev || !y_dev || x_dev == y_dev) return SMOE_EINVAL;
  if (!aligned16(w_codes_dev) || !aligned16(w_scales_dev) || !aligned16(x_dev) || !aligned16(idx_dev) || !aligned16(y_dev)) return SMOE_EALIGN;
  ON_DEVICE_OF(ctx);
  const MatvecArgs a{w_codes_dev, w_scales_dev, x_dev, idx_dev, y_dev, E, N, K, T, k, x_slots, swiglu, T > 1 && E < T * k};
  // Rows of a work-group.  Four tiles share one fetch and one splitting of the activations between four waves, one unit of columns in flight each, so that many
  // work-groups fit a CU; where that leaves too few work-groups, one tile and eight waves.  Microseconds with four tiles / with one, K 2048, by work-groups of four:
  //   fp32   dense 32: 16 tokens 10.9 / 7.4; dense 128: 1 token 9.2 / 8.7, 4 tokens 11.0 / 8.8, 16 tokens 11.9 / 12.3 (K 8192, 1 token: 33.7 / 24.1); dense 256: 1 token 10.0 / 14.7;
  //          top-6 of 64, 264: 1 token 11.5 / 16.6; 2048 (K 1408): 16 tokens 28.6 / 64.5
  //   bf16   dense 128: 16 tokens 8.9 / 8.3; dense 256: 1 token 8.6 / 8.6, 4 tokens 8.4 / 9.7, 16 tokens 9.4 / 13.6; dense 512: 1 token 11.9 / 14.4, 4 tokens 12.8 / 16.1;
  //          top-6 of 64, 264: 1 token 10.9 / 9.3, 4 tokens 10.6 / 8.9; 528: 1 token 14.7 / 14.3; top-4 of 60, 704: 4 tokens 15.6 / 18.3; 2048 (K 1408): 16 tokens 21.9 / 32.8
  // The limit in fp32 is somewhat low for long rows and few tokens, that of bf16 somewhat high for a dense matrix.
  const long long wgs = (long long)((N + 63) / 64) * (!idx_dev ? 1 : T * k < E ? T * k : E);
  if (act_dtype == SMOE_F32) {
    if (wgs < 128) launch_matvec<SMOE_F32, 1, 8>(ctx, a);
    else launch_matvec<SMOE_F32, 4, 4>(ctx, a);
  } else {
    if (wgs < (T > 4 ? 256 : 512)) launch_matvec<SMOE_BF16, 1, 8>(ctx, a);
    else launch_matvec<SMOE_BF16, 4, 4>(ctx, a);
  }
  HIPCHK(ctx, hipGetLastError());
  return SMOE_OK;
}
