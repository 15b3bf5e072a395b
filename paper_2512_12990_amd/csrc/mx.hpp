// Microscaled 4-bit floats: what quantiser and products share.
//
// A row of K numbers is K / 2 bytes of codes (two e2m1 codes a byte, the even column in the low nibble) and K / 32 bytes
// of scales: a block of 32 columns is 16 bytes of codes and one e8m0 byte X + 127, X the block's power of two.  e2m1:
// sign, then 0 .5 1 1.5 2 3 4 6.  Scale byte 255 makes its block NaN.
#pragma once
#include "common.hpp"

// 2^X as a float; X = -127 is a subnormal
__device__ __forceinline__ float mx_scale(uint32_t byte) {
  const uint32_t u = byte == 0 ? 0x00400000u : byte == 255 ? 0x7FC00000u : byte << 23;
  return __uint_as_float(u);
}

// silu(g) * u for gates from -76 on.  e^-g = 2^(t + r), t = -g log2 e rounded and r what that rounding left, so that the exponential keeps its last
// bits at any g; the limits of +-200 keep infinities out of r.  Off by at most 9 half steps: exponential 4, sum 1,
// reciprocal 2, two products 2.
#define SWIGLU_FAR -76.0f
__device__ __forceinline__ float swiglu_near(float g, float u) {
  const float x = __builtin_amdgcn_fmed3f(-g, -200.0f, 200.0f);
  const float t = x * 1.44269502f, r = fmaf(x, 1.92596299e-8f, fmaf(x, 1.44269502f, -t));
  const float e = __builtin_amdgcn_exp2f(t) * fmaf(r, 0.693147182f, 1.0f);
  return g * __builtin_amdgcn_rcpf(1.0f + e) * u;
}
// For any gate.  Below -76 1 + e^-g is e^-g to the last bit but may pass fp32, and its reciprocal may be subnormal, where a large u still makes a normal
// number of it: there m = 2^160 e^g stands for the quotient, and 2^-160 comes in two halves with u (which only a result of less than the smallest
// subnormal can make subnormal).  Past the limit of -220 m is 0, and so is the result at any u (2^-317 * 2^128).  Off by fewer half steps, and by a
// subnormal's step.
__device__ __forceinline__ float swiglu(float g, float u) {
  if (!(g < SWIGLU_FAR)) return swiglu_near(g, u);
  const float x = fmaxf(g, -220.0f);
  float t, at;
  {
#pragma clang fp contract(off)
    t = x * 1.44269502f;
    at = t + 160.0f;                                         // (exact; from x itself r would not be what is left)
  }
  const float r = fmaf(x, 1.92596299e-8f, fmaf(x, 1.44269502f, -t));
  const float m = __builtin_amdgcn_exp2f(at) * fmaf(r, 0.693147182f, 1.0f);
  return u * 0x1p-80f * (g * m) * 0x1p-80f;
}

// one expert's matrix [N, K]: byte offsets inside it stay below 2^31
static inline int check_mx_matrix(int N, int K) {
  if (N <= 0 || N % 16 || N > (1 << 20) || K <= 0 || K % 32 || K > (1 << 16) || (long long)N * (K / 2) >= (1ll << 31)) return SMOE_ESHAPE;
  return SMOE_OK;
}
