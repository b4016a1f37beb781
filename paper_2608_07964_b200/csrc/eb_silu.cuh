// The activation of the 8-bit expert kernels, whose results are scaled by the largest of their block: each has to be right to its own size.
#pragma once

namespace {

__device__ __forceinline__ float exp2f_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rcp_approx(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// silu(g) * u for two values.  With e = exp(-|g|), at most 1, silu(g) = max(g, g e) / (1 + e): g / (1 + e) from 0 on, g e / (1 + e) below.  So
// nothing is made that is larger than g before u comes in, and silu falls with e to 0 (e below 2^-126 counts as 0: g below -87.3).
// Not by tanh.approx: its 2^-11 would send one value in a hundred to the other e4m3 neighbour; this is within (|g| + 3) 2^-22 of its size.
// The special function unit bounds the epilogue of a tile, so two quotients share one reciprocal: of the product of two numbers from 1 to 2.
// A gate that is NaN is taken out of its e by the maximum, and stays in its own result.
__device__ __forceinline__ void silu_mul2(float g0, float u0, float g1, float u1, float* h0, float* h1) {
  const float e0 = exp2f_approx(fmaxf(fabsf(g0) * -1.442695041f, -150.f)), e1 = exp2f_approx(fmaxf(fabsf(g1) * -1.442695041f, -150.f));
  const float d0 = 1.f + e0, d1 = 1.f + e1, r = rcp_approx(d0 * d1);
  *h0 = fmaxf(g0, g0 * e0) * (r * d1) * u0;
  *h1 = fmaxf(g1, g1 * e1) * (r * d0) * u1;
}

}  // namespace
