// Blocks of 128 elements as e4m3 values with one scale: q = round(x * 448 / m), scale = m / 448, m = max |x| of the block.
//
// The quotient has to be the true one rounded once: bf16 elements often lie halfway between two e4m3 values (x * 448 / m with
// m a power of two, say), and a quotient that is off in its last bit sends such an element to the other neighbour.  With
// a = 448 x and b = m, both scaled by a power of two, a and b have 11 and 8 significant bits, so a / b is either a
// midpoint exactly or further from it than 2^-14 relative; t = a * (1 / b) with one residual step t + (a - t b) / b is within
// 2^-44 of it before its last rounding, which a midpoint (5 bits) survives unchanged.  Four instructions an element and one
// reciprocal a block.
#pragma once

#include <cuda_fp8.h>

#include "eb_internal.cuh"

namespace {

constexpr float kE4M3Max = 448.f;

struct BlockScale {
  float mul, b, inv;   // a = x * mul; a / b by inv
  float scale;         // m / 448; NaN if the block holds an infinity or NaN, so that all that is made from it is NaN
};

// m16: the largest |x| of the block as bf16 bits
__device__ __forceinline__ BlockScale block_scale(unsigned m16) {
  const float m = __uint_as_float(m16 << 16);
  // power of two that brings m near 1: exponent 254 - e, kept where neither it nor 448 times it leaves the normal range
  const int e = (int)(m16 >> 7), fe = min(max(254 - e, 1), 237);
  const float f = __uint_as_float((unsigned)fe << 23);
  BlockScale s;
  s.mul = kE4M3Max * f;
  s.b = m * f;
  s.inv = m16 ? __frcp_rn(s.b) : 0.f;
  s.scale = e == 255 ? __uint_as_float(0x7fc00000u) : __fdiv_rn(m, kE4M3Max);
  return s;
}
__device__ __forceinline__ float block_quotient(const BlockScale& s, float x) {
  const float a = x * s.mul, t = a * s.inv;
  return fmaf(fmaf(-t, s.b, a), s.inv, t);
}
__device__ __forceinline__ unsigned pack_e4m3(float lo, float hi) {
  return (unsigned)__nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ float low_bf16(unsigned v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float high_bf16(unsigned v) { return __uint_as_float(v & 0xffff0000u); }

// largest |x| of the eight bf16 elements of a vector, as bf16 bits
__device__ __forceinline__ unsigned abs_max8(const uint4& v) {
  const unsigned k = 0x7fff7fffu;
  const unsigned m = __vmaxu2(__vmaxu2(v.x & k, v.y & k), __vmaxu2(v.z & k, v.w & k));
  return max(m & 0xffffu, m >> 16);
}
// eight elements to eight e4m3 values
__device__ __forceinline__ uint2 quantise8(const BlockScale& s, const uint4& v) {
  uint2 q;
  q.x = pack_e4m3(block_quotient(s, low_bf16(v.x)), block_quotient(s, high_bf16(v.x))) |
        pack_e4m3(block_quotient(s, low_bf16(v.y)), block_quotient(s, high_bf16(v.y))) << 16;
  q.y = pack_e4m3(block_quotient(s, low_bf16(v.z)), block_quotient(s, high_bf16(v.z))) |
        pack_e4m3(block_quotient(s, low_bf16(v.w)), block_quotient(s, high_bf16(v.w))) << 16;
  return q;
}
// The scale of a block whose sixteen vectors lie in sixteen neighbouring lanes (`lanes` 8: rows of one block at most, in eight).  Whole
// warps call it; lanes without elements hold zeros.
__device__ __forceinline__ BlockScale warp_block_scale(const uint4& v, int lanes) {
  unsigned m = abs_max8(v);
  if (lanes > 8) m = max(m, __shfl_xor_sync(0xffffffffu, m, 8));
#pragma unroll
  for (int o = 4; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
  return block_scale(m);
}

}  // namespace
