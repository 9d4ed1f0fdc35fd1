// FP8 E4M3 codes of float32 values, for the kernels that write an FP8 cache.
#pragma once

#include "attn_common.hpp"

namespace rl {

// OCP E4M3 code of a float32 value, from the format's bit layout: nearest
// value, ties to the even code; magnitudes of 448 and above (infinity
// included) saturate to 448; NaN gives the NaN code. The sign is kept.
__device__ __forceinline__ uint32_t e4m3_from_f32(float f) {
  const uint32_t u = __float_as_uint(f);
  const uint32_t sign = (u >> 24) & 0x80u;
  const uint32_t a = u & 0x7FFFFFFFu;
  uint32_t code;
  if (a > 0x7F800000u) {
    code = 0x7Fu;                                   // NaN
  } else if (a >= 0x43E00000u) {
    code = 0x7Eu;                                   // >= 448: saturate
  } else if (a < 0x3C800000u) {
    // below 2^-6: the subnormal step is 2^-9, so the code is the value in
    // steps, rounded to nearest even (8 is the smallest normal, code 0x08)
    code = (uint32_t)__builtin_rintf(__uint_as_float(a) * 512.f);
  } else {
    const uint32_t e = (a >> 23) - 127u + 7u;       // biased E4M3 exponent, 1..15
    uint32_t r = (a >> 20) & 7u;                    // top three mantissa bits
    const uint32_t rest = a & 0xFFFFFu;
    if (rest > 0x80000u || (rest == 0x80000u && (r & 1u))) ++r;
    code = (e << 3) + r;                            // r == 8 carries into the exponent
    if (code > 0x7Eu) code = 0x7Eu;
  }
  return code | sign;
}

// E4M3 codes of eight float32 values divided by the positive scale s (inv: the
// correctly rounded 1/s), four per word. The code is the E4M3 value nearest
// to the correctly rounded float32 quotient. Fast path: q0 = x * inv, then
// one residual correction q0 + (x - q0 s) inv, which is the correctly rounded
// quotient for normal results (Markstein's theorem: the residual is exact in
// an FMA and the reciprocal is correctly rounded); subnormal quotients, where
// it may be off, all encode to zero, and the sign is taken from x so that -0
// stays -0. The clamped value is then converted by the hardware E4M3
// conversion (round to nearest even), which matches the format's definition
// on every input in that range. Non-finite inputs, or a product that
// overflows, take the IEEE division and the bit-level encoder instead.
__device__ __forceinline__ uint2 e4m3_pack8(const float (&x)[8], float s, float inv) {
  float q[8];
  bool special = false;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float xf = x[e];
    const float q0 = xf * inv;
    const float r = __builtin_fmaf(-q0, s, xf);
    q[e] = __builtin_copysignf(__builtin_fmaf(r, inv, q0), xf);
    special |= (__float_as_uint(q0) & 0x7F800000u) == 0x7F800000u;
  }
  uint2 w;
  if (!special) {
    auto c = [&](int e) { return __builtin_amdgcn_fmed3f(q[e], -448.f, 448.f); };
    w.x = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c(0), c(1), 0, false);
    w.x = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c(2), c(3), (int)w.x, true);
    w.y = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c(4), c(5), 0, false);
    w.y = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c(6), c(7), (int)w.y, true);
  } else {
    w.x = w.y = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t code = e4m3_from_f32(x[e] / s);
      if (e < 4) w.x |= code << (8 * e); else w.y |= code << (8 * (e - 4));
    }
  }
  return w;
}
// (bf16 rows)
__device__ __forceinline__ uint2 e4m3_pack8(const bf16x8& x, float s, float inv) {
  float f[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = (float)x[e];
  return e4m3_pack8(f, s, inv);
}

}  // namespace rl
