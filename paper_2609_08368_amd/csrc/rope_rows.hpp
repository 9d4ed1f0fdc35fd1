// Head rows as the rotary kernels hold them: angles, chunks and what turns them.
#pragma once

#include "attn_common.hpp"
#include "e4m3.hpp"

namespace rl {

// cos and sin of 2 pi t for t in turns, any size: t is reduced in 64 bits to
// x in [-1/8, 1/8] turns around a quarter k, and |2 pi x| <= pi/4 leaves the
// first dropped Taylor terms below 2e-9 (sine) and 2e-9 (cosine).
__device__ __forceinline__ float2 cos_sin_turns(double t) {
  const double r = t - __builtin_rint(t);           // [-1/2, 1/2]
  const double k4 = __builtin_rint(4.0 * r);        // quarter, -2..2
  const float y = (float)((r - 0.25 * k4) * 6.283185307179586476925);
  const int k = (int)k4 & 3;
  const float z = y * y;
  const float s = y * fmaf(z, fmaf(z, fmaf(z, fmaf(z, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), 1.f);
  const float c = fmaf(
      z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
  const float a = (k & 1) ? s : c, b = (k & 1) ? c : s;
  // quarter 0: (c, s), 1: (-s, c), 2: (-c, -s), 3: (s, -c)
  return {(k == 1 || k == 2) ? -a : a, (k >= 2) ? -b : b};
}

typedef float f32x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ f32x8 widen(bf16x8 x) {
  f32x8 y;
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] = (float)x[e];
  return y;
}
__device__ __forceinline__ bf16x8 narrow(f32x8 x) {
  bf16x8 y;
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] = (__bf16)x[e];
  return y;
}
__device__ __forceinline__ uint2 codes(f32x8 x, float s, float inv) {
  float f[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = x[e];
  return e4m3_pack8(f, s, inv);
}

// First elements of the two chunks of duplet d: with F frequencies, duplets
// below F / 8 are rotated, the others hold 16 neighbours behind them.
struct Chunks {
  int lo, hi;
  bool turned;
};
__device__ __forceinline__ Chunks chunks_of(int d, int F, bool interleaved) {
  const bool turned = 8 * d < F;
  if (turned && !interleaved) return {8 * d, F + 8 * d, true};
  return {16 * d, 16 * d + 8, turned};
}

// cs: cos and sin of the duplet's eight frequencies. (x cos a - y sin a, y cos a +
// x sin a), with the fused products written out: left to the compiler they differ
// between the kernels, and a row's bits with the size of its call.
__device__ __forceinline__ void turn_pair(float& x, float& y, float2 cs) {
  const float u = x, w = y;
  x = fmaf(u, cs.x, -(w * cs.y));
  y = fmaf(w, cs.x, u * cs.y);
}
__device__ __forceinline__ void turn(f32x8& a, f32x8& b, const float2 (&cs)[8], bool interleaved) {
  if (interleaved) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      f32x8& z = e < 4 ? a : b;
      const int i = 2 * (e & 3);
      float x = z[i], y = z[i + 1];
      turn_pair(x, y, cs[e]);
      z[i] = x;
      z[i + 1] = y;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float x = a[e], y = b[e];
      turn_pair(x, y, cs[e]);
      a[e] = x;
      b[e] = y;
    }
  }
}

template <bool kNt, typename T>
__device__ __forceinline__ void store_chunk(void* dst, T x) {
  typedef unsigned int words __attribute__((ext_vector_type(sizeof(T) / 4)));
  if constexpr (kNt)
    __builtin_nontemporal_store(__builtin_bit_cast(words, x), static_cast<words*>(dst));
  else
    *static_cast<words*>(dst) = __builtin_bit_cast(words, x);
}


// Mean square of a head row held by eight neighbouring lanes, 16 elements each; all
// of them receive it. The sum's order is written out: a row's bits are the same in
// every kernel.
__device__ __forceinline__ float row_sum8(float v) {
  v += dpp<kDppXor1>(v);
  v += dpp<kDppXor2>(v);
  return v + dpp<kDppHalfMirror>(v);
}
__device__ __forceinline__ float dot16(f32x8 a, f32x8 b, f32x8 c, f32x8 d) {   // a.b + c.d
  float s = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) s = fmaf(a[e], b[e], s);
#pragma unroll
  for (int e = 0; e < 8; ++e) s = fmaf(c[e], d[e], s);
  return s;
}
__device__ __forceinline__ float inv_rms(f32x8 a, f32x8 b, float eps) {
  return __builtin_amdgcn_rsqf(fmaf(row_sum8(dot16(a, a, b, b)), 1.f / kHeadDim, eps));
}

// Eight of a norm's weights from dimension i on.
__device__ __forceinline__ f32x8 load_weights(const void* w, int i, bool f32) {
  if (!f32) return widen(*reinterpret_cast<const bf16x8*>(static_cast<const __bf16*>(w) + i));
  typedef f32x8 f32x8_of16 __attribute__((aligned(16)));
  return *reinterpret_cast<const f32x8_of16*>(static_cast<const float*>(w) + i);
}

}  // namespace rl
