// Rotary positions: each pair of a query or key row's rotated dimensions turns
// by its frequency times the row's position on the frequency's axis (time,
// height, width; one axis for text). Alone (q and k rows to rows), or in one
// pass with the KV append: rotated keys and the values go straight to their
// slots in the pages, as bf16 or as E4M3 codes of the quotient by the KV
// head's scale, so keys are not written as rows and read again.
//
// The angle is formed in 64 bits (in 32 a position of 60,000 would leave 12
// bits behind the point, 2e-3 rad at the fastest frequency), reduced to an
// eighth of a turn there, and its sine and cosine are Taylor polynomials in 32
// bits: a wave does the frequencies of a row at once, one a lane, and the
// row's heads share them through LDS. A row is rounded once, from 32 bits to
// what is stored.
//
// The pass is a copy with a few multiplies: HBM-bound at 2 x 256 bytes a head
// row. A thread holds two 8-element chunks that the rotation maps onto
// themselves (dimensions i and freqs + i, or 16 neighbours), which is why the
// outputs may be the inputs.
#include "attn_common.hpp"
#include "e4m3.hpp"
#include "kernels.hpp"

namespace rl {

namespace {

constexpr int kRopeThreads = 256;
constexpr int kRopeRows = 4;                        // rows of a workgroup: one a wave for the angles
constexpr int kRopeHeads = kRopeThreads / 8;        // head rows of a step (8 threads each)

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

// cs: cos and sin of the duplet's eight frequencies
__device__ __forceinline__ void turn(f32x8& a, f32x8& b, const float2 (&cs)[8], bool interleaved) {
  if (interleaved) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      f32x8& x = e < 4 ? a : b;
      const int i = 2 * (e & 3);
      const float u = x[i], w = x[i + 1];
      x[i] = u * cs[e].x - w * cs[e].y;
      x[i + 1] = w * cs[e].x + u * cs[e].y;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float u = a[e], w = b[e];
      a[e] = u * cs[e].x - w * cs[e].y;
      b[e] = w * cs[e].x + u * cs[e].y;
    }
  }
}

template <bool kAppend, bool kFp8>
__global__ __launch_bounds__(kRopeThreads) void rope_kernel(RopeArgs a) {
  __shared__ float2 cs[kRopeRows][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int row0 = blockIdx.x * kRopeRows;
  const int n = min(kRopeRows, a.rows - row0);
  if (wave < n && lane < a.freqs) {
    int axis = a.axes ? a.axes[(int64_t)lane * a.axes_s] : 0;
    if ((unsigned)axis >= (unsigned)a.n_axes) {
      atomicOr(a.err, kErrAxis);
      axis = axis < 0 ? 0 : a.n_axes - 1;
    }
    const int p = a.pos[(int64_t)axis * a.pos_sa + (int64_t)(row0 + wave) * a.pos_st];
    const double f = (double)a.inv_freq[(int64_t)lane * a.freq_s] * (a.inverse ? -1.0 : 1.0);
    cs[wave][lane] = cos_sin_turns((double)p * f * 0.15915494309189533577);
  }
  __syncthreads();
  const int per_row = a.Hq + (kAppend ? 2 : 1) * a.Hkv;
  const int d = threadIdx.x & 7;
  const Chunks turned = chunks_of(d, a.freqs, a.interleaved), plain = chunks_of(d, 0, false);
  for (int i = threadIdx.x >> 3; i < n * per_row; i += kRopeHeads) {
    const int w = i / per_row, h = i - w * per_row;
    const int64_t r = row0 + w;
    int64_t slot = 0;
    if constexpr (kAppend) {
      slot = a.slots[r * a.slots_s];
      if (slot < 0) continue;                       // a row behind the last request's: nothing of it is touched
    }
    const bool is_v = kAppend && h >= a.Hq + a.Hkv;
    const bool is_k = !is_v && h >= a.Hq;
    const int g = h - a.Hq - (is_v ? a.Hkv : 0);    // KV head
    const Chunks c = is_v ? plain : turned;
    const __bf16* src = is_v   ? (const __bf16*)a.v + r * a.v_st + g * a.v_sh
                        : is_k ? (const __bf16*)a.k + r * a.k_st + g * a.k_sh
                               : (const __bf16*)a.q + r * a.q_st + h * a.q_sh;
    const bf16x8 xa = load_nt<bf16x8>(src + c.lo), xb = load_nt<bf16x8>(src + c.hi);
    f32x8 fa = widen(xa), fb = widen(xb);
    if (c.turned) {
      float2 t[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) t[e] = cs[w][8 * d + e];
      turn(fa, fb, t, a.interleaved);
    }
    if (!is_v && (!is_k || a.k_out)) {
      __bf16* dst = is_k ? (__bf16*)a.k_out + r * a.ko_st + g * a.ko_sh : (__bf16*)a.q_out + r * a.qo_st + h * a.qo_sh;
      *reinterpret_cast<bf16x8*>(dst + c.lo) = narrow(fa);
      *reinterpret_cast<bf16x8*>(dst + c.hi) = narrow(fb);
    }
    if constexpr (kAppend) {
      if (!is_v && !is_k) continue;
      const int64_t page = slot >> a.log2_page;
      if (page >= a.num_pages) {                    // never write outside the pool
        atomicOr(a.err, kErrSlot);
        continue;
      }
      const int in_page = (int)(slot & (a.page_size - 1));
      const int64_t at = is_v ? page * a.vp_sp + in_page * a.vp_ss + g * a.vp_sh
                              : page * a.kp_sp + in_page * a.kp_ss + g * a.kp_sh;
      if constexpr (!kFp8) {
        __bf16* dst = (__bf16*)(is_v ? a.v_pages : a.k_pages) + at;
        *reinterpret_cast<bf16x8*>(dst + c.lo) = is_v ? xa : narrow(fa);
        *reinterpret_cast<bf16x8*>(dst + c.hi) = is_v ? xb : narrow(fb);
      } else {
        const float s = is_v ? a.v_scale[g * a.vs_s] : a.k_scale[g * a.ks_s];
        if (!scale_ok(s)) {
          atomicOr(a.err, kErrScale);
          continue;
        }
        uint8_t* dst = (uint8_t*)(is_v ? a.v_pages : a.k_pages) + at;
        const float inv = 1.0f / s;
        *reinterpret_cast<uint2*>(dst + c.lo) = codes(fa, s, inv);
        *reinterpret_cast<uint2*>(dst + c.hi) = codes(fb, s, inv);
      }
    }
  }
}

}  // namespace

hipError_t launch_rope(const RopeArgs& a, hipStream_t stream, KernelTimer* timer) {
  const unsigned grid = (unsigned)((a.rows + kRopeRows - 1) / kRopeRows);
  if (timer) (void)hipEventRecord(timer->start, stream);
  if (!a.slots)
    rope_kernel<false, false><<<grid, kRopeThreads, 0, stream>>>(a);
  else if (!a.k_scale)
    rope_kernel<true, false><<<grid, kRopeThreads, 0, stream>>>(a);
  else
    rope_kernel<true, true><<<grid, kRopeThreads, 0, stream>>>(a);
  if (timer) (void)hipEventRecord(timer->stop, stream);
  return hipGetLastError();
}

}  // namespace rl
