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
// bits: a wave does the frequencies of its row at once, one a lane, and each
// lane takes its eight from LDS. A row is rounded once, from 32 bits to what
// is stored.
//
// The pass is a copy with a few multiplies: HBM-bound at 2 x 256 bytes a head
// row. A thread holds two 8-element chunks that the rotation maps onto
// themselves (dimensions i and freqs + i, or 16 neighbours), which is why the
// outputs may be the inputs; eight threads have a head row.
//
// A wave takes 8 or 16 head rows of one row, which repeats the angles for
// every part of a row, but keeps the reads of neighbouring waves together.
// 32768 rows of 64 + 8 + 8 heads into bf16 pages took 260 us with a whole row a
// wave, 242 with 16 head rows and 222 with those stored nontemporally (6.0
// TB/s; a large copy runs at 4.9), 208 into FP8 pages. A call whose parts of 8
// heads all fit the device at once is bound by its launch, its loads' latency
// and the angles: 128 rows of 96 + 8 + 8 heads take 4.3 us (13.0 with four
// rows a workgroup, 5.6 with parts of 16).
//
// The nontemporal stores are for a call's own time, and the attention that reads
// its rows next pays for them: 2500 rows of 64 + 8 + 8 heads take 19.1 us (20.8
// with ordinary stores) but 69.6 together with the prefill behind them (66.7),
// 8000 rows 56.8 (53.5) and 182 (177), 36000 rows 258 (269) and 805 (791).
#include <algorithm>
#include <type_traits>

#include "attn_common.hpp"
#include "e4m3.hpp"
#include "kernels.hpp"

namespace rl {

namespace {

constexpr int kRopeThreads = 256;
constexpr int kWavesPerCu = 32;                     // that fit at once

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

// A wave has eight head rows of a row (kLarge: sixteen, stored nontemporally),
// which it loads before it forms the row's angles.
template <bool kAppend, bool kFp8, bool kLarge>
__global__ __launch_bounds__(kRopeThreads) void rope_kernel(RopeArgs a) {
  constexpr int kBatch = kLarge ? 2 : 1;            // eights of head rows
  __shared__ __attribute__((aligned(16))) float2 cs[kRopeThreads / 64][64];
  const int lane = threadIdx.x & 63, d = lane & 7;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int unit = blockIdx.x * (kRopeThreads / 64) + wave;
  const int r32 = unit / a.parts;
  if (r32 >= a.rows) return;                        // (no barrier follows: a wave is alone)
  const int64_t r = r32;
  const int per_row = a.Hq + (kAppend ? 2 : 1) * a.Hkv;
  const int h0 = (unit - r32 * a.parts) * (8 * kBatch) + (lane >> 3);
  const Chunks turned = chunks_of(d, a.freqs, a.interleaved), plain = chunks_of(d, 0, false);
  // position of this lane's axis and frequency of this lane: the axis picks the lane
  const int at = a.pos[(int64_t)min(lane, a.n_axes - 1) * a.pos_sa + r * a.pos_st];
  const int f = min(lane, a.freqs - 1);
  const float freq = a.inv_freq[(int64_t)f * a.freq_s];
  int axis = a.axes ? a.axes[(int64_t)f * a.axes_s] : 0;
  int64_t slot = 0;
  if constexpr (kAppend) slot = a.slots[r * a.slots_s];

  enum { kQ, kK, kV };
  auto kind_of = [&](int h) { return h < a.Hq ? kQ : !kAppend || h < a.Hq + a.Hkv ? kK : kV; };
  bf16x8 xa[kBatch], xb[kBatch];
#pragma unroll
  for (int i = 0; i < kBatch; ++i) {
    const int h = h0 + 8 * i;
    if (h >= per_row) continue;
    const int kind = kind_of(h);
    const __bf16* src = kind == kQ   ? (const __bf16*)a.q + r * a.q_st + h * a.q_sh
                        : kind == kK ? (const __bf16*)a.k + r * a.k_st + (h - a.Hq) * a.k_sh
                                     : (const __bf16*)a.v + r * a.v_st + (h - a.Hq - a.Hkv) * a.v_sh;
    xa[i] = load_nt<bf16x8>(src + (kind == kV ? plain.lo : turned.lo));
    xb[i] = load_nt<bf16x8>(src + (kind == kV ? plain.hi : turned.hi));
  }

  if ((unsigned)axis >= (unsigned)a.n_axes) {
    atomicOr(a.err, kErrAxis);
    axis = axis < 0 ? 0 : a.n_axes - 1;
  }
  const int p = __shfl(at, axis);
  cs[wave][lane] = cos_sin_turns((double)p * ((double)freq * (a.inverse ? -1.0 : 1.0)) * 0.15915494309189533577);
  __builtin_amdgcn_wave_barrier();
  float2 t[8];                                      // of this lane's frequencies
#pragma unroll
  for (int e = 0; e < 8; ++e) t[e] = cs[wave][8 * d + e];
  int64_t kat = 0, vat = 0;                         // the slot's places in the pages
  bool in_pool = false;
  if constexpr (kAppend) {
    if (slot < 0) return;                           // a row behind the last request's: nothing of it is written
    const int64_t page = slot >> a.log2_page;
    const int in_page = (int)(slot & (a.page_size - 1));
    in_pool = page < a.num_pages;                   // never write outside the pool
    if (!in_pool) atomicOr(a.err, kErrSlot);
    kat = page * a.kp_sp + in_page * a.kp_ss;
    vat = page * a.vp_sp + in_page * a.vp_ss;
  }
#pragma unroll
  for (int i = 0; i < kBatch; ++i) {
    const int h = h0 + 8 * i;
    if (h >= per_row) continue;
    const int kind = kind_of(h), g = h - a.Hq - (kind == kV ? a.Hkv : 0);   // g: KV head
    const Chunks c = kind == kV ? plain : turned;
    f32x8 fa = widen(xa[i]), fb = widen(xb[i]);
    if (c.turned) turn(fa, fb, t, a.interleaved);
    if (kind == kQ || (kind == kK && a.k_out)) {
      __bf16* dst = kind == kK ? (__bf16*)a.k_out + r * a.ko_st + g * a.ko_sh
                               : (__bf16*)a.q_out + r * a.qo_st + h * a.qo_sh;
      store_chunk<kLarge>(dst + c.lo, narrow(fa));
      store_chunk<kLarge>(dst + c.hi, narrow(fb));
    }
    if constexpr (kAppend) {
      if (kind == kQ || !in_pool) continue;
      const int64_t at = kind == kV ? vat + g * a.vp_sh : kat + g * a.kp_sh;
      if constexpr (!kFp8) {
        __bf16* dst = (__bf16*)(kind == kV ? a.v_pages : a.k_pages) + at;
        store_chunk<kLarge>(dst + c.lo, kind == kV ? xa[i] : narrow(fa));
        store_chunk<kLarge>(dst + c.hi, kind == kV ? xb[i] : narrow(fb));
      } else {
        const float s = kind == kV ? a.v_scale[g * a.vs_s] : a.k_scale[g * a.ks_s];
        if (!scale_ok(s)) {
          atomicOr(a.err, kErrScale);
          continue;
        }
        uint8_t* dst = (uint8_t*)(kind == kV ? a.v_pages : a.k_pages) + at;
        const float inv = 1.0f / s;
        store_chunk<kLarge>(dst + c.lo, codes(fa, s, inv));
        store_chunk<kLarge>(dst + c.hi, codes(fb, s, inv));
      }
    }
  }
}

}  // namespace

hipError_t launch_rope(const RopeArgs& args, int cus, hipStream_t stream, KernelTimer* timer) {
  RopeArgs a = args;
  // parts of 8 heads if all of them fit at once (see the top)
  const int64_t eights = (a.Hq + (a.slots ? 2 : 1) * a.Hkv + 7) / 8;
  const bool large = a.rows * eights > (int64_t)kWavesPerCu * cus;
  a.parts = (int)(large ? (eights + 1) / 2 : eights);
  const unsigned grid = (unsigned)(((int64_t)a.rows * a.parts + kRopeThreads / 64 - 1) / (kRopeThreads / 64));
  auto run = [&](auto append, auto fp8) {
    if (large)
      rope_kernel<append, fp8, true><<<grid, kRopeThreads, 0, stream>>>(a);
    else
      rope_kernel<append, fp8, false><<<grid, kRopeThreads, 0, stream>>>(a);
  };
  if (timer) (void)hipEventRecord(timer->start, stream);
  if (!a.slots)
    run(std::false_type{}, std::false_type{});
  else if (!a.k_scale)
    run(std::true_type{}, std::false_type{});
  else
    run(std::true_type{}, std::true_type{});
  if (timer) (void)hipEventRecord(timer->stop, stream);
  return hipGetLastError();
}

}  // namespace rl
