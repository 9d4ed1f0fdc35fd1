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
// With the norms of q and k in the pass (kNorm), the eight threads of a head row add
// their squares: 16384 rows of 64 + 8 heads 99 us, 6.1 TB/s; 20K rows of 64 + 8 + 8 into
// FP8 pages 139 us, 5.9 TB/s; 128 rows of 96 + 8 + 8 4.7 us.
//
// The nontemporal stores are for a call's own time, and the attention that reads
// its rows next pays for them: 2500 rows of 64 + 8 + 8 heads take 19.1 us (20.8
// with ordinary stores) but 69.6 together with the prefill behind them (66.7),
// 8000 rows 56.8 (53.5) and 182 (177), 36000 rows 258 (269) and 805 (791).
#include <algorithm>
#include <type_traits>

#include "kernels.hpp"
#include "rope_rows.hpp"

namespace rl {

namespace {

constexpr int kRopeThreads = 256;
constexpr int kWavesPerCu = 32;                     // that fit at once

// A wave has eight head rows of a row (kLarge: sixteen, stored nontemporally),
// which it loads before it forms the row's angles.
template <bool kAppend, bool kFp8, bool kLarge, bool kNorm>
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
    if (kNorm && kind != kV) {
      const void* w = kind == kQ ? a.q_weight : a.k_weight;
      const float rms = inv_rms(fa, fb, a.eps);
      fa = fa * rms * load_weights(w, c.lo, a.weights_f32);
      fb = fb * rms * load_weights(w, c.hi, a.weights_f32);
    }
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
  auto launch = [&](auto append, auto fp8, auto norm) {
    if (large)
      rope_kernel<append, fp8, true, norm><<<grid, kRopeThreads, 0, stream>>>(a);
    else
      rope_kernel<append, fp8, false, norm><<<grid, kRopeThreads, 0, stream>>>(a);
  };
  auto run = [&](auto append, auto fp8) {
    if (a.q_weight)
      launch(append, fp8, std::true_type{});
    else
      launch(append, fp8, std::false_type{});
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
