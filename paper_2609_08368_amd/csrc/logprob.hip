// Log probabilities of given tokens, with the entropy of their distribution and
// its likeliest tokens, from a step's logits; and the gradient of the logits.
//
// With z_j = s x_j (s the row's scale), lse = ln sum_j exp z_j:
//   logprob = z_token - lse,   entropy = lse - sum_j p_j z_j,   p_j = exp(z_j - lse).
// A row is cut into segments of kSegment logits. A wave holds a whole segment in
// registers: it takes the segment's maximum m first, then S = sum_j 2^y_j and
// Y = sum_j 2^y_j y_j with y_j = (x_j - m) s log2 e, so nothing is rescaled on the
// way. The segments' (m, S, Y) are folded in one fixed tree whatever workgroup
// made them, so that a row's bits depend on its logits alone: not on the size of
// the call, on how its rows are shared out or on where they lie.
//   lse = s M + ln 2 log2 S,  entropy = ln 2 (log2 S - Y / S)
// Y is taken around a base within half a power of two of the maximum, so neither term is
// larger than 1/2 or the entropy. The entropy of a sure row is what is left of the two,
// and of a sum next to 1: off by 1e-7 on average and 4e-7 at most over 1024 rows with
// entropies from 1e-6 to 4e-3. (With y = (x - m) c, so that the maximum adds 1 and 0, by
// 1e-7 and 2.3e-6, as small powers added to 1 one by one all round the same way, and
// 6e-7 with those added in pairs; both took 2-5% longer.)
//
// Alternatives: a bound that K of a workgroup's threads' largest logits reach bounds
// the K-th largest logit from below, so only those threads hold any of the K
// likeliest. Their logits are looked at again (in registers, or read again, and then
// only those of the segments whose largest reaches the bound), and the few that reach
// the bound are ranked. A row of which more than kCand logits reach it (equal ones, most
// of all a constant row) or that has a NaN or +inf is searched K times instead, a pass over a
// workgroup's segments for each: 128 constant rows of 131072 with 20 alternatives take 250
// us (19 otherwise), 2048 of them 7.5 ms (0.1).
//
// A row of a large call is one workgroup's: one pass over the logits, HBM-bound at 6.3
// TB/s (4096 rows of 131072 bf16 logits, a third left out, 118 us; a large copy runs
// at 4.9, a read at 7.2). Rows that would not fill the device are shared by up to 16
// workgroups, the last of which to arrive answers (two launches took 3-4 us more): 128
// rows of 131072 take 12.6 us, with 20 alternatives 17.1 (38 with a first form that
// counted larger maxima thread by thread), one row of 32000 6.1 and 10.5, a chain of
// dependent steps of about 1 us. The gradient is a copy with an exponential: 5.7 TB/s.
#include <algorithm>

#include "attn_common.hpp"
#include "kernels.hpp"

namespace rl {

namespace {

constexpr int kLpThreads = 256, kLpWaves = kLpThreads / 64;
constexpr int kSegment = kLogprobSegment;
constexpr int kCand = 512;                          // candidates that are ranked at once
constexpr int kHeldCand = 64;                       // of a wave, from its registers
constexpr int kCellRounds = 16;                     // rounds of segments whose largest logits are kept, at most
constexpr uint32_t kKeyNegInf = 0x007fffffu;        // key_of(-inf)

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
// (rows may start at any element: a vocabulary need not be a multiple of 16 bytes)
typedef u32x4 u32x4_any __attribute__((aligned(2)));

// 128 registers: left alone the compiler takes 168 and three waves a SIMD fit (512 rows
// of 131072 bf16 logits with 20 alternatives 43 us, 49 so; 4096 of 32000 68 and 75); 80
// or 64 leave it spilling (72 and 94).
constexpr int kLpWavesPerSimd = 4;

// Logits of type X in sixteen bytes, and those as fp32.
template <typename X>
constexpr int kPer = 16 / (int)sizeof(X);
template <typename X>
__device__ __forceinline__ void unpack(u32x4 w, float (&f)[kPer<X>]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(X) == 2) {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    } else {
      f[i] = __uint_as_float(w[i]);
    }
  }
}
template <typename X>
__device__ __forceinline__ u32x4 pack(const float (&f)[kPer<X>]) {
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(X) == 2)
      w[i] = __builtin_bit_cast(u16, (__bf16)f[2 * i]) | (uint32_t)__builtin_bit_cast(u16, (__bf16)f[2 * i + 1]) << 16;
    else
      w[i] = __float_as_uint(f[i]);
  }
  return w;
}
// Sixteen bytes of logits from element e of n on; those behind the end are -inf.
template <typename X>
__device__ __forceinline__ u32x4 load_logits(const X* x, int e, int n) {
  if (e + kPer<X> <= n) return __builtin_nontemporal_load(reinterpret_cast<const u32x4_any*>(x + e));
  float f[kPer<X>];
#pragma unroll
  for (int i = 0; i < kPer<X>; ++i) f[i] = e + i < n ? (float)x[e + i] : kNegInf;
  return pack<X>(f);
}

// An order of floats as whole numbers: NaN lowest, both zeros one.
__device__ __forceinline__ uint32_t key_of(float f) {
  uint32_t u = __float_as_uint(f);
  if ((u & 0x7fffffffu) > 0x7f800000u) return 0;
  if (u == 0x80000000u) u = 0;
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float float_of(uint32_t key) {
  return __uint_as_float((key & 0x80000000u) ? key ^ 0x80000000u : ~key);
}
// The larger logit first, of equal ones the lower index. Never 0.
__device__ __forceinline__ uint64_t rank_of(uint32_t key, int index) {
  return (uint64_t)key << 32 | (0xffffffffu - (uint32_t)index);
}

// A row's token and scale; token < 0: the row is left out.
struct RowInput {
  int token;
  float scale;
};
__device__ __forceinline__ RowInput read_row(const LogprobArgs& a, int64_t r, int* bad) {
  const int64_t t = a.tok64 ? static_cast<const int64_t*>(a.tokens)[r * a.tok_s]
                            : (int64_t)static_cast<const int*>(a.tokens)[r * a.tok_s];
  RowInput in{t < 0 ? -1 : (int)min(t, (int64_t)a.vocab), a.scale ? a.scale[r * a.scale_s] : 1.f};
  if (in.token == a.vocab) {
    *bad |= kErrToken;
    in.token = -1;
  }
  if (!scale_ok(in.scale)) {
    if (t >= 0) *bad |= kErrRowScale;
    in.token = -1;
  }
  return in;
}

// One segment's maximum and sums. y is taken around base(m) instead of m c (c = s
// log2 e): a whole number where that is near, so that y = x c - base is one fused
// product, rounded once; c itself is rounded, but the same for all logits of the row.
struct Part {
  float m, s, y;
};
constexpr float kNear = 1048576.f;
// m c - base(m)
__device__ __forceinline__ float above_base(float m, float c) {
  const float z = m * c;
  return fabsf(z) <= kNear ? fmaf(m, c, -__builtin_rintf(z)) : 0.f;
}

// Loads of a lane for a segment.
template <typename X>
constexpr int kLoads = kSegment / 64 / kPer<X>;

// A wave's segment of n logits at x, to registers.
template <typename X>
__device__ __forceinline__ void load_segment(const X* x, int n, u32x4 (&w)[kLoads<X>]) {
  const int at = (threadIdx.x & 63) * kPer<X>;
  if (n == kSegment) {
#pragma unroll
    for (int i = 0; i < kLoads<X>; ++i)
      w[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_any*>(x + at + i * 64 * kPer<X>));
  } else {
#pragma unroll
    for (int i = 0; i < kLoads<X>; ++i) w[i] = load_logits(x, at + i * 64 * kPer<X>, n);
  }
}

// The sums of a wave's segment; *lane_max is the largest of this lane's logits.
template <typename X>
__device__ __forceinline__ Part segment_part(const u32x4 (&w)[kLoads<X>], float c, float* lane_max) {
  float top = kNegInf;
#pragma unroll
  for (int i = 0; i < kLoads<X>; ++i) {
    float f[kPer<X>];
    unpack<X>(w[i], f);
#pragma unroll
    for (int e = 0; e < kPer<X>; ++e) top = fmaxf(top, f[e]);
  }
  *lane_max = top;
  Part p{wave_max(top), 0.f, 0.f};
  const float m = p.m == kNegInf ? 0.f : p.m;       // (excluded tokens alone: every term is 0)
  const float z = m * c;
  auto sums = [&](auto y_of) {
#pragma unroll
    for (int i = 0; i < kLoads<X>; ++i) {
      float f[kPer<X>];
      unpack<X>(w[i], f);
#pragma unroll
      for (int e = 0; e < kPer<X>; ++e) {
        const float y = y_of(f[e]), t = exp2_fast(y);
        p.s += t;
        p.y = fmaf(t, fmaxf(y, -1000.f), p.y);      // (0 times -inf)
      }
    }
  };
  if (fabsf(z) <= kNear) {
    const float base = -__builtin_rintf(z);
    sums([&](float v) { return fmaf(v, c, base); });
  } else {
    sums([&](float v) { return (v - m) * c; });     // (a product may overflow)
  }
  p.s = wave_sum(p.s);
  p.y = wave_sum(p.y);
  return p;
}

// The row's sums from its segments' (a wave; every lane receives them). kShared: they
// were handed over by several workgroups.
template <bool kShared>
__device__ __forceinline__ Part fold_parts(const Part* parts, int n, float c) {
  const int lane = threadIdx.x & 63;
  auto at = [&](int i) {
    if constexpr (!kShared) return parts[i];
    return Part{handed_over(&parts[i].m), handed_over(&parts[i].s), handed_over(&parts[i].y)};
  };
  Part first{kNegInf, 0.f, 0.f};
  if (lane < n) first = at(lane);                   // (mostly all there is)
  float m = first.m;
  for (int i = lane + 64; i < n; i += 64) m = fmaxf(m, at(i).m);
  Part row{wave_max(m), 0.f, 0.f};
  const float r = above_base(row.m, c);
  for (int i = lane; i < n; i += 64) {
    const Part p = i == lane ? first : at(i);
    // between the bases
    const float d = p.m == kNegInf ? 0.f : fmaxf(fmaf(p.m - row.m, c, r - above_base(p.m, c)), -1000.f);
    const float f = exp2_fast(d);
    row.s = fmaf(f, p.s, row.s);
    row.y = fmaf(f, fmaf(d, p.s, p.y), row.y);
  }
  row.s = wave_sum(row.s);
  row.y = wave_sum(row.y);
  return row;
}

// What a row answers with, from its sums: log probabilities are (x - m) scale + rest.
struct RowStats {
  float m, rest;
  bool none;                                        // every token is excluded
};
__device__ __forceinline__ float log_prob(const RowStats& r, float x, float scale) {
  return r.none ? kNegInf : fmaf(x - r.m, scale, r.rest);
}

// x: the token's logit.
__device__ __forceinline__ RowStats write_row(const LogprobArgs& a, int64_t r, float x, float scale, float c,
                                              const Part& p) {
  const float log2s = __builtin_amdgcn_logf(p.s);
  // (bits, not comparisons: the device code is compiled as if there were no NaN)
  const RowStats st{p.m, kLn2 * (above_base(p.m, c) - log2s), (__float_as_uint(p.s) << 1) == 0};
  if ((threadIdx.x & 63) == 0) {
    a.logprobs[r * a.lp_s] = log_prob(st, x, scale);
    if (a.lse) a.lse[r * a.lse_s] = st.none ? kNegInf : fmaf(p.m, scale, -st.rest);
    if (a.entropy) {
      float h = kLn2 * (log2s - p.y / p.s);
      const uint32_t u = __float_as_uint(h);
      if (st.none || (u >= 0x80000000u && u <= 0xff800000u)) h = 0.f;     // (a rounding below 0)
      a.entropy[r * a.ent_s] = h;
    }
  }
  return st;
}

// A row without a token.
__device__ __forceinline__ void write_masked(const LogprobArgs& a, int64_t r) {
  const int tid = threadIdx.x;
  if (tid == 0) {
    a.logprobs[r * a.lp_s] = 0.f;
    if (a.lse) a.lse[r * a.lse_s] = 0.f;
    if (a.entropy) a.entropy[r * a.ent_s] = 0.f;
  }
  if (tid < a.top) {
    a.top_ids[r * a.ti_s + tid] = -1;
    a.top_lps[r * a.tl_s + tid] = kNegInf;
  }
}

struct TopLds {
  __attribute__((aligned(16))) uint32_t keys[kLpThreads];
  __attribute__((aligned(16))) uint64_t cand[kCand];
  uint64_t best[kLogprobTop];
  uint32_t tau;
  union __attribute__((aligned(16))) {
    int winners[kCand];                             // rounds << 8 | threads whose logits are read again
    uint64_t mine[kLpWaves][kHeldCand];             // of each wave
  };
  int n_winners, n_cand;
};

// The `top` largest of list[0 .. n) to t.best, in order; 0 behind the last. (Each
// counts the larger ones; reads of a fixed number at a time overlap. The list has room
// for a multiple of sixteen.)
__device__ __forceinline__ void rank_candidates(TopLds& t, uint64_t* list, int n, int top) {
  typedef unsigned long long u64x2 __attribute__((ext_vector_type(2)));
  const int tid = threadIdx.x;
  const int padded = (n + 15) & ~15;
  if (tid < top) t.best[tid] = 0;
  if (tid < padded - n) list[n + tid] = 0;
  __syncthreads();
  for (int i = tid; i < n; i += kLpThreads) {
    const uint64_t mine = list[i];
    int rank = 0;
    for (int j = 0; j < padded; j += 16) {
#pragma unroll
      for (int k = 0; k < 16; k += 2) {
        const u64x2 two = *reinterpret_cast<const u64x2*>(&list[j + k]);
        rank += (two.x > mine) + (two.y > mine);
      }
    }
    if (mine != 0 && rank < top) t.best[rank] = mine;
  }
  __syncthreads();
}

// The same of `chunks` lists of `top` in order, in t.cand: each has top / chunks, rounded
// up, entries that reach the least of those entries, so only what reaches it is ranked,
// some 40 of 160 (128 rows of 131072, 20 alternatives 18.6 -> 18.1 us, 32 of them 20.9 ->
// 18.8; lists of fewer than 96 entries in all would take 0.3 longer than ranking them).
__device__ __forceinline__ void rank_lists(TopLds& t, int chunks, int top) {
  const int tid = threadIdx.x, lane = tid & 63, n = chunks * top, each = (top + chunks - 1) / chunks;
  if (n < 96) {
    rank_candidates(t, t.cand, n, top);
    return;
  }
  uint64_t* some = &t.mine[0][0];
  if (tid == 0) t.n_cand = 0;
  uint64_t bound = ~0ull;
#pragma unroll 4
  for (int c = 0; c < chunks; ++c) bound = min(bound, t.cand[c * top + each - 1]);
  __syncthreads();
  for (int i0 = 0; i0 < n; i0 += kLpThreads) {
    const int i = i0 + tid;
    const uint64_t v = i < n ? t.cand[i] : 0;
    const bool in = v != 0 && v >= bound;
    const uint64_t m = __builtin_amdgcn_ballot_w64(in);
    int at = 0;
    if (lane == 0 && m != 0) at = atomicAdd(&t.n_cand, __popcll(m));
    at = __builtin_amdgcn_readfirstlane(at) +
         __builtin_amdgcn_mbcnt_hi((unsigned)(m >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)m, 0));
    if (in && at < kLpWaves * kHeldCand) some[at] = v;
  }
  __syncthreads();
  const int found = t.n_cand;
  if (found <= kLpWaves * kHeldCand)
    rank_candidates(t, some, found, top);
  else
    rank_candidates(t, t.cand, n, top);
}

// A bound that at least `top` of the workgroup's threads' largest logits reach, and
// hardly more: two bits after two from the top, until the count is near enough.
__device__ __forceinline__ void find_bound(TopLds& t, float lane_max, int top) {
  constexpr int kSlack = 8;                         // (a few more to look at cost less than more bits)
  const int tid = threadIdx.x;
  t.keys[tid] = key_of(lane_max);
  __syncthreads();
  if (tid < 64) {
    const u32x4 w = *reinterpret_cast<const u32x4*>(&t.keys[4 * tid]);
    // from the highest pair of bits in which they differ
    uint32_t all = w[0] & w[1] & w[2] & w[3], some = w[0] | w[1] | w[2] | w[3];
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
      all &= __shfl_xor(all, m);
      some |= __shfl_xor(some, m);
    }
    all = __builtin_amdgcn_readfirstlane(all);
    some = __builtin_amdgcn_readfirstlane(some);
    const int from = all == some ? 0 : (31 - __builtin_clz(all ^ some)) & ~1;
    uint32_t lo = some & ~((4u << from) - 1);       // (the shared bits; 4 << 30 is 0)
    for (int shift = from; shift >= 0; shift -= 2) {
      int n[4];                                     // threads that reach lo + k steps
#pragma unroll
      for (int k = 1; k < 4; ++k) {
        const uint32_t next = lo | (uint32_t)k << shift;
        n[k] = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) n[k] += __popcll(__builtin_amdgcn_ballot_w64(w[i] >= next));
      }
      const int k = n[3] >= top ? 3 : n[2] >= top ? 2 : n[1] >= top ? 1 : 0;
      lo |= (uint32_t)k << shift;
      if (k > 0 && (k == 3 ? n[3] : k == 2 ? n[2] : n[1]) <= top + kSlack) break;
    }
    if (tid == 0) {
      t.tau = max(lo, kKeyNegInf + 1);              // excluded tokens are no alternatives
      t.n_winners = t.n_cand = 0;
    }
  }
  __syncthreads();
}

// Those of sixteen bytes of logits from element e on that reach the bound, to the list.
template <typename X>
__device__ __forceinline__ void add_candidates(TopLds& t, u32x4 w, int e, uint32_t tau) {
  const float bound = float_of(tau);
  float f[kPer<X>];
  unpack<X>(w, f);
#pragma unroll
  for (int j = 0; j < kPer<X>; ++j) {
    if (!(f[j] >= bound)) continue;                 // (cheaper than its key; NaN may pass, and its key does not)
    const uint32_t k = key_of(f[j]);
    if (k < tau) continue;
    const int at = atomicAdd(&t.n_cand, 1);
    if (at < kCand) t.cand[at] = rank_of(k, e + j);
  }
}

// The workgroup's likeliest tokens to t.best: of segments seg0 .. seg1-1 of row x,
// where wave w has seg0 + w, seg0 + w + kLpWaves, ... and lane_max is this
// thread's largest logit of those. kHeld: each wave has one, which is in w. odd: the
// wave met a NaN or +inf (a maximum with a signaling NaN may lose what it held, so the
// bounds do not count then).
template <typename X, bool kHeld>
__device__ __forceinline__ void find_top(TopLds& t, const X* x, int vocab, int seg0, int seg1, float lane_max, bool odd,
                                         const u32x4 (&w)[kLoads<X>], const u16* cells, int top) {
  const int tid = threadIdx.x;
  find_bound(t, lane_max, top);
  if (odd && (tid & 63) == 0) atomicAdd(&t.n_cand, kCand + 1);
  const uint32_t tau = t.tau;
  const bool wins = key_of(lane_max) >= tau;
  static_assert(kCand >= kLpWaves * kHeldCand, "every wave's list fits");
  if constexpr (kHeld) {
    // a wave lists its own side by side, and then takes room for them at once
    const int lane = tid & 63, wave = tid >> 6;
    int n = 0;
    if (__builtin_amdgcn_ballot_w64(wins) != 0) {
      const float bound = float_of(tau);
      const int e = (seg0 + wave) * kSegment + lane * kPer<X>;
#pragma unroll
      for (int i = 0; i < kLoads<X>; ++i) {
        float f[kPer<X>];
        unpack<X>(w[i], f);
#pragma unroll
        for (int j = 0; j < kPer<X>; ++j) {
          if (__builtin_amdgcn_ballot_w64(wins && f[j] >= bound) == 0) continue;
          const uint32_t k = key_of(f[j]);          // (NaN may pass the bound, and its key does not)
          const bool in = wins && k >= tau;
          const uint64_t m = __builtin_amdgcn_ballot_w64(in);
          const int at = n + __builtin_amdgcn_mbcnt_hi((unsigned)(m >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)m, 0));
          if (in && at < kHeldCand) t.mine[wave][at] = rank_of(k, e + i * 64 * kPer<X> + j);
          n += __popcll(m);
        }
      }
      int at = 0;
      if (lane == 0) at = atomicAdd(&t.n_cand, n > kHeldCand ? kCand + 1 : n);
      at = __builtin_amdgcn_readfirstlane(at);
      __builtin_amdgcn_wave_barrier();
      if (lane < n && at + lane < kCand) t.cand[at + lane] = t.mine[wave][lane];
    }
  } else {
    // a thread's logits of those rounds whose largest reaches the bound, if that is
    // kept (cells: its upper half), else of all
    const int rounds = (seg1 - seg0 + kLpWaves - 1) / kLpWaves;
    if (wins)
      for (int i = 0; i < (cells ? rounds : 1); ++i) {
        if (seg0 + (tid >> 6) + i * kLpWaves >= seg1) break;
        if (cells && cells[i * kLpThreads + tid] < (tau >> 16)) continue;
        const int at = atomicAdd(&t.n_winners, 1);
        if (at < kCand) t.winners[at] = i << 8 | tid;
      }
    __syncthreads();
    const int per = (cells ? 1 : rounds) * kLoads<X>, n = min(t.n_winners, kCand) * per;
    if (t.n_winners > kCand && tid == 0) atomicAdd(&t.n_cand, kCand + 1);
    constexpr int kAgain = 4;                       // loads that are under way at once
    for (int p0 = tid; p0 < n; p0 += kAgain * kLpThreads) {
      u32x4 again[kAgain];
      int e[kAgain];
#pragma unroll
      for (int k = 0; k < kAgain; ++k) {
        const int p = p0 + k * kLpThreads;
        e[k] = vocab;
        if (p < n) {
          const int entry = t.winners[p / per], i = p % per, who = entry & (kLpThreads - 1);
          const int seg = seg0 + (who >> 6) + ((entry >> 8) + i / kLoads<X>) * kLpWaves;
          if (seg < seg1) e[k] = seg * kSegment + ((i % kLoads<X>) * 64 + (who & 63)) * kPer<X>;
        }
        again[k] = load_logits(x, e[k], vocab);
      }
#pragma unroll
      for (int k = 0; k < kAgain; ++k)
        if (e[k] < vocab) add_candidates<X>(t, again[k], e[k], tau);
    }
  }
  __syncthreads();
  int found = t.n_cand;
  if (found <= kCand) {
    rank_candidates(t, t.cand, found, top);
    return;
  }
  // odd values, or so many equal logits that the list does not hold them: one after the
  // other, each the largest below the last
  const int lo = seg0 * kSegment, hi = min(vocab, seg1 * kSegment);
  uint64_t below = ~0ull;
  for (found = 0; found < top; ++found) {
    uint64_t most = 0;
    for (int e = lo + tid; e < hi; e += kLpThreads) {
      const uint64_t v = rank_of(key_of((float)x[e]), e);
      if (v < below && v > most) most = v;
    }
    __syncthreads();                                // (the last round's list has been read)
    t.cand[tid] = most;
    __syncthreads();
    for (int s = kLpThreads / 2; s > 0; s >>= 1) {
      if (tid < s && t.cand[tid + s] > t.cand[tid]) t.cand[tid] = t.cand[tid + s];
      __syncthreads();
    }
    below = t.cand[0];
    if ((uint32_t)(below >> 32) <= kKeyNegInf) break;
    if (tid == 0) t.best[found] = below;
  }
  if (tid < top && tid >= found) t.best[tid] = 0;
  __syncthreads();
}

// t.best as the row's alternatives.
__device__ __forceinline__ void write_top(const LogprobArgs& a, int64_t r, const TopLds& t, const RowStats& st,
                                          float scale) {
  const int i = threadIdx.x;
  if (i >= a.top) return;
  const uint64_t b = t.best[i];
  a.top_ids[r * a.ti_s + i] = b ? (int)(0xffffffffu - (uint32_t)b) : -1;
  a.top_lps[r * a.tl_s + i] = b ? log_prob(st, float_of((uint32_t)(b >> 32)), scale) : kNegInf;
}

// Workgroup: segments of one row. Where a row is shared, its workgroups leave the
// segments' sums and their likeliest tokens in memory, and the last of them to
// arrive answers. kHeld: a wave has one segment at most.
template <typename X, bool kTop, bool kHeld>
__global__ __launch_bounds__(kLpThreads, kLpWavesPerSimd) void logprob_kernel(LogprobArgs a) {
  extern __shared__ Part parts[];                   // a workgroup for each row: [segs]; behind them, cells
  __shared__ TopLds top;
  __shared__ int last;
  const int row32 = blockIdx.x / a.chunks, chunk = blockIdx.x - row32 * a.chunks;
  const int64_t r = row32;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const X* x = static_cast<const X*>(a.x) + r * a.x_s;
  const int seg0 = chunk * a.segs_chunk, seg1 = min(a.segs, seg0 + a.segs_chunk);
  Part* shared = a.chunks > 1 ? static_cast<Part*>(a.parts) + r * a.segs : nullptr;
  u32x4 w[kLoads<X>];
  auto load = [&](int s) { load_segment(x + s * kSegment, min(kSegment, a.vocab - s * kSegment), w); };
  // (calls of few rows do not wait for the token before they load; of many, rows that
  // are left out are not loaded)
  int s = seg0 + wave;
  if (shared && s < seg1) load(s);
  int bad = 0;
  const RowInput in = read_row(a, r, &bad);
  if (in.token < 0) {
    if (chunk != 0) return;
    if (bad && tid == 0) atomicOr(a.err, bad);
    write_masked(a, r);
    return;
  }
  const float c = in.scale * kLog2e, x_token = (float)x[in.token];
  if (!shared && s < seg1) load(s);
  float most = kNegInf;
  bool odd = false;
  u16* cells = nullptr;                             // upper halves of the threads' largest of each round
  if (kTop && !kHeld && a.segs_chunk <= kLpWaves * kCellRounds)
    cells = reinterpret_cast<u16*>(parts + (shared ? 0 : a.segs)) + tid;
  while (s < seg1) {
    float lane_max;
    const Part p = segment_part<X>(w, c, &lane_max);
    most = fmaxf(most, lane_max);
    odd |= (__float_as_uint(p.s) & 0x7fffffffu) > 0x7f800000u;
    if (kTop && !kHeld && cells) {
      *cells = (u16)(key_of(lane_max) >> 16);
      cells += kLpThreads;
    }
    if ((tid & 63) == 0) {
      if (shared) {
        hand_over(&shared[s].m, p.m);
        hand_over(&shared[s].s, p.s);
        hand_over(&shared[s].y, p.y);
      } else {
        parts[s] = p;
      }
    }
    if (kHeld) break;
    s += kLpWaves;
    if (s < seg1) load(s);
  }
  if (kTop && !kHeld && cells) cells = reinterpret_cast<u16*>(parts + (shared ? 0 : a.segs));
  if constexpr (kTop) find_top<X, kHeld>(top, x, a.vocab, seg0, seg1, most, odd, w, cells, a.top);
  Part sums;
  if (shared) {
    uint64_t* cands = a.cands + r * a.chunks * a.top;
    if (kTop && tid < a.top) hand_over(cands + chunk * a.top + tid, top.best[tid]);
    if (!arrive(a.arrived + r, a.chunks, &last)) return;
    // (one wave folds the sums while the others fetch the tokens)
    if (wave == 0) sums = fold_parts<true>(shared, a.segs, c);
    if constexpr (kTop) {
      const int n = a.chunks * a.top;
      if (wave != 0)
        for (int i = tid - 64; i < n; i += kLpThreads - 64) top.cand[i] = handed_over(cands + i);
      __syncthreads();
      rank_lists(top, a.chunks, a.top);
    }
  } else {
    __syncthreads();
    if (wave == 0) sums = fold_parts<false>(parts, a.segs, c);
  }
  if (wave == 0) {
    const RowStats st = write_row(a, r, x_token, in.scale, c, sums);
    if (kTop) write_top(a, r, top, st, in.scale);
  }
}

// Gradient: d_x_j = s (g (delta_j - p_j) - h p_j (ln p_j + H)), an element-wise pass with
// ln p_j = s x_j - lse. That lse is rounded, so p is off by half a step of it, relatively:
// 2^-19 below kLseNear, no more than the products and powers of a token with |ln p| = 10
// are off by, but 3e-5 at 1000 and everything at 1e7. Rows past kLseNear are therefore one
// workgroup's, which sums their powers again, around their largest logit m, and takes
// ln p_j = (x_j - m) s + rest as the forward call does; behind the row's last load, as the
// row may be in place. They cost a second read, 4096 rows of 131072 bf16 logits 702 us
// (343 with lse in every workgroup), and calls of few rows are as slow as one workgroup:
// 128 rows 158 us (13; 71 of 151936 logits, whose rows do not all begin on one channel).
constexpr int kGradLoads = 4;
constexpr float kLseNear = 64.f;

// A row's largest logit and -ln of the sum of exp((x_j - m) scale), by a workgroup: one
// read of the row. A thread's sum is taken around one of its logits, another one only
// when a logit is 2^kAhead times as likely, so that what is rounded then fades.
template <typename X>
__device__ __forceinline__ void sum_again(const X* x, int vocab, float scale, float* m_out, float* rest_out) {
  __shared__ float most[kLpWaves], sums[kLpWaves];
  constexpr float kAhead = 8.f;
  const int tid = threadIdx.x;
  const float c = scale * kLog2e;
  float base = kNegInf;
  double sum = 0.0;                                 // (of up to 2^21 / 256 logits)
  for (int e0 = tid * kPer<X>; e0 < vocab; e0 += kGradLoads * kLpThreads * kPer<X>) {
    u32x4 w[kGradLoads];
#pragma unroll
    for (int i = 0; i < kGradLoads; ++i) w[i] = load_logits(x, e0 + i * kLpThreads * kPer<X>, vocab);
    float top = kNegInf;
#pragma unroll
    for (int i = 0; i < kGradLoads; ++i) {
      float f[kPer<X>];
      unpack<X>(w[i], f);
#pragma unroll
      for (int j = 0; j < kPer<X>; ++j) top = fmaxf(top, f[j]);
    }
    if (top == kNegInf && base == kNegInf) continue;                      // (excluded tokens alone)
    if (base == kNegInf) base = top;
    if ((top - base) * c > kAhead) {
      sum *= (double)exp2_fast((base - top) * c);
      base = top;
    }
#pragma unroll
    for (int i = 0; i < kGradLoads; ++i) {
      float f[kPer<X>], t = 0.f;
      unpack<X>(w[i], f);
#pragma unroll
      for (int j = 0; j < kPer<X>; ++j) t += exp2_fast((f[j] - base) * c);
      sum += (double)t;
    }
  }
  const float wave_top = wave_max(base);
  if ((tid & 63) == 0) most[tid >> 6] = wave_top;
  __syncthreads();
  float m = most[0];
#pragma unroll
  for (int i = 1; i < kLpWaves; ++i) m = fmaxf(m, most[i]);
  const float mine = wave_sum(base == kNegInf ? 0.f : (float)sum * exp2_fast((base - m) * c));
  if ((tid & 63) == 0) sums[tid >> 6] = mine;
  __syncthreads();
  float all = 0.f;
#pragma unroll
  for (int i = 0; i < kLpWaves; ++i) all += sums[i];
  *m_out = m;
  *rest_out = -kLn2 * __builtin_amdgcn_logf(all);
}

// The workgroup of a row that has all of it: workgroups go to the eight dies in turn, and
// these should too, whatever number of them a row has.
__device__ __forceinline__ int far_chunk(int row, int chunks) {
  const int even = chunks % 8 == 0 ? 8 : chunks % 4 == 0 ? 4 : chunks % 2 == 0 ? 2 : 1;
  return (int)((int64_t)row * even / 8 % chunks);
}

template <typename X>
__global__ __launch_bounds__(kLpThreads) void logprob_grad_kernel(LogprobArgs a) {
  const int row32 = blockIdx.x / a.chunks, chunk = blockIdx.x - row32 * a.chunks;
  const int64_t r = row32;
  int bad = 0;
  const RowInput in = read_row(a, r, &bad);
  if (bad && chunk == 0 && threadIdx.x == 0) atomicOr(a.err, bad);
  const X* x = static_cast<const X*>(a.x) + r * a.x_s;
  X* d = static_cast<X*>(a.d_x) + r * a.dx_s;
  const int e0 = (chunk * kGradLoads * kLpThreads + threadIdx.x) * kPer<X>;
  float lse = 0.f, g = 0.f, h = 0.f, ent = 0.f;
  if (in.token >= 0) {
    lse = a.lse[r * a.lse_s];
    if (a.d_lp) g = a.d_lp[r * a.dlp_s];
    if (a.d_ent) {
      h = a.d_ent[r * a.dent_s];
      ent = a.entropy[r * a.ent_s];
    }
  }
  if (in.token < 0 || lse == kNegInf) {             // left out, or every token excluded
#pragma unroll
    for (int i = 0; i < kGradLoads; ++i) {
      const int e = e0 + i * kLpThreads * kPer<X>;
      if (e + kPer<X> <= a.vocab)
        __builtin_nontemporal_store(u32x4{0, 0, 0, 0}, reinterpret_cast<u32x4_any*>(d + e));
      else
        for (int j = e; j < a.vocab; ++j) d[j] = (X)0.f;
    }
    return;
  }
  // the gradient of the logits from element e on, with ln p = (x - m) s + rest
  auto pass = [&](int e0, float m, float rest) {
    u32x4 w[kGradLoads];
#pragma unroll
    for (int i = 0; i < kGradLoads; ++i) w[i] = load_logits(x, e0 + i * kLpThreads * kPer<X>, a.vocab);
#pragma unroll
    for (int i = 0; i < kGradLoads; ++i) {
      const int e = e0 + i * kLpThreads * kPer<X>;
      float f[kPer<X>];
      unpack<X>(w[i], f);
#pragma unroll
      for (int j = 0; j < kPer<X>; ++j) {
        const float lp = fmaf(f[j] - m, in.scale, rest), p = exp2_fast(lp * kLog2e);
        const float v = -p * fmaf(h, fmaxf(lp, -1000.f) + ent, g);        // (0 times -inf)
        f[j] = in.scale * (e + j == in.token ? v + g : v);
      }
      if (e + kPer<X> <= a.vocab)
        __builtin_nontemporal_store(pack<X>(f), reinterpret_cast<u32x4_any*>(d + e));
      else
#pragma unroll
        for (int j = 0; j < kPer<X>; ++j)
          if (e + j < a.vocab) d[e + j] = (X)f[j];
    }
  };
  // (by bits: a NaN is near, as lse carries it to the whole row and sums that skip
  // stretches of nothing else would not)
  const uint32_t size = __float_as_uint(lse) & 0x7fffffffu;
  if (size <= __builtin_bit_cast(uint32_t, kLseNear) || size > 0x7f800000u) {
    pass(e0, 0.f, -lse);
    return;
  }
  if (chunk != far_chunk(row32, a.chunks)) return;
  float m, rest;
  sum_again(x, a.vocab, in.scale, &m, &rest);
  for (int e = threadIdx.x * kPer<X>; e < a.vocab; e += kGradLoads * kLpThreads * kPer<X>) pass(e, m, rest);
}

}  // namespace

// Workgroups of a row: one where the rows fill the device, else as many as that
// takes, of four segments at least.
int logprob_chunks(int64_t rows, int vocab, int cus) {
  const int segs = (vocab + kSegment - 1) / kSegment;
  if (rows > kLogprobSharedRows) return 1;
  const int64_t want = std::max<int64_t>(1, (8 * (int64_t)cus + rows - 1) / std::max<int64_t>(rows, 1));
  const int most = std::min(kLogprobChunks, (segs + kLpWaves - 1) / kLpWaves);
  const int chunks = (int)std::min<int64_t>(want, std::max(1, most));
  const int each = ((segs + chunks - 1) / chunks + kLpWaves - 1) / kLpWaves * kLpWaves;
  return std::max(1, (segs + each - 1) / each);
}

hipError_t launch_logprob(const LogprobArgs& args, hipStream_t stream) {
  LogprobArgs a = args;
  a.segs = (a.vocab + kSegment - 1) / kSegment;
  a.segs_chunk = ((a.segs + a.chunks - 1) / a.chunks + kLpWaves - 1) / kLpWaves * kLpWaves;
  const unsigned grid = (unsigned)((int64_t)a.rows * a.chunks);
  const size_t lds_parts = a.chunks == 1 ? sizeof(Part) * (size_t)a.segs : 0;
  const int rounds = a.segs_chunk / kLpWaves;
  const size_t lds = lds_parts + (a.top && rounds > 1 && rounds <= kCellRounds ? rounds * kLpThreads * sizeof(u16) : 0);
  auto run = [&](auto type, auto top, auto held) {
    logprob_kernel<decltype(type), decltype(top)::value, decltype(held)::value>
        <<<grid, kLpThreads, lds, stream>>>(a);
  };
  auto run_type = [&](auto type) {
    const bool held = a.segs_chunk <= kLpWaves;
    if (!a.top)
      run(type, std::false_type{}, std::false_type{});
    else if (held)
      run(type, std::true_type{}, std::true_type{});
    else
      run(type, std::true_type{}, std::false_type{});
  };
  if (a.f32)
    run_type(float{});
  else
    run_type(__bf16{});
  return hipGetLastError();
}

hipError_t launch_logprob_grad(const LogprobArgs& args, hipStream_t stream) {
  LogprobArgs a = args;
  const int64_t each = (int64_t)kGradLoads * kLpThreads * (a.f32 ? kPer<float> : kPer<__bf16>);
  a.chunks = (int)((a.vocab + each - 1) / each);
  const unsigned grid = (unsigned)((int64_t)a.rows * a.chunks);
  if (a.f32)
    logprob_grad_kernel<float><<<grid, kLpThreads, 0, stream>>>(a);
  else
    logprob_grad_kernel<__bf16><<<grid, kLpThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace rl
