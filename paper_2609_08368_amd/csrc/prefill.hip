// Causal attention over whole packed prompts: row i of a prompt attends to its
// rows 0 .. i, whose K and V are packed rows too (no pages).
//
// A unit of work is (prompt b, KV head g, block of query heads, run of tokens):
// up to 256 query rows, token-major (row r -> token r / RB, head r % RB), which
// all read the same keys in steps of 64.
//
// S^T = K Q^T and O^T += V^T P^T on 32x32x16 MFMAs, so that a row is a column:
// its scores, maximum and sums are in two lanes, and P^T is an operand of the
// second product as it comes. Four waves, one a SIMD with all 512 registers, of
// 64 rows each: an operand read from LDS serves two MFMAs (with 32 rows, and
// eight waves, a 16K prompt of 64 + 8 heads took 4.0-4.4 ms against 3.6, bound
// by those reads). A wave's step is one stream: values of step j - 1, softmax of
// step j and scores of step j + 1, in which each MFMA is followed by the four or
// five vector instructions of a softmax slot, which run beside it. Rows of K and
// V go from memory to LDS by the load, two and three steps ahead, one barrier a
// step.
//
// There is no running maximum: a row's probabilities are taken against the
// maximum of its first keys, which in 32-bit floats is as good unless a later
// score is 88 above it. Then a sum or O is infinite or NaN at the end, as it is
// where a masked value is (0 times infinity), and the wave computes its rows
// again, slowly and with a running maximum (attend_again); so it does where a sum
// is below 1/2, which scores of 1e7 and more can do. Where two waves split
// a tile's keys, each has such a maximum of its own, and the weights that join
// them are kept in range whatever the distance of the two. A running maximum
// everywhere cost 7-10% of a 16K prompt. The second attempt is dear: with all rows
// of prompts of 300 to 16384 a call takes 7.6-8.7 times as long, and a lone wave's
// 64 rows with 4K (16K) keys, as for an infinity in the last value, add 0.7 ms
// (3.3 ms) to it.
//
// Probabilities are rounded to bf16 for the second product, as in the extend
// kernels: the MFMAs that keep 32 bits run at a fraction of the rate, and two bf16
// halves would be half as many MFMAs again. A result is off by 2^-8 of the mean
// magnitude of its values at most, as much as its own rounding to bf16 (rms of the
// two together 2.1e-3, of the rounding alone 1.6e-3), also where the output has 32
// bits. Row sums are of the unrounded ones, in 32 bits.
//
// Workgroups stay, one a CU, and take units from a longest-first order that each
// of them works out alike (plan_levels); a unit's first rows are requested in
// the last step of the one before.
//
// MFMA-bound: a 16384-row prompt of 64 + 8 heads runs at 1.20-1.27 PFLOP/s
// (3.45-3.67 ms, box to box; a large bf16 matrix product of the library runs at
// 1.22). Its cycles and those of 16 prompts of 2-4K rows are 3,130 a step of 256
// rows, of which the MFMAs take 2,048, and 20,000 a unit around the steps
// (operands and scores of the first one, the last values, rows out, and what the
// CUs wait for each other at the end). With 4.5 steps a unit that is most of it:
// 24 prompts of up to 701 rows of 96 + 8 heads run at 0.49-0.51 PFLOP/s (202-213
// us, 2.1-2.3 TB/s), MFMAs busy 24%.
//
// The grid is a multiple of the head groups (KV heads times blocks of query
// heads), since a unit's order is worked out for one: of 256 CUs, 96 groups use
// 192 and 129 use 129 (2000 rows of 128 heads of their own take 157 us, of 129
// 254).
#include <algorithm>
#include <type_traits>

#include "kernels.hpp"
#include "tile_attn.hpp"

namespace rl {

namespace {

constexpr int kPreThreads = 256;       // four waves, one a SIMD
constexpr int kStep = 64;              // keys of a step
constexpr int kAhead = 4, kRing = 8;   // LDS operands read ahead of a pair's MFMAs, and their registers
constexpr int kKPitch = 1024 + 16;     // LDS blocks of four 256-byte rows
constexpr int kVPitch = 1024 + 64;
constexpr int kKSize = 16 * kKPitch, kVSize = 16 * kVPitch;
constexpr int kKBufs = 3, kVBufs = 4;
constexpr int kLevels = 1024;          // chunk levels of the longest-first order
constexpr int kSorted = kPreThreads;   // prompts that are sorted, a thread each

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

template <int kFrom, int kTo, typename F>
__device__ __forceinline__ void each(F&& f) {
  if constexpr (kFrom < kTo) {
    f(std::integral_constant<int, kFrom>{});
    each<kFrom + 1, kTo>(f);
  }
}

// The first and a further MFMA of a score chain, with the scores in VGPRs and q
// in AGPRs. As assembly, since the compiler would put every accumulator of this
// kernel into AGPRs and copy the scores out of them, an instruction for each. It
// does not know these as MFMAs, so what their hazards ask for is done by hand:
// q is in place two instructions before the first (body), and no result is read
// before 12 wait states after the last (body, and the scores' first use), which
// is what the compiler leaves behind the same product as a builtin.
__device__ __forceinline__ void mfma_first(f32x16& c, const bf16x8& a, const bf16x8& b) {
  asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(c) : "v"(a), "a"(b));
}
__device__ __forceinline__ void mfma_next(f32x16& c, const bf16x8& a, const bf16x8& b) {
  asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(c) : "v"(a), "a"(b));
}

// The last one of a chain has its result elsewhere: were it the same registers,
// the compiler might copy the sums to the next iteration's before it, unseen. Its
// sums stay as they are for 7 wait states more (kept).
__device__ __forceinline__ void mfma_last(f32x16& d, const f32x16& c, const bf16x8& a, const bf16x8& b) {
  asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %3" : "=&v"(d) : "v"(a), "a"(b), "v"(c));
}

// The same value, as far as the compiler knows known only from here on: what is
// formed from it is formed here, and not kept in registers over a loop.
__device__ __forceinline__ int here(int x) {
  asm volatile("" : "+v"(x));
  return x;
}
__device__ __forceinline__ uint32_t here(uint32_t uniform) {
  asm volatile("" : "+s"(uniform));
  return uniform;
}

__device__ __forceinline__ void kept(const f32x16& c) { asm volatile("" ::"v"(c)); }

// Rows [q0, q0 + n) of prompt b, clamped into the call's rows.
struct Prompt {
  int q0, n;
};
__device__ __forceinline__ Prompt prompt_of(const PrefillArgs& a, int b, int* bad) {
  int q0 = a.indptr[(int64_t)b * a.indptr_s], q1 = a.indptr[(int64_t)(b + 1) * a.indptr_s];
  if (q0 < 0 || q1 < q0 || q1 > a.rows) {
    *bad |= kErrIndptr;
    q0 = min(max(q0, 0), a.rows);
    q1 = min(max(q1, q0), a.rows);
  }
  return {q0, q1 - q0};
}
__device__ __forceinline__ int tiles_of(const PrefillArgs& a, int n) { return (n + a.tile_tokens - 1) / a.tile_tokens; }

constexpr int kUnit = 1, kNoTile = 0, kEnd = -1;
struct Plan {
  int count[kLevels + 1];              // chunks of a level or above
  int with[kLevels];                   // prompts that have a level
  int4 chunks[kSorted / 4];            // chunks of each prompt
  int2 sorted[kSorted];                // (first row, rows) of the prompts, those with most chunks first
  int4 units[kPreThreads + 1];         // (first row of the prompt, its rows, tile, kUnit ..) of the workgroup's next units
  int wave_tot[16];
};

// Inclusive sums from the end of a[0 .. kLevels), kLevels / kPreThreads entries a thread.
__device__ __forceinline__ void suffix_sums(int* x, int* wave_tot) {
  constexpr int kPer = kLevels / kPreThreads;
  int v[kPer], sum = 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    v[i] = x[kLevels - 1 - (threadIdx.x * kPer + i)];
    sum += v[i];
  }
  int total, before = block_exclusive_scan(sum, &total, wave_tot);
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    before += v[i];
    x[kLevels - 1 - (threadIdx.x * kPer + i)] = before;
  }
  __syncthreads();
}

// Longest first: chunks of 2^chunk_log neighbouring tiles by descending index
// (level) in their prompt, which is their key range; within a level the prompts
// with most chunks first, equal ones in order (every workgroup makes the same
// plan). Two prefix sums over the levels give the place of every chunk: count[l]
// of them have level l or above, and the prompts that have a level are the first
// ones of `sorted`.
__device__ __forceinline__ void plan_levels(const PrefillArgs& a, Plan& p, int* bad) {
  const int tid = threadIdx.x;
  if (a.B == 1) {
    if (tid == 0) {
      const Prompt x = prompt_of(a, 0, bad);
      p.sorted[0] = make_int2(x.q0, x.n);
    }
    return;                              // (the caller synchronises)
  }
  for (int i = tid; i < kLevels; i += kPreThreads) p.with[i] = 0;
  int mine = 0;
  Prompt x{0, 0};
  if (tid < a.B) {
    x = prompt_of(a, tid, bad);
    mine = min(((tiles_of(a, x.n) - 1) >> a.chunk_log) + 1, kLevels);
  }
  reinterpret_cast<int*>(p.chunks)[tid] = mine;
  __syncthreads();
  if (mine > 0) atomicAdd(&p.with[mine - 1], 1);
  int place = 0;
  for (int i = 0; i < (a.B + 3) >> 2; ++i) {
    const int4 c = p.chunks[i];
    auto before = [&](int x, int b) { return x > mine || (x == mine && b < tid); };
    place += before(c.x, 4 * i) + before(c.y, 4 * i + 1) + before(c.z, 4 * i + 2) + before(c.w, 4 * i + 3);
  }
  if (tid < a.B) p.sorted[place] = make_int2(x.q0, x.n);
  __syncthreads();
  suffix_sums(p.with, p.wave_tot);
  for (int i = tid; i < kLevels; i += kPreThreads) p.count[i] = p.with[i];
  if (tid == 0) p.count[kLevels] = 0;
  __syncthreads();
  suffix_sums(p.count, p.wave_tot);
}

// The unit of rank `rank` of a head group.
__device__ __forceinline__ int4 unit_of(const PrefillArgs& a, const Plan& p, int rank) {
  int bad = 0, tile;
  Prompt x;
  if (a.B <= kSorted) {
    const int c = rank >> a.chunk_log;
    int level, k = 0;
    if (a.B == 1) {                      // (a lone prompt needs no sums)
      const int2 y = p.sorted[0];
      level = ((tiles_of(a, y.y) - 1) >> a.chunk_log) - c;
      if (level < 0 || y.y == 0) return make_int4(0, 0, 0, kEnd);
    } else {
      if (c >= p.count[0]) return make_int4(0, 0, 0, kEnd);
      level = 0;                         // the last level with count above c
#pragma unroll
      for (int step = kLevels / 2; step > 0; step >>= 1)
        if (p.count[level + step] > c) level += step;
      k = c - p.count[level + 1];
    }
    const int2 y = p.sorted[k];
    x = {y.x, y.y};
    tile = (level << a.chunk_log) + (1 << a.chunk_log) - 1 - (rank & ((1 << a.chunk_log) - 1));
  } else {
    // Too many prompts to sort (and no one of them is much of the call): in the
    // order of the rows. Prompt b's tiles take the places from q0 / tt + b on,
    // which are enough for them whatever the prompts' bounds, so no sum is needed.
    const int places = a.rows / a.tile_tokens + a.B;
    if (rank >= places) return make_int4(0, 0, 0, kEnd);
    auto base = [&](int i) { return min(max(a.indptr[(int64_t)i * a.indptr_s], 0), a.rows) / a.tile_tokens + i; };
    int lo = 0, hi = a.B - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (base(mid) <= rank) lo = mid; else hi = mid - 1;
    }
    tile = rank - base(lo);
    x = prompt_of(a, lo, &bad);
  }
  return make_int4(x.q0, x.n, tile, tile >= 0 && tile < tiles_of(a, x.n) ? kUnit : kNoTile);
}

// Whether a lane's part of O^T or of a row sum holds an infinity or a NaN (by the
// bits: device code is compiled assuming no NaN operands).
template <int NRB>
__device__ __forceinline__ bool odd_values(const f32x16 (&o)[NRB][4], const float (&l)[NRB]) {
  uint32_t top = 0;
#pragma unroll
  for (int rb = 0; rb < NRB; ++rb) {
    top = max(top, __float_as_uint(l[rb]) & 0x7fffffffu);
#pragma unroll
    for (int jd = 0; jd < 4; ++jd)
#pragma unroll
      for (int e = 0; e < 16; ++e) top = max(top, __float_as_uint(o[rb][jd][e]) & 0x7fffffffu);
  }
  return top >= 0x7f800000u;
}

// A block of 32 rows of a unit (row r0 on) again, without the two shortcuts of the
// fast path: the running maximum follows every step, and a masked key's value
// takes no part at all (0 times an infinity or a NaN is NaN). Its maximum is of
// the raw scores and subtracted before the scale, which is exact for the largest
// one: minus a scaled and rounded maximum, a score of 1e10 powers of two would
// leave hundreds of them. By one wave, operands
// straight from memory; keys below `whole`, which every row sees, by MFMA, the
// others one by one. Not inlined: the fast path's registers are its own.
typedef __attribute__((address_space(4))) const PrefillArgs ConstPrefillArgs;
__device__ __attribute__((noinline)) void attend_again(ConstPrefillArgs* ap, int r0, int q0, int i0, int cnt, int g,
                                                       int hb) {
  const PrefillArgs a = *(const PrefillArgs*)ap;
  const int lane = threadIdx.x & 63, col = lane & 31, kg = lane >> 5;
  const int r = r0 + col, ti = r / a.rows_head, hr = r - ti * a.rows_head;
  const bool ok = ti < cnt && hb * a.rows_head + hr < a.R;
  const int head = g * a.R + hb * a.rows_head + (ok ? hr : 0);
  const int64_t row = q0 + i0 + (ok ? ti : 0);
  const int keys = i0 + cnt, limit = ok ? i0 + ti : keys - 1, whole = (i0 + 1) / 32 * 32;
  const __bf16* kb = (const __bf16*)a.k + (int64_t)q0 * a.k_st + g * a.k_sh;
  const __bf16* vb = (const __bf16*)a.v + (int64_t)q0 * a.v_st + g * a.v_sh;
  bf16x8 qv[8];
  load_q_operand((const __bf16*)a.q + row * a.q_st + (int64_t)head * a.q_sh, ok, qv);
  const float sl2 = a.scale * kLog2e;
  const f32x16 zero = {};
  f32x16 o[4] = {zero, zero, zero, zero};
  float m = -__FLT_MAX__, l = 0.f;
#pragma unroll 1
  for (int t0 = 0; t0 < whole; t0 += 32) {
    f32x16 s = zero;
#pragma unroll
    for (int c = 0; c < 8; ++c)
      s = mfma_32x32x16(load_bf16x8(kb + (int64_t)(t0 + col) * a.k_st + 16 * c + 8 * kg), qv[c], s);
    float mx = s[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) mx = fmaxf(mx, s[e]);
    const float m_new = fmaxf(m, max_l32(mx)), alpha = exp2_fast((m - m_new) * sl2);
    m = m_new;
    l *= alpha;
#pragma unroll
    for (int jd = 0; jd < 4; ++jd) o[jd] *= alpha;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      bf16x8 p;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x = exp2_fast((s[8 * h + e] - m) * sl2);
        l += x;
        p[e] = (__bf16)x;
      }
#pragma unroll
      for (int jd = 0; jd < 4; ++jd) {
        bf16x8 v;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          v[e] = vb[(int64_t)(t0 + 16 * h + 8 * (e >> 2) + 4 * kg + (e & 3)) * a.v_st + 32 * jd + col];
        o[jd] = mfma_32x32x16(v, p, o[jd]);
      }
    }
  }
#pragma unroll 1
  for (int t = whole; t < keys; ++t) {
    const __bf16* kr = kb + (int64_t)t * a.k_st;
    const __bf16* vr = vb + (int64_t)t * a.v_st + 4 * kg;
    float s = 0.f;
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      const bf16x8 x = load_bf16x8(kr + 16 * c + 8 * kg);
#pragma unroll
      for (int e = 0; e < 8; ++e) s = fmaf((float)x[e], (float)qv[c][e], s);
    }
    s = sum_l32(s);
    if (t > limit) continue;
    const float m_new = fmaxf(m, s), alpha = exp2_fast((m - m_new) * sl2), p = exp2_fast((s - m_new) * sl2);
    m = m_new;
    l = l * alpha + (kg ? 0.f : p);
#pragma unroll
    for (int jd = 0; jd < 4; ++jd)
#pragma unroll
      for (int e = 0; e < 16; ++e)
        o[jd][e] = fmaf(p, (float)vr[32 * jd + 8 * (e >> 2) + (e & 3)], o[jd][e] * alpha);
  }
  const float l_tot = sum_l32(l);
  if (!ok) return;
  const float inv = 1.f / l_tot;
  if (a.out_f32)
    store_o_row((float*)a.out + row * a.out_st + (int64_t)head * a.out_sh, o, inv);
  else
    store_o_row((__bf16*)a.out + row * a.out_st + (int64_t)head * a.out_sh, o, inv);
  if (a.lse && lane < 32)
    a.lse[row * a.lse_st + (int64_t)head * a.lse_sh] = fmaf(m, sl2, __builtin_amdgcn_logf(l_tot)) * kLn2;
}

// A wave's 32 rows to memory. O^T has a row's dimensions in two lanes, four
// neighbours at a time; through LDS (wave-private, 128 bytes of each row at once)
// a store instruction writes whole lines of eight rows instead of 16 bytes of 32.
// row(i, ok): address of row i.
constexpr int kOutPitch = 128 + 16;
template <typename T, typename RowOf>
__device__ __forceinline__ void store_block(const f32x16 (&o)[4], float inv, char* lds, int lane, RowOf&& row) {
  constexpr int kJd = 4 / sizeof(T);               // 32-dimension blocks in 128 bytes
  typedef T t4 __attribute__((ext_vector_type(4)));
  const int col = lane & 31, kg = lane >> 5;
  T* to[4];
  bool ok[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) to[i] = row(8 * i + (lane >> 3), &ok[i]);
#pragma unroll
  for (int part = 0; part < 4 / kJd; ++part) {
#pragma unroll
    for (int jd = 0; jd < kJd; ++jd)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        t4 x;
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = (T)(o[part * kJd + jd][4 * q + i] * inv);
        *reinterpret_cast<t4*>(lds + col * kOutPitch + (32 * jd + 8 * q + 4 * kg) * (int)sizeof(T)) = x;
      }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(lds + (8 * i + (lane >> 3)) * kOutPitch + 16 * (lane & 7));
      if (ok[i]) *reinterpret_cast<u32x4*>(to[i] + 32 * kJd * part + (16 / (int)sizeof(T)) * (lane & 7)) = x;
    }
  }
}

// NRB blocks of 32 rows a wave; kParts = 2: the waves are two row groups times
// two halves of a step's keys, joined at a unit's end, so that a tile has half
// of the rows and an operand from LDS still serves as many MFMAs.
template <int NRB, int kParts>
__global__ __launch_bounds__(kPreThreads, 1) void prefill_kernel(PrefillArgs a) {
  __shared__ __attribute__((aligned(16))) char kl[kKBufs * kKSize], vl[kVBufs * kVSize];
  __shared__ __attribute__((aligned(16))) char outl[4][32 * kOutPitch];
  __shared__ Plan plan;
  __shared__ int64_t q_off[kPreThreads], out_off[kPreThreads];   // elements from a tile's first row of its first head
  constexpr int kBlocks = 2 / kParts;              // 32-key blocks of a step for a wave
  constexpr int kOps = 8 * kBlocks;                // operands of V, and of K, of a step
  constexpr int kSlots = 2 * kOps * NRB;           // MFMAs of a step
  constexpr int kGroups = 4 / kParts;              // row groups
  const int tid = threadIdx.x, lane = tid & 63, col = lane & 31, kg = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int part = wave / kGroups;                 // of the keys
  const int heads = a.Hkv * a.head_blocks, gh = blockIdx.x % heads;
  const int g = gh / a.head_blocks, hb = gh % a.head_blocks;
  const int w = blockIdx.x / heads, ws = gridDim.x / heads;   // workgroups of this head group
  const float sl2 = a.scale * kLog2e;
  const int row0 = wave % kGroups * (32 * NRB);    // of the wave in the tile
  const int64_t head0 = g * a.R + hb * a.rows_head;
  {
    const int ti = tid / a.rows_head, hr = tid - ti * a.rows_head;
    const bool head_ok = hb * a.rows_head + hr < a.R;
    q_off[tid] = head_ok ? ti * a.q_st + hr * a.q_sh : 0;
    out_off[tid] = head_ok ? ti * a.out_st + hr * a.out_sh : -1;
  }
  int bad = 0;
  if (a.B <= kSorted) {
    plan_levels(a, plan, &bad);
    if (blockIdx.x != 0) bad = 0;                  // (the first workgroup reports the prompts' bounds)
  } else {
    for (int b = blockIdx.x * kPreThreads + tid; b < a.B; b += gridDim.x * kPreThreads) prompt_of(a, b, &bad);
  }
  if (bad) atomicOr(a.err, bad);

  // rows of a step go from memory to LDS by the load itself: block b of 16 holds
  // rows b + 16 s (s = lane / 16), wave w fills blocks 4 w .. 4 w + 3
  const uint32_t kss = 2u * (uint32_t)a.k_st, vss = 2u * (uint32_t)a.v_st;
  const std::integral_constant<int, kKPitch> kpitch{};
  const std::integral_constant<int, kVPitch> vpitch{};
  auto load_row = [&](int t) { return 16 * ((t & 63) >> 4) + 4 * wave; };
  auto load_chunk = [&](int t) { return 16u * (t & 15); };
  const uint32_t kvo = (uint32_t)load_row(tid) * kss + load_chunk(tid), vvo = (uint32_t)load_row(tid) * vss + load_chunk(tid);
  auto load_step = [&](const char* rows, uint32_t ss, uint32_t vo, char* dst, auto pitch_, int last) {
    constexpr int kPitch = decltype(pitch_)::value;
    const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)(dst + 4 * wave * kPitch);
    ss = here(ss);
    uint32_t at[4];
    if (last >= kStep - 1) {
#pragma unroll
      for (int i = 0; i < 4; ++i) at[i] = vo + i * ss;
    } else {                                       // rows past the last key load that key again
      const int t = here(tid);
#pragma unroll
      for (int i = 0; i < 4; ++i) at[i] = (uint32_t)min(load_row(t) + i, last) * ss + load_chunk(t);
    }
    // As assembly: see the 128-key routine in tile_attn.hpp. In one statement, since
    // the compiler does not know it as loads: an SGPR that a vector instruction
    // wrote (the reload of a spilled one) needs 5 wait states, and m0 needs 1. It
    // says that it sets m0, of which the compiler warns (it keeps nothing there).
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
    asm volatile(
        "s_mov_b32 m0, %5\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %0, %4\n\t"
        "s_add_u32 m0, m0, %6\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %4\n\t"
        "s_add_u32 m0, m0, %6\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %4\n\t"
        "s_add_u32 m0, m0, %6\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %3, %4" ::"v"(at[0]),
        "v"(at[1]), "v"(at[2]), "v"(at[3]), "s"(rows), "s"(lds), "i"(kPitch)
        : "memory", "m0", "scc");
#pragma clang diagnostic pop
  };
  auto barrier = [&]() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  auto barrier_lds = [&]() {                       // what was written to LDS is read behind it
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    barrier();
  };
  auto after = [&](int x, int size, int bufs) { return x + size == bufs * size ? 0 : x + size; };

  struct Unit {
    int q0, i0, cnt, keys;
    const char *k, *v;
  };
  auto unit_at = [&](int i) {
    const int4 x = plan.units[i];
    Unit u;
    u.q0 = __builtin_amdgcn_readfirstlane(x.x);
    const int n = __builtin_amdgcn_readfirstlane(x.y);
    u.i0 = __builtin_amdgcn_readfirstlane(x.z) * a.tile_tokens;
    u.cnt = min(a.tile_tokens, n - u.i0);
    u.keys = u.i0 + u.cnt;                         // keys [0, keys) are visible to some row, [0, i0] to every row
    u.k = (const char*)((const __bf16*)a.k + (int64_t)u.q0 * a.k_st + g * a.k_sh);
    u.v = (const char*)((const __bf16*)a.v + (int64_t)u.q0 * a.v_st + g * a.v_sh);
    return u;
  };
  struct Row {
    bool ok;
    int ti, head;
    int64_t row;
  };
  auto row_of = [&](const Unit& u, int thread, int rb) {
    const int r = ((thread >> 6) % kGroups) * (32 * NRB) + 32 * rb + (thread & 31);
    // r / rows_head for r < 256: r + 1/2 is at least 2^-9 of it away from a multiple
    const int ti = (int)(((float)r + 0.5f) * a.rows_head_inv), hr = r - ti * a.rows_head;
    const bool ok = ti < u.cnt && hb * a.rows_head + hr < a.R;
    return Row{ok, ti, g * a.R + hb * a.rows_head + (ok ? hr : 0), (int64_t)(u.q0 + u.i0 + (ok ? ti : 0))};
  };

  bf16x8 qv[NRB][8];
  int k0 = 0, v0 = 0;                              // buffers of a unit's first step
  // what a unit needs before its first step; its query rows as they lie in memory, 16 lanes a row
  auto request = [&](const Unit& u, int kb, int vb) {
    const int last = u.keys - 1;
    load_step(u.k, kss, kvo, kl + kb, kpitch, last);
    if (last >= kStep) load_step(u.k + kStep * (int64_t)kss, kss, kvo, kl + after(kb, kKSize, kKBufs), kpitch, last - kStep);
    load_step(u.v, vss, vvo, vl + vb, vpitch, last);
    if (last >= 2 * kStep)
      load_step(u.k + 2 * kStep * (int64_t)kss, kss, kvo, kl + after(after(kb, kKSize, kKBufs), kKSize, kKBufs), kpitch,
                last - 2 * kStep);
    if (last >= kStep) load_step(u.v + kStep * (int64_t)vss, vss, vvo, vl + after(vb, kVSize, kVBufs), vpitch, last - kStep);
    const int t = here(tid), rows = u.cnt * a.rows_head;
    const __bf16* qb = (const __bf16*)a.q + (int64_t)(u.q0 + u.i0) * a.q_st + head0 * a.q_sh + 8 * (t & 15);
    const int r0 = row0 + ((t & 63) >> 4);
#pragma unroll
    for (int rb = 0; rb < NRB; ++rb) {
      int64_t off[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) off[i] = q_off[r0 + 32 * rb + 4 * i];
#pragma unroll
      for (int i = 0; i < 8; ++i)                  // (a row past the tile's is its first one again, and not stored)
        qv[rb][i] = load_bf16x8(qb + (r0 + 32 * rb + 4 * i < rows ? off[i] : 0));
    }
  };

  const int kread = (col & 15) * kKPitch + (col >> 4) * 256 + 16 * kg + 512 * part;
  const int tr_row = 4 * kg + ((lane & 15) >> 2), tr_col = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
  const int vread = tr_row * kVPitch + 2 * tr_col + 512 * part;
  // operand i of an iteration: below kOps of V (16 keys i / 4, 32 dimensions i % 4), then of K (32 keys, 16 dimensions)
  auto read = [&](auto i_, const char* vb, const char* kb) -> bf16x8 {
    constexpr int i = decltype(i_)::value;
    if constexpr (i < kOps) {
      const char* vp = vb + 256 * (i >> 2) + 64 * (i & 3);
      const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)vp);
      const i16x4 up = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(vp + 8 * kVPitch));
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, up, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
      return *reinterpret_cast<const bf16x8*>(kb + 512 * ((i - kOps) >> 3) + 32 * (i & 7));
    }
  };
  const std::true_type yes{};
  const std::false_type no{};

  for (int base = 0;; base += kPreThreads) {
    // this workgroup's next units: every second round in opposite order, so that the sums of a longest-first list even out
    __syncthreads();
    {
      const int k = base + tid;
      plan.units[tid] = unit_of(a, plan, k * ws + ((k & 1) ? ws - 1 - w : w));
      if (tid == 0) plan.units[kPreThreads] = make_int4(0, 0, 0, kNoTile);
    }
    __syncthreads();
    auto next_of = [&](int i) {                    // the next entry that is a unit; kPreThreads if none
      while (i < kPreThreads && __builtin_amdgcn_readfirstlane(plan.units[i].w) == kNoTile) ++i;
      return i;
    };
    int at = next_of(0);
    if (at < kPreThreads && __builtin_amdgcn_readfirstlane(plan.units[at].w) == kEnd) break;
    if (at == kPreThreads) continue;
    Unit u = unit_at(at);
    request(u, k0, v0);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    bool end = false;
    for (;;) {
      at = next_of(at + 1);
      end = at < kPreThreads && __builtin_amdgcn_readfirstlane(plan.units[at].w) == kEnd;
      const bool more = at < kPreThreads && !end;
      Unit un = u;
      if (more) un = unit_at(at);
      const int n = (u.keys + kStep - 1) / kStep;
      const int n_full = (u.i0 + 1) / kStep;       // steps [0, n_full) need no mask
      int limit[NRB];
#pragma unroll
      for (int rb = 0; rb < NRB; ++rb) {
        const Row r = row_of(u, tid, rb);
        limit[rb] = (r.ok ? u.i0 + r.ti : u.keys - 1) - 32 * part - 4 * kg;
      }
      barrier();                                   // the first steps' rows are in LDS
      int v_cur = v0, v_next2 = after(after(v0, kVSize, kVBufs), kVSize, kVBufs), v_prev = after(v_next2, kVSize, kVBufs);
      {
        // The query rows become MFMA operands through the V buffers that nothing is in, half of one a wave. (Loaded as
        // operands, 32 rows with 16 bytes of each lane, they kept the load path busy for 4 times as long.)
        constexpr int kPitch = 256 + 16;
        static_assert(64 * kPitch == kVSize, "two waves' rows in a buffer");
        const int t = here(tid) & 63;
        char* const own = vl + (wave & 2 ? v_prev : v_next2) + (wave & 1) * (32 * kPitch);
        char* const to = own + (t >> 4) * kPitch + 16 * (t & 15);
        const char* const from = own + (t & 31) * kPitch + 16 * (t >> 5);
#pragma unroll
        for (int rb = 0; rb < NRB; ++rb) {
#pragma unroll
          for (int i = 0; i < 8; ++i) *reinterpret_cast<bf16x8*>(to + 4 * i * kPitch) = qv[rb][i];
#pragma unroll
          for (int c = 0; c < 8; ++c) qv[rb][c] = *reinterpret_cast<const bf16x8*>(from + 32 * c);
        }
      }
#pragma unroll
      for (int rb = 0; rb < NRB; ++rb)
#pragma unroll
        for (int c = 0; c < 8; ++c) asm volatile("" : "+a"(qv[rb][c]));
      const f32x16 zero = {};
      f32x16 o[NRB][4], s[kBlocks][NRB];                 // O^T, and S^T(j) of the current step [32 keys][row block]
      bf16x8 pb[NRB][2 * kBlocks];                           // P^T(j - 1)
      bf16x8 ring[kRing];
      float nm[NRB], l[NRB], l2[NRB];              // minus the maximum, and two sums
#pragma unroll
      for (int rb = 0; rb < NRB; ++rb) {
        l[rb] = l2[rb] = 0.f;
#pragma unroll
        for (int jd = 0; jd < 4; ++jd) o[rb][jd] = zero;
      }
      {
        const char* kb = kl + k0 + kread;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
          for (int c = 0; c < 8; ++c) {
            const bf16x8 x = *reinterpret_cast<const bf16x8*>(kb + 512 * b + 32 * c);
#pragma unroll
            for (int rb = 0; rb < NRB; ++rb) s[b][rb] = mfma_32x32x16(x, qv[rb][c], c == 0 ? zero : s[b][rb]);
          }
#pragma unroll
        for (int rb = 0; rb < NRB; ++rb) {
          float mx = kNegInf;
          const int lim = here(limit[rb]);         // (else the compiler keeps these comparisons for the softmax)
#pragma unroll
          for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e)
              mx = fmaxf(mx, 32 * b + 8 * (e >> 2) + (e & 3) <= lim ? s[b][rb][e] : kNegInf);
          // (a row without a key in this part's half of the first step has none in it at all)
          nm[rb] = kParts == 2 && lim + 4 * kg < 0 ? 0.f : -max_l32(mx) * sl2;
        }
      }
      barrier();                                   // K(0)'s buffer is free
      // buffers of V(j - 1), V(j), V(j + 2), K(j + 1), K(j + 3), and the rows that come next
      int k_next = after(k0, kKSize, kKBufs), k_next3 = k0;
      const char* kp = u.k + 3 * kStep * (int64_t)kss;
      const char* vp = u.v + 2 * kStep * (int64_t)vss;
      // iteration j: the values of step j - 1, the softmax of step j, the scores of step j + 1
      auto body = [&](int j, auto pv_tag, auto s_tag, auto mask_tag) {
        constexpr bool kPV = decltype(pv_tag)::value, kS = decltype(s_tag)::value, kMask = decltype(mask_tag)::value;
        const char* vb = vl + v_prev + vread;
        const char* vb_next = vl + v_cur + vread;
        const char* kb = kl + k_next + kread;
        f32x16 sn[kBlocks][NRB], sf[kBlocks][NRB];
        u32x4 pn[NRB][2 * kBlocks];
        float t1, p0, p1, q0, q1;
        auto finish = [&](auto x_, int part) {     // sums and conversion of pair x
          constexpr int x = decltype(x_)::value;
          if constexpr (x >= 0) {
            constexpr int h = x / (4 * NRB), rb = (x >> 2) % NRB, e = x & 3;
            if (part == 0) {
              l[rb] += q0;
            } else {
              l2[rb] += q1;
              uint32_t w2 = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)q0, (__bf16)q1});
              asm volatile("" : "+v"(w2));
              pn[rb][h][e] = w2;
            }
          }
        };
        auto soft = [&](auto slot_) {
          constexpr int slot = decltype(slot_)::value, x = slot >> 1;
          constexpr int h = x / (4 * NRB), rb = (x >> 2) % NRB, e = 2 * (x & 3);
          if constexpr ((slot & 1) == 0) {
            float t0 = fmaf(s[h >> 1][rb][8 * (h & 1) + e], sl2, nm[rb]);
            t1 = fmaf(s[h >> 1][rb][8 * (h & 1) + e + 1], sl2, nm[rb]);
            if constexpr (kMask) {
              constexpr int z = 8 * (h & 1) + e, key = 32 * (h >> 1) + 8 * (z >> 2) + (z & 3);
              const int d = limit[rb] - j * kStep;
              if (key > d) t0 = kNegInf;
              if (key + 1 > d) t1 = kNegInf;
            }
            q0 = p0;
            q1 = p1;
            p0 = exp2_fast(t0);
            finish(std::integral_constant<int, x - 1>{}, 0);
          } else {
            p1 = exp2_fast(t1);
            finish(std::integral_constant<int, x - 1>{}, 1);
          }
        };
        if constexpr (kS) {
          if (j + 2 < n) load_step(vp, vss, vvo, vl + v_next2, vpitch, u.keys - 1 - (j + 2) * kStep);
          if (j + 3 < n) load_step(kp, kss, kvo, kl + k_next3, kpitch, u.keys - 1 - (j + 3) * kStep);
          vp += kStep * (int64_t)vss;
          kp += kStep * (int64_t)kss;
          asm volatile("s_nop 1" ::"a"(qv[0][0]), "a"(qv[0][1]), "a"(qv[0][2]), "a"(qv[0][3]), "a"(qv[0][4]),
                       "a"(qv[0][5]), "a"(qv[0][6]), "a"(qv[0][7]));
          if constexpr (NRB == 2)
            asm volatile("s_nop 1" ::"a"(qv[NRB - 1][0]), "a"(qv[NRB - 1][1]), "a"(qv[NRB - 1][2]), "a"(qv[NRB - 1][3]),
                         "a"(qv[NRB - 1][4]), "a"(qv[NRB - 1][5]), "a"(qv[NRB - 1][6]), "a"(qv[NRB - 1][7]));
          __builtin_amdgcn_sched_barrier(0);
        } else if (more) {
          request(un, k_next, after(v_cur, kVSize, kVBufs));
        }
        constexpr int i0 = kPV ? 0 : kOps, i1 = kS ? 2 * kOps : kOps;
        if constexpr (!kPV && kS) each<kOps, kOps + kAhead>([&](auto i) { ring[i % kRing] = read(i, vb, kb); });
        if constexpr (!kPV) each<0, kSlots / 2>([&](auto i) { soft(i); });
        each<i0, i1>([&](auto i) {
          // (behind the last, the first of the next iteration: values of step j)
          // Two at a time, with one wait for both (17 waits a step instead of 33: 0.7% of a 16K prompt, 4% of short steps;
          // four at a time spilled registers): the counter falls in order, and behind the second are the reads of the
          // next four operands (two for one of V).
          if constexpr ((i & 1) == 0) {
            each<i + kAhead, i + kAhead + 2>([&](auto k) {
              if constexpr (k < i1)
                ring[k % kRing] = read(k, vb, kb);
              else
                ring[k % kRing] = read(std::integral_constant<int, k - i1>{}, vb_next, kb);
            });
            constexpr auto reads = [](int k) { return k % i1 >= i0 && k % i1 < kOps ? 2 : 1; };
            constexpr int behind = reads(i + 2) + reads(i + 3) + reads(i + 4) + reads(i + 5);
            __builtin_amdgcn_s_waitcnt(0xc07f | behind << 8);
          }
          __builtin_amdgcn_sched_barrier(0);
          each<0, NRB>([&](auto rb) {
            if constexpr (i < kOps)
              o[rb][i & 3] = mfma_32x32x16(ring[i % kRing], pb[rb][i >> 2], o[rb][i & 3]);
            else if constexpr ((i & 7) == 0)
              mfma_first(sn[(i - kOps) >> 3][rb], ring[i % kRing], qv[rb][0]);
            else if constexpr ((i & 7) == 7)
              mfma_last(sf[(i - kOps) >> 3][rb], sn[(i - kOps) >> 3][rb], ring[i % kRing], qv[rb][7]);
            else
              mfma_next(sn[(i - kOps) >> 3][rb], ring[i % kRing], qv[rb][i & 7]);
            __builtin_amdgcn_sched_barrier(0);
            soft(std::integral_constant<int, NRB * i + rb>{});
            __builtin_amdgcn_sched_barrier(0);
          });
          if constexpr (kBlocks == 2 && i == kOps + 8) each<0, NRB>([&](auto rb) { kept(sn[0][rb]); });
        });
        if constexpr (!kS) each<kSlots / 2, kSlots>([&](auto i) { soft(i); });
        q0 = p0;
        q1 = p1;
        finish(std::integral_constant<int, kSlots / 2 - 1>{}, 0);
        finish(std::integral_constant<int, kSlots / 2 - 1>{}, 1);
#pragma unroll
        for (int rb = 0; rb < NRB; ++rb) asm volatile("" : "+v"(l[rb]), "+v"(l2[rb]));
        if constexpr (i0 == i1) each<0, kAhead>([&](auto i) { ring[i] = read(i, vb_next, kb); });
        if constexpr (kS) {
          asm volatile("s_nop 11" ::: "memory");   // S^T(j + 1) is complete
          each<0, NRB>([&](auto rb) { kept(sn[kBlocks - 1][rb]); });
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int rb = 0; rb < NRB; ++rb)
#pragma unroll
          for (int h = 0; h < 2 * kBlocks; ++h) pb[rb][h] = __builtin_bit_cast(bf16x8, pn[rb][h]);
        if constexpr (kS) {
#pragma unroll
          for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int rb = 0; rb < NRB; ++rb) s[b][rb] = sf[b][rb];
        }
      };
      auto turn = [&](int j) {
        // the rows of V(j + 1) and K(j + 2), requested an iteration ago, have come
        if (j + 3 < n)
          asm volatile("s_waitcnt vmcnt(8)" ::: "memory");
        else
          asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        barrier();
        v_prev = v_cur;
        v_cur = after(v_cur, kVSize, kVBufs);
        v_next2 = after(v_next2, kVSize, kVBufs);
        k_next = after(k_next, kKSize, kKBufs);
        k_next3 = after(k_next3, kKSize, kKBufs);
      };
      if (n == 1) {
        body(0, no, no, yes);
      } else {
        if (n_full > 0)
          body(0, no, yes, no);
        else
          body(0, no, yes, yes);
        turn(0);
        int j = 1;
        for (; j + 1 < n && j < n_full; ++j) {
          body(j, yes, yes, no);
          turn(j);
        }
        for (; j + 1 < n; ++j) {
          body(j, yes, yes, yes);
          turn(j);
        }
        body(j, yes, no, yes);
      }
      // the values of the last step (its first operands are read)
      {
        const char* vb = vl + v_cur + vread;
        each<0, kOps>([&](auto i) {
          if constexpr (i + kAhead < kOps)
            ring[(i + kAhead) % kRing] = read(std::integral_constant<int, i + kAhead>{}, vb, vb);
#pragma unroll
          for (int rb = 0; rb < NRB; ++rb)
            o[rb][i & 3] = mfma_32x32x16(ring[i % kRing], pb[rb][i >> 2], o[rb][i & 3]);
        });
      }
      k0 = k_next;
      v0 = after(v_cur, kVSize, kVBufs);
#pragma unroll
      for (int rb = 0; rb < NRB; ++rb) l[rb] += l2[rb];
      if constexpr (kParts == 2) {
        // The second parts' sums join the first's, 16 KB of a row block at a time
        // through the V buffers that hold nothing any more (of the last two steps).
        float* const buf = reinterpret_cast<float*>(vl + (wave % kGroups ? v_cur : v_prev)) + 4 * lane;
        float* const ml = reinterpret_cast<float*>(outl[2 + wave % kGroups]) + 2 * lane;
#pragma unroll
        for (int rb = 0; rb < NRB; ++rb) {
          barrier_lds();
          if (part == 1) {
            const Row r = row_of(u, here(tid), rb);
            const bool sees = (r.ok ? u.i0 + r.ti : u.keys - 1) >= 32;
            const float l1 = sum_l32(l[rb]);
            ml[0] = sees && l1 < 0.5f ? -kNegInf : l1;   // (see below: again)
            ml[1] = -nm[rb];
#pragma unroll
            for (int jd = 0; jd < 4; ++jd)
#pragma unroll
              for (int q = 0; q < 4; ++q)
                *reinterpret_cast<f32x4*>(buf + 256 * (4 * jd + q)) =
                    f32x4{o[rb][jd][4 * q], o[rb][jd][4 * q + 1], o[rb][jd][4 * q + 2], o[rb][jd][4 * q + 3]};
          }
          barrier_lds();
          if (part == 0) {
            // The bases are of the first keys only, so a sum may be up to 2^128 times its part's weight and the lower
            // part still count where 2^(m0 - m1) is flushed to zero (below 2^-126). Far parts are joined 2^96 higher,
            // where it is not down to a distance of 222 (and a part that much lower does not count).
            const float l1 = ml[0], m0 = -nm[rb], m1 = l1 == 0.f ? kNegInf : ml[1], m = fmaxf(m0, m1);
            const float up = l1 != 0.f && m - fminf(m0, m1) > 120.f ? 96.f : 0.f;
            const float w0 = exp2_fast(m0 - m + up), w1 = exp2_fast(m1 - m + up);
            l[rb] = l[rb] * w0 + (kg ? 0.f : l1 * w1);
            nm[rb] = up - m;
#pragma unroll
            for (int jd = 0; jd < 4; ++jd)
#pragma unroll
              for (int q = 0; q < 4; ++q) {
                const f32x4 x = *reinterpret_cast<const f32x4*>(buf + 256 * (4 * jd + q));
#pragma unroll
                for (int i = 0; i < 4; ++i) o[rb][jd][4 * q + i] = fmaf(x[i], w1, o[rb][jd][4 * q + i] * w0);
              }
          }
        }
      }
      const int t = here(tid);
      const bool mine = kParts == 1 || part == 0;  // these rows are this wave's to store
      bool odd = false;
#pragma unroll
      for (int rb = 0; rb < NRB; ++rb) {
        l[rb] = sum_l32(l[rb]);
        // The first keys' maximum has a probability of 1 but for its rounding. That is half a power of two from 2^24
        // powers on and past all of them from 2^32 on, where nothing may be left of a sum.
        odd |= l[rb] < 0.5f;
      }
      const bool again = __builtin_amdgcn_ballot_w64(odd || odd_values<NRB>(o, l)) != 0;
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // the next unit's rows have come (before the stores, which need not)
#pragma unroll
      for (int rb = 0; rb < NRB; ++rb) {
        const float l_tot = l[rb];
        const Row r = row_of(u, t, rb);
        if (again || !mine) continue;
        const float inv = 1.f / l_tot;
        const int64_t at = (int64_t)(u.q0 + u.i0) * a.out_st + head0 * a.out_sh;
        auto row = [&](auto* out, int i, bool* ok) {
          const int x = row0 + 32 * rb + i;
          const int64_t off = out_off[x];
          *ok = x < u.cnt * a.rows_head && off >= 0;
          return out + at + off;
        };
        if (a.out_f32)
          store_block<float>(o[rb], inv, outl[wave], t & 63, [&](int i, bool* ok) { return row((float*)a.out, i, ok); });
        else
          store_block<__bf16>(o[rb], inv, outl[wave], t & 63, [&](int i, bool* ok) { return row((__bf16*)a.out, i, ok); });
        if (a.lse && r.ok && (t & 63) < 32)
          a.lse[r.row * a.lse_st + (int64_t)r.head * a.lse_sh] = (__builtin_amdgcn_logf(l_tot) - nm[rb]) * kLn2;
      }
      if (again && mine) {
        for (int rb = 0; rb < NRB; ++rb)
          attend_again((ConstPrefillArgs*)__builtin_amdgcn_kernarg_segment_ptr(), row0 + 32 * rb, u.q0, u.i0,
                       u.cnt, g, hb);
      }
      if (!more) break;
      u = un;
    }
    if (end) break;
  }
}

}  // namespace

hipError_t launch_prefill(const PrefillArgs& args, int cus, hipStream_t stream, KernelTimer* timer) {
  PrefillArgs a = args;
  const int64_t tiles = a.rows / a.tile_tokens;
  a.chunk_log = a.rows / a.B >= 16 * a.tile_tokens ? 2 : 0;
  while ((tiles >> a.chunk_log) + 1 > kLevels) ++a.chunk_log;
  const int64_t heads = (int64_t)a.Hkv * a.head_blocks;
  const int64_t most = tiles + ((int64_t)a.B << a.chunk_log);    // ranks of a head group, at most
  const unsigned grid = (unsigned)(heads * std::max<int64_t>(1, std::min<int64_t>(cus / heads, most)));
  a.rows_head_inv = 1.f / (float)a.rows_head;
  if (timer) (void)hipEventRecord(timer->start, stream);
  if (a.tile_rows == 256)
    prefill_kernel<2, 1><<<grid, kPreThreads, 0, stream>>>(a);
  else if (a.tile_rows == 128)
    prefill_kernel<2, 2><<<grid, kPreThreads, 0, stream>>>(a);
  else
    prefill_kernel<1, 2><<<grid, kPreThreads, 0, stream>>>(a);
  if (timer) (void)hipEventRecord(timer->stop, stream);
  return hipGetLastError();
}

}  // namespace rl
