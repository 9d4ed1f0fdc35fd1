// Causal attention over whole packed prompts: row i of a prompt attends to its
// rows 0 .. i, whose K and V are packed rows too (no pages).
//
// A unit of work is (prompt b, KV head g, block of query heads, run of tokens):
// up to 256 query rows, token-major (row r -> token r / RB, head r % RB), which
// all read the same keys; one workgroup computes it.
#include <algorithm>

#include "kernels.hpp"
#include "tile_attn.hpp"

namespace rl {

namespace {

constexpr int kPreWaves = 8;

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

// Prompt b's tiles take places tile_base(b), tile_base(b) + 1, ...: a prompt of
// n rows from row q0 on has at most (q0 + n) / tt + 1 - q0 / tt of them, so
// places need no sum over the prompts.
__device__ __forceinline__ int tile_base(const PrefillArgs& a, int b) {
  const int q0 = min(max(a.indptr[(int64_t)b * a.indptr_s], 0), a.rows);
  return q0 / a.tile_tokens + b;
}

// Whether a lane's part of O^T holds an infinity or a NaN (by the bits: device
// code is compiled assuming no NaN operands).
__device__ __forceinline__ bool odd_values(const f32x16 (&o)[4]) {
  uint32_t top = 0;
#pragma unroll
  for (int jd = 0; jd < 4; ++jd)
#pragma unroll
    for (int e = 0; e < 16; ++e) top = max(top, __float_as_uint(o[jd][e]) & 0x7fffffffu);
  return top >= 0x7f800000u;
}

// A masked key has probability 0, and 0 times an infinity or a NaN in its value
// row is NaN: only such values bring one into a row that does not see them. So a
// unit whose result holds one is computed again, with the tiles only up to the
// first masked key and the others here, key by key, each for the rows that see it.
__device__ __forceinline__ void attend_keys(const PrefillArgs& a, int q0, int g, int t0, int keys, int limit,
                                            float sl2, const bf16x8 (&qv)[8], f32x16 (&o)[4], float& m, float& l) {
  const int kg = (threadIdx.x & 63) >> 5;
#pragma unroll 1
  for (int t = t0; t < keys; ++t) {
    const __bf16* kr = (const __bf16*)a.k + (int64_t)(q0 + t) * a.k_st + g * a.k_sh;
    const __bf16* vr = (const __bf16*)a.v + (int64_t)(q0 + t) * a.v_st + g * a.v_sh + 4 * kg;
    float s = 0.f;
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      const bf16x8 x = load_bf16x8(kr + 16 * c + 8 * kg);
#pragma unroll
      for (int e = 0; e < 8; ++e) s = fmaf((float)x[e], (float)qv[c][e], s);
    }
    s = sum_l32(s) * sl2;
    if (t > limit) continue;
    const float m_new = fmaxf(m, s), alpha = exp2_fast(m - m_new), p = exp2_fast(s - m_new);
    m = m_new;
    l = l * alpha + (kg ? 0.f : p);
#pragma unroll
    for (int jd = 0; jd < 4; ++jd)
#pragma unroll
      for (int e = 0; e < 16; ++e)
        o[jd][e] = fmaf(p, (float)vr[32 * jd + 8 * (e >> 2) + (e & 3)], o[jd][e] * alpha);
  }
}

__global__ __launch_bounds__(kPreWaves * 64, 2) void prefill_kernel(PrefillArgs a) {
  __shared__ u16 ks[kKeys][kKStride];
  __shared__ u16 vs[kKeys][kVStride];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int col = lane & 31, kg = lane >> 5;
  const int heads = a.Hkv * a.head_blocks;
  const int place = blockIdx.x / heads, gh = blockIdx.x % heads;
  const int g = gh / a.head_blocks, hb = gh % a.head_blocks;
  int bad = 0;
  if (gh == 0 && place < a.B) {          // (some workgroup checks each prompt's bounds)
    prompt_of(a, place, &bad);
    if (bad && tid == 0) atomicOr(a.err, bad);
  }
  int lo = 0, hi = a.B - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (tile_base(a, mid) <= place) lo = mid; else hi = mid - 1;
  }
  const Prompt p = prompt_of(a, lo, &bad);
  const int64_t i0_64 = (int64_t)(place - tile_base(a, lo)) * a.tile_tokens;
  if (i0_64 < 0 || i0_64 >= p.n) return;
  const int i0 = (int)i0_64;
  const int cnt = min(a.tile_tokens, p.n - i0);
  const int keys = i0 + cnt;             // keys [0, keys) are visible to some row, [0, i0] to every row

  const int RB = a.rows_head, r = wave * kWaveRows + col;
  const int ti = r / RB, hr = r - ti * RB;
  const bool ok = ti < cnt && hb * RB + hr < a.R;
  const int limit = ok ? i0 + ti : keys - 1;
  const int64_t row = p.q0 + i0 + (ok ? ti : 0);
  const int head = g * a.R + hb * RB + (ok ? hr : 0);
  bf16x8 qv[8];
  load_q_operand((const __bf16*)a.q + row * a.q_st + (int64_t)head * a.q_sh, ok, qv);
  const float sl2 = a.scale * kLog2e;
  f32x16 o[4];
  float m, l;
  const int ld_row = tid >> 4, ld_chunk = (tid & 15) * 8;
  const int tr_row = 4 * kg + ((lane & 15) >> 2);
  const int tr_col = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
  auto attend = [&](int t_end) {
#pragma unroll
  for (int jd = 0; jd < 4; ++jd)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[jd][e] = 0.f;
  m = kNoKey;
  l = 0.f;
  for (int t0 = 0; t0 < t_end; t0 += kKeys) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int t = min(t0 + ld_row + 32 * i, keys - 1);
      const int64_t kr = p.q0 + t;
      *reinterpret_cast<bf16x8*>(&ks[ld_row + 32 * i][ld_chunk]) =
          load_bf16x8((const __bf16*)a.k + kr * a.k_st + g * a.k_sh + ld_chunk);
      *reinterpret_cast<bf16x8*>(&vs[ld_row + 32 * i][ld_chunk]) =
          load_bf16x8((const __bf16*)a.v + kr * a.v_st + g * a.v_sh + ld_chunk);
    }
    __syncthreads();
    f32x16 sc[2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
      for (int e = 0; e < 16; ++e) sc[kb][e] = 0.f;
#pragma unroll
      for (int c = 0; c < 8; ++c)
        sc[kb] = mfma_32x32x16(*reinterpret_cast<const bf16x8*>(&ks[32 * kb + col][16 * c + 8 * kg]), qv[c], sc[kb]);
    }
    float mt = kNegInf;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        if (t0 + 32 * kb + 8 * (e >> 2) + 4 * kg + (e & 3) > limit) sc[kb][e] = kNegInf;
        mt = fmaxf(mt, sc[kb][e]);
      }
    const float m_new = fmaxf(m, max_l32(mt) * sl2);
    const float alpha = exp2_fast(m - m_new);
    m = m_new;
    l *= alpha;
#pragma unroll
    for (int jd = 0; jd < 4; ++jd) o[jd] *= alpha;
    bf16x8 pb[4];
#pragma unroll
    for (int h = 0; h < 4; ++h)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x = exp2_fast(fmaf(sc[h >> 1][8 * (h & 1) + e], sl2, -m));
        l += x;
        pb[h][e] = (__bf16)x;
      }
#pragma unroll
    for (int h = 0; h < 4; ++h)
#pragma unroll
      for (int jd = 0; jd < 4; ++jd) {
        const u16* vp = &vs[16 * h + tr_row][32 * jd + tr_col];
        const i16x4 x0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)vp);
        const i16x4 x1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(vp + 8 * kVStride));
        const i16x8 v8 = __builtin_shufflevector(x0, x1, 0, 1, 2, 3, 4, 5, 6, 7);
        o[jd] = mfma_32x32x16(__builtin_bit_cast(bf16x8, v8), pb[h], o[jd]);
      }
  }
  };
  attend(keys);
  if (__syncthreads_or(odd_values(o))) {
    const int whole = (i0 + 1) / kKeys * kKeys;
    attend(whole);
    attend_keys(a, p.q0, g, whole, keys, limit, sl2, qv, o, m, l);
  }
  const float l_tot = sum_l32(l);
  if (!ok) return;
  const float inv = 1.f / l_tot;
  if (a.out_f32)
    store_o_row((float*)a.out + row * a.out_st + (int64_t)head * a.out_sh, o, inv);
  else
    store_o_row((__bf16*)a.out + row * a.out_st + (int64_t)head * a.out_sh, o, inv);
  if (a.lse && lane < 32)
    a.lse[row * a.lse_st + (int64_t)head * a.lse_sh] = (m + __builtin_amdgcn_logf(l_tot)) * kLn2;
}

}  // namespace

hipError_t launch_prefill(const PrefillArgs& a, hipStream_t stream, KernelTimer* timer) {
  const int64_t places = a.rows / a.tile_tokens + a.B;
  const unsigned grid = (unsigned)(places * a.Hkv * a.head_blocks);
  if (timer) (void)hipEventRecord(timer->start, stream);
  prefill_kernel<<<grid, kPreWaves * 64, 0, stream>>>(a);
  if (timer) (void)hipEventRecord(timer->stop, stream);
  return hipGetLastError();
}

}  // namespace rl
