// Gradient of normed and rotated head rows. With x a row of 128, r = (mean x^2 +
// eps)^(-1/2), n = r x and out = turn(w n):
//   g = turned back gradient of out,  u = w g,
//   d_x = r (u - n mean(u n)),  d_w = sum over rows and heads of g n.
//
// A pass over two rows in and one out, HBM-bound at 3 x 256 bytes a head row, beside
// some 350 VALU instructions for eight of them (46% busy). A wave takes eight
// head rows of a row at a time and loads the next ones before it uses these, a
// workgroup rows of q or of k only, and its sums of the weights' gradients stay in
// registers until it is through; they are added up in one order by a second launch, so
// that the same call gives the same bits. 16384 rows of 64 + 8 heads take 165 us (5.5
// TB/s) with eight workgroups a CU, 185 with four, and 3.4-6 for the sums.
#include <algorithm>

#include "kernels.hpp"
#include "rope_rows.hpp"

namespace rl {

namespace {

constexpr int kGradThreads = 256, kGradWaves = kGradThreads / 64;

__global__ __launch_bounds__(kGradThreads) void rope_grad_kernel(RopeGradArgs a) {
  __shared__ __attribute__((aligned(16))) float2 cs[kGradWaves][64];
  __shared__ float sums[kGradWaves][kHeadDim];
  const int lane = threadIdx.x & 63, d = lane & 7;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool is_k = blockIdx.x >= (unsigned)a.q_groups;
  const int group = is_k ? blockIdx.x - a.q_groups : blockIdx.x, groups = is_k ? a.k_groups : a.q_groups;
  const int heads = is_k ? a.r.Hkv : a.r.Hq, parts = (heads + 7) / 8, units = a.r.rows * parts;
  const __bf16* x = static_cast<const __bf16*>(is_k ? a.r.k : a.r.q);
  const __bf16* dy = static_cast<const __bf16*>(is_k ? a.dk_out : a.dq_out);
  __bf16* dx = static_cast<__bf16*>(is_k ? a.r.k_out : a.r.q_out);
  const int64_t x_st = is_k ? a.r.k_st : a.r.q_st, x_sh = is_k ? a.r.k_sh : a.r.q_sh;
  const int64_t dy_st = is_k ? a.gk_st : a.gq_st, dy_sh = is_k ? a.gk_sh : a.gq_sh;
  const int64_t dx_st = is_k ? a.r.ko_st : a.r.qo_st, dx_sh = is_k ? a.r.ko_sh : a.r.qo_sh;
  const Chunks c = chunks_of(d, a.r.freqs, a.r.interleaved);
  const void* w = is_k ? a.r.k_weight : a.r.q_weight;
  const f32x8 wa = load_weights(w, c.lo, a.r.weights_f32), wb = load_weights(w, c.hi, a.r.weights_f32);
  const int f = min(lane, a.r.freqs - 1);
  const double turns = -0.15915494309189533577 * (double)a.r.inv_freq[(int64_t)f * a.r.freq_s];   // (turned back)
  int axis = a.r.axes ? a.r.axes[(int64_t)f * a.r.axes_s] : 0;
  if ((unsigned)axis >= (unsigned)a.r.n_axes) {
    atomicOr(a.r.err, kErrAxis);
    axis = axis < 0 ? 0 : a.r.n_axes - 1;
  }
  // a unit's rows and position; those of the next are loaded before this one's are used
  struct Unit {
    bf16x8 xa, xb, ga, gb;
    int64_t r;
    int h, at;
    bool has;
  };
  auto load = [&](int u) {
    Unit t;
    const int r32 = u / parts;
    t.r = r32;
    t.h = (u - r32 * parts) * 8 + (lane >> 3);
    t.has = t.h < heads;
    t.xa = t.xb = t.ga = t.gb = zero_bf16x8();
    t.at = a.r.pos[(int64_t)min(lane, a.r.n_axes - 1) * a.r.pos_sa + t.r * a.r.pos_st];
    if (t.has) {
      const __bf16* px = x + t.r * x_st + t.h * x_sh;
      const __bf16* pg = dy + t.r * dy_st + t.h * dy_sh;
      t.xa = load_nt<bf16x8>(px + c.lo);
      t.xb = load_nt<bf16x8>(px + c.hi);
      t.ga = load_nt<bf16x8>(pg + c.lo);
      t.gb = load_nt<bf16x8>(pg + c.hi);
    }
    return t;
  };
  f32x8 sa = {}, sb = {};
  const int step = groups * kGradWaves;
  int u = group * kGradWaves + wave;
  Unit next;
  if (u < units) next = load(u);
  for (; u < units; u += step) {
    const Unit t = next;
    if (u + step < units) next = load(u + step);
    const int p = __shfl(t.at, axis);
    __builtin_amdgcn_wave_barrier();                // (the last unit's angles have been read)
    cs[wave][lane] = cos_sin_turns((double)p * turns);
    __builtin_amdgcn_wave_barrier();
    f32x8 na = widen(t.xa), nb = widen(t.xb), ya = widen(t.ga), yb = widen(t.gb);
    if (c.turned) {
      float2 cosines[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) cosines[e] = cs[wave][8 * d + e];
      turn(ya, yb, cosines, a.r.interleaved);
    }
    const float rms = inv_rms(na, nb, a.r.eps);
    na *= rms;
    nb *= rms;
    const f32x8 ua = ya * wa, ub = yb * wb;
    const float mean = row_sum8(dot16(ua, na, ub, nb)) * (1.f / kHeadDim);
    if (t.has) {
      __bf16* pd = dx + t.r * dx_st + t.h * dx_sh;
      store_chunk<true>(pd + c.lo, narrow((ua - na * mean) * rms));
      store_chunk<true>(pd + c.hi, narrow((ub - nb * mean) * rms));
      sa += ya * na;
      sb += yb * nb;
    }
  }
  // over the wave's eight rows of lanes, then over the waves
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    sa[e] += __shfl_xor(sa[e], 8);
    sb[e] += __shfl_xor(sb[e], 8);
    sa[e] = group_sum(sa[e]);
    sb[e] = group_sum(sb[e]);
    if (lane < 8) {
      sums[wave][c.lo + e] = sa[e];
      sums[wave][c.hi + e] = sb[e];
    }
  }
  __syncthreads();
  if (threadIdx.x < kHeadDim) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < kGradWaves; ++i) s += sums[i][threadIdx.x];
    a.parts[(int64_t)blockIdx.x * kHeadDim + threadIdx.x] = s;
  }
}

// Workgroup: sixteen columns of the sums of q (y = 0) or k; a thread's loads are in
// flight together, as few workgroups have much to read.
constexpr int kSumThreads = 1024, kSumCols = 16, kSumRows = kSumThreads / kSumCols;
__global__ __launch_bounds__(kSumThreads) void rope_grad_sum_kernel(RopeGradArgs a) {
  __shared__ float sums[kSumRows][kSumCols + 1];
  const int i = threadIdx.x % kSumCols, j = threadIdx.x / kSumCols, col = blockIdx.x * kSumCols + i;
  const bool is_k = blockIdx.y != 0;
  const int first = is_k ? a.q_groups : 0, end = is_k ? a.q_groups + a.k_groups : a.q_groups;
  float s = 0.f;
#pragma unroll 16
  for (int g = first + j; g < end; g += kSumRows) s += a.parts[(int64_t)g * kHeadDim + col];
  sums[j][i] = s;
  __syncthreads();
  for (int n = kSumRows / 2; n > 0; n >>= 1) {
    if (j < n) sums[j][i] += sums[j + n][i];
    __syncthreads();
  }
  if (j != 0) return;
  if (is_k)
    a.dk_weight[col * a.dkw_s] = sums[0][i];
  else
    a.dq_weight[col * a.dqw_s] = sums[0][i];
}

}  // namespace

hipError_t launch_rope_grad(const RopeGradArgs& a, hipStream_t stream, KernelTimer* timer) {
  if (timer) (void)hipEventRecord(timer->start, stream);
  if (a.q_groups + a.k_groups > 0) rope_grad_kernel<<<a.q_groups + a.k_groups, kGradThreads, 0, stream>>>(a);
  if (timer) (void)hipEventRecord(timer->stop, stream);
  rope_grad_sum_kernel<<<dim3(kHeadDim / kSumCols, a.dk_weight ? 2 : 1), kSumThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace rl
