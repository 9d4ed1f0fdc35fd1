// Gradient of normed and rotated head rows. With x a row of 128, r = (mean x^2 +
// eps)^(-1/2), n = r x and out = turn(w n):
//   g = turned back gradient of out,  u = w g,
//   d_x = r (u - n mean(u n)),  d_w = sum over rows and heads of g n.
//
// A pass over two rows in and one out, HBM-bound at 3 x 256 bytes a head row. A
// wave takes eight head rows of a row at a time, a workgroup rows of q or of k
// only, and its sums of the weights' gradients stay in registers until it is
// through; they are added up in one order by a second launch, so that the same
// call gives the same bits.
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
  f32x8 sa = {}, sb = {};
  for (int u = group * kGradWaves + wave; u < units; u += groups * kGradWaves) {
    const int r32 = u / parts;
    const int64_t r = r32;
    const int h = (u - r32 * parts) * 8 + (lane >> 3);
    const bool has = h < heads;
    const int at = a.r.pos[(int64_t)min(lane, a.r.n_axes - 1) * a.r.pos_sa + r * a.r.pos_st];
    bf16x8 xa = zero_bf16x8(), xb = xa, ga = xa, gb = xa;
    if (has) {
      const __bf16* px = x + r * x_st + h * x_sh;
      const __bf16* pg = dy + r * dy_st + h * dy_sh;
      xa = load_nt<bf16x8>(px + c.lo);
      xb = load_nt<bf16x8>(px + c.hi);
      ga = load_nt<bf16x8>(pg + c.lo);
      gb = load_nt<bf16x8>(pg + c.hi);
    }
    const int p = __shfl(at, axis);
    __builtin_amdgcn_wave_barrier();                // (the last unit's angles have been read)
    cs[wave][lane] = cos_sin_turns((double)p * turns);
    __builtin_amdgcn_wave_barrier();
    f32x8 na = widen(xa), nb = widen(xb), ya = widen(ga), yb = widen(gb);
    if (c.turned) {
      float2 t[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) t[e] = cs[wave][8 * d + e];
      turn(ya, yb, t, a.r.interleaved);
    }
    const float rms = inv_rms(na, nb, a.r.eps);
    na *= rms;
    nb *= rms;
    const f32x8 ua = ya * wa, ub = yb * wb;
    const float mean = row_sum8(dot16(ua, na, ub, nb)) * (1.f / kHeadDim);
    if (has) {
      __bf16* pd = dx + r * dx_st + h * dx_sh;
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

// Workgroup 0: the weights of q; 1: those of k.
constexpr int kSumThreads = 1024, kSumRows = kSumThreads / kHeadDim;
__global__ __launch_bounds__(kSumThreads) void rope_grad_sum_kernel(RopeGradArgs a) {
  __shared__ float sums[kSumRows][kHeadDim];
  const int i = threadIdx.x % kHeadDim, j = threadIdx.x / kHeadDim;
  const bool is_k = blockIdx.x != 0;
  const int first = is_k ? a.q_groups : 0, end = is_k ? a.q_groups + a.k_groups : a.q_groups;
  float s = 0.f;
#pragma unroll 8
  for (int g = first + j; g < end; g += kSumRows) s += a.parts[(int64_t)g * kHeadDim + i];
  sums[j][i] = s;
  __syncthreads();
  if (j != 0) return;
  s = 0.f;
#pragma unroll
  for (int k = 0; k < kSumRows; ++k) s += sums[k][i];
  if (is_k)
    a.dk_weight[i * a.dkw_s] = s;
  else
    a.dq_weight[i * a.dqw_s] = s;
}

}  // namespace

hipError_t launch_rope_grad(const RopeGradArgs& a, hipStream_t stream, KernelTimer* timer) {
  if (timer) (void)hipEventRecord(timer->start, stream);
  if (a.q_groups + a.k_groups > 0) rope_grad_kernel<<<a.q_groups + a.k_groups, kGradThreads, 0, stream>>>(a);
  if (timer) (void)hipEventRecord(timer->stop, stream);
  rope_grad_sum_kernel<<<a.dk_weight ? 2 : 1, kSumThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace rl
