// Requests that begin as copies of others, and requests that end: what happens to
// a table of pages between the steps that rl::map_kernel plans.
//
// Fork: a request takes over the first n tokens of another. Its full pages become
// the other's (block-table entries are copied), the rest n mod P of the last one
// needs a page of its own, from the list of free ones, and its rows a copy in every
// layer. One prefix sum over the requests places the pages.
//
// Drop: a request keeps its first n tokens. A page is free when no request's table
// holds it within the request's tokens, so the tables themselves say which pages
// are shared, and there are no counts to keep in step with them.
//
// The bytes are few; both are chains of dependent loads on top of a launch.
#include <algorithm>

#include "attn_common.hpp"
#include "kernels.hpp"

namespace rl {

namespace {

__device__ __forceinline__ int read_used(const int* free_used, int n_free, int* bad) {
  const int used = *free_used;
  if (used >= 0 && used <= n_free) return used;
  *bad |= kErrPool;
  return used < 0 ? 0 : n_free;
}

constexpr int kForkPer = 4;                         // requests of a thread in a pass

// What request b begins with.
struct Fork {
  int parent;                                       // negative: not forked, or not validly
  int len, kv;                                      // tokens it takes over, tokens it holds without
};
__device__ __forceinline__ Fork read_fork(const ForkArgs& a, int b, int* bad) {
  const int kv = a.kv_lens[(int64_t)b * a.kv_s];
  const int p = a.parents[(int64_t)b * a.par_s];
  if (p < 0) return {-1, 0, kv};
  // from another request that is not forked itself, into one that holds nothing
  if (p >= a.B || p == b || kv != 0 || a.parents[(int64_t)p * a.par_s] >= 0) {
    *bad |= kErrParent;
    return {-1, 0, kv};
  }
  const int n = a.fork_lens[(int64_t)b * a.fl_s], theirs = a.kv_lens[(int64_t)p * a.kv_s];
  if (n < 0 || n > theirs || theirs > a.max_pages * a.page_size) {
    *bad |= kErrLen;
    return {-1, 0, kv};
  }
  return {p, n, kv};
}

// Each workgroup sums over all requests and writes its own `block` of them.
template <int kThreads>
__global__ __launch_bounds__(kThreads) void fork_kernel(ForkArgs a) {
  constexpr int kPass = kThreads * kForkPer;
  // of a pass's requests: parent (negative: nothing to write), tokens, own page
  __shared__ int parent[kPass], len[kPass], fresh[kPass];
  __shared__ int wave_tot[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int lo = blockIdx.x * a.block, hi = min(a.B, lo + a.block);
  int bad = 0;
  const int used = read_used(a.free_used, a.n_free, &bad), room = a.n_free - used;
  int taken = 0;                                    // pages of the passes before
  for (int b0 = 0; b0 < a.B; b0 += kPass) {
    Fork q[kForkPer];
    int mine = 0;
#pragma unroll
    for (int i = 0; i < kForkPer; ++i) {
      const int b = b0 + tid * kForkPer + i;
      q[i] = b < a.B ? read_fork(a, b, &bad) : Fork{-1, 0, 0};
      mine += (q[i].len & (a.page_size - 1)) != 0;
    }
    int total;
    int at = taken + block_exclusive_scan(mine, &total, wave_tot);
#pragma unroll
    for (int i = 0; i < kForkPer; ++i) {
      const int s = tid * kForkPer + i, b = b0 + s;
      const bool need = (q[i].len & (a.page_size - 1)) != 0;
      at += need;
      int page = -1;
      bool ok = q[i].parent >= 0;
      if (ok && at > room) {                        // in order, until the list has no page left
        bad |= kErrPool;
        ok = false;
      }
      if (ok && need) {
        page = a.free_pages[(int64_t)(used + at - 1) * a.free_s];
        if ((unsigned)page >= (unsigned)a.num_pages) {
          bad |= kErrPage;
          ok = false;
        }
      }
      parent[s] = ok ? q[i].parent : -1;
      len[s] = q[i].len;
      fresh[s] = page;
      if (a.lengths && blockIdx.x == 0 && b < a.B) a.kv_out[(int64_t)b * a.kv_out_s] = ok ? q[i].len : q[i].kv;
    }
    taken += total;
    __syncthreads();
    if (a.entries) {
      const int end = min(hi - b0, kPass);
      for (int s = max(lo - b0, 0) + wave; s < end; s += kThreads / 64) {   // a wave has a request
        const int b = b0 + s, p = parent[s], n = p < 0 ? 0 : len[s];
        const int full = n >> a.log2_page, rest = n & (a.page_size - 1);
        const int* from = a.bt + (int64_t)max(p, 0) * a.bt_sb;
        int* to = a.bt + (int64_t)b * a.bt_sb;
        for (int j = lane; j < full; j += 64) to[(int64_t)j * a.bt_sj] = from[(int64_t)j * a.bt_sj];
        if (lane == 0) {
          int* c = a.copies + (int64_t)b * a.cp_s;
          c[0] = rest ? from[(int64_t)full * a.bt_sj] : -1;
          c[1] = rest ? fresh[s] : -1;
          c[2] = rest;
          if (rest) to[(int64_t)full * a.bt_sj] = fresh[s];
        }
      }
    }
    __syncthreads();                                // the lists are rebuilt for the next pass
  }
  if (blockIdx.x != 0) return;                      // (each workgroup meets the errors)
  if (a.lengths && tid == 0) *a.used_out = used + min(taken, room);
  if (a.entries && bad) atomicOr(a.err, bad);
}

// Workgroup: some rows of one copy, of K or of V.
constexpr int kCopyThreads = 256, kCopyLoads = 4;   // 16 bytes each
__global__ __launch_bounds__(kCopyThreads) void copy_pages_kernel(CopyArgs a) {
  typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
  const int* c = a.copies + (int64_t)blockIdx.x * a.cp_s;
  const int src = c[0], dst = c[1], rows = c[2];
  if (rows <= 0) return;
  if ((unsigned)src >= (unsigned)a.num_pages || (unsigned)dst >= (unsigned)a.num_pages || rows > a.page_size) {
    if (threadIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0)
      atomicOr(a.err, rows > a.page_size ? kErrLen : kErrPage);
    return;
  }
  if (src == dst) return;
  char* base = blockIdx.z ? a.v : a.k;
  const int64_t sp = blockIdx.z ? a.vp_sp : a.kp_sp, ss = blockIdx.z ? a.vp_ss : a.kp_ss;
  const int64_t sh = blockIdx.z ? a.vp_sh : a.kp_sh;
  const int per_head = a.row_bytes / 16, per_row = a.Hkv * per_head, n = rows * per_row;
  const int i0 = blockIdx.y * kCopyThreads * kCopyLoads + threadIdx.x;
  const char* from = base + src * sp;
  char* to = base + dst * sp;
  u32x4 x[kCopyLoads];
  int64_t off[kCopyLoads];
#pragma unroll
  for (int k = 0; k < kCopyLoads; ++k) {
    const int i = min(i0 + k * kCopyThreads, n - 1);
    const int t = i / per_row, rem = i - t * per_row, h = rem / per_head;
    off[k] = t * ss + h * sh + (rem - h * per_head) * 16;
    x[k] = *reinterpret_cast<const u32x4*>(from + off[k]);
  }
#pragma unroll
  for (int k = 0; k < kCopyLoads; ++k)
    if (i0 + k * kCopyThreads < n) *reinterpret_cast<u32x4*>(to + off[k]) = x[k];
}

// Drop: one workgroup marks the pages that requests keep and those they drop, in
// LDS, and lists the ones dropped and not kept, in the order of their ids.
constexpr int kDropThreads = 1024;
constexpr int kDropBits = 7680 * 32;                // pages of a pass (two marks each: 60 KB)
__global__ __launch_bounds__(kDropThreads) void drop_kernel(DropArgs a) {
  extern __shared__ unsigned marks[];               // kept, dropped
  __shared__ int wave_tot[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int bad = 0;
  const int used = read_used(a.free_used, a.n_free, &bad);
  const int room = a.max_pages * a.page_size;
  int found = 0;                                    // pages of all passes
  // two turns over the pool where it takes several passes: their number first, which says
  // where the list begins
  const int passes = max(1, (a.num_pages + kDropBits - 1) / kDropBits);
  for (int turn = passes > 1 ? 0 : 1, at = 0; turn < 2; ++turn, at = 0)
    for (int pass = 0; pass < passes; ++pass) {
      const int first = pass * kDropBits, pages = min(a.num_pages - first, kDropBits);
      const int words = (pages + 31) / 32;
      for (int i = tid; i < 2 * words; i += kDropThreads) marks[i] = 0;
      __syncthreads();
      for (int b = wave; b < a.B; b += kDropThreads / 64) {       // a wave has a request
        const int kv = a.kv_lens[(int64_t)b * a.kv_s], k = a.keep_lens[(int64_t)b * a.keep_s];
        if (kv < 0 || kv > room || k < 0) bad |= kErrLen;
        const int len = kv < 0 ? 0 : min(kv, room), keep = k < 0 ? len : min(k, len);
        const int held = (int)(((unsigned)len + a.page_size - 1) >> a.log2_page);
        const int kept = (int)(((unsigned)keep + a.page_size - 1) >> a.log2_page);
        for (int j = lane; j < held; j += 64) {
          const int page = a.bt[(int64_t)b * a.bt_sb + (int64_t)j * a.bt_sj];
          if ((unsigned)page >= (unsigned)a.num_pages) {
            bad |= kErrPage;
            continue;
          }
          const int i = page - first;
          if ((unsigned)i < (unsigned)pages) atomicOr(&marks[(j < kept ? 0 : words) + (i >> 5)], 1u << (i & 31));
        }
      }
      __syncthreads();
      const int each = (words + kDropThreads - 1) / kDropThreads;
      const int w0 = min(words, tid * each), w1 = min(words, w0 + each);
      int mine = 0;
      for (int i = w0; i < w1; ++i) mine += __popc(marks[words + i] & ~marks[i]);
      int total;
      int rank = at + block_exclusive_scan(mine, &total, wave_tot);
      at += total;
      if (passes == 1) found = total;
      if (turn == 0) {
        found += total;
      } else {
        for (int i = w0; i < w1; ++i)
          for (unsigned m = marks[words + i] & ~marks[i]; m; m &= m - 1, ++rank) {
            const int to = used - found + rank;
            if (to >= 0) a.free_pages[(int64_t)to * a.free_s] = first + 32 * i + __ffs(m) - 1;
          }
      }
      __syncthreads();
    }
  for (int b = tid; b < a.B; b += kDropThreads) {
    const int kv = a.kv_lens[(int64_t)b * a.kv_s], k = a.keep_lens[(int64_t)b * a.keep_s];
    a.kv_out[(int64_t)b * a.kv_out_s] = k < 0 ? kv : min(kv, k);
  }
  if (found > used) bad |= kErrPool;                // more than the list has lost
  if (tid == 0) *a.used_out = max(0, used - found);
  if (bad) atomicOr(a.err, bad);
}

}  // namespace

hipError_t launch_fork(const ForkArgs& args, hipStream_t stream) {
  ForkArgs a = args;
  const int groups = std::max(1, std::min(256, (a.B + 3) / 4));
  a.block = (a.B + groups - 1) / groups;
  const bool in_place = a.kv_out == a.kv_lens || a.used_out == a.free_used;
  auto run = [&](int n, bool lengths, bool entries) {
    a.lengths = lengths;
    a.entries = entries;
    if (a.B <= 256 * kForkPer)
      fork_kernel<256><<<n, 256, 0, stream>>>(a);
    else
      fork_kernel<1024><<<n, 1024, 0, stream>>>(a);
  };
  run(groups, groups == 1 || !in_place, true);
  // in place, the lengths that every workgroup reads are written behind them all
  if (groups > 1 && in_place) run(1, true, false);
  return hipGetLastError();
}

hipError_t launch_copy_pages(const CopyArgs& a, hipStream_t stream) {
  const int most = a.page_size * a.Hkv * (a.row_bytes / 16), each = kCopyThreads * kCopyLoads;
  const dim3 grid((unsigned)a.n, (unsigned)((most + each - 1) / each), 2);
  copy_pages_kernel<<<grid, kCopyThreads, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_drop(const DropArgs& a, hipStream_t stream) {
  const int words = (std::min(a.num_pages, kDropBits) + 31) / 32;
  drop_kernel<<<1, kDropThreads, 2 * sizeof(unsigned) * (size_t)words, stream>>>(a);
  return hipGetLastError();
}

}  // namespace rl
