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
// The bytes are few; both are chains of dependent loads on top of a launch: 128 forks
// take 6.2 us, drops of 128 requests with 44K table entries 14, of 3000 with 86K 20.5.
// The copies are bound by their launch and ramp: 128 times 32 rows of 8 heads, K and V,
// 6.0 us for 16.8 MB written and 2.1 MB read (eight requests copy one page), 3.1 TB/s.
#include <algorithm>
#include <type_traits>

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
  const int kv = a.kv_lens[(int64_t)b * a.kv_s], n = a.fork_lens[(int64_t)b * a.fl_s];
  const int p = a.parents[(int64_t)b * a.par_s];
  if (p < 0) return {-1, 0, kv};
  const int q = min(p, a.B - 1);                    // (read at once with the parent's length)
  const int theirs = a.kv_lens[(int64_t)q * a.kv_s], grandparent = a.parents[(int64_t)q * a.par_s];
  // from another request that is not forked itself, into one that holds nothing
  if (p >= a.B || p == b || kv != 0 || grandparent >= 0) {
    *bad |= kErrParent;
    return {-1, 0, kv};
  }
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
  // (the rows of a page mostly lie side by side)
  const bool dense = ss == (int64_t)a.Hkv * a.row_bytes && (sh == a.row_bytes || a.Hkv == 1);
  const int i0 = blockIdx.y * kCopyThreads * kCopyLoads + threadIdx.x;
  if (i0 >= n) return;
  const char* from = base + src * sp;
  char* to = base + dst * sp;
  u32x4 x[kCopyLoads];
  int64_t off[kCopyLoads];
#pragma unroll
  for (int k = 0; k < kCopyLoads; ++k) {
    const int i = min(i0 + k * kCopyThreads, n - 1);
    off[k] = (int64_t)i * 16;
    if (!dense) {
      const int t = i / per_row, rem = i - t * per_row, h = rem / per_head;
      off[k] = t * ss + h * sh + (rem - h * per_head) * 16;
    }
    x[k] = *reinterpret_cast<const u32x4*>(from + off[k]);
  }
#pragma unroll
  for (int k = 0; k < kCopyLoads; ++k)
    if (i0 + k * kCopyThreads < n) *reinterpret_cast<u32x4*>(to + off[k]) = x[k];
}

// The calling waves' requests, first, first + step, ...: a wave calls mark(page, kept)
// for their pages, and writes the length each keeps (which nobody else reads). Eight
// loads are under way at once, of one request's entries or of several requests'.
template <typename Mark>
__device__ __forceinline__ void for_pages(const DropArgs& a, int first, int step, bool write, int* bad, Mark mark) {
  constexpr int kAhead = 8;
  const int lane = threadIdx.x & 63, room = a.max_pages * a.page_size;
  const int log2_each = a.max_pages <= 64 ? 0 : a.max_pages <= 128 ? 1 : a.max_pages <= 256 ? 2 : 3;
  const int each = 1 << log2_each, together = kAhead >> log2_each;        // loads of a request, requests
  for (int b0 = first; b0 < a.B; b0 += step * together) {
    int page[kAhead], held[kAhead], kept[kAhead];
    // (entries past a request's are read and not used: one round trip less)
    if (a.max_pages > 0)
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int b = min(b0 + (i >> log2_each) * step, a.B - 1), j = lane + 64 * (i & (each - 1));
        page[i] = a.bt[(int64_t)b * a.bt_sb + (int64_t)min(j, a.max_pages - 1) * a.bt_sj];
      }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int b = b0 + (i >> log2_each) * step, at = min(b, a.B - 1);
      const int kv = a.kv_lens[(int64_t)at * a.kv_s], k = a.keep_lens[(int64_t)at * a.keep_s];
      if (kv < 0 || kv > room || k < 0) *bad |= kErrLen;
      const int len = kv < 0 || b >= a.B ? 0 : min(kv, room), keep = k < 0 ? len : min(k, len);
      held[i] = (int)(((unsigned)len + a.page_size - 1) >> a.log2_page);
      kept[i] = (int)(((unsigned)keep + a.page_size - 1) >> a.log2_page);
    }
    auto mark_all = [&](int j0) {
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int j = j0 + 64 * (i & (each - 1));
        if (j >= held[i]) continue;
        if ((unsigned)page[i] >= (unsigned)a.num_pages)
          *bad |= kErrPage;
        else
          mark(page[i], j < kept[i]);
      }
    };
    mark_all(lane);
    for (int j0 = lane + 64 * kAhead; j0 < held[0]; j0 += 64 * kAhead) {  // (then each == kAhead)
#pragma unroll
      for (int i = 0; i < kAhead; ++i)
        page[i] = a.bt[(int64_t)b0 * a.bt_sb + (int64_t)min(j0 + 64 * i, held[0] - 1) * a.bt_sj];
      mark_all(j0);
    }
    if (write && lane < together) {                 // (behind the reads: in place)
      const int b = b0 + lane * step;
      if (b < a.B) {
        const int kv = a.kv_lens[(int64_t)b * a.kv_s], k = a.keep_lens[(int64_t)b * a.keep_s];
        a.kv_out[(int64_t)b * a.kv_out_s] = k < 0 ? kv : min(kv, k);
      }
    }
  }
}

// Lists the pages of n words (64 bits each, in LDS) of marks, the first of which is
// page `first`, in the order of their ids up to entry end - 1; returns how many there
// are. A wave has a word at a time, a lane a bit, so the entries leave it side by side
// (a thread that had a word and a bit after the other took twice the call's time).
// base: n ints of LDS. All threads call it.
constexpr int kDropThreads = 1024, kDropWaves = kDropThreads / 64;
__device__ __forceinline__ int list_pages(const DropArgs& a, const uint64_t* marks, int n, int* base, int first, int end,
                                          int* wave_tot) {
  const int tid = threadIdx.x, lane = tid & 63, each = (n + kDropThreads - 1) / kDropThreads;
  const int i0 = min(n, tid * each), i1 = min(n, i0 + each);
  int mine = 0, total;
  for (int i = i0; i < i1; ++i) mine += __popcll(marks[i]);
  int at = block_exclusive_scan(mine, &total, wave_tot);
  for (int i = i0; i < i1; ++i) {
    base[i] = at;
    at += __popcll(marks[i]);
  }
  __syncthreads();
  const int start = end - total;
  const unsigned bit = 1u << (lane & 31);
  // (the list is mostly dense: without a 64-bit product an id)
  auto list = [&](auto stride) {
#pragma unroll 4
    for (int i = tid >> 6; i < n; i += kDropWaves) {
      const uint64_t x = marks[i];
      const unsigned lo = (unsigned)x, hi = (unsigned)(x >> 32);
      const int to = start + base[i] + __builtin_amdgcn_mbcnt_hi(hi, __builtin_amdgcn_mbcnt_lo(lo, 0));
      if (((lane < 32 ? lo : hi) & bit) && to >= 0) a.free_pages[to * stride] = first + 64 * i + lane;
    }
  };
  if (a.free_s == 1)
    list(std::integral_constant<int, 1>{});
  else
    list(a.free_s);
  return total;
}

__device__ __forceinline__ void finish_drop(const DropArgs& a, int used, int listed, int bad) {
  if (listed > used) bad |= kErrPool;               // more than the list has lost
  if (threadIdx.x == 0) *a.used_out = max(0, used - listed);
  if (bad) atomicOr(a.err, bad);
}

// The workgroups mark the pages that their requests keep and those they drop, in LDS,
// and hand the marks to the last one to arrive, which lists the pages dropped and not
// kept. (Marking in memory took 17 us where this takes 14: an atomic on
// memory that eight dies share leaves at 3.5 a ns.)
__global__ __launch_bounds__(kDropThreads) void drop_kernel(DropArgs a) {
  extern __shared__ uint64_t marks[];               // n words of kept pages, n of dropped ones
  __shared__ int wave_tot[16];
  __shared__ int last;
  const int tid = threadIdx.x, wave = tid >> 6, n = (a.num_pages + 127) / 128 * 2, groups = gridDim.x;
  unsigned* bits = reinterpret_cast<unsigned*>(marks);
  int bad = 0;
  const int used = read_used(a.free_used, a.n_free, &bad);
  for (int i = tid; i < 2 * n; i += kDropThreads) marks[i] = 0;
  __syncthreads();
  for_pages(a, blockIdx.x * kDropWaves + wave, groups * kDropWaves, true, &bad,
            [&](int page, bool keep) { atomicOr(&bits[(keep ? 0 : 2 * n) + (page >> 5)], 1u << (page & 31)); });
  __syncthreads();
  if (groups > 1) {
    uint64_t* mine = a.marks + (int64_t)blockIdx.x * 2 * n;
    for (int i = tid; i < 2 * n; i += kDropThreads) hand_over(mine + i, marks[i]);
    if (!arrive(a.arrived, groups, &last)) {
      if (bad) atomicOr(a.err, bad);
      return;
    }
  }
  if (groups > 1) {
    for (int i = tid; i < 2 * n; i += kDropThreads) {
      uint64_t x = 0;
#pragma unroll
      for (int g = 0; g < kDropGroups; ++g)         // (all under way at once; the last one again where there are fewer)
        x |= handed_over(a.marks + (int64_t)min(g, groups - 1) * 2 * n + i);
      marks[i] = x;
    }
    __syncthreads();
  }
  for (int i = tid; i < n; i += kDropThreads) marks[i] = marks[n + i] & ~marks[i];
  __syncthreads();
  const int listed = list_pages(a, marks, n, reinterpret_cast<int*>(marks + n), 0, used, wave_tot);
  finish_drop(a, used, listed, bad);
}

// Larger pools: one workgroup, a part of the pool after the other, from the highest ids
// down (so that their number need not be known before).
__global__ __launch_bounds__(kDropThreads) void drop_large_kernel(DropArgs a) {
  extern __shared__ uint64_t marks[];               // kept, dropped
  __shared__ int wave_tot[16];
  const int tid = threadIdx.x, wave = tid >> 6;
  constexpr int n = kDropPart / 64;
  unsigned* bits = reinterpret_cast<unsigned*>(marks);
  int bad = 0;
  const int used = read_used(a.free_used, a.n_free, &bad);
  int listed = 0;
  for (int part = (a.num_pages - 1) / kDropPart; part >= 0; --part) {
    const int first = part * kDropPart;
    for (int i = tid; i < 2 * n; i += kDropThreads) marks[i] = 0;
    __syncthreads();
    // (in place, the lengths are there until the last part has been read)
    for_pages(a, wave, kDropWaves, part == 0, &bad, [&](int page, bool keep) {
      const int i = page - first;
      if ((unsigned)i < (unsigned)kDropPart) atomicOr(&bits[(keep ? 0 : 2 * n) + (i >> 5)], 1u << (i & 31));
    });
    __syncthreads();
    for (int i = tid; i < n; i += kDropThreads) marks[i] = marks[n + i] & ~marks[i];
    __syncthreads();
    listed += list_pages(a, marks, n, reinterpret_cast<int*>(marks + n), first, used - listed, wave_tot);
    __syncthreads();
  }
  finish_drop(a, used, listed, bad);
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
  if (a.num_pages <= kDropPart) {
    const int bytes = (a.num_pages + 127) / 128 * 32;
    // as many workgroups as there are requests for, and room for their marks
    const int groups = std::max(1, std::min({kDropGroups, (a.B + 15) / 16, kDropMarkBytes / std::max(bytes, 1)}));
    drop_kernel<<<groups, kDropThreads, (size_t)bytes, stream>>>(a);
  } else {
    drop_large_kernel<<<1, kDropThreads, kDropPart / 4, stream>>>(a);
  }
  return hipGetLastError();
}

}  // namespace rl
