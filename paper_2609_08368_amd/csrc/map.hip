// Slot maps: the block-table entries, slots and positions of a step's new rows
// from the lengths of its requests, so that a step needs no host between two
// others and can be captured.
//
// Request b holds c_b tokens and adds n_b. It takes ceil((c_b + n_b) / P) -
// ceil(c_b / P) pages from the list of free ones, behind those of the requests
// before it; two prefix sums over the requests (rows and pages) place
// everything. Every new page holds the row of its first token, so the thread of
// that row writes the block-table entry, and rows are all there is to share out.
//
// The bytes are nothing; a call is a chain of dependent loads (lengths, sums,
// table or free list, stores) on top of a launch. So each workgroup sums over
// all requests again and then writes its share of the rows, where a launch of
// its own for the sums would cost more: 128 decoding requests take one
// workgroup 3.8 us, 32 requests with 38K rows 5.6 us, and 3001 with 50K rows
// 7.8-8.5 us, in one pass of 1024 threads (9.7 in three of 256 threads). In place,
// the lengths of more than 1024 rows are written by a second launch: in a graph
// 2.0 us more for 32 requests and 2.7 for 3001, 4 us in eager calls.
#include <algorithm>

#include "attn_common.hpp"
#include "kernels.hpp"

namespace rl {

namespace {

constexpr int kMapPer = 4;                          // requests of a thread in a pass

// Rows and pages that requests take (64 bits: a refused request may ask for any number).
struct Need {
  long long rows, pages;
};

// A request's lengths; rows = 0 and bad set where they are out of range.
struct Request {
  int cached, rows, pages, first;                   // first: pages it holds before the step
};
__device__ __forceinline__ Request read_request(const MapArgs& a, int b, int* bad) {
  const int c = a.kv_lens[(int64_t)b * a.kv_s], n = a.new_lens[(int64_t)b * a.new_s];
  const int room = a.max_pages * a.page_size;
  if (c < 0 || n < 0 || c > room || n > room - c) {
    *bad |= kErrLen;
    return {c, 0, 0, 0};
  }
  const int before = (int)(((unsigned)c + a.page_size - 1) >> a.log2_page);
  const int after = (int)(((unsigned)(c + n) + a.page_size - 1) >> a.log2_page);
  return {c, n, after - before, before};
}

// Pages of the free list that earlier steps took, clamped into the list.
__device__ __forceinline__ int read_used(const MapArgs& a, int* bad) {
  const int used = *a.free_used;
  if (used >= 0 && used <= a.n_free) return used;
  *bad |= kErrPool;
  return used < 0 ? 0 : a.n_free;
}

// Exclusive prefix sums of a thread's need over the workgroup, and its totals.
template <int kThreads>
__device__ __forceinline__ Need scan_need(Need x, Need* total, Need* wave_tot) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const Need s{wave_inclusive_scan64(x.rows), wave_inclusive_scan64(x.pages)};
  if (lane == 63) wave_tot[wave] = s;
  __syncthreads();
  Need before{0, 0}, all{0, 0};
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) {
    const Need t = wave_tot[w];
    if (w < wave) before = {before.rows + t.rows, before.pages + t.pages};
    all = {all.rows + t.rows, all.pages + t.pages};
  }
  *total = all;
  return {before.rows + s.rows - x.rows, before.pages + s.pages - x.pages};
}

template <int kThreads>
__global__ __launch_bounds__(kThreads) void map_kernel(MapArgs a) {
  constexpr int kPass = kThreads * kMapPer;
  // of a pass's requests: first row, tokens before the step, pages before it,
  // and (free entry of the first new page) - (pages before it)
  __shared__ int row0[kPass], cached[kPass], before[kPass], taken[kPass];
  __shared__ Need wave_tot[kThreads / 64];
  __shared__ Need stop;                             // rows and pages of the requests served
  __shared__ int stopped;
  const int tid = threadIdx.x;
  const bool first_wg = blockIdx.x == 0;
  const int lo = blockIdx.x * a.rows_block, hi = min(a.rows, lo + a.rows_block);
  int bad = 0;
  const int used = read_used(a, &bad);
  if (tid == 0) stopped = 0;
  __syncthreads();
  Need at{0, 0};                                    // what the passes before took
  for (int b0 = 0; b0 < a.B; b0 += kPass) {
    Request q[kMapPer];
    Need mine{0, 0};
#pragma unroll
    for (int i = 0; i < kMapPer; ++i) {
      const int b = b0 + tid * kMapPer + i;
      q[i] = b < a.B ? read_request(a, b, &bad) : Request{0, 0, 0, 0};
      mine = {mine.rows + q[i].rows, mine.pages + q[i].pages};
    }
    Need total;
    const Need off = scan_need<kThreads>(mine, &total, wave_tot);
    // Requests are served in order until one does not fit; that one sees the
    // sums of all before it fit and its own not, and no other does.
    Need x{at.rows + off.rows, at.pages + off.pages};
    const Need x0 = x;
    auto fits = [&](const Need& s) { return s.rows <= a.rows && s.pages <= a.n_free - used; };
#pragma unroll
    for (int i = 0; i < kMapPer; ++i) {
      const Need y{x.rows + q[i].rows, x.pages + q[i].pages};
      if (fits(x) && !fits(y)) {
        stop = x;
        stopped = 1;
        bad |= y.rows > a.rows ? kErrRows : kErrPool;
      }
      x = y;
    }
    __syncthreads();
    const Need served{at.rows + total.rows, at.pages + total.pages};
    const Need end = stopped ? stop : served;
    x = x0;
#pragma unroll
    for (int i = 0; i < kMapPer; ++i) {
      const int s = tid * kMapPer + i, b = b0 + s;
      const Need y{x.rows + q[i].rows, x.pages + q[i].pages};
      const bool ok = fits(y);
      const int r = (int)(ok ? x.rows : end.rows);
      row0[s] = r;
      cached[s] = q[i].cached;
      before[s] = q[i].first;
      taken[s] = used + (int)(ok ? x.pages : 0) - q[i].first;
      if (first_wg && b < a.B) {
        a.indptr[(int64_t)b * a.indptr_s] = r;
        if (!a.late) a.kv_out[(int64_t)b * a.kv_out_s] = q[i].cached + (ok ? q[i].rows : 0);
      }
      x = y;
    }
    __syncthreads();
    // this workgroup's rows of the pass
    const int p0 = (int)min(at.rows, end.rows), p1 = (int)end.rows;
    for (int r = max(lo, p0) + tid; r < min(hi, p1); r += kThreads) {
      // the last request that starts at or before r (the ones without rows share
      // the start of the next)
      int s = 0;
#pragma unroll
      for (int step = kPass / 2; step > 0; step >>= 1)
        if (row0[s + step] <= r) s += step;
      const int b = b0 + s, t = cached[s] + (r - row0[s]), j = t >> a.log2_page;
      const bool fresh = j >= before[s];
      int* entry = a.bt + (int64_t)b * a.bt_sb + (int64_t)j * a.bt_sj;
      const int page = fresh ? a.free_pages[(int64_t)(taken[s] + j) * a.free_s] : *entry;
      const bool ok = (unsigned)page < (unsigned)a.num_pages;
      const int in_page = t & (a.page_size - 1);
      if (!ok) bad |= kErrPage;
      if (fresh && ok && in_page == 0) *entry = page;
      a.slots[(int64_t)r * a.slots_s] = ok ? ((int64_t)page << a.log2_page) | in_page : -1;
      const int d = a.delta ? a.delta[(int64_t)b * a.delta_s] : 0;
      a.pos[(int64_t)r * a.pos_s] = (int)((unsigned)t + (unsigned)d);
    }
    at = served;
    __syncthreads();                                // the lists are rebuilt for the next pass
  }
  const Need end = stopped ? stop : at;
  for (int r = max(lo, (int)end.rows) + tid; r < hi; r += kThreads) {   // rows behind the last request's
    a.slots[(int64_t)r * a.slots_s] = -1;
    a.pos[(int64_t)r * a.pos_s] = 0;
  }
  if (first_wg) {
    if (tid == 0) {
      a.indptr[(int64_t)a.B * a.indptr_s] = (int)end.rows;
      if (!a.late) *a.used_out = used + (int)end.pages;
    }
  }
  // (each workgroup meets the requests' errors; the first reports them)
  if (bad & (first_wg ? ~0 : kErrPage)) atomicOr(a.err, bad);
}

// The step's lengths and free entries in place, behind the workgroups that all
// read the ones before it: what each request got is in the row bounds.
constexpr int kLateThreads = 1024;
__global__ __launch_bounds__(kLateThreads) void map_lengths_kernel(MapArgs a) {
  __shared__ long long wave_tot[16];
  long long pages = 0;
  for (int b = threadIdx.x; b < a.B; b += kLateThreads) {
    const int c = a.kv_lens[(int64_t)b * a.kv_s];
    const int n = a.indptr[(int64_t)(b + 1) * a.indptr_s] - a.indptr[(int64_t)b * a.indptr_s];
    if (n > 0) pages += (((unsigned)(c + n) + a.page_size - 1) >> a.log2_page) -
                        (((unsigned)c + a.page_size - 1) >> a.log2_page);
    a.kv_out[(int64_t)b * a.kv_out_s] = c + n;
  }
  long long total;
  block_exclusive_scan64(pages, &total, wave_tot);
  if (threadIdx.x == 0) {
    int bad = 0;
    *a.used_out = read_used(a, &bad) + (int)total;
  }
}

}  // namespace

hipError_t launch_map(const MapArgs& args, hipStream_t stream) {
  MapArgs a = args;
  // a workgroup per 512 rows, at most one per CU or so; up to 1024 rows are left to one, which
  // then writes the lengths itself whether in place or not
  const int groups = a.rows <= 1024 ? 1 : std::min(256, (a.rows + 511) / 512);
  a.rows_block = (a.rows + groups - 1) / groups;
  a.late = groups > 1 && (a.kv_out == a.kv_lens || a.used_out == a.free_used);
  if (a.B <= 256 * kMapPer)                         // one pass (see the top)
    map_kernel<256><<<groups, 256, 0, stream>>>(a);
  else
    map_kernel<1024><<<groups, 1024, 0, stream>>>(a);
  if (a.late) map_lengths_kernel<<<1, kLateThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace rl
