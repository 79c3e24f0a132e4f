// Page tables, slot maps and the free list for one change of lengths, in one launch.
//
// Every block computes the three prefix sums (pages taken, pages given back, new rows) over all sequences into its
// shared memory: 8 K sequences are 64 KB of lengths from L2, and doing it in every block costs no more time than doing it
// in one, while it saves a second launch and the scratch between the two.  After that each entry written is a
// function of its index alone: the j-th page taken is the j-th page given back, or the free list's entry behind
// its front; a row's slot follows from its page.  No entry that is read is written in the same launch (the table
// entries read are pages the sequences already hold, the ones written are new; the list's entries read lie behind its
// front, the ones written before it), so blocks need no order among themselves.
// The unit of work is a page that gets new rows: a lane finds its page, the warp's 32 pages then cover one run of the slot
// map, which the warp writes in full lines (a slot's page comes from the lane that holds it, by a search over the lanes).
// Bound by latency: a launch, the lengths, a scan, two searches, one look-up (1,792 sequences growing by a row: 7.2 us; 448
// prompts admitted and 336 released, 1.3 million slots of 8 bytes: 7.3 us, of which the bytes are 1.6).
#pragma once

#include "pages_common.cuh"

namespace meda {

constexpr int kTabThreads = 1024;
constexpr int kTabPer = kPagesMaxSeqs / kTabThreads;     // sequences of a thread, at most

struct TablesParams {
  const int32_t* lens;
  const int32_t* new_lens;
  int32_t* free_pages;
  const int32_t* free_top;
  int32_t* free_top_out;
  int32_t* table;
  int32_t* cu_new;
  int64_t* slots;
  int* status;
  int lens_stride, new_stride, n_seqs, n_pages, width, page_shift, slots_capacity;
};

// Shared memory: six arrays over the sequences, but more than half of an SM's: the next launch's blocks come in while this
// one's run, and have to spread over the SMs as they free up rather than pile up on the first ones (14.3 us without, 7.8 with, for 448 prompts back to back).
__host__ __device__ inline size_t tables_smem(int n_seqs) {
  const size_t need = (size_t)(n_seqs + 1) * 24, half = 116 * 1024;
  return need > half ? need : half;
}

__device__ __forceinline__ int pages_of(int rows, int shift) { return (int)(((unsigned)rows + (1u << shift) - 1u) >> shift); }

__global__ void __launch_bounds__(kTabThreads)
page_tables_kernel(TablesParams p) {
  begin_grid();
  extern __shared__ __align__(16) int tab_smem[];
  __shared__ long long warp_moves[kTabThreads / 32], warp_rows[kTabThreads / 32];
  __shared__ int warp_touched[kTabThreads / 32];
  const int n = p.n_seqs, lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  int* pops = tab_smem;                 // [n + 1] pages taken before sequence i
  int* pushes = pops + n + 1;           // [n + 1] pages given back before sequence i
  int* fresh = pushes + n + 1;          // [n + 1] new rows before sequence i
  int* units = fresh + n + 1;           // [n + 1] pages with new rows before sequence i
  int* was = units + n + 1;             // [n] rows before
  int* will = was + n + 1;              // [n] rows after
  const int max_rows = p.width << p.page_shift;

#pragma unroll 4
  for (int i = threadIdx.x; i < n; i += kTabThreads) {
    was[i] = p.lens ? p.lens[(size_t)i * p.lens_stride] : 0;
    will[i] = p.new_lens[(size_t)i * p.new_stride];
  }
  const int top = *p.free_top;
  __syncthreads();
  // a thread's consecutive sequences, then the block: pages taken and given back (below 2^31 each: see meda_pages_create) share
  // one 64-bit sum
  const int per = (n + kTabThreads - 1) / kTabThreads;
  const int lo = min(n, (int)threadIdx.x * per), hi = min(n, lo + per);
  long long moves = 0, rows = 0;
  int touched = 0, bad = 0;
  int step[kTabPer], more[kTabPer], pages[kTabPer];             // pages taken (given back: negative), new rows, pages they touch
#pragma unroll
  for (int y = 0; y < kTabPer; ++y) {
    step[y] = more[y] = pages[y] = 0;
    if (lo + y < hi) {
      const int a = was[lo + y], b = will[lo + y];
      if (a < 0 || b < 0 || a > max_rows || b > max_rows) {
        bad = 1;
      } else {
        step[y] = pages_of(b, p.page_shift) - pages_of(a, p.page_shift);
        more[y] = max(0, b - a);
        pages[y] = more[y] ? pages_of(b, p.page_shift) - (a >> p.page_shift) : 0;
      }
    }
    moves += ((long long)max(0, step[y]) << 32) + max(0, -step[y]);
    rows += more[y];
    touched += pages[y];
  }
  long long incl_moves = moves, incl_rows = rows;
  int incl_touched = touched;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, incl_moves, o), z = __shfl_up_sync(0xffffffffu, incl_rows, o);
    const int t = __shfl_up_sync(0xffffffffu, incl_touched, o);
    if (lane >= o) {
      incl_moves += y;
      incl_rows += z;
      incl_touched += t;
    }
  }
  if (lane == 31) {
    warp_moves[warp] = incl_moves;
    warp_rows[warp] = incl_rows;
    warp_touched[warp] = incl_touched;
  }
  bad = __syncthreads_or(bad);
  // every warp scans the warps' sums by itself, one per lane
  constexpr int kWarps = kTabThreads / 32;
  long long sum_moves = lane < kWarps ? warp_moves[lane] : 0, sum_rows = lane < kWarps ? warp_rows[lane] : 0;
  int sum_touched = lane < kWarps ? warp_touched[lane] : 0;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, sum_moves, o), z = __shfl_up_sync(0xffffffffu, sum_rows, o);
    const int t = __shfl_up_sync(0xffffffffu, sum_touched, o);
    if (lane >= o) {
      sum_moves += y;
      sum_rows += z;
      sum_touched += t;
    }
  }
  const long long all_moves = __shfl_sync(0xffffffffu, sum_moves, 31), n_fresh = __shfl_sync(0xffffffffu, sum_rows, 31);
  const int total_units = __shfl_sync(0xffffffffu, sum_touched, 31);
  const long long before_moves = __shfl_sync(0xffffffffu, sum_moves, (warp + 31) % 32);
  const long long before_rows = __shfl_sync(0xffffffffu, sum_rows, (warp + 31) % 32);
  const int before_touched = __shfl_sync(0xffffffffu, sum_touched, (warp + 31) % 32);
  incl_moves += (warp ? before_moves : 0) - moves;
  incl_rows += (warp ? before_rows : 0) - rows;
  incl_touched += (warp ? before_touched : 0) - touched;
  const long long n_pops = all_moves >> 32, n_pushes = all_moves & 0xffffffffll;
  const bool first = blockIdx.x == 0 && threadIdx.x == 0;
  int code = MEDA_OK;
  if (bad || top < 0 || top > p.n_pages || top + n_pops - n_pushes < 0) code = MEDA_ERR_INVALID_ARG;
  else if (top + n_pops - n_pushes > p.n_pages || n_fresh > (p.slots ? p.slots_capacity : INT32_MAX)) code = MEDA_ERR_WORKSPACE;
  const int stride = gridDim.x * kTabThreads;
  if (code != MEDA_OK) {
#pragma unroll 1
    for (long long i = blockIdx.x * kTabThreads + threadIdx.x; i < p.slots_capacity; i += stride) p.slots[i] = -1;
#pragma unroll 1
    for (int i = blockIdx.x * kTabThreads + threadIdx.x; i <= n; i += stride) p.cu_new[i] = 0;
    if (first) {
      *p.free_top_out = top;
      set_status(p.status, code);
    }
    return;
  }
  int r_pop = (int)(incl_moves >> 32), r_push = (int)(incl_moves & 0xffffffffll), r_new = (int)incl_rows, r_unit = incl_touched;
#pragma unroll
  for (int y = 0; y < kTabPer; ++y)
    if (lo + y < hi) {
      r_pop += max(0, step[y]);
      r_push += max(0, -step[y]);
      r_new += more[y];
      r_unit += pages[y];
      pops[lo + y + 1] = r_pop;
      pushes[lo + y + 1] = r_push;
      fresh[lo + y + 1] = r_new;
      units[lo + y + 1] = r_unit;
      if (blockIdx.x == 0) p.cu_new[lo + y + 1] = r_new;
    }
  if (threadIdx.x == 0) pops[0] = pushes[0] = fresh[0] = units[0] = 0;
  if (first) {
    p.cu_new[0] = 0;
    *p.free_top_out = (int)(top + n_pops - n_pushes);
  }
  __syncthreads();
  const int total_pops = (int)n_pops, total_pushes = (int)n_pushes, total_new = (int)n_fresh;

  // (entries are looked at where they are moved: to look at all of them beforehand, every block would have to)
  auto checked = [&](int page) {
    if ((unsigned)page >= (unsigned)p.n_pages) {
      set_status(p.status, MEDA_ERR_INVALID_ARG);
      return -1;
    }
    return page;
  };
  const int top_bit = n > 1 ? 1 << (31 - __clz(n - 1)) : 0;    // first step of a search over n entries
  auto find = [&](const int* pre, int x) {                     // largest i < n with pre[i] <= x
    int i = 0;
#pragma unroll 1
    for (int step = top_bit; step > 0; step >>= 1)
      if (i + step < n && pre[i + step] <= x) i += step;
    return i;
  };
  auto pushed = [&](int j) -> const int32_t* {                 // where the j-th page given back stands
    const int i = find(pushes, j);
    return p.table + (size_t)i * p.width + pages_of(will[i], p.page_shift) + (j - pushes[i]);
  };

  // pages that get new rows: the page, its table entry if it was taken, and its rows' slots
  const int mask = (1 << p.page_shift) - 1;
  const int warps = gridDim.x * (kTabThreads / 32);
#pragma unroll 1
  for (long long u0 = (long long)(warp * gridDim.x + blockIdx.x) * 32; u0 < total_units; u0 += (long long)warps * 32) {
    const int u = (int)u0 + lane;
    int first_slot = total_new, rows_here = 0, page = -1, row0 = 0;
    if (u < total_units) {
      const int i = find(units, u);
      const int a = was[i], b = will[i], col = (a >> p.page_shift) + (u - units[i]), held = pages_of(a, p.page_shift);
      const int32_t* src = p.table + (size_t)i * p.width + col;
      if (col >= held) {
        const int j = pops[i] + (col - held);
        src = j < total_pushes ? pushed(j) : p.free_pages + top + (j - total_pushes);
      }
      page = checked(*src);
      if (col >= held) p.table[(size_t)i * p.width + col] = page;
      const int r0 = max(a, col << p.page_shift), r1 = min(b, (col + 1) << p.page_shift);
      row0 = r0 & mask;
      rows_here = r1 - r0;
      first_slot = fresh[i] + (r0 - a);
    }
    if (!p.slots) continue;
    const unsigned begin = (unsigned)__shfl_sync(0xffffffffu, first_slot, 0);      // (t0 and t may pass 2^31 behind the last slot)
    const int last = 31 - __clz(__ballot_sync(0xffffffffu, rows_here > 0));
    const unsigned end = (unsigned)__shfl_sync(0xffffffffu, first_slot + rows_here, last);
#pragma unroll 1
    for (unsigned t0 = begin; t0 < end; t0 += 128) {           // four slots of a lane at a time: their searches run side by side
      int owner[4] = {0, 0, 0, 0};                             // the lane whose page holds the slot
#pragma unroll
      for (int step = 16; step > 0; step >>= 1)
#pragma unroll
        for (int y = 0; y < 4; ++y)
          if ((unsigned)__shfl_sync(0xffffffffu, first_slot, owner[y] + step) <= t0 + 32 * y + lane) owner[y] += step;
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        const unsigned t = t0 + 32 * y + lane;
        const int pg = __shfl_sync(0xffffffffu, page, owner[y]);
        const int r = __shfl_sync(0xffffffffu, row0 - first_slot, owner[y]) + (int)t;
        if (t < end) p.slots[t] = pg < 0 ? -1 : ((int64_t)pg << p.page_shift) + r;
      }
    }
  }
  // pages given back that nobody took onto the list; nothing in the slots behind the last row
#pragma unroll 1
  for (long long j = (long long)total_pops + blockIdx.x * kTabThreads + threadIdx.x; j < total_pushes; j += stride)
    p.free_pages[top - 1 - (j - total_pops)] = checked(*pushed((int)j));
#pragma unroll 1
  for (long long t = (long long)total_new + blockIdx.x * kTabThreads + threadIdx.x; t < p.slots_capacity; t += stride) p.slots[t] = -1;
}

}  // namespace meda
