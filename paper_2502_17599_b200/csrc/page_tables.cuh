// Page tables, slot maps and the free list for one change of lengths, in one launch.
//
// Every block computes the three prefix sums (pages taken, pages given back, new rows) over all sequences into its
// shared memory: 8 K sequences are 64 KB of lengths from L2, and doing it in every block costs no more time than doing it
// in one, while it saves a second launch and the scratch between the two.  After that each entry written is a
// function of its index alone: the j-th page taken is the j-th page given back, or the free list's entry behind
// its front; a row's slot follows from its page.  No entry that is read is written in the same launch (the table
// entries read are pages the sequences already hold, the ones written are new; the list's entries read lie behind its
// front, the ones written before it), so blocks need no order among themselves.
// Bound by latency for decoding steps (a launch, the lengths, two scans), by the 8-byte slots for whole prompts.
#pragma once

#include "pages_common.cuh"

namespace meda {

constexpr int kTabThreads = 512;
constexpr int kTabWarpRows = 256;        // consecutive new rows whose slots one warp writes

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

__device__ __forceinline__ int pages_of(int rows, int shift) { return (int)(((unsigned)rows + (1u << shift) - 1u) >> shift); }

__global__ void __launch_bounds__(kTabThreads)
page_tables_kernel(TablesParams p) {
  extern __shared__ __align__(16) int tab_smem[];
  __shared__ long long scratch[kTabThreads / 32 + 1];
  const int n = p.n_seqs;
  int* pops = tab_smem;                 // [n + 1] pages taken before sequence i
  int* pushes = pops + n + 1;           // [n + 1] pages given back before sequence i
  int* fresh = pushes + n + 1;          // [n + 1] new rows before sequence i
  const int max_rows = p.width << p.page_shift;

  auto old_len = [&](int i) { return p.lens ? p.lens[(size_t)i * p.lens_stride] : 0; };
  auto new_len = [&](int i) { return p.new_lens[(size_t)i * p.new_stride]; };

  const int per = (n + kTabThreads - 1) / kTabThreads;
  const int lo = min(n, (int)threadIdx.x * per), hi = min(n, lo + per);
  long long s_pop = 0, s_push = 0, s_new = 0;
  int bad = 0;
  for (int i = lo; i < hi; ++i) {
    const int a = old_len(i), b = new_len(i);
    const bool off = a < 0 || b < 0 || a > max_rows || b > max_rows;
    bad |= off;
    const int have = off ? 0 : pages_of(a, p.page_shift), need = off ? 0 : pages_of(b, p.page_shift);
    const int up = max(0, need - have), down = max(0, have - need), rows = off ? 0 : max(0, b - a);
    pops[i + 1] = up;
    pushes[i + 1] = down;
    fresh[i + 1] = rows;
    s_pop += up;
    s_push += down;
    s_new += rows;
  }
  const int top = *p.free_top;
  long long n_pops, n_pushes, n_fresh;
  long long r_pop = block_prefix<kTabThreads>(s_pop, scratch, n_pops);
  long long r_push = block_prefix<kTabThreads>(s_push, scratch, n_pushes);
  long long r_new = block_prefix<kTabThreads>(s_new, scratch, n_fresh);
  bad = __syncthreads_or(bad);
  const bool first = blockIdx.x == 0 && threadIdx.x == 0;
  int code = MEDA_OK;
  if (bad || top < 0 || top > p.n_pages || top + n_pops - n_pushes < 0) code = MEDA_ERR_INVALID_ARG;
  else if (top + n_pops - n_pushes > p.n_pages || n_fresh > (p.slots ? p.slots_capacity : INT32_MAX)) code = MEDA_ERR_WORKSPACE;
  const int stride = gridDim.x * kTabThreads;
  if (code != MEDA_OK) {
    for (int i = blockIdx.x * kTabThreads + threadIdx.x; i < p.slots_capacity; i += stride) p.slots[i] = -1;
    for (int i = blockIdx.x * kTabThreads + threadIdx.x; i <= n; i += stride) p.cu_new[i] = 0;
    if (first) {
      *p.free_top_out = top;
      set_status(p.status, code);
    }
    return;
  }
  for (int i = lo; i < hi; ++i) {
    r_pop += pops[i + 1];
    r_push += pushes[i + 1];
    r_new += fresh[i + 1];
    pops[i + 1] = (int)r_pop;
    pushes[i + 1] = (int)r_push;
    fresh[i + 1] = (int)r_new;
    if (blockIdx.x == 0) p.cu_new[i + 1] = (int)r_new;
  }
  if (threadIdx.x == 0) pops[0] = pushes[0] = fresh[0] = 0;
  if (first) {
    p.cu_new[0] = 0;
    *p.free_top_out = (int)(top + n_pops - n_pushes);
  }
  __syncthreads();
  const int total_pops = (int)n_pops, total_pushes = (int)n_pushes, total_new = (int)n_fresh;

  auto checked = [&](int page) {
    if ((unsigned)page >= (unsigned)p.n_pages) {
      set_status(p.status, MEDA_ERR_INVALID_ARG);
      return -1;
    }
    return page;
  };
  auto pushed = [&](int j) {            // j-th page given back
    const int i = ragged_find(pushes, n, j);
    return checked(p.table[(size_t)i * p.width + pages_of(new_len(i), p.page_shift) + (j - pushes[i])]);
  };
  auto popped = [&](int j) {            // j-th page taken
    return j < total_pushes ? pushed(j) : checked(p.free_pages[top + (j - total_pushes)]);
  };

  // pages taken into the table, pages left over onto the list
  for (int j = blockIdx.x * kTabThreads + threadIdx.x; j < total_pops; j += stride) {
    const int i = ragged_find(pops, n, j);
    p.table[(size_t)i * p.width + pages_of(old_len(i), p.page_shift) + (j - pops[i])] = popped(j);
  }
  for (int j = total_pops + blockIdx.x * kTabThreads + threadIdx.x; j < total_pushes; j += stride)
    p.free_pages[top - 1 - (j - total_pops)] = pushed(j);

  // slots of the new rows: a warp finds the sequence of its first row and walks on from there
  const int lane = threadIdx.x % 32;
  const int mask = (1 << p.page_shift) - 1;
  const int warps = gridDim.x * (kTabThreads / 32);
  for (long long c0 = (long long)(blockIdx.x * (kTabThreads / 32) + threadIdx.x / 32) * kTabWarpRows; c0 < p.slots_capacity;
       c0 += (long long)warps * kTabWarpRows) {
    const int end = (int)min(c0 + kTabWarpRows, (long long)p.slots_capacity);
    int i = c0 < total_new ? ragged_find(fresh, n, (int)c0) : 0;
    for (int t = (int)c0 + lane; t < end; t += 32) {
      int64_t slot = -1;
      if (t < total_new) {
        while (t >= fresh[i + 1]) ++i;
        const int have = old_len(i);
        const int row = have + (t - fresh[i]), col = row >> p.page_shift, held = pages_of(have, p.page_shift);
        const int page = col < held ? checked(p.table[(size_t)i * p.width + col]) : popped(pops[i] + (col - held));
        if (page >= 0) slot = ((int64_t)page << p.page_shift) + (row & mask);
      }
      p.slots[t] = slot;
    }
  }
}

}  // namespace meda
