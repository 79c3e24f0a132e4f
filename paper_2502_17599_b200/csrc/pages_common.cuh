// Shared parts of the paged-cache kernels: the handle, and the block-wide prefix sums by which every block finds
// its share of a ragged batch.  Lengths live on the device, so no launch can be sized by them: grids are fixed by
// the GPU, every block reads all lengths (8 K at most, from L2) and takes an equal part of the work they add up to.
#pragma once

#include "meda_common.cuh"

struct meda_pages {
  meda_pages_config cfg;
  int device = 0;
  int sm_count = 0;
  int group = 1;                       // query heads per KV head
  int page_shift = 4;                  // log2(page_size)
  int64_t launches = 0;
  int64_t bytes = 0;
  void* slab = nullptr;                // the one allocation all pointers below lead into
  int* status = nullptr;               // device status word (first error wins)
  unsigned long long* rope_freq = nullptr;   // [half] turns per position, as a 64-bit fraction
  int* rope_axis = nullptr;            // [half]
  float* attn_partial = nullptr;       // [blocks][2][group][head_dim + 2] softmax states of segments that cross blocks
  int4* attn_split = nullptr;          // [blocks] segments that go on behind a block
  float* select_scratch = nullptr;     // [sequences][n_kv_heads][max_seq_pages] scores, then four floats per eight pages: bound, largest, smallest, unused
  int attn_blocks = 0;                 // blocks of the attention kernel that are resident at once
};

namespace meda {

constexpr int kPagesMaxSeqs = 8192;
constexpr int kPagesMaxSeqPages = 262144;

// Every kernel of the paged caches starts with this.  The launches are programmatic (see launch_after): the next kernel of
// the stream may be set up while this one still runs, and waits here, before it touches any memory, until all before it
// has finished and its writes are visible.  A kernel takes 3 to 10 us on a decoding step; 1 to 2 of them were the gap.
__device__ __forceinline__ void begin_grid() {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
}

// Exclusive prefix of `v` over a block of THREADS threads (1024 at most) in thread order, and the block total.
// `scratch` holds THREADS / 32 values; two barriers.  Every warp scans the warps' sums by itself, one value per lane: reading
// them all in every thread would keep the shared memory busy for THREADS cycles.
template <int THREADS, typename V>
__device__ __forceinline__ V block_prefix(V v, V* scratch, V& total) {
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  V incl = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const V y = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += y;
  }
  __syncthreads();                      // previous users of scratch are done
  if (lane == 31) scratch[warp] = incl;
  __syncthreads();
  V sums = lane < THREADS / 32 ? scratch[lane] : 0;
#pragma unroll
  for (int o = 1; o < THREADS / 32; o <<= 1) {
    const V y = __shfl_up_sync(0xffffffffu, sums, o);
    if (lane >= o) sums += y;
  }
  total = __shfl_sync(0xffffffffu, sums, 31);
  const V before = __shfl_sync(0xffffffffu, sums, (warp + 31) % 32);
  return (warp ? before : 0) + incl - v;
}

// A sequence's length as the kernels use it: out-of-range values are cut to the nearest valid one.
__device__ __forceinline__ int clamped_len(const int32_t* lens, int stride, int i, int max_rows, bool& bad) {
  const int len = lens[(size_t)i * stride];
  bad |= len < 0 || len > max_rows;
  return min(max(len, 0), max_rows);
}

// pre[0 .. n] (shared memory) <- exclusive prefix sums of units(length of sequence i).  A thread takes consecutive
// sequences, so one block-wide scan serves any n.  Afterwards every thread may read pre (and what units() wrote of its
// own sequences, as long as every warp writes the same).
template <int THREADS, typename F>
__device__ __forceinline__ void ragged_prefix(int n, int* pre, int* scratch, F units) {
  if (n <= 32) {                        // few sequences: every warp for itself (they write the same values), no barrier
    const int lane = threadIdx.x % 32;
    int u = lane < n ? units(lane) : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, u, o);
      if (lane >= o) u += y;
    }
    if (lane < n) pre[lane + 1] = u;
    if (lane == 0) pre[0] = 0;
    __syncwarp();
    return;
  }
#pragma unroll 4
  for (int i = threadIdx.x; i < n; i += THREADS) pre[i + 1] = units(i);         // neighbouring threads, neighbouring lengths
  __syncthreads();
  const int per = (n + THREADS - 1) / THREADS;
  const int lo = min(n, (int)threadIdx.x * per), hi = min(n, lo + per);
  int sum = 0;
#pragma unroll 1
  for (int i = lo; i < hi; ++i) sum += pre[i + 1];
  int total;
  int run = block_prefix<THREADS>(sum, scratch, total);
#pragma unroll 1
  for (int i = lo; i < hi; ++i) {
    run += pre[i + 1];
    pre[i + 1] = run;
  }
  if (threadIdx.x == 0) pre[0] = 0;
  __syncthreads();
}

// Largest i in [0, n) with pre[i] <= x, for pre[0] = 0 <= x < pre[n]: the sequence unit x belongs to
// (sequences without units are passed over).
__device__ __forceinline__ int ragged_find(const int* pre, int n, int x) {
  int lo = 0, hi = n;                   // pre[lo] <= x < pre[hi]
#pragma unroll 1
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (pre[mid] <= x) lo = mid;
    else hi = mid;
  }
  return lo;
}

}  // namespace meda
