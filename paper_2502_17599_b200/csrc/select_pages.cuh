// Pages worth reading for one new token: per (sequence, KV head) the `keep` pages with the highest score, the largest
// logit a page's key bounds allow any of the head's queries, max_h sum_d (q >= 0 ? q * max : q * min).
//
// One cluster of blocks per (sequence, KV head), in one launch: the blocks score equal parts of the sequence's pages into
// sort keys in their shared memory, find the keep-th largest key by radix passes over it (histograms added up through
// distributed shared memory) and write their kept pages in order.  Scores never go to global memory.
//
// Four lanes share a page (each a quarter of every 64 bytes of its bounds), eight pages side by side in a warp and PP
// deep, so that one read of the queries from shared memory serves PP pages; two shuffles finish a sum.  The sum is taken in
// 64 bits and rounded once: which of two near pages is kept must not hang on the order of an fp32 sum, because the
// whole output follows from it.  That arithmetic, not the bounds' bytes, is what bounds the kernel when few clusters run.
#pragma once

#include <cooperative_groups.h>

#include "pages_common.cuh"
#include "rope_append.cuh"   // RopeVec
#include "select.cuh"        // block_exclusive_sum

namespace meda {

constexpr int kPselBins = 2048;          // 11-bit digits: 11 + 11 + 10 bits of a key

struct SelectPagesParams {
  const void* q;
  const void* bounds;
  const int32_t* table;
  const int32_t* lens;
  int32_t* sel;
  int* status;
  int lens_stride, n_seqs, n_heads, group, n_pages, width, page_shift, keep, n_first, n_last;
};

struct SelectPagesSmem {
  int keys_off, hist_off, q_off, misc_off, total;
};
__host__ __device__ inline SelectPagesSmem select_pages_smem(int width, int cluster_size, int gp, int d) {
  SelectPagesSmem L;
  int off = 0;
  L.q_off = off;     off += gp * d * 8;
  L.hist_off = off;  off += 2 * kPselBins * 4;
  L.misc_off = off;  off += 64 * 4;
  L.keys_off = off;  off += ((width + cluster_size - 1) / cluster_size + 3) / 4 * 16;
  L.total = off;
  return L;
}

__device__ __forceinline__ unsigned int page_key(float score) {
  if (score != score) return 0xfffffffeu;                      // NaN ranks above every number, below a forced page
  const unsigned int b = __float_as_uint(score + 0.f);         // -0 counts as 0
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}

// D = head_dim, GP = query heads per KV head rounded up to a power of two.
template <typename T, int D, int GP>
__global__ void __launch_bounds__(kSelThreads, 1)
select_pages_kernel(SelectPagesParams p) {
  namespace cg = cooperative_groups;
  constexpr int E = RopeVec<T>::E;                             // elements per 16-byte vector
  constexpr int X = D / (4 * E);                               // vectors of a bound per lane
  constexpr int PP = GP <= 4 ? 2 : 1;                          // pages per lane and step (registers: 64-bit sums per head)
  extern __shared__ __align__(16) unsigned char psel_smem[];
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = (int)cluster.block_rank(), CS = (int)cluster.num_blocks();
  const SelectPagesSmem L = select_pages_smem(p.width, CS, GP, D);
  unsigned int* keys = reinterpret_cast<unsigned int*>(psel_smem + L.keys_off);
  unsigned int* hist = reinterpret_cast<unsigned int*>(psel_smem + L.hist_off);
  double* qs = reinterpret_cast<double*>(psel_smem + L.q_off); // [GP][D]
  int* misc = reinterpret_cast<int*>(psel_smem + L.misc_off);  // [0..32] scan scratch, [41] kept for sure, [42] equal, [44] digit, [45] remaining
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const int pair = blockIdx.x / CS, i = pair / p.n_heads, g = pair % p.n_heads;
  const int page_size = 1 << p.page_shift;
  bool bad = false;
  const int len = clamped_len(p.lens, p.lens_stride, i, p.width << p.page_shift, bad);
  if (bad && threadIdx.x == 0) set_status(p.status, MEDA_ERR_INVALID_ARG);
  const int n = (len + page_size - 1) >> p.page_shift;         // pages of the sequence
  int32_t* out = p.sel + ((size_t)i * p.n_heads + g) * p.keep;
  if (n <= p.keep) {                                           // uniform over the cluster: every page is kept
    for (int c = rank * kSelThreads + threadIdx.x; c < n; c += CS * kSelThreads) out[c] = c;
    return;
  }
  const int chunk = (n + CS - 1) / CS;
  const int lo = min(n, rank * chunk), hi = min(n, lo + chunk);

  // ---- scores
  for (int x = threadIdx.x; x < GP * D; x += kSelThreads)
    qs[x] = x < p.group * D ? (double)to_f32<T>(static_cast<const T*>(p.q)[((size_t)i * p.n_heads + g) * p.group * D + x]) : 0.0;
  __syncthreads();
  const int sub = lane / 4, quarter = lane % 4;
  for (int c0 = lo + warp * 8 * PP; c0 < hi; c0 += kSelThreads / 4 * PP) {
    const uint4* src[PP];
    bool ok[PP];
#pragma unroll
    for (int y = 0; y < PP; ++y) {
      const int c = c0 + y * 8 + sub;
      const int page = c < hi ? p.table[(size_t)i * p.width + c] : 0;
      ok[y] = c < hi && (unsigned)page < (unsigned)p.n_pages;
      if (c < hi && !ok[y] && quarter == 0) set_status(p.status, MEDA_ERR_INVALID_ARG);
      src[y] = static_cast<const uint4*>(p.bounds) + ((size_t)(ok[y] ? page : 0) * p.n_heads + g) * 2 * (D / E) + quarter;
    }
    double acc[PP][GP];
#pragma unroll
    for (int y = 0; y < PP; ++y)
#pragma unroll
      for (int h = 0; h < GP; ++h) acc[y][h] = 0.0;
#pragma unroll
    for (int x = 0; x < X; ++x) {
      float mn[PP][E], mx[PP][E];
#pragma unroll
      for (int y = 0; y < PP; ++y) {
        const uint4 zero = make_uint4(0, 0, 0, 0);
        RopeVec<T>::unpack(ok[y] ? src[y][x * 4] : zero, mn[y]);
        RopeVec<T>::unpack(ok[y] ? src[y][D / E + x * 4] : zero, mx[y]);
      }
#pragma unroll
      for (int e = 0; e < E; e += 2) {
        double dn[PP][2], dx[PP][2];
#pragma unroll
        for (int y = 0; y < PP; ++y)
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            dn[y][b] = (double)mn[y][e + b];
            dx[y][b] = (double)mx[y][e + b];
          }
#pragma unroll
        for (int h = 0; h < GP; ++h) {
          const double2 qv = *reinterpret_cast<const double2*>(qs + h * D + x * 4 * E + quarter * E + e);
#pragma unroll
          for (int y = 0; y < PP; ++y) {
            acc[y][h] = fma(qv.x, qv.x >= 0.0 ? dx[y][0] : dn[y][0], acc[y][h]);
            acc[y][h] = fma(qv.y, qv.y >= 0.0 ? dx[y][1] : dn[y][1], acc[y][h]);
          }
        }
      }
    }
#pragma unroll
    for (int y = 0; y < PP; ++y) {
      float best = -INFINITY;
      bool nan = false;
#pragma unroll
      for (int h = 0; h < GP; ++h) {
        double s = acc[y][h];
        s += __shfl_xor_sync(0xffffffffu, s, 1);
        s += __shfl_xor_sync(0xffffffffu, s, 2);
        const float f = (float)s;
        if (h < p.group) {
          nan |= f != f;
          best = fmaxf(best, f);
        }
      }
      const int c = c0 + y * 8 + sub;
      if (quarter == 0 && c < hi)
        keys[c - lo] = c < p.n_first || c >= n - p.n_last ? 0xffffffffu : page_key(nan ? NAN : best);
    }
  }
  __syncthreads();

  // ---- the keep-th largest key, most significant digit first (alternate passes count into alternate histograms,
  // so that one cluster barrier per pass is enough)
  unsigned int prefix = 0u, mask = 0u;
  int remaining = p.keep;
#pragma unroll 1
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : (pass == 1 ? 10 : 0);
    const unsigned int bins = pass == 2 ? 1024u : 2048u;
    unsigned int* h = hist + (pass & 1) * kPselBins;
    for (int b = threadIdx.x; b < kPselBins; b += kSelThreads) h[b] = 0u;
    __syncthreads();
    for (int c = threadIdx.x; c < hi - lo; c += kSelThreads) {
      const unsigned int key = keys[c];
      if ((key & mask) == prefix) atomicAdd(&h[(key >> shift) & (bins - 1u)], 1u);
    }
    cluster.sync();
    const int b0 = (int)bins - 1 - 2 * (int)threadIdx.x, b1 = b0 - 1;
    int n0 = 0, n1 = 0;
    if (b1 >= 0) {
#pragma unroll 8
      for (int r = 0; r < CS; ++r) {
        const uint2 two = *reinterpret_cast<const uint2*>(cluster.map_shared_rank(h, r) + b1);
        n1 += (int)two.x;
        n0 += (int)two.y;
      }
    }
    int all;
    const int above = block_exclusive_sum(n0 + n1, misc, all);
    if (above < remaining && above + n0 + n1 >= remaining) {
      if (above + n0 >= remaining) { misc[44] = b0; misc[45] = remaining - above; }
      else { misc[44] = b1; misc[45] = remaining - above - n0; }
    }
    __syncthreads();
    prefix |= (unsigned int)misc[44] << shift;
    mask |= (bins - 1u) << shift;
    remaining = misc[45];
  }
  const unsigned int threshold = prefix;
  const int take_equal = remaining;                            // keys equal to the threshold that are kept, lowest pages first

  // ---- kept pages, in order
  int sure = 0, equal = 0;
  for (int c = threadIdx.x; c < hi - lo; c += kSelThreads) {
    sure += keys[c] > threshold;
    equal += keys[c] == threshold;
  }
  sure = __reduce_add_sync(0xffffffffu, sure);
  equal = __reduce_add_sync(0xffffffffu, equal);
  if (threadIdx.x == 0) { misc[41] = 0; misc[42] = 0; }
  __syncthreads();
  if (lane == 0) { atomicAdd(&misc[41], sure); atomicAdd(&misc[42], equal); }
  cluster.sync();
  int kept_before = 0, equal_before = 0;
  for (int r = 0; r < rank; ++r) {
    const int* m = cluster.map_shared_rank(misc, r);
    const int e = m[42];
    kept_before += m[41] + min(max(take_equal - equal_before, 0), e);
    equal_before += e;
  }
  for (int c0 = 0; c0 < hi - lo; c0 += kSelThreads) {
    const int c = c0 + (int)threadIdx.x;
    const unsigned int key = c < hi - lo ? keys[c] : 0u;
    const bool is_equal = c < hi - lo && key == threshold;
    int eq_total, keep_total;
    const int eq_rank = equal_before + block_exclusive_sum(is_equal, misc, eq_total);
    const bool kept = c < hi - lo && (key > threshold || (is_equal && eq_rank < take_equal));
    const int pos = kept_before + block_exclusive_sum(kept, misc, keep_total);
    if (kept) out[pos] = lo + c;
    kept_before += keep_total;
    equal_before += eq_total;
  }
  cluster.sync();                                              // no block leaves while another may still read its counters
}

}  // namespace meda
