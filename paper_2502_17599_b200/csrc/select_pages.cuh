// Pages worth reading for one new token: per (sequence, KV head) the `keep` pages with the highest score, the largest
// logit a page's key bounds allow any of the head's queries, max_h sum_d (q >= 0 ? q * max : q * min).
//
// The sum is taken in 64 bits and rounded once: which of two near pages is kept must not hang on the order of an fp32
// sum, because the whole output follows from it.  64-bit arithmetic on every page would cost several times what reading
// the bounds does (100 us instead of 4 for 8,064 pages and 28 heads), so bf16 caches go two ways at once:
//   - every page gets an approximate score from the matrix instructions, max(q, 0) . max + min(q, 0) . min (products of bf16
//     are exact, the fp32 sum is off by at most eps);
//   - radix passes over those find the keep-th largest to 22 bits; pages above it by more than 2 eps are kept, pages below it
//     by more than 2 eps are not (the true keep-th score lies within eps of it), and the few in between are scored
//     again in 64 bits and ranked among themselves.
// Where that cannot decide (an infinity or a NaN, more than kPselMaxDoubt pages in between) and for fp32 caches every page is
// scored in 64 bits and the radix passes go to the last bit.
//
// One cluster of blocks per (sequence, KV head), in one launch: the blocks hold the sort keys of equal parts of the
// sequence's pages in shared memory, add up their histograms through distributed shared memory, and write their kept
// pages in order.  Scores never go to global memory.
#pragma once

#include <cooperative_groups.h>

#include "paged_attention.cuh"   // mma_bf16
#include "pages_common.cuh"
#include "rope_append.cuh"       // RopeVec

namespace meda {

constexpr int kPselThreads = 512;
constexpr int kPselBins = 2048;          // 11-bit digits: 11 + 11 + 10 bits of a key
constexpr int kPselMaxDoubt = 256;       // pages scored again in 64 bits

struct SelectPagesParams {
  const void* q;
  const void* bounds;
  const int32_t* table;
  const int32_t* lens;
  int32_t* sel;
  int* status;
  int lens_stride, n_seqs, n_heads, group, n_pages, width, page_shift, keep, n_first, n_last;
};

// Block-shared counters; other blocks of the cluster read some of them.
struct SelectPagesShared {
  int scan[kPselThreads / 32 + 1];
  int digit, remaining;
  int sure, equal, doubtful;             // this block's pages
  int undecided;                         // a NaN or an infinity among this block's approximate scores
  int listed;                            // doubtful pages written to the list (block 0)
  unsigned int max_abs;                  // largest |bound| of this block's pages, as float bits
  float q_norm;                          // largest sum |q| over the heads
};

struct SelectPagesSmem {
  int keys_off, hist_off, q_off, list_off, total;
};
__host__ __device__ inline SelectPagesSmem select_pages_smem(int width, int cluster_size, int gp, int d) {
  SelectPagesSmem L;
  int off = 0;
  L.q_off = off;     off += gp * d * 8;
  L.hist_off = off;  off += 2 * kPselBins * 4;
  L.list_off = off;  off += kPselMaxDoubt * 8;
  L.keys_off = off;  off += ((width + cluster_size - 1) / cluster_size + 3) / 4 * 16;
  L.total = off;
  return L;
}

__device__ __forceinline__ unsigned int page_key(float score) {
  if (score != score) return 0xfffffffeu;                      // NaN ranks above every number, below a forced page
  const unsigned int b = __float_as_uint(score + 0.f);         // -0 counts as 0
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ float key_score(unsigned int key) {
  return __uint_as_float((key & 0x80000000u) ? (key & 0x7fffffffu) : ~key);
}

// The score of one page for one KV head by a whole warp, in 64 bits.  qs: the head's queries [group][D] as doubles.
template <typename T, int D>
__device__ __forceinline__ float page_score_warp(const T* lo, const T* hi, const double* qs, int group, int lane) {
  constexpr int E = D / 32;
  double mn[E], mx[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    mn[e] = (double)to_f32<T>(lo[e * 32 + lane]);
    mx[e] = (double)to_f32<T>(hi[e * 32 + lane]);
  }
  float best = -INFINITY;
  bool nan = false;
  for (int h = 0; h < group; ++h) {
    double s = 0.0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const double q = qs[h * D + e * 32 + lane];
      s = fma(q, q >= 0.0 ? mx[e] : mn[e], s);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    const float f = (float)s;
    nan |= f != f;
    best = fmaxf(best, f);
  }
  return nan ? NAN : best;
}

// D = head_dim, GP = query heads per KV head rounded up to a power of two.
template <typename T, int D, int GP>
__global__ void __launch_bounds__(kPselThreads, 1)
select_pages_kernel(SelectPagesParams p) {
  namespace cg = cooperative_groups;
  constexpr bool kBf16 = sizeof(T) == 2;
  constexpr int kWarps = kPselThreads / 32;
  constexpr int E = RopeVec<T>::E;                             // elements per 16-byte vector
  constexpr int X = D / (4 * E);                               // vectors of a bound per lane, four lanes to a page
  extern __shared__ __align__(16) unsigned char psel_smem[];
  __shared__ SelectPagesShared sh;
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = (int)cluster.block_rank(), CS = (int)cluster.num_blocks();
  const SelectPagesSmem L = select_pages_smem(p.width, CS, GP, D);
  unsigned int* keys = reinterpret_cast<unsigned int*>(psel_smem + L.keys_off);
  unsigned int* hist = reinterpret_cast<unsigned int*>(psel_smem + L.hist_off);
  uint2* list = reinterpret_cast<uint2*>(psel_smem + L.list_off);   // (key, page) of doubtful pages, in block 0
  double* qs = reinterpret_cast<double*>(psel_smem + L.q_off); // [GP][D]
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const int pair = blockIdx.x / CS, i = pair / p.n_heads, g = pair % p.n_heads;
  const int page_size = 1 << p.page_shift;
  bool bad = false;
  const int len = clamped_len(p.lens, p.lens_stride, i, p.width << p.page_shift, bad);
  if (bad && threadIdx.x == 0) set_status(p.status, MEDA_ERR_INVALID_ARG);
  const int n = (len + page_size - 1) >> p.page_shift;         // pages of the sequence
  int32_t* out = p.sel + ((size_t)i * p.n_heads + g) * p.keep;
  if (n <= p.keep) {                                           // uniform over the cluster: every page is kept
    for (int c = rank * kPselThreads + threadIdx.x; c < n; c += CS * kPselThreads) out[c] = c;
    return;
  }
  const int chunk = (n + CS - 1) / CS;
  const int lo = min(n, rank * chunk), hi = min(n, lo + chunk);
  const T* qh = static_cast<const T*>(p.q) + ((size_t)i * p.n_heads + g) * p.group * D;
  const int32_t* table = p.table + (size_t)i * p.width;
  const T* bounds = static_cast<const T*>(p.bounds);
  auto forced = [&](int c) { return c < p.n_first || c >= n - p.n_last; };
  // page (column of the table) c's place in the pool of bounds; a page outside the pool is reported and scores as page 0
  auto place = [&](int c) {
    const int page = table[c];
    const bool ok = (unsigned)page < (unsigned)p.n_pages;
    if (!ok) set_status(p.status, MEDA_ERR_INVALID_ARG);
    return ((size_t)(ok ? page : 0) * p.n_heads + g) * 2 * D;
  };

  if (threadIdx.x == 0) {
    sh.undecided = kBf16 ? 0 : 1;
    sh.listed = 0;
    sh.max_abs = 0u;
    sh.q_norm = 0.f;
  }
  for (int x = threadIdx.x; x < GP * D; x += kPselThreads) qs[x] = x < p.group * D ? (double)to_f32<T>(qh[x]) : 0.0;
  for (int b = threadIdx.x; b < 2 * kPselBins; b += kPselThreads) hist[b] = 0u;
  __syncthreads();

  // One radix pass over this block's keys and the cluster's sum of its histogram: narrows prefix / mask / remaining by a digit.
  unsigned int prefix = 0u, mask = 0u;
  int remaining = p.keep;
  auto radix_pass = [&](int pass) {
    const int shift = pass == 0 ? 21 : (pass == 1 ? 10 : 0);
    const unsigned int bins = pass == 2 ? 1024u : 2048u;
    unsigned int* h = hist + (pass & 1) * kPselBins;           // alternate passes count into alternate histograms: one cluster
    for (int c = threadIdx.x; c < hi - lo; c += kPselThreads) {    // barrier per pass is enough
      const unsigned int key = keys[c];
      if ((key & mask) == prefix) atomicAdd(&h[(key >> shift) & (bins - 1u)], 1u);
    }
    cluster.sync();
    // a thread owns four bins, from the top down
    const int b0 = (int)bins - 4 - 4 * (int)threadIdx.x;
    int c[4] = {0, 0, 0, 0};
    if (b0 >= 0) {
#pragma unroll 8
      for (int r = 0; r < CS; ++r) {
        const uint4 four = *reinterpret_cast<const uint4*>(cluster.map_shared_rank(h, r) + b0);
        c[0] += (int)four.w;
        c[1] += (int)four.z;
        c[2] += (int)four.y;
        c[3] += (int)four.x;
      }
    }
    int all;
    int above = block_prefix<kPselThreads>(c[0] + c[1] + c[2] + c[3], sh.scan, all);
    if (above < remaining && above + c[0] + c[1] + c[2] + c[3] >= remaining) {
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        if (above < remaining && above + c[y] >= remaining) {
          sh.digit = b0 + 3 - y;
          sh.remaining = remaining - above;
        }
        above += c[y];
      }
    }
    // the other histogram is free again (its readers have passed the barrier above): cleared for the next pass
    unsigned int* other = hist + ((pass + 1) & 1) * kPselBins;
    if (pass > 0)
      for (int b = threadIdx.x; b < kPselBins; b += kPselThreads) other[b] = 0u;
    __syncthreads();
    prefix |= (unsigned int)sh.digit << shift;
    mask |= (bins - 1u) << shift;
    remaining = sh.remaining;
  };

  unsigned int threshold = 0u;           // pages with a larger key are kept, and the first take_equal of those with this one
  int take_equal = 0;
  bool decided = false;
  if constexpr (kBf16) {
    // ---- approximate scores: eight pages side by side, A = the queries' positive and negative parts (row: head), B = a page's
    // bounds (column: page), the contraction index permuted as in paged_attention.cuh
    constexpr int NH = GP > 8 ? 2 : 1;
    constexpr int KC = D / 32;
    uint4 pos[NH][KC], neg[NH][KC];
    {
      const __nv_bfloat162 zero = __floats2bfloat162_rn(0.f, 0.f);
      const int r = lane / 4, c = lane % 4;
#pragma unroll
      for (int y = 0; y < NH; ++y) {
        const int h = r + 8 * y;
        float norm = 0.f;
#pragma unroll
        for (int x = 0; x < KC; ++x) {
          const uint4 v = h < p.group ? *reinterpret_cast<const uint4*>(qh + (size_t)h * D + x * 32 + c * 8) : make_uint4(0, 0, 0, 0);
          const uint32_t w[4] = {v.x, v.y, v.z, v.w};
          uint32_t a[4], b[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            __nv_bfloat162 t;
            memcpy(&t, &w[e], 4);
            const __nv_bfloat162 up = __hmax2_nan(t, zero), down = __hmin2_nan(t, zero);
            memcpy(&a[e], &up, 4);
            memcpy(&b[e], &down, 4);
            norm += fabsf(__low2float(t)) + fabsf(__high2float(t));
          }
          pos[y][x] = make_uint4(a[0], a[1], a[2], a[3]);
          neg[y][x] = make_uint4(b[0], b[1], b[2], b[3]);
        }
        norm += __shfl_xor_sync(0xffffffffu, norm, 1);
        norm += __shfl_xor_sync(0xffffffffu, norm, 2);
        norm = warp_max(norm);
        if (warp == 0 && lane == 0) sh.q_norm = fmaxf(sh.q_norm, norm);
      }
    }
    __nv_bfloat162 top2 = __floats2bfloat162_rn(0.f, 0.f);     // running max |bound| of this lane's pieces
    bool odd = false;
    for (int c0 = lo + warp * 8; c0 < hi; c0 += kWarps * 8) {
      const int r = lane / 4, c = lane % 4;
      const T* src = bounds + place(min(c0 + r, hi - 1)) + c * 8;
      uint4 mn[KC], mx[KC];
#pragma unroll
      for (int x = 0; x < KC; ++x) {
        mn[x] = load_stream(reinterpret_cast<const uint4*>(src + x * 32));
        mx[x] = load_stream(reinterpret_cast<const uint4*>(src + D + x * 32));
      }
      float up[4] = {0.f, 0.f, 0.f, 0.f}, down[4] = {0.f, 0.f, 0.f, 0.f};        // two chains of dependent instructions
#pragma unroll
      for (int x = 0; x < KC; ++x) {
        mma_bf16(up, pos[0][x].x, NH > 1 ? pos[NH - 1][x].x : 0u, pos[0][x].y, NH > 1 ? pos[NH - 1][x].y : 0u, mx[x].x, mx[x].y);
        mma_bf16(down, neg[0][x].x, NH > 1 ? neg[NH - 1][x].x : 0u, neg[0][x].y, NH > 1 ? neg[NH - 1][x].y : 0u, mn[x].x, mn[x].y);
        mma_bf16(up, pos[0][x].z, NH > 1 ? pos[NH - 1][x].z : 0u, pos[0][x].w, NH > 1 ? pos[NH - 1][x].w : 0u, mx[x].z, mx[x].w);
        mma_bf16(down, neg[0][x].z, NH > 1 ? neg[NH - 1][x].z : 0u, neg[0][x].w, NH > 1 ? neg[NH - 1][x].w : 0u, mn[x].z, mn[x].w);
      }
#pragma unroll
      for (int x = 0; x < KC; ++x) {
        const uint32_t w[8] = {mn[x].x, mn[x].y, mn[x].z, mn[x].w, mx[x].x, mx[x].y, mx[x].z, mx[x].w};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          __nv_bfloat162 t;
          memcpy(&t, &w[e], 4);
          top2 = __hmax2_nan(top2, __habs2(t));
        }
      }
      // the best head of pages 2c and 2c + 1
      float best[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float a = r < p.group ? up[e] + down[e] : -INFINITY;
        const float b = NH > 1 && r + 8 < p.group ? up[2 + e] + down[2 + e] : -INFINITY;
        odd |= a != a || b != b;
        best[e] = fmaxf(a, b);
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) best[e] = fmaxf(best[e], __shfl_xor_sync(0xffffffffu, best[e], o));
      }
      if (r < 2) {
        const int at = c0 + 2 * c + r;
        if (at < hi) keys[at - lo] = forced(at) ? 0xffffffffu : page_key(best[r]);
      }
    }
    const float top_abs = fmaxf(__low2float(top2), __high2float(top2));
    odd |= __low2float(top2) != __low2float(top2) || __high2float(top2) != __high2float(top2) || top_abs == INFINITY;
    const unsigned int top_bits = __reduce_max_sync(0xffffffffu, __float_as_uint(top_abs));
    odd = __any_sync(0xffffffffu, odd);
    if (lane == 0) {
      atomicMax(&sh.max_abs, top_bits);
      if (odd) atomicOr(&sh.undecided, 1);
    }
    __syncthreads();
    radix_pass(0);
    radix_pass(1);
    // The bounds of all blocks: eps = 2^-16 max_h sum |q| max |bound| covers 2 D products summed in fp32 by two chains of
    // D / 16 instructions (each off by 2^-21 of the partial sums at most, which stay below sum |q| max |bound|).
    float top_all = 0.f;
    bool undecided = false;
    for (int r = 0; r < CS; ++r) {
      const SelectPagesShared* o = cluster.map_shared_rank(&sh, r);
      top_all = fmaxf(top_all, __uint_as_float(o->max_abs));
      undecided |= o->undecided != 0;
    }
    const float eps = 1.52587890625e-5f * sh.q_norm * top_all;
    const unsigned int k0 = prefix, k1 = prefix | 1023u;        // the keep-th approximate score lies in [k0, k1]
    undecided |= !(eps < 1e30f) || k1 >= 0xff7fffffu || k0 <= 0x00800000u;
    if (!undecided) {
      const unsigned int low = page_key(key_score(k0) - 2.01f * eps), high = page_key(key_score(k1) + 2.01f * eps);
      int sure = 0, doubt = 0;
      for (int c = threadIdx.x; c < hi - lo; c += kPselThreads) {
        sure += keys[c] > high;
        doubt += keys[c] >= low && keys[c] <= high;
      }
      int all_sure, all_doubt;
      block_prefix<kPselThreads>(sure, sh.scan, all_sure);
      const int my_doubt = block_prefix<kPselThreads>(doubt, sh.scan, all_doubt);
      if (threadIdx.x == 0) {
        sh.sure = all_sure;
        sh.doubtful = all_doubt;
      }
      cluster.sync();
      int need = p.keep, before = 0, total = 0;
      for (int r = 0; r < CS; ++r) {
        const SelectPagesShared* o = cluster.map_shared_rank(&sh, r);
        need -= o->sure;
        if (r < rank) before += o->doubtful;
        total += o->doubtful;
      }
      if (total <= kPselMaxDoubt) {                            // uniform over the cluster
        // own doubtful pages onto block 0's list (any order), scored there by its owner's warps
        uint2* all = cluster.map_shared_rank(list, 0);
        int at = before + my_doubt;
        for (int c = threadIdx.x; c < hi - lo; c += kPselThreads)
          if (keys[c] >= low && keys[c] <= high) list[at++ - before].y = (unsigned int)c;      // staged here first
        __syncthreads();
        const int mine = all_doubt;
        unsigned int my_page[(kPselMaxDoubt + kWarps - 1) / kWarps];
#pragma unroll
        for (int y = 0; y < (kPselMaxDoubt + kWarps - 1) / kWarps; ++y)
          my_page[y] = y * kWarps + warp < mine ? list[y * kWarps + warp].y : 0u;
        cluster.sync();                                        // block 0's own staging has been read
#pragma unroll
        for (int y = 0; y < (kPselMaxDoubt + kWarps - 1) / kWarps; ++y) {
          const int e = y * kWarps + warp;
          if (e < mine) {
            const int c = lo + (int)my_page[y];
            const T* src = bounds + place(c);
            const float s = page_score_warp<T, D>(src, src + D, qs, p.group, lane);
            if (lane == 0) all[before + e] = make_uint2(page_key(s), (unsigned int)c);
          }
        }
        cluster.sync();
        // the `need` best of the list, ties to the lowest page: the kept ones get the highest key, the others the lowest
        for (int e = warp; e < mine; e += kWarps) {
          const uint2 me = all[before + e];
          int better = 0;
          for (int o = lane; o < total; o += 32) {
            const uint2 x = all[o];
            better += x.x > me.x || (x.x == me.x && x.y < me.y);
          }
          better = __reduce_add_sync(0xffffffffu, better);
          if (lane == 0) keys[(int)me.y - lo] = better < need ? 0xffffffffu : 0u;
        }
        threshold = high;
        decided = true;
        __syncthreads();
      }
    }
  }
  if (!decided) {
    // ---- every page in 64 bits: four lanes to a page, eight pages side by side
    if constexpr (kBf16) {
      cluster.sync();                                          // nobody still reads the histograms
      for (int b = threadIdx.x; b < 2 * kPselBins; b += kPselThreads) hist[b] = 0u;
      prefix = mask = 0u;
      remaining = p.keep;
    }
    const int sub = lane / 4, quarter = lane % 4;
    for (int c0 = lo + warp * 8; c0 < hi; c0 += kWarps * 8) {
      const uint4* src = reinterpret_cast<const uint4*>(bounds + place(min(c0 + sub, hi - 1))) + quarter;
      double acc[GP];
#pragma unroll
      for (int h = 0; h < GP; ++h) acc[h] = 0.0;
#pragma unroll 1
      for (int x = 0; x < X; ++x) {
        float mn[E], mx[E];
        RopeVec<T>::unpack(src[x * 4], mn);
        RopeVec<T>::unpack(src[D / E + x * 4], mx);
#pragma unroll
        for (int e = 0; e < E; e += 2) {
          const double n0 = (double)mn[e], n1 = (double)mn[e + 1], x0 = (double)mx[e], x1 = (double)mx[e + 1];
#pragma unroll
          for (int h = 0; h < GP; ++h) {
            const double2 qv = *reinterpret_cast<const double2*>(qs + h * D + x * 4 * E + quarter * E + e);
            acc[h] = fma(qv.x, qv.x >= 0.0 ? x0 : n0, acc[h]);
            acc[h] = fma(qv.y, qv.y >= 0.0 ? x1 : n1, acc[h]);
          }
        }
      }
      float best = -INFINITY;
      bool nan = false;
#pragma unroll
      for (int h = 0; h < GP; ++h) {
        double s = acc[h];
        s += __shfl_xor_sync(0xffffffffu, s, 1);
        s += __shfl_xor_sync(0xffffffffu, s, 2);
        const float f = (float)s;
        if (h < p.group) {
          nan |= f != f;
          best = fmaxf(best, f);
        }
      }
      const int c = c0 + sub;
      if (quarter == 0 && c < hi) keys[c - lo] = forced(c) ? 0xffffffffu : page_key(nan ? NAN : best);
    }
    __syncthreads();
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) radix_pass(pass);
    threshold = prefix;
    take_equal = remaining;                                    // keys equal to the threshold that are kept, lowest pages first
  }

  // ---- kept pages, in order
  int sure = 0, equal = 0;
  for (int c = threadIdx.x; c < hi - lo; c += kPselThreads) {
    sure += keys[c] > threshold;
    equal += keys[c] == threshold;
  }
  int all_sure, all_equal;
  block_prefix<kPselThreads>(sure, sh.scan, all_sure);
  block_prefix<kPselThreads>(equal, sh.scan, all_equal);
  if (threadIdx.x == 0) {
    sh.sure = all_sure;
    sh.equal = all_equal;
  }
  cluster.sync();
  int kept_before = 0, equal_before = 0;
  for (int r = 0; r < rank; ++r) {
    const SelectPagesShared* o = cluster.map_shared_rank(&sh, r);
    const int e = o->equal;
    kept_before += o->sure + min(max(take_equal - equal_before, 0), e);
    equal_before += e;
  }
  for (int c0 = 0; c0 < hi - lo; c0 += kPselThreads) {
    const int c = c0 + (int)threadIdx.x;
    const unsigned int key = c < hi - lo ? keys[c] : 0u;
    const bool is_equal = c < hi - lo && key == threshold;
    int eq_total, keep_total;
    const int eq_rank = equal_before + block_prefix<kPselThreads>((int)is_equal, sh.scan, eq_total);
    const bool kept = c < hi - lo && (key > threshold || (is_equal && eq_rank < take_equal));
    const int pos = kept_before + block_prefix<kPselThreads>((int)kept, sh.scan, keep_total);
    if (kept) out[pos] = lo + c;
    kept_before += keep_total;
    equal_before += eq_total;
  }
  cluster.sync();                                              // no block leaves while another may still read its counters
}

}  // namespace meda
