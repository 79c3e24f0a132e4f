// Pages worth reading for one new token: per (sequence, KV head) the `keep` pages with the highest score, the largest
// logit a page's key bounds allow any of the head's queries, max_h sum_d (q >= 0 ? q * max : q * min).
//
// The sum is taken in 64 bits and rounded once: which of two near pages is kept must not hang on the order of an fp32
// sum, because the whole output follows from it.  64-bit arithmetic on every page would cost far more than reading
// the bounds does (100 us instead of 4 for 8,067 pages of 4 KV heads with 7 query heads each), so bf16 caches go
// two ways at once:
//   - page_scores_kernel gives every page an approximate score from the matrix instructions, max(q, 0) . max + min(q, 0) . min
//     (products of bf16 are exact, the fp32 sum is off by eps at most), with the whole GPU; the same instructions on |min| and |max|
//     give sum |q| |bound|, which eps is proportional to;
//   - choose_pages_kernel, one block per (sequence, KV head), finds the keep-th largest of them to one of 2,048 equal bins
//     between the smallest and the largest score.  A page more than 2 eps above that bin is kept, one more than 2 eps below it
//     is not (the true keep-th score lies within eps of the approximate one), and the few in between are scored again
//     in 64 bits and ranked among themselves.
// Where that cannot decide (an infinity or a NaN, more than kPselMaxDoubt pages in between) the block scores all its
// pages in 64 bits and finds the keep-th by radix passes to the last bit.  fp32 caches get 64-bit scores at once, and are bound by them
// (those 8,067 pages, 33 MB of bounds: 40 us with the choice, against 14 in bf16).
//
// One block chooses because its work is a handful of block-wide steps over keys in registers; a cluster of blocks per
// sequence with histograms in distributed shared memory spent 6,000 cycles on each step (31 us against 14 for both launches at
// 129,072 rows, keep 404, where the bounds are 16.5 MB).  Bound by latency: two launches, each a chain of dependent reads and
// block-wide steps; with 256 pairs of 1,000 pages (131 MB of bounds) 38 us, at head_dim 256 (262 MB; registers spill) 84.
#pragma once

#include "paged_attention.cuh"   // mma_bf16, InvariantDiv, div_small
#include "pages_common.cuh"
#include "rope_append.cuh"       // RopeVec

namespace meda {

constexpr int kPscoreThreads = 384;
constexpr int kPscoreUnit = 8;           // pages side by side in a warp
constexpr int kPselItems = 8;            // scores per thread held in registers in one round
constexpr int kPselBins = 2048;
constexpr int kPselMaxDoubt = 512;       // pages scored again in 64 bits

struct SelectPagesParams {
  const void* q;
  const void* bounds;
  const int32_t* table;
  const int32_t* lens;
  int32_t* sel;
  float* scores;                         // [n_seqs * n_heads][width]
  float4* units;                         // [n_seqs * n_heads][width / kPscoreUnit, rounded up]: of a unit's pages the largest sum |q| |bound|
                                         // (not finite where a score is not; 0 where the scores are exact), the largest and the smallest score
  int* status;
  int lens_stride, n_seqs, n_heads, group, n_pages, width, page_shift, keep, n_first, n_last;
  InvariantDiv heads_div;
};

__host__ __device__ inline int pscore_units(int pages) { return (pages + kPscoreUnit - 1) / kPscoreUnit; }

__device__ __forceinline__ unsigned int page_key(float score) {
  if (score != score) return 0xffffffffu;                      // NaN ranks highest
  const unsigned int b = __float_as_uint(score + 0.f);         // -0 counts as 0
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}

// Place of a page's bounds for KV head g; a page outside the pool is reported and scores as page 0.
__device__ __forceinline__ size_t bounds_place(const SelectPagesParams& p, int page, int g, int d) {
  const bool ok = (unsigned)page < (unsigned)p.n_pages;
  if (!ok) set_status(p.status, MEDA_ERR_INVALID_ARG);
  return ((size_t)(ok ? page : 0) * p.n_heads + g) * 2 * d;
}

// ---- scores of all pages ---------------------------------------------------------------------------------
// A unit is eight neighbouring pages of one (sequence, KV head); a warp takes a run of units.  It looks up four of them at
// a time (lane l: page l % 8 of unit l / 8), fetches a unit's bounds while it works on the one before, and reads the queries
// again where the pair changes.  Four lanes share a page.  D = head_dim, GP = query heads per KV head rounded up to a power of two.
template <typename T, int D, int GP>
__global__ void __launch_bounds__(kPscoreThreads, sizeof(T) == 4 ? 2 : 1)
page_scores_kernel(SelectPagesParams p) {
  constexpr bool kBf16 = sizeof(T) == 2;
  constexpr int E = RopeVec<T>::E;                             // elements per 16-byte vector
  constexpr int X = D / (4 * E);                               // vectors of a bound per lane
  constexpr int NH = GP > 8 ? 2 : 1;
  begin_grid();
  extern __shared__ __align__(16) int pscore_smem[];
  __shared__ int scratch[kPscoreThreads / 32 + 1];
  int* pre = pscore_smem;                                      // [n + 1] units before sequence i (of one KV head)
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, r = lane / 4, c = lane % 4;
  const int page_size = 1 << p.page_shift, max_rows = p.width << p.page_shift, row_units = pscore_units(p.width);
  const T* bounds = static_cast<const T*>(p.bounds);
  ragged_prefix<kPscoreThreads>(p.n_seqs, pre, scratch, [&](int i) {
    bool bad = false;
    const int len = clamped_len(p.lens, p.lens_stride, i, max_rows, bad);
    if (bad && blockIdx.x == 0) set_status(p.status, MEDA_ERR_INVALID_ARG);
    const int pages = (len + page_size - 1) >> p.page_shift;
    return pages > p.keep ? pscore_units(pages) : 0;           // (a sequence that keeps everything needs no scores)
  });
  const int total = pre[p.n_seqs] * p.n_heads;
  const int warps = gridDim.x * (kPscoreThreads / 32), me = blockIdx.x * (kPscoreThreads / 32) + warp;
  const int base = total / warps, extra = total - base * warps;
  const int u0 = base * me + min(me, extra), u1 = u0 + base + (me < extra);

  uint4 mn[kBf16 ? X : 1], mx[kBf16 ? X : 1];                  // bf16: the bounds of the next unit
  uint4 pos[NH][kBf16 ? X : 1], neg[NH][kBf16 ? X : 1];        // bf16: the queries' positive and negative parts as fragments
  int held = -1;
  // this lane's page of the four units from `from` on: its bounds' place, its (sequence, KV head), its number in the sequence and that one's pages
  size_t l_at = 0;
  int l_pair = 0, l_c0 = 0, l_n = 0;
  auto look_up = [&](int from) {
    const int u = min(from + lane / 8, u1 - 1);
    const int i = ragged_find(pre, p.n_seqs, p.heads_div.of(u)), units = pre[i + 1] - pre[i];
    const int g = div_small(u - pre[i] * p.n_heads, units);
    bool bad = false;
    l_n = (clamped_len(p.lens, p.lens_stride, i, max_rows, bad) + page_size - 1) >> p.page_shift;
    l_pair = i * p.n_heads + g;
    l_c0 = (u - pre[i] * p.n_heads - g * units) * kPscoreUnit;
    l_at = bounds_place(p, p.table[(size_t)i * p.width + min(l_c0 + lane % 8, l_n - 1)], g, D);
  };
  auto fetch = [&](int u) {                                    // the bounds of unit u, one of the four looked up
    if constexpr (kBf16) {
      const T* src = bounds + __shfl_sync(0xffffffffu, l_at, ((u - u0) % 4) * 8 + r) + c * 8;
#pragma unroll
      for (int x = 0; x < X; ++x) {
        mn[x] = load_stream(reinterpret_cast<const uint4*>(src + x * 32));
        mx[x] = load_stream(reinterpret_cast<const uint4*>(src + D + x * 32));
      }
    }
  };
  if (u0 < u1) {
    look_up(u0);
    fetch(u0);
  }
#pragma unroll 1
  for (int u = u0; u < u1; ++u) {
    const int from = ((u - u0) % 4) * 8;
    const int pair = __shfl_sync(0xffffffffu, l_pair, from), c0 = __shfl_sync(0xffffffffu, l_c0, from);
    const int n = __shfl_sync(0xffffffffu, l_n, from);
    const size_t at = __shfl_sync(0xffffffffu, l_at, from + r);
    const T* qh = static_cast<const T*>(p.q) + (size_t)pair * p.group * D;
    float size, best[2];                                       // best: bf16, of pages 2c and 2c + 1; fp32, best[0] of page r
    bool odd = false;
    if constexpr (kBf16) {
      if (pair != held) {
        held = pair;
        const __nv_bfloat162 zero = __floats2bfloat162_rn(0.f, 0.f);
#pragma unroll
        for (int y = 0; y < NH; ++y) {
          const int h = r + 8 * y;
#pragma unroll
          for (int x = 0; x < X; ++x) {
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
            }
            pos[y][x] = make_uint4(a[0], a[1], a[2], a[3]);
            neg[y][x] = make_uint4(b[0], b[1], b[2], b[3]);
          }
        }
      }
      // A = queries (row: head), B = bounds (column: page), the contraction index permuted as in paged_attention.cuh
      float up[4] = {0.f, 0.f, 0.f, 0.f}, down[4] = {0.f, 0.f, 0.f, 0.f};        // four chains of dependent instructions
      float abs_up[4] = {0.f, 0.f, 0.f, 0.f}, abs_down[4] = {0.f, 0.f, 0.f, 0.f};
      constexpr uint32_t kAbs = 0x7fff7fffu;
      auto fragment = [&](float(&s)[4], const uint4(&a)[NH][X], int x, const uint4& b, uint32_t keep) {
        mma_bf16(s, a[0][x].x, NH > 1 ? a[NH - 1][x].x : 0u, a[0][x].y, NH > 1 ? a[NH - 1][x].y : 0u, b.x & keep, b.y & keep);
        mma_bf16(s, a[0][x].z, NH > 1 ? a[NH - 1][x].z : 0u, a[0][x].w, NH > 1 ? a[NH - 1][x].w : 0u, b.z & keep, b.w & keep);
      };
#pragma unroll
      for (int x = 0; x < X; ++x) {
        fragment(up, pos, x, mx[x], 0xffffffffu);
        fragment(down, neg, x, mn[x], 0xffffffffu);
        fragment(abs_up, pos, x, mx[x], kAbs);
        fragment(abs_down, neg, x, mn[x], kAbs);
      }
      if (u + 1 < u1) {
        if ((u + 1 - u0) % 4 == 0) look_up(u + 1);
        fetch(u + 1);
      }
      size = 0.f;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float a = r < p.group ? up[e] + down[e] : -INFINITY;
        const float b = NH > 1 && r + 8 < p.group ? up[2 + e] + down[2 + e] : -INFINITY;
        const float s = fmaxf(abs_up[e] - abs_down[e], abs_up[2 + e] - abs_down[2 + e]);         // (0 for heads there are none of)
        odd |= a != a || b != b || !(s < INFINITY);
        size = fmaxf(size, s);
        best[e] = fmaxf(a, b);
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) best[e] = fmaxf(best[e], __shfl_xor_sync(0xffffffffu, best[e], o));
      }
      if (r < 2 && c0 + 2 * c + r < n) p.scores[(size_t)pair * p.width + c0 + 2 * c + r] = best[r];
    } else {
      const uint4* src = reinterpret_cast<const uint4*>(bounds + at) + c;
      double acc[GP];
#pragma unroll
      for (int h = 0; h < GP; ++h) acc[h] = 0.0;
#pragma unroll 2
      for (int x = 0; x < X; ++x) {
        float lo[E], hi[E];
        RopeVec<T>::unpack(src[x * 4], lo);
        RopeVec<T>::unpack(src[D / E + x * 4], hi);
#pragma unroll
        for (int h = 0; h < GP; ++h)
          if (h < p.group) {
            float qv[E];
            RopeVec<T>::unpack(*reinterpret_cast<const uint4*>(qh + (size_t)h * D + (x * 4 + c) * E), qv);
#pragma unroll
            for (int e = 0; e < E; ++e) acc[h] = fma((double)qv[e], (double)(qv[e] >= 0.f ? hi[e] : lo[e]), acc[h]);
          }
      }
      float top = -INFINITY;
      bool nan = false;
#pragma unroll
      for (int h = 0; h < GP; ++h)
        if (h < p.group) {
          double s = acc[h];
          s += __shfl_xor_sync(0xffffffffu, s, 1);
          s += __shfl_xor_sync(0xffffffffu, s, 2);
          const float f = (float)s;
          nan |= f != f;
          top = fmaxf(top, f);
        }
      odd = nan || fabsf(top) == INFINITY;
      size = 0.f;
      best[0] = best[1] = top;
      if (c == 0 && c0 + r < n) p.scores[(size_t)pair * p.width + c0 + r] = nan ? NAN : top;
      if (u + 1 < u1 && (u + 1 - u0) % 4 == 0) look_up(u + 1);
    }
    // (pages behind the last repeat it)
    const float high = warp_max(fmaxf(best[0], best[1])), low = -warp_max(-fminf(best[0], best[1]));
    size = warp_max(size);
    odd = __any_sync(0xffffffffu, odd);
    if (lane == 0) p.units[(size_t)pair * row_units + c0 / kPscoreUnit] = make_float4(odd ? NAN : size, high, low, 0.f);
  }
}

// The score of one page for one KV head by a whole warp, in 64 bits.  qs: the head's queries [group][D] as floats.  A lane
// holds D / 32 dimensions; the sums of eight heads are exchanged so that four lanes end up with each.
template <typename T, int D>
__device__ __noinline__ float page_score_warp(const T* lo, const float* qs, int group, int lane) {
  constexpr int N = D / 32;
  double mn[N], mx[N];
#pragma unroll
  for (int e = 0; e < N; ++e) {
    mn[e] = (double)to_f32<T>(lo[e * 32 + lane]);
    mx[e] = (double)to_f32<T>(lo[D + e * 32 + lane]);
  }
  float best = -INFINITY;
  bool nan = false;
#pragma unroll 1
  for (int h0 = 0; h0 < group; h0 += 8) {
    double s[8];
#pragma unroll
    for (int y = 0; y < 8; ++y) {
      s[y] = 0.0;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const double q = (double)qs[min(h0 + y, group - 1) * D + e * 32 + lane];
        s[y] = fma(q, q >= 0.0 ? mx[e] : mn[e], s[y]);
      }
    }
#pragma unroll
    for (int o = 4; o >= 1; o >>= 1) {                         // lanes 4 o apart keep the upper or the lower half of what is left
      const bool upper = (lane & (4 * o)) != 0;
#pragma unroll
      for (int y = 0; y < o; ++y) {
        const double give = upper ? s[y] : s[y + o], keep = upper ? s[y + o] : s[y];
        s[y] = keep + __shfl_xor_sync(0xffffffffu, give, 4 * o);
      }
    }
    s[0] += __shfl_xor_sync(0xffffffffu, s[0], 2);
    s[0] += __shfl_xor_sync(0xffffffffu, s[0], 1);
    const float f = (float)s[0];                               // of head h0 + lane / 4 (of the last head again behind it)
    nan |= f != f;
    best = fmaxf(best, f);
  }
  best = warp_max(best);
  return __any_sync(0xffffffffu, nan) ? NAN : best;
}

// ---- the choice, one block per (sequence, KV head) ---------------------------------------------------------
// Shared memory: the queries as floats, two bits per page.
__host__ __device__ inline int choose_smem(int width, int group, int d) { return (group * d + 2 * ((width + 31) / 32)) * 4; }

template <typename T, int D, int kPselThreads>
__global__ void __launch_bounds__(kPselThreads, 1024 / kPselThreads)
choose_pages_kernel(SelectPagesParams p) {
  constexpr bool kExact = sizeof(T) == 4;                      // the scores are the 64-bit ones already
  constexpr int kWarps = kPselThreads / 32;
  begin_grid();
  extern __shared__ __align__(16) float choose_smem_base[];
  __shared__ unsigned int hist[kPselBins];
  __shared__ uint2 list[kPselMaxDoubt];                        // (key, page) of the pages in doubt
  __shared__ int listed_page[kPselMaxDoubt];                   // their table entries
  __shared__ int scan[kWarps];
  __shared__ float red[3][kWarps];
  __shared__ int s_bin, s_need, s_sure, s_listed;
  float* qs = choose_smem_base;                                // [group][D]
  unsigned int* kept = reinterpret_cast<unsigned int*>(qs + p.group * D);      // [words]
  unsigned int* equal = kept + (p.width + 31) / 32;            // [words], the fallback's
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const int pair = blockIdx.x, i = p.heads_div.of(pair), g = pair - i * p.n_heads;
  const int page_size = 1 << p.page_shift;
  // a thread's scores: page (round * items + y) * threads + thread, so that a warp's 32 pages are one word of the bit maps;
  // what the first round needs is fetched before the sequence's length is known
  const float* scores = p.scores + (size_t)pair * p.width;
  const float4* units = p.units + (size_t)pair * pscore_units(p.width);
  float v[kPselItems];
  auto page_at = [&](int round, int y) { return (round * kPselItems + y) * kPselThreads + (int)threadIdx.x; };
  auto load_round = [&](int round) {
#pragma unroll
    for (int y = 0; y < kPselItems; ++y) {
      const int c = page_at(round, y);
      v[y] = c < p.width ? scores[c] : 0.f;
    }
  };
  load_round(0);
  const float4 first_unit = (int)threadIdx.x < pscore_units(p.width) ? units[threadIdx.x] : make_float4(0.f, 0.f, 0.f, 0.f);
  bool bad = false;
  const int len = clamped_len(p.lens, p.lens_stride, i, p.width << p.page_shift, bad);
  const int n = (len + page_size - 1) >> p.page_shift;         // pages of the sequence
  int32_t* out = p.sel + (size_t)pair * p.keep;
  if (n <= p.keep) {                                           // every page is kept
#pragma unroll 1
    for (int c = threadIdx.x; c < n; c += kPselThreads) out[c] = c;
    return;
  }
  const T* qh = static_cast<const T*>(p.q) + (size_t)pair * p.group * D;
  const T* bounds = static_cast<const T*>(p.bounds);
  const int32_t* table = p.table + (size_t)i * p.width;
  const int want = p.keep - p.n_first - p.n_last;              // pages to choose among those that are not kept anyway
  const int words = (n + 31) / 32, rounds = (n + kPselThreads * kPselItems - 1) / (kPselThreads * kPselItems);
  auto forced = [&](int c) { return c < p.n_first || c >= n - p.n_last; };
  auto open_page = [&](int c) { return c < n && !forced(c); };

  auto any_at = [&](int round, int y) { return (round * kPselItems + y) * kPselThreads < n; };       // uniform
  // pages kept anyway count as +inf from here on, what lies behind the last page as -inf
  auto settle = [&](int round) {
#pragma unroll
    for (int y = 0; y < kPselItems; ++y) {
      const int c = page_at(round, y);
      if (any_at(round, y)) v[y] = c >= n ? -INFINITY : (forced(c) ? INFINITY : v[y]);
    }
  };
  float top = -INFINITY, bottom = INFINITY, limit = 0.f;       // limit: largest sum |q| |bound|
  bool odd = false;
#pragma unroll 1
  for (int x = threadIdx.x; x < pscore_units(n); x += kPselThreads) {
    const float4 f = x == (int)threadIdx.x ? first_unit : units[x];
    odd |= f.x != f.x;
    limit = fmaxf(limit, f.x);
    top = fmaxf(top, f.y);
    bottom = fminf(bottom, f.z);
  }
  if constexpr (!kExact)
#pragma unroll 1
    for (int x = threadIdx.x; x < p.group * D; x += kPselThreads) qs[x] = to_f32<T>(qh[x]);
#pragma unroll 1
  for (int x = threadIdx.x; x < kPselBins; x += kPselThreads) hist[x] = 0u;
  if (threadIdx.x == 0) s_sure = s_listed = 0;
  top = warp_max(top);
  bottom = -warp_max(-bottom);
  limit = warp_max(limit);
  if (lane == 0) {
    red[0][warp] = top;
    red[1][warp] = -bottom;
    red[2][warp] = limit;
  }
  odd = __syncthreads_or(odd);
  top = warp_max(red[0][lane % kWarps]);
  bottom = -warp_max(red[1][lane % kWarps]);
  limit = warp_max(red[2][lane % kWarps]);
  // eps: a score is 2 D products summed by D / 8 instructions; each adds 16 products to a sum in fp32, cutting every addend to
  // 24 bits of the largest at worst, 17 * 2^-24 of sum |q| |bound| in all: D / 8 * 17 * 2^-24 < D 2^-22.  (That sum itself is known to
  // as much: the 1 % on top covers it.)
  const float slack = 2.f * 1.01f * (float)D * 2.384185791015625e-7f * limit;
  const float scale = top > bottom ? (kPselBins - 1) / (top - bottom) : 0.f;
  const float scale_or_one = scale > 0.f ? scale : 1.f;
  // bin 0 holds the best scores; fp32 rounding keeps the order
  auto bin_of = [&](float s) { return (int)fminf(fmaxf((top - s) * scale, 0.f), (float)(kPselBins - 1)); };
  bool decided = !odd && slack < 1e30f && scale < 1e30f && top < 1e30f && bottom > -1e30f;
  if (want == 0) {                                             // nothing to choose
#pragma unroll 1
    for (int w = threadIdx.x; w < words; w += kPselThreads) kept[w] = 0u;
    __syncthreads();
#pragma unroll 1
    for (int c = threadIdx.x; c < p.n_first + p.n_last; c += kPselThreads) {
      const int page = c < p.n_first ? c : n - p.n_last + (c - p.n_first);
      atomicOr(&kept[page / 32], 1u << (page % 32));
    }
    __syncthreads();
  } else if (decided) {
#pragma unroll 1
    for (int round = 0; round < rounds; ++round) {
      if (round > 0) load_round(round);
      settle(round);
#pragma unroll
      for (int y = 0; y < kPselItems; ++y)
        if (any_at(round, y) && v[y] != -INFINITY) atomicAdd(&hist[bin_of(v[y])], 1u);
    }
    __syncthreads();
    {
      constexpr int kOwn = kPselBins / kPselThreads;           // a thread's bins
      int own[kOwn], sum = 0;
#pragma unroll
      for (int y = 0; y < kOwn; ++y) {
        own[y] = (int)hist[kOwn * threadIdx.x + y];
        sum += own[y];
      }
      int all;
      int before = block_prefix<kPselThreads>(sum, scan, all);
#pragma unroll
      for (int y = 0; y < kOwn; ++y) {
        if (before < p.keep && before + own[y] >= p.keep) s_bin = kOwn * threadIdx.x + y;
        before += own[y];
      }
    }
    __syncthreads();
    // the bin of the keep-th largest approximate score, widened by the rounding of its own borders, and 2 eps on each side
    const float round_off = 1e-6f * (fabsf(top) + fabsf(bottom));
    const float high = top - (float)s_bin / scale_or_one + round_off + slack, low = top - (float)(s_bin + 1) / scale_or_one - round_off - slack;
    int sure = 0;                                              // of the warp's pages (lane 0 counts)
#pragma unroll 1
    for (int round = 0; round < rounds; ++round) {
      if (rounds > 1) {
        load_round(round);
        settle(round);
      }
#pragma unroll
      for (int y = 0; y < kPselItems; ++y) {
        const int c = page_at(round, y);
        if (any_at(round, y) && c - lane < n) {                // uniform over the warp
          const unsigned int word = __ballot_sync(0xffffffffu, v[y] > high);
          if (lane == 0) {
            kept[c / 32] = word;
            sure += __popc(word);
          }
          if (v[y] <= high && v[y] >= low) {
            const int e = atomicAdd(&s_listed, 1);
            if (e < kPselMaxDoubt) {
              list[e] = make_uint2(page_key(v[y]), (unsigned int)c);
              if constexpr (!kExact) listed_page[e] = table[c];
            }
          }
        }
      }
    }
    if (lane == 0) atomicAdd(&s_sure, sure);
    __syncthreads();
    const int listed = s_listed, need = p.keep - s_sure;
    decided = listed <= kPselMaxDoubt;
    if (decided) {
      if constexpr (!kExact) {
#pragma unroll 1
        for (int e = warp; e < listed; e += kWarps) {
          const float s = page_score_warp<T, D>(bounds + bounds_place(p, listed_page[e], g, D), qs, p.group, lane);
          if (lane == 0) list[e].x = page_key(s);
        }
        __syncthreads();
      }
#pragma unroll 1
      for (int e = threadIdx.x; e < listed; e += kPselThreads) {     // the `need` best of the list, ties to the lowest page
        const uint2 me = list[e];
        int better = 0;
#pragma unroll 4
        for (int o = 0; o < listed; ++o) {
          const uint2 x = list[o];
          better += x.x > me.x || (x.x == me.x && x.y < me.y);
        }
        if (better < need) atomicOr(&kept[me.y / 32], 1u << (me.y % 32));
      }
      __syncthreads();
    }
  }
  if (want > 0 && !decided) {
    // ---- every page in 64 bits (into the scores' place), and radix passes to the last bit
    float* exact = p.scores + (size_t)pair * p.width;
    if constexpr (!kExact) {
#pragma unroll 1
      for (int c = warp; c < n; c += kWarps) {
        const float s = page_score_warp<T, D>(bounds + bounds_place(p, table[c], g, D), qs, p.group, lane);
        if (lane == 0) exact[c] = s;
      }
    }
    __syncthreads();
    unsigned int prefix = 0u, mask = 0u;
    int remaining = want;
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 21 : (pass == 1 ? 10 : 0);
      const unsigned int bins = pass == 2 ? 1024u : 2048u;
#pragma unroll 1
      for (int x = threadIdx.x; x < kPselBins; x += kPselThreads) hist[x] = 0u;
      __syncthreads();
#pragma unroll 1
      for (int c = threadIdx.x; c < n; c += kPselThreads) {
        const unsigned int key = page_key(exact[c]);
        if (!forced(c) && (key & mask) == prefix) atomicAdd(&hist[(key >> shift) & (bins - 1u)], 1u);
      }
      __syncthreads();
      constexpr int kOwn = kPselBins / kPselThreads;           // a thread's bins, from the top down
      const int b0 = (int)bins - 1 - kOwn * (int)threadIdx.x;
      int sum = 0, all;
#pragma unroll 1
      for (int y = 0; y < kOwn; ++y) sum += b0 - y >= 0 ? (int)hist[b0 - y] : 0;
      int above = block_prefix<kPselThreads>(sum, scan, all);
#pragma unroll 1
      for (int y = 0; y < kOwn && b0 - y >= 0; ++y) {
        const int here = (int)hist[b0 - y];
        if (above < remaining && above + here >= remaining) {
          s_bin = b0 - y;
          s_need = remaining - above;
        }
        above += here;
      }
      __syncthreads();
      prefix |= (unsigned int)s_bin << shift;
      mask |= (bins - 1u) << shift;
      remaining = s_need;
      __syncthreads();
    }
#pragma unroll 1
    for (int c = threadIdx.x; c < words * 32; c += kPselThreads) {             // words * 32 and the stride keep warps whole
      const unsigned int key = c < n ? page_key(exact[c]) : 0u;
      const unsigned int above = __ballot_sync(0xffffffffu, c < n && (forced(c) || key > prefix));
      const unsigned int same = __ballot_sync(0xffffffffu, open_page(c) && key == prefix);
      if (lane == 0) {
        kept[c / 32] = above;
        equal[c / 32] = same;
      }
    }
    __syncthreads();
    int before = 0;
#pragma unroll 1
    for (int w0 = 0; w0 < words; w0 += kPselThreads) {         // of equal keys the lowest pages
      const int w = w0 + (int)threadIdx.x;
      unsigned int same = w < words ? equal[w] : 0u;
      int all;
      int rank = before + block_prefix<kPselThreads>(__popc(same), scan, all);
      before += all;
#pragma unroll 1
      while (same && rank < remaining) {
        const unsigned int bit = same & (0u - same);
        kept[w] |= bit;
        same ^= bit;
        ++rank;
      }
    }
    __syncthreads();
  }

  // ---- kept pages, in order
  int before = 0;
#pragma unroll 1
  for (int w0 = 0; w0 < words; w0 += kPselThreads) {
    const int w = w0 + (int)threadIdx.x;
    unsigned int bits = w < words ? kept[w] : 0u;
    int all;
    int at = before + block_prefix<kPselThreads>(__popc(bits), scan, all);
    before += all;
#pragma unroll 1
    while (bits) {
      const int b = __ffs((int)bits) - 1;
      bits &= bits - 1u;
      out[at++] = w * 32 + b;
    }
  }
}

}  // namespace meda
