// Attention of one new token per sequence over paged caches of ragged lengths (Eq. 3), in one launch.
//
// Work split.  All (sequence, KV head, 16-row tile) triples form one list; block c of C takes the c-th equal part of
// it, so a batch of one 128K cache and a batch of 64 very different ones load the GPU alike, without the host
// knowing any length.  Inside a block the warps take tiles in turn.  A segment (sequence, KV head) that lies in one
// block is finished there; the at most two segments of a block that cross its borders leave softmax states (max, sum,
// weighted values) in scratch, and the block that arrives last at such a segment joins the states in block order:
// no second launch, no atomics on values, the same bits every run.
//
// Inner loop, bf16.  One pass over K and V with the running maximum and sum.  A warp's tile goes straight from
// global memory into matrix-instruction fragments: the contraction index of Q K^T may be permuted freely as
// long as Q and K agree, so a lane's 16-byte piece of a key row serves as four fragments; the same holds for the
// value rows with P V written as (V^T)(P^T), where two byte permutes pair neighbouring rows.  So there is no shared
// memory, barrier or bulk copy in the loop; latency is covered by the next tile's loads, issued before this tile's
// arithmetic, in all the warps of an SM.  The kernel is bound by reading the cache; the matrix instructions only have
// to keep up (24 to 32 of them for 8 KB at head_dim 128), so the warp-level ones are used: eight query heads fill
// their narrow side, where the tensor-memory instructions would want 128 rows of queries.
// Probabilities enter P V as a sum of two bf16 numbers (16 bits of mantissa, 2^-17 relative), so that rounding
// them stays below the rounding of the output; logits, maxima, sums and accumulators are fp32.
//
// fp32 caches: the same walk with the products on the CUDA cores (see DecodeShape in decode.cuh for the reduction).
#pragma once

#include "decode.cuh"        // transpose_reduce
#include "page_rows.cuh"     // load_stream
#include "pages_common.cuh"

namespace meda {

constexpr int kAttTile = 16;             // rows per tile; a page holds whole tiles

struct AttnParams {
  const void* q;
  const void* k;
  const void* v;
  const int32_t* table;
  const int32_t* lens;
  const int32_t* sel;
  void* out;
  float* lse;
  float* partial;
  unsigned int* counters;
  int* status;
  int lens_stride, n_seqs, n_heads, group, n_pages, width, page_shift, keep;
  float scale_log2;                      // log2(e) / sqrt(head_dim)
};

__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t word_of(const uint4& x, int i) { return i == 0 ? x.x : i == 1 ? x.y : i == 2 ? x.z : x.w; }

// ---- bf16: D = head_dim, NH = groups of eight query heads ------------------------------------------------
// Lane l: r = l / 4, c = l % 4.  Q K^T has A = queries (row r: head r, row r + 8: head r + 8), B = keys (column r: row r of
// the tile's half); P V has A = V^T, B = P^T (row pairs 2c, 2c + 1 of both halves; column r: head r).
template <int D, int NH>
struct AttnTileBf16 {
  using T = __nv_bfloat16;
  static constexpr int kHeads = 8 * NH;
  static constexpr int KC = D / 32, VC = D / 64;
  uint4 q[NH][KC];
  uint4 k[2][KC];
  uint4 v[4][VC];
  float o[VC][4][NH][4];
  float m[NH], l[NH];

  __device__ __forceinline__ void begin(const T* qh, int heads, int lane) {      // qh: the segment's first query head
    const int r = lane / 4, c = lane % 4;
#pragma unroll
    for (int n = 0; n < NH; ++n) {
      const int h = r + 8 * n;
#pragma unroll
      for (int x = 0; x < KC; ++x)
        q[n][x] = h < heads ? *reinterpret_cast<const uint4*>(qh + (size_t)h * D + x * 32 + c * 8) : make_uint4(0, 0, 0, 0);
      m[n] = -INFINITY;
      l[n] = 0.f;
    }
#pragma unroll
    for (int y = 0; y < VC; ++y)
#pragma unroll
      for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int n = 0; n < NH; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[y][x][n][e] = 0.f;
  }
  __device__ __forceinline__ void load_k(const T* rows, int nv, int lane) {
    const int r = lane / 4, c = lane % 4;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const bool on = t * 8 + r < nv;
#pragma unroll
      for (int x = 0; x < KC; ++x)
        k[t][x] = on ? load_stream(reinterpret_cast<const uint4*>(rows + (t * 8 + r) * D + x * 32 + c * 8)) : make_uint4(0, 0, 0, 0);
    }
  }
  __device__ __forceinline__ void load_v(const T* rows, int nv, int lane) {
    const int r = lane / 4, c = lane % 4;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int row = 2 * c + (t & 1) + (t >> 1) * 8;
      const bool on = row < nv;
#pragma unroll
      for (int y = 0; y < VC; ++y)
        v[t][y] = on ? load_stream(reinterpret_cast<const uint4*>(rows + row * D + y * 64 + r * 8)) : make_uint4(0, 0, 0, 0);
    }
  }
  // logits of the tile in k, in the log2 domain: s[t][0..1] head r, rows t * 8 + 2c, + 1; s[t][2..3] head r + 8
  __device__ __forceinline__ void logits(float (&s)[2][4], float scale_log2, int nv, int lane) {
    const int c = lane % 4;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      float even[4] = {0.f, 0.f, 0.f, 0.f}, odd[4] = {0.f, 0.f, 0.f, 0.f};       // two chains of dependent instructions
#pragma unroll
      for (int x = 0; x < KC; ++x) {
        mma_bf16(even, q[0][x].x, NH > 1 ? q[NH - 1][x].x : 0u, q[0][x].y, NH > 1 ? q[NH - 1][x].y : 0u, k[t][x].x, k[t][x].y);
        mma_bf16(odd, q[0][x].z, NH > 1 ? q[NH - 1][x].z : 0u, q[0][x].w, NH > 1 ? q[NH - 1][x].w : 0u, k[t][x].z, k[t][x].w);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[t][e] = (even[e] + odd[e]) * scale_log2;
        if (t * 8 + 2 * c + (e & 1) >= nv) s[t][e] = -INFINITY;
      }
    }
  }
  __device__ __forceinline__ void attend(float (&s)[2][4], int lane) {
    const int c = lane % 4;
    uint32_t hi[NH][2], lo[NH][2];
#pragma unroll
    for (int n = 0; n < NH; ++n) {
      float top = fmaxf(fmaxf(s[0][2 * n], s[0][2 * n + 1]), fmaxf(s[1][2 * n], s[1][2 * n + 1]));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const float mn = fmaxf(m[n], top);
      const float ref = mn == -INFINITY ? 0.f : mn;
      if (__any_sync(0xffffffffu, mn > m[n])) {                // the maximum moved: bring the sums to the new one
        const float f = exp2f(m[n] - ref);
        m[n] = mn;
        l[n] *= f;
        const float f0 = __shfl_sync(0xffffffffu, f, 8 * c), f1 = __shfl_sync(0xffffffffu, f, 8 * c + 4);   // heads 2c, 2c + 1
#pragma unroll
        for (int y = 0; y < VC; ++y)
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            o[y][x][n][0] *= f0;
            o[y][x][n][1] *= f1;
            o[y][x][n][2] *= f0;
            o[y][x][n][3] *= f1;
          }
      }
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const float p0 = exp2f(s[t][2 * n] - ref), p1 = exp2f(s[t][2 * n + 1] - ref);
        l[n] += p0 + p1;
        const __nv_bfloat162 h2 = __floats2bfloat162_rn(p0, p1);
        const __nv_bfloat162 l2 = __floats2bfloat162_rn(p0 - __low2float(h2), p1 - __high2float(h2));
        memcpy(&hi[n][t], &h2, 4);
        memcpy(&lo[n][t], &l2, 4);
      }
    }
#pragma unroll
    for (int y = 0; y < VC; ++y)
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const uint32_t w0 = word_of(v[0][y], x), w1 = word_of(v[1][y], x), w2 = word_of(v[2][y], x), w3 = word_of(v[3][y], x);
        const uint32_t a0 = __byte_perm(w0, w1, 0x5410), a1 = __byte_perm(w0, w1, 0x7632);
        const uint32_t a2 = __byte_perm(w2, w3, 0x5410), a3 = __byte_perm(w2, w3, 0x7632);
#pragma unroll
        for (int n = 0; n < NH; ++n) {
          mma_bf16(o[y][x][n], a0, a1, a2, a3, hi[n][0], hi[n][1]);
          mma_bf16(o[y][x][n], a0, a1, a2, a3, lo[n][0], lo[n][1]);
        }
      }
  }
  // state to shared memory: sm [kHeads], sl [kHeads], so [kHeads][ld]
  __device__ __forceinline__ void put(float* sm, float* sl, float* so, int ld, int heads, int lane) {
    const int r = lane / 4, c = lane % 4;
#pragma unroll
    for (int n = 0; n < NH; ++n) {
      float sum = l[n];
      sum += __shfl_xor_sync(0xffffffffu, sum, 1);
      sum += __shfl_xor_sync(0xffffffffu, sum, 2);
      if (c == 0) {
        sm[r + 8 * n] = m[n];
        sl[r + 8 * n] = sum;
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int h = 2 * c + e + 8 * n;
        if (h < heads) {
#pragma unroll
          for (int y = 0; y < VC; ++y) {
            float4* d = reinterpret_cast<float4*>(so + h * ld + y * 64 + r * 8);
            d[0] = make_float4(o[y][0][n][e], o[y][0][n][2 + e], o[y][1][n][e], o[y][1][n][2 + e]);
            d[1] = make_float4(o[y][2][n][e], o[y][2][n][2 + e], o[y][3][n][e], o[y][3][n][2 + e]);
          }
        }
      }
    }
  }
};

// ---- fp32: GP = query heads handled together (1, 2, 4 or 8) -------------------------------------------------
// Lane l owns dimensions [l * E, l * E + E).  A tile is worked through four rows at a time; lane h * 4 + b of the
// transposing reduction owns the logit of (row b, head h).
template <int D, int GP>
struct AttnTileF32 {
  using T = float;
  static constexpr int kHeads = GP;
  static constexpr int E = D / 32, B = 4;
  static constexpr int P = GP * B <= 8 ? 8 : (GP * B <= 16 ? 16 : 32);
  float q[GP][E];
  float kx[2][B][E], vx[2][B][E];
  float acc[GP][E];
  float m, l;                            // of this lane's head

  __device__ __forceinline__ void begin(const T* qh, int heads, int lane) {
#pragma unroll
    for (int h = 0; h < GP; ++h)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        q[h][e] = h < heads ? qh[(size_t)h * D + lane * E + e] : 0.f;
        acc[h][e] = 0.f;
      }
    m = -INFINITY;
    l = 0.f;
  }
  __device__ __forceinline__ static void load_rows(float (&x)[B][E], const T* rows, int r0, int nv, int lane) {
#pragma unroll
    for (int b = 0; b < B; ++b) {
      const bool on = r0 + b < nv;
      const T* src = rows + (r0 + b) * D + lane * E;
      if constexpr (E == 2) {
        const float2 t = on ? *reinterpret_cast<const float2*>(src) : make_float2(0.f, 0.f);
        x[b][0] = t.x;
        x[b][1] = t.y;
      } else {
#pragma unroll
        for (int e = 0; e < E; e += 4) {
          const float4 t = on ? *reinterpret_cast<const float4*>(src + e) : make_float4(0.f, 0.f, 0.f, 0.f);
          x[b][e] = t.x;
          x[b][e + 1] = t.y;
          x[b][e + 2] = t.z;
          x[b][e + 3] = t.w;
        }
      }
    }
  }
  // One group of four rows, already in kx[cur], vx[cur], of which rows r0 + b < nv count.
  __device__ __forceinline__ void rows4(int cur, int r0, int nv, float scale_log2, int lane) {
    float part[P];
#pragma unroll
    for (int i = 0; i < P; ++i) part[i] = 0.f;
#pragma unroll
    for (int h = 0; h < GP; ++h)
#pragma unroll
      for (int b = 0; b < B; ++b) {
        float dot = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) dot = fmaf(q[h][e], kx[cur][b][e], dot);
        part[h * B + b] = dot;
      }
    float s = transpose_reduce<P>(part, lane) * scale_log2;
    const int pair = lane % P;
    if (pair >= GP * B || r0 + pair % B >= nv) s = -INFINITY;
    float mn = s;
    mn = fmaxf(mn, __shfl_xor_sync(0xffffffffu, mn, 1));
    mn = fmaxf(mn, __shfl_xor_sync(0xffffffffu, mn, 2));
    mn = fmaxf(mn, m);
    const float ref = mn == -INFINITY ? 0.f : mn;
    const float pr = exp2f(s - ref), f = exp2f(m - ref);
    float sum = pr;
    sum += __shfl_xor_sync(0xffffffffu, sum, 1);
    sum += __shfl_xor_sync(0xffffffffu, sum, 2);
    l = l * f + sum;
    m = mn;
#pragma unroll
    for (int h = 0; h < GP; ++h) {
      const float fh = __shfl_sync(0xffffffffu, f, h * B);
#pragma unroll
      for (int e = 0; e < E; ++e) acc[h][e] *= fh;
#pragma unroll
      for (int b = 0; b < B; ++b) {
        const float w = __shfl_sync(0xffffffffu, pr, h * B + b);
#pragma unroll
        for (int e = 0; e < E; ++e) acc[h][e] = fmaf(w, vx[cur][b][e], acc[h][e]);
      }
    }
  }
  __device__ __forceinline__ void put(float* sm, float* sl, float* so, int ld, int heads, int lane) {
#pragma unroll
    for (int h = 0; h < GP; ++h) {
      const float mh = __shfl_sync(0xffffffffu, m, h * B), lh = __shfl_sync(0xffffffffu, l, h * B);
      if (lane == 0) {
        sm[h] = mh;
        sl[h] = lh;
      }
      if (h < heads)
#pragma unroll
        for (int e = 0; e < E; ++e) so[h * ld + lane * E + e] = acc[h][e];
    }
  }
};

template <typename T>
__device__ __forceinline__ void store4(T* dst, const float4& x);
template <>
__device__ __forceinline__ void store4<float>(float* dst, const float4& x) { *reinterpret_cast<float4*>(dst) = x; }
template <>
__device__ __forceinline__ void store4<__nv_bfloat16>(__nv_bfloat16* dst, const float4& x) {
  const __nv_bfloat162 a = __floats2bfloat162_rn(x.x, x.y), b = __floats2bfloat162_rn(x.z, x.w);
  uint2 w;
  memcpy(&w.x, &a, 4);
  memcpy(&w.y, &b, 4);
  *reinterpret_cast<uint2*>(dst) = w;
}

// Floats of one softmax state in scratch: values of every head, then maxima, then sums (padded to 16 bytes).
__host__ __device__ inline int attn_state_floats(int heads, int d) { return heads * (d + 4); }
// Shared memory: prefix of tiles, and the larger of the warps' states and the weights of a join.
__host__ __device__ inline int attn_prefix_floats(int n_seqs) { return (n_seqs + 1 + 3) / 4 * 4; }
__host__ __device__ inline int attn_merge_floats(int warps, int heads, int d, int blocks) {
  const int states = warps * heads * (d + 4 + 2), join = blocks * heads + 2 * heads;
  return states > join ? states : join;
}

template <typename Tile, int D, int W>
__global__ void __launch_bounds__(W * 32, 1)
paged_attention_kernel(AttnParams p) {
  using T = typename Tile::T;
  constexpr bool kBf16 = sizeof(T) == 2;
  constexpr int HP = Tile::kHeads;
  constexpr int LD = D + 4;
  extern __shared__ __align__(16) float att_smem[];
  __shared__ int scratch[W + 1];
  __shared__ int s_last;
  int* pre = reinterpret_cast<int*>(att_smem);
  float* sm_m = att_smem + attn_prefix_floats(p.n_seqs);       // [W][HP]
  float* sm_l = sm_m + W * HP;                                 // [W][HP]
  float* sm_o = sm_l + W * HP;                                 // [W][HP][LD]
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const int max_rows = p.width << p.page_shift, page_size = 1 << p.page_shift;
  const int tile_shift = p.page_shift - 4;                     // log2(tiles per page)
  const int chunks = (p.group + HP - 1) / HP;                  // segments per KV head
  const int H = p.n_heads * chunks;
  const int state_heads = min(p.group, HP);
  const int state_floats = attn_state_floats(state_heads, D);
  const int n_q_heads = p.n_heads * p.group;

  ragged_prefix<W * 32>(p.n_seqs, pre, scratch, [&](int i) {
    bool bad = false;
    const int len = clamped_len(p.lens, p.lens_stride, i, max_rows, bad);
    if (bad && blockIdx.x == 0) set_status(p.status, MEDA_ERR_INVALID_ARG);
    if (!p.sel) return (len + kAttTile - 1) / kAttTile;
    return min(p.keep, (len + page_size - 1) >> p.page_shift) << tile_shift;
  });

  // sequences without rows
  for (int i = blockIdx.x; i < p.n_seqs; i += gridDim.x)
    if (pre[i] == pre[i + 1]) {
      for (int x = threadIdx.x; x < n_q_heads * D / 4; x += W * 32)
        store4<T>(static_cast<T*>(p.out) + (size_t)i * n_q_heads * D + x * 4, make_float4(0.f, 0.f, 0.f, 0.f));
      if (p.lse)
        for (int h = threadIdx.x; h < n_q_heads; h += W * 32) p.lse[(size_t)i * n_q_heads + h] = -INFINITY;
    }

  const long long total = (long long)pre[p.n_seqs] * H;
  const long long C = min((long long)gridDim.x, (total + W - 1) / W);        // blocks with work: a tile per warp at least
  if ((long long)blockIdx.x >= C) return;
  const long long t0 = total * blockIdx.x / C, t1 = total * (blockIdx.x + 1) / C;

  // a tile's first row in the pools and the number of its rows that count (0: nothing to read)
  auto lookup = [&](long long x, long long& row, int& nv) {
    row = 0;
    nv = 0;
    if (x >= t1) return;
    const int i = ragged_find(pre, p.n_seqs, (int)(x / H));
    const int tiles = pre[i + 1] - pre[i];
    const int local = (int)(x - (long long)pre[i] * H);
    const int sh = local / tiles, tile = local - sh * tiles, g = sh / chunks;
    bool bad = false;
    const int len = clamped_len(p.lens, p.lens_stride, i, max_rows, bad);
    int col = tile >> tile_shift;
    const int r0 = (tile & ((1 << tile_shift) - 1)) * kAttTile;
    bool ok = true;
    if (p.sel) {
      col = p.sel[((size_t)i * p.n_heads + g) * p.keep + col];
      ok = col >= 0 && col < (len + page_size - 1) >> p.page_shift;
    }
    if (ok) {
      nv = min(kAttTile, max(0, len - ((col << p.page_shift) + r0)));
      if (nv > 0) {
        const int page = p.table[(size_t)i * p.width + col];
        ok = (unsigned)page < (unsigned)p.n_pages;
        row = (((long long)page * p.n_heads + g) << p.page_shift) + r0;
      }
    }
    if (!ok) {
      nv = 0;
      set_status(p.status, MEDA_ERR_INVALID_ARG);
    }
  };

  // lane y holds the look-up of the warp's y-th tile from here, and of the 32 tiles after those
  const T* kp = static_cast<const T*>(p.k);
  const T* vp = static_cast<const T*>(p.v);
  long long x = t0 + warp;
  long long row_now, row_next;
  int nv_now, nv_next;
  lookup(x + (long long)lane * W, row_now, nv_now);
  lookup(x + (long long)(32 + lane) * W, row_next, nv_next);
  int at = 0;
  Tile tile;
  long long row = __shfl_sync(0xffffffffu, row_now, 0);
  int nv = __shfl_sync(0xffffffffu, nv_now, 0);
  if constexpr (kBf16) {
    tile.load_k(kp + row * D, nv, lane);
    tile.load_v(vp + row * D, nv, lane);
  } else {
    tile.load_rows(tile.kx[0], kp + row * D, 0, nv, lane);
    tile.load_rows(tile.vx[0], vp + row * D, 0, nv, lane);
  }

  int seq = ragged_find(pre, p.n_seqs, (int)(t0 / H));
  int sh = (int)(t0 - (long long)pre[seq] * H) / (pre[seq + 1] - pre[seq]);
  long long seg0 = (long long)pre[seq] * H + (long long)sh * (pre[seq + 1] - pre[seq]);
  while (seg0 < t1) {
    const int tiles = pre[seq + 1] - pre[seq];
    const long long seg1 = seg0 + tiles;
    const long long end = min(seg1, t1);
    const int g = sh / chunks, h0 = (sh % chunks) * HP;
    const int heads = min(HP, p.group - h0);
    const size_t first_head = (size_t)seq * n_q_heads + (size_t)g * p.group + h0;
    tile.begin(static_cast<const T*>(p.q) + first_head * D, heads, lane);

    while (x < end) {
      // where the warp's next tile lies
      ++at;
      if (at == 32) {
        row_now = row_next;
        nv_now = nv_next;
        at = 0;
        lookup(x + (long long)(33 + lane) * W, row_next, nv_next);
      }
      const long long row_after = __shfl_sync(0xffffffffu, row_now, at);
      const int nv_after = __shfl_sync(0xffffffffu, nv_now, at);
      if constexpr (kBf16) {
        float s[2][4];
        tile.logits(s, p.scale_log2, nv, lane);
        tile.load_k(kp + row_after * D, nv_after, lane);
        if (nv > 0) tile.attend(s, lane);
        tile.load_v(vp + row_after * D, nv_after, lane);
      } else {
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          const T* nk = b < 3 ? kp + row * D : kp + row_after * D;
          const T* nvp = b < 3 ? vp + row * D : vp + row_after * D;
          const int r0 = b < 3 ? 4 * (b + 1) : 0, n = b < 3 ? nv : nv_after;
          tile.load_rows(tile.kx[(b + 1) & 1], nk, r0, n, lane);
          tile.load_rows(tile.vx[(b + 1) & 1], nvp, r0, n, lane);
          if (4 * b < nv) tile.rows4(b & 1, 4 * b, nv, p.scale_log2, lane);
        }
      }
      row = row_after;
      nv = nv_after;
      x += W;
    }

    // ---- the warps' states of this segment, joined in warp order
    tile.put(sm_m + warp * HP, sm_l + warp * HP, sm_o + warp * HP * LD, LD, heads, lane);
    __syncthreads();
    const bool whole = seg0 >= t0 && seg1 <= t1;
    float* state = p.partial + ((size_t)blockIdx.x * 2 + (seg0 < t0 ? 0 : 1)) * state_floats;
    for (int e = threadIdx.x; e < heads * (D / 4); e += W * 32) {
      const int h = e / (D / 4), d = (e % (D / 4)) * 4;
      float mm = -INFINITY;
#pragma unroll
      for (int w = 0; w < W; ++w) mm = fmaxf(mm, sm_m[w * HP + h]);
      const float ref = mm == -INFINITY ? 0.f : mm;
      float ll = 0.f;
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < W; ++w) {
        const float f = exp2f(sm_m[w * HP + h] - ref);
        const float4 y = *reinterpret_cast<const float4*>(sm_o + (w * HP + h) * LD + d);
        ll = fmaf(f, sm_l[w * HP + h], ll);
        acc.x = fmaf(f, y.x, acc.x);
        acc.y = fmaf(f, y.y, acc.y);
        acc.z = fmaf(f, y.z, acc.z);
        acc.w = fmaf(f, y.w, acc.w);
      }
      if (whole) {
        const float inv = ll == 0.f ? 0.f : 1.f / ll;
        store4<T>(static_cast<T*>(p.out) + (first_head + h) * D + d, make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv));
        if (p.lse && d == 0) p.lse[first_head + h] = (mm + log2f(ll)) * 0.6931471805599453f;
      } else {
        *reinterpret_cast<float4*>(state + h * D + d) = acc;
        if (d == 0) {
          state[state_heads * D + h] = mm;
          state[state_heads * D + state_heads + h] = ll;
        }
      }
    }
    if (!whole) {
      __threadfence();
      __syncthreads();
      const int c0 = (int)(((seg0 + 1) * C + total - 1) / total - 1), c1 = (int)((seg1 * C + total - 1) / total - 1);
      const int parts = c1 - c0 + 1;
      unsigned int* counter = p.counters + (size_t)seq * H + sh;
      if (threadIdx.x == 0) s_last = atomicAdd(counter, 1u) == (unsigned)(parts - 1);
      __syncthreads();
      if (s_last) {
        __threadfence();
        // state of part y: the first block's segment starts inside it (slot 1) unless it starts exactly at its border too
        auto part_state = [&](int y) {
          const long long b0 = total * (c0 + y) / C;
          return p.partial + ((size_t)(c0 + y) * 2 + (seg0 < b0 ? 0 : 1)) * state_floats;
        };
        float* weight = sm_m;                                  // [parts][heads]
        for (int h = warp; h < heads; h += W) {
          float mm = -INFINITY;
          for (int y = lane; y < parts; y += 32) mm = fmaxf(mm, __ldcg(part_state(y) + state_heads * D + h));
          mm = warp_max(mm);
          const float ref = mm == -INFINITY ? 0.f : mm;
          float ll = 0.f;
          for (int y = lane; y < parts; y += 32) {
            const float* st = part_state(y) + state_heads * D + h;
            const float f = exp2f(__ldcg(st) - ref);
            weight[y * heads + h] = f;
            ll = fmaf(f, __ldcg(st + state_heads), ll);
          }
          ll = warp_sum(ll);
          const float inv = ll == 0.f ? 0.f : 1.f / ll;
          for (int y = lane; y < parts; y += 32) weight[y * heads + h] *= inv;
          if (p.lse && lane == 0) p.lse[first_head + h] = (mm + log2f(ll)) * 0.6931471805599453f;
        }
        __syncthreads();
        for (int e = threadIdx.x; e < heads * (D / 4); e += W * 32) {
          const int h = e / (D / 4), d = (e % (D / 4)) * 4;
          float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
          for (int y = 0; y < parts; ++y) {
            const float4 z = __ldcg(reinterpret_cast<const float4*>(part_state(y) + h * D + d));
            const float f = weight[y * heads + h];
            acc.x = fmaf(f, z.x, acc.x);
            acc.y = fmaf(f, z.y, acc.y);
            acc.z = fmaf(f, z.z, acc.z);
            acc.w = fmaf(f, z.w, acc.w);
          }
          store4<T>(static_cast<T*>(p.out) + (first_head + h) * D + d, acc);
        }
        if (threadIdx.x == 0) *counter = 0u;
      }
    }
    // next segment with tiles
    seg0 = seg1;
    if (++sh == H) {
      sh = 0;
      do ++seq; while (seq < p.n_seqs && pre[seq] == pre[seq + 1]);
    }
    __syncthreads();                                           // the states' shared memory is written again
  }
}

}  // namespace meda
