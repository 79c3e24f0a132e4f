// Attention of one new token per sequence over paged caches of ragged lengths (Eq. 3).
//
// Work split.  All (sequence, KV head, 16-row tile) triples form one list; block c of C takes the c-th equal part of
// it, so a batch of one 128K cache and a batch of 64 very different ones load the GPU alike, without the host
// knowing any length.  Inside a block the warps take tiles in turn.  A segment (sequence, KV head) that lies in one
// block is finished there; the at most two segments of a block that cross its borders leave softmax states (max, sum,
// weighted values) in scratch, and a second, small launch joins the states of a segment in block order: the same bits
// every run.  (Joining them in the block that arrives last cost more: a fence and an atomic of 1.3 us, and then one SM
// reads 37 states of 3.6 KB for each KV head of a long cache in 5 us; the second launch is set up during the first.)
//
// Inner loop, bf16.  One pass over K and V with the running maximum and sum.  A warp's tile goes straight from
// global memory into matrix-instruction fragments: the contraction index of Q K^T may be permuted freely as
// long as Q and K agree, so a lane's 16-byte piece of a key row serves as four fragments; the same holds for the
// value rows with P V written as (V^T)(P^T), where two byte permutes pair neighbouring rows.  So there is no shared
// memory, barrier or bulk copy in the loop; latency is covered by the next tile's loads, issued before this tile's
// arithmetic, in all the warps of an SM.  (A plain stream of such reads reaches 6.3 to 6.5 TB/s here, one through
// cp.async rings 6.0 to 6.3, through tiled or bulk TMA rings 5.3 to 6.1.)  The kernel is bound by reading the cache; the matrix instructions only have
// to keep up (24 to 32 of them for 8 KB at head_dim 128), so the warp-level ones are used: eight query heads fill
// their narrow side, where the tensor-memory instructions would want 128 rows of queries.
// Probabilities enter P V as a sum of two bf16 numbers (2^-16 relative), so that rounding them stays below the rounding
// of the output; logits, maxima, sums and accumulators are fp32.  Both parts of a positive probability are positive: an infinite
// value then adds infinities of one sign (0 * inf and inf - inf are NaN).
//
// Measured with its second launch, calls back to back, 28 query and 4 KV heads of 128, bf16: one cache of 129,072 rows (264 MB) 48.7 us,
// 5.4 TB/s or 84 % of a plain copy, about 7 us of it launches, look-ups and joining; 64 caches of 36 to 18,944 rows (410 MB) 72.8 us,
// 87 %; one of 947 rows 8.2 us, latency alone (7.5 replayed from a graph).  400 MB with 16 heads per KV head: 5.1 TB/s at head_dim 128,
// 4.7 at 64; with 7 heads at head_dim 256 5.0, with 16, which read the cache twice there, 2.7.
//
// fp32 caches: the same walk with the products on the CUDA cores (see DecodeShape in decode.cuh for the reduction), whose
// shuffles bound it from four query heads per KV head on (400 MB of caches, head_dim 128: 5.9 TB/s with one, 4.1 with four, 3.3 with
// seven, 1.7 with sixteen, which read the cache twice).
#pragma once

#include "decode.cuh"        // transpose_reduce
#include "page_rows.cuh"     // load_stream
#include "pages_common.cuh"

namespace meda {

constexpr int kAttTile = 16;             // rows per tile; a page holds whole tiles
// Empty tiles counted with every segment of a batch of sequences: what starting one and joining its warps' states takes,
// in tiles of a block's time.  Without them a block whose share is many short segments works far longer than one inside
// a long one (64 sequences of 36 to 18,944 rows: 96 us; 8 tiles: 87, 12: 80, 20: 71, 28: 72; seven bf16 heads of 128 to a KV head,
// the one shape it was measured on: other tiles take another time each, and would want another number).
constexpr int kAttSegment = 20;
// Tiles per block where the GPU has more blocks than that fills.  One sequence of 947 rows, 4 KV heads, replayed from a graph: 4 tiles
// 7.2 us, 8: 7.6, 16: 9.1; of 4,000 rows: 9.0, 8.5, 9.3.
constexpr int kAttLeast = 8;

// x / d for 0 <= x < 2^31 by a multiplication: with 2^s < d < 2^(s+1), mul = ceil(2^(32+s) / d) is off by less than d / 2^(32+s),
// which x below 2^31 cannot turn into a whole unit; powers of two are shifts.
struct InvariantDiv {
  unsigned mul = 0;
  int shift = 0;
  __host__ void set(unsigned d) {
    shift = 0;
    while ((2ull << shift) <= d) ++shift;                      // floor(log2(d))
    mul = (d & (d - 1)) == 0 ? 0u : (unsigned)(((1ull << (32 + shift)) + d - 1) / d);
  }
  __device__ __forceinline__ int of(int x) const { return (mul ? (int)__umulhi((unsigned)x, mul) : x) >> shift; }
};

struct AttnParams {
  const void* q;
  const void* k;
  const void* v;
  const int32_t* table;
  const int32_t* lens;
  const int32_t* sel;
  void* out;
  float* lse;
  float* partial;                        // [blocks][2] softmax states of segments that cross borders
  int4* split;                           // [blocks]: (blocks, first query head of [n_seqs][n_q_heads], query heads) of the segment that
                                         // starts in the block and goes on behind it; 0 blocks: there is none
  int* status;
  int lens_stride, n_seqs, n_heads, group, n_pages, width, page_shift, keep;
  float scale_log2;                      // log2(e) / sqrt(head_dim)
  InvariantDiv heads_div, grid_div;      // by the segments of a sequence, by the blocks of the launch
};

__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ float exp2_fast(float x) {              // 2^x, off by 2^-22 at most; 0 for x below -126
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// What cutting p to a bf16 leaves; where that is nothing, 2^-126 (0 for p = 0, which exp2_fast gives below 2^-126), far below the
// rounding of a sum whose largest probability is 1.
__device__ __forceinline__ float low_part(float p) {
  const float rest = p - __uint_as_float(__float_as_uint(p) & 0xffff0000u);
  return fmaxf(rest, fminf(p, 1.17549435e-38f));
}

__device__ __forceinline__ uint32_t word_of(const uint4& x, int i) { return i == 0 ? x.x : i == 1 ? x.y : i == 2 ? x.z : x.w; }

// ---- bf16: D = head_dim, NH = groups of eight query heads, R = rows worked on at a time (16 or 8) -----------------
// Lane l: r = l / 4, c = l % 4.  Q K^T has A = queries (row r: head r, row r + 8: head r + 8), B = keys (column r: row r of
// the tile's half); P V has A = V^T, B = P^T (row pairs 2c, 2c + 1 of both halves; column r: head r).  With R = 8
// there is one half: its P V takes both parts of the probabilities in one instruction, the values' fragment twice.
template <int D, int NH, int R = 16>
struct AttnTileBf16 {
  using T = __nv_bfloat16;
  static constexpr int kHeads = 8 * NH;
  static constexpr int KC = D / 32, VC = D / 64, KT = R / 8, kRows = R;
  uint4 q[NH][KC];
  uint4 k[KT][KC];
  uint4 v[2 * KT][VC];
  float o[VC][4][NH][4];
  float m[NH], l[NH];

  __device__ __forceinline__ void load_q(const T* qh, int heads, int lane) {     // qh: the segment's first query head
    const int r = lane / 4, c = lane % 4;
#pragma unroll
    for (int n = 0; n < NH; ++n) {
      const int h = r + 8 * n;
#pragma unroll
      for (int x = 0; x < KC; ++x)
        q[n][x] = h < heads ? *reinterpret_cast<const uint4*>(qh + (size_t)h * D + x * 32 + c * 8) : make_uint4(0, 0, 0, 0);
    }
  }
  __device__ __forceinline__ void reset() {
#pragma unroll
    for (int n = 0; n < NH; ++n) {
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
  // Rows behind the nv that count are not read: their lanes read the last one that does, its logit is set to -inf and its
  // value to 0 (an infinite one times a probability of 0 would be NaN).
  __device__ __forceinline__ void load_k(const T* rows, int r0, int nv, int lane) {
    const int r = lane / 4, c = lane % 4;
#pragma unroll
    for (int t = 0; t < KT; ++t) {
      const T* src = rows + min(r0 + t * 8 + r, nv - 1) * D + c * 8;
#pragma unroll
      for (int x = 0; x < KC; ++x) k[t][x] = load_stream(reinterpret_cast<const uint4*>(src + x * 32));
    }
  }
  __device__ __forceinline__ void load_v(const T* rows, int r0, int nv, int lane) {
    const int r = lane / 4, c = lane % 4;
#pragma unroll
    for (int t = 0; t < 2 * KT; ++t) {
      const T* src = rows + min(r0 + 2 * c + (t & 1) + (t >> 1) * 8, nv - 1) * D + r * 8;
#pragma unroll
      for (int y = 0; y < VC; ++y) v[t][y] = load_stream(reinterpret_cast<const uint4*>(src + y * 64));
    }
  }
  // logits of the rows in k (r0 and on of the tile), in the log2 domain: s[t][0..1] head r, rows t * 8 + 2c, + 1; s[t][2..3] head r + 8
  __device__ __forceinline__ void logits(float (&s)[KT][4], float scale_log2, int r0, int nv, int lane) {
    const int c = lane % 4;
#pragma unroll
    for (int t = 0; t < KT; ++t) {
      float even[4] = {0.f, 0.f, 0.f, 0.f}, odd[4] = {0.f, 0.f, 0.f, 0.f};       // two chains of dependent instructions
#pragma unroll
      for (int x = 0; x < KC; ++x) {
        mma_bf16(even, q[0][x].x, NH > 1 ? q[NH - 1][x].x : 0u, q[0][x].y, NH > 1 ? q[NH - 1][x].y : 0u, k[t][x].x, k[t][x].y);
        mma_bf16(odd, q[0][x].z, NH > 1 ? q[NH - 1][x].z : 0u, q[0][x].w, NH > 1 ? q[NH - 1][x].w : 0u, k[t][x].z, k[t][x].w);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) s[t][e] = (even[e] + odd[e]) * scale_log2;
    }
    if (nv < r0 + R) {
#pragma unroll
      for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (r0 + t * 8 + 2 * c + (e & 1) >= nv) s[t][e] = -INFINITY;
    }
  }
  __device__ __forceinline__ void attend(float (&s)[KT][4], int r0, int nv, int lane) {
    const int c = lane % 4;
    uint32_t hi[NH][KT], lo[NH][KT];
    if (nv < r0 + R) {
#pragma unroll
      for (int t = 0; t < 2 * KT; ++t)
        if (r0 + 2 * c + (t & 1) + (t >> 1) * 8 >= nv)
#pragma unroll
          for (int y = 0; y < VC; ++y) v[t][y] = make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int n = 0; n < NH; ++n) {
      float top = fmaxf(fmaxf(s[0][2 * n], s[0][2 * n + 1]), fmaxf(s[KT - 1][2 * n], s[KT - 1][2 * n + 1]));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const float mn = fmaxf(m[n], top);
      const float ref = mn == -INFINITY ? 0.f : mn;
      if (__any_sync(0xffffffffu, mn > m[n])) {                // the maximum moved: bring the sums to the new one
        const float f = exp2_fast(m[n] - ref);
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
      for (int t = 0; t < KT; ++t) {
        const float p0 = exp2_fast(s[t][2 * n] - ref), p1 = exp2_fast(s[t][2 * n + 1] - ref);
        l[n] += p0 + p1;
        hi[n][t] = __byte_perm(__float_as_uint(p0), __float_as_uint(p1), 0x7632);         // the upper 16 bits: cut, not rounded
        const __nv_bfloat162 l2 = __floats2bfloat162_rn(low_part(p0), low_part(p1));
        memcpy(&lo[n][t], &l2, 4);
      }
    }
#pragma unroll
    for (int y = 0; y < VC; ++y)
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const uint32_t w0 = word_of(v[0][y], x), w1 = word_of(v[1][y], x);
        const uint32_t a0 = __byte_perm(w0, w1, 0x5410), a1 = __byte_perm(w0, w1, 0x7632);
        if constexpr (KT == 2) {
          const uint32_t w2 = word_of(v[2 * KT - 2][y], x), w3 = word_of(v[2 * KT - 1][y], x);
          const uint32_t a2 = __byte_perm(w2, w3, 0x5410), a3 = __byte_perm(w2, w3, 0x7632);
#pragma unroll
          for (int n = 0; n < NH; ++n) {
            mma_bf16(o[y][x][n], a0, a1, a2, a3, hi[n][0], hi[n][KT - 1]);
            mma_bf16(o[y][x][n], a0, a1, a2, a3, lo[n][0], lo[n][KT - 1]);
          }
        } else {                                               // both parts of the probabilities in one: the eight rows twice
#pragma unroll
          for (int n = 0; n < NH; ++n) mma_bf16(o[y][x][n], a0, a1, a0, a1, hi[n][0], lo[n][0]);
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

  __device__ __forceinline__ void load_q(const T* qh, int heads, int lane) {
#pragma unroll
    for (int h = 0; h < GP; ++h)
#pragma unroll
      for (int e = 0; e < E; ++e) q[h][e] = h < heads ? qh[(size_t)h * D + lane * E + e] : 0.f;
  }
  __device__ __forceinline__ void reset() {
#pragma unroll
    for (int h = 0; h < GP; ++h)
#pragma unroll
      for (int e = 0; e < E; ++e) acc[h][e] = 0.f;
    m = -INFINITY;
    l = 0.f;
  }
  // Rows r0 .. r0 + 3 of the tile; behind the last of nv that one again (see AttnTileBf16::load_k; rows4 sets its value to 0).
  __device__ __forceinline__ static void load_rows(float (&x)[B][E], const T* rows, int r0, int nv, int lane) {
#pragma unroll
    for (int b = 0; b < B; ++b) {
      const T* src = rows + min(r0 + b, nv - 1) * D + lane * E;
      if constexpr (E == 2) {
        const float2 t = *reinterpret_cast<const float2*>(src);
        x[b][0] = t.x;
        x[b][1] = t.y;
      } else {
#pragma unroll
        for (int e = 0; e < E; e += 4) {
          const float4 t = *reinterpret_cast<const float4*>(src + e);
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
    if (nv < r0 + B) {
#pragma unroll
      for (int b = 1; b < B; ++b)
        if (r0 + b >= nv)
#pragma unroll
          for (int e = 0; e < E; ++e) vx[cur][b][e] = 0.f;
    }
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
    const float pr = exp2_fast(s - ref), f = exp2_fast(m - ref);
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

// Floats of one softmax state in scratch: values of every head, then (maximum, sum) of every head.
__host__ __device__ inline int attn_state_floats(int heads, int d) { return heads * (d + 4); }
// Shared memory: prefix of tiles and row counts, and two sets of the warps' states.
__host__ __device__ inline int attn_prefix_floats(int n_seqs) { return (2 * n_seqs + 1 + 3) / 4 * 4; }
__host__ __device__ constexpr int attn_merge_floats(int warps, int heads, int d) { return warps * heads * (d + 4 + 2); }

// a / b for 0 <= a < 2^31, b > 0 and a quotient below 2^20: the fp32 estimate is off by one at most.
__device__ __forceinline__ int div_small(int a, int b) {
  float inverse;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inverse) : "f"((float)b));             // off by 2^-23 at most
  int q = (int)((float)a * inverse);
  const int r = a - q * b;
  q -= r < 0;
  q += r >= b;
  return q;
}

template <typename Tile, int D, int W>
__global__ void __launch_bounds__(W * 32, 1)
paged_attention_kernel(AttnParams p) {
  using T = typename Tile::T;
  constexpr bool kBf16 = sizeof(T) == 2;
  constexpr int HP = Tile::kHeads;
  constexpr int LD = D + 4;
  constexpr int kStates = attn_merge_floats(W, HP, D);
  begin_grid();
  extern __shared__ __align__(16) float att_smem[];
  __shared__ int scratch[W + 1];
  int* pre = reinterpret_cast<int*>(att_smem);                 // [n + 1] tiles before sequence i
  int* rows_of = pre + p.n_seqs + 1;                           // [n] rows of sequence i
  float* merge = att_smem + attn_prefix_floats(p.n_seqs);      // two sets of [W][HP] maxima, [W][HP] sums, [W][HP][LD] values
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const int max_rows = p.width << p.page_shift, page_size = 1 << p.page_shift;
  const int tile_shift = p.page_shift - 4;                     // log2(tiles per page)
  const int chunks = (p.group + HP - 1) / HP;                  // segments per KV head
  const int H = p.n_heads * chunks;
  const int state_heads = min(p.group, HP);
  const int state_floats = attn_state_floats(state_heads, D);
  const int n_q_heads = p.n_heads * p.group;
  const int gap = p.n_seqs > 1 ? kAttSegment : 0;

  ragged_prefix<W * 32>(p.n_seqs, pre, scratch, [&](int i) {
    bool bad = false;
    const int len = clamped_len(p.lens, p.lens_stride, i, max_rows, bad);
    if (bad && blockIdx.x == 0) set_status(p.status, MEDA_ERR_INVALID_ARG);
    rows_of[i] = len;
    const int tiles = p.sel ? min(p.keep, (len + page_size - 1) >> p.page_shift) << tile_shift : (len + kAttTile - 1) / kAttTile;
    return tiles ? tiles + gap : 0;
  });

  // (All tile counts stay below 2^31: see meda_pages_create.)
  const int total = pre[p.n_seqs] * H;
  // Blocks with work: as many to a segment as give each kAttLeast tiles on average, so that segments of one length are cut
  // alike and no block works on two of them needlessly.  Block b's first tile is b / C of the total, rounded down.
  const int most = max(p.n_seqs * H, 1), each = most * kAttLeast;
  const int C = total == 0 ? 0 : min((int)gridDim.x, total <= (long long)each * gridDim.x ? most * (div_small(total - 1, each) + 1) : (int)gridDim.x);
  const int base = C == (int)gridDim.x ? p.grid_div.of(total) : (C > 0 ? div_small(total, C) : 0), extra = total - base * C;
  auto block_start = [&](int b) { return base * b + div_small(extra * b, C); };
  auto block_of = [&](int x) {
    int b = min((int)((float)x * ((float)C / (float)total)), C - 1);
    while (block_start(b) > x) --b;
    while (b + 1 < C && block_start(b + 1) <= x) ++b;
    return b;
  };
  const bool has_work = (int)blockIdx.x < C;
  const int t0 = has_work ? block_start(blockIdx.x) : 0, t1 = has_work ? block_start(blockIdx.x + 1) : 0;

  // a tile's first row in the pools and the number of its rows that count (0: nothing to read)
  auto lookup = [&](int x, long long& row, int& nv) {
    row = 0;
    nv = 0;
    if (x >= t1) return;
    const int i = ragged_find(pre, p.n_seqs, p.heads_div.of(x));
    const int tiles = pre[i + 1] - pre[i];
    const int local = x - pre[i] * H;
    const int sh = div_small(local, tiles), tile = local - sh * tiles, g = chunks == 1 ? sh : sh / chunks;
    if (tile >= tiles - gap) return;
    const int len = rows_of[i];
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

  int seq = 0, sh = 0, seg0 = 0;
  auto next_segment = [&] {                                    // the next one with tiles
    seg0 += pre[seq + 1] - pre[seq];
    if (++sh == H) {
      sh = 0;
#pragma unroll 1
      do ++seq; while (seq < p.n_seqs && pre[seq] == pre[seq + 1]);
    }
  };
  if (has_work) {
    seq = ragged_find(pre, p.n_seqs, p.heads_div.of(t0));
    const int tiles = pre[seq + 1] - pre[seq];
    sh = div_small(t0 - pre[seq] * H, tiles);
    seg0 = pre[seq] * H + sh * tiles;
    if (t0 >= seg0 + tiles - gap) next_segment();      // nothing but empty tiles of it here
  }
  const T* kp = static_cast<const T*>(p.k);
  const T* vp = static_cast<const T*>(p.v);
  Tile tile;
  auto load_q = [&] {
    const int g = chunks == 1 ? sh : sh / chunks, h0 = (sh - g * chunks) * HP;
    tile.load_q(static_cast<const T*>(p.q) + ((size_t)seq * n_q_heads + (size_t)g * p.group + h0) * D, min(HP, p.group - h0), lane);
  };
  if (seg0 < t1) load_q();                                     // (a block may hold nothing but the last segment's empty tiles)
  tile.reset();

  // One iteration works on tile x, whose keys and values are in registers, and fetches tile x + W; the first one only
  // fetches.  Lane y holds the look-up of tile y of the 32 the warp is going through; the next 32 are looked up half
  // way through them.
  int x = t0 + warp - W, at = -1, buffer = 0, nv = 0;
  long long row = 0, row_now = 0, row_next = 0;
  int nv_now = 0, nv_next = 0;
  bool worked = false;
  int4 split = make_int4(0, 0, 0, 0);
#pragma unroll 1
  while (seg0 < t1) {
    ++at;
    if (at == 32) {
      row_now = row_next;
      nv_now = nv_next;
      at = 0;
    }
    if (at == 16 || x < t0) {
      lookup(x + (at == 16 ? 17 : 1) * W + lane * W, row_next, nv_next);
      if (at != 16) {
        row_now = row_next;
        nv_now = nv_next;
      }
    }
    const long long row_after = __shfl_sync(0xffffffffu, row_now, at);
    const int nv_after = __shfl_sync(0xffffffffu, nv_now, at);
    if constexpr (kBf16) {
      constexpr int R = Tile::kRows;
#pragma unroll
      for (int b = 0; b < kAttTile; b += R) {
        float s[R / 8][4];
        const bool last = b + R == kAttTile;                   // of this tile; then comes the next one's first
        const int n = last ? nv_after : nv, r0 = last ? 0 : b + R;
        if (b < nv) tile.logits(s, p.scale_log2, b, nv, lane);
        if (r0 < n) tile.load_k(kp + (last ? row_after : row) * D, r0, n, lane);
        if (b < nv) tile.attend(s, b, nv, lane);
        if (r0 < n) tile.load_v(vp + (last ? row_after : row) * D, r0, n, lane);
      }
    } else {
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const int r0 = b < 3 ? 4 * (b + 1) : 0, n = b < 3 ? nv : nv_after;
        if (r0 < n) {
          tile.load_rows(tile.kx[(b + 1) & 1], kp + (b < 3 ? row : row_after) * D, r0, n, lane);
          tile.load_rows(tile.vx[(b + 1) & 1], vp + (b < 3 ? row : row_after) * D, r0, n, lane);
        }
        if (4 * b < nv) tile.rows4(b & 1, 4 * b, nv, p.scale_log2, lane);
      }
    }
    worked |= x >= t0;
    row = row_after;
    nv = nv_after;
    x += W;

    // (empty tiles do not count, so a border among them splits nothing)
#pragma unroll 1
    while (seg0 < t1 && x >= min(seg0 + pre[seq + 1] - pre[seq] - gap, t1)) {
      const int seg1 = seg0 + pre[seq + 1] - pre[seq] - gap, was_seg0 = seg0;
      const int g = chunks == 1 ? sh : sh / chunks, h0 = (sh - g * chunks) * HP;
      const int heads = min(HP, p.group - h0);
      const size_t first_head = (size_t)seq * n_q_heads + (size_t)g * p.group + h0;
      next_segment();                                          // its queries can come already
      if (seg0 < t1) load_q();

      // ---- the warps' states of this segment, joined in warp order.  The buffers alternate, so that one barrier per
      // segment is enough.  A warp without tiles leaves a maximum of -inf, a sum of 0 and no values; nobody reads those.
      float* sm_m = merge + buffer * kStates;
      float* sm_l = sm_m + W * HP;
      float* sm_o = sm_l + W * HP;
      buffer ^= 1;
      if (worked) tile.put(sm_m + warp * HP, sm_l + warp * HP, sm_o + warp * HP * LD, LD, heads, lane);
      else if (lane < HP) {
        sm_m[warp * HP + lane] = -INFINITY;
        sm_l[warp * HP + lane] = 0.f;
      }
      __syncthreads();
      tile.reset();
      const bool whole = was_seg0 >= t0 && seg1 <= t1;
      const int slot = was_seg0 < t0 ? 0 : 1;
      float* state = p.partial + ((size_t)blockIdx.x * 2 + slot) * state_floats;
#pragma unroll 1
      for (int e = threadIdx.x; e < heads * (D / 4); e += W * 32) {
        const int h = e / (D / 4), d = (e % (D / 4)) * 4;
        float mm = -INFINITY;
#pragma unroll
        for (int w = 0; w < W; ++w) mm = fmaxf(mm, sm_m[w * HP + h]);
        float ll = 0.f;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int w = 0; w < W; ++w) {
          const float mw = sm_m[w * HP + h], lw = sm_l[w * HP + h];
          if (mw != -INFINITY || lw != 0.f) {                    // (a sum that is NaN has a maximum of -inf when all logits are)
            const float f = exp2_fast(mw - mm);
            const float4 y = *reinterpret_cast<const float4*>(sm_o + (w * HP + h) * LD + d);
            ll = fmaf(f, lw, ll);
            acc.x = fmaf(f, y.x, acc.x);
            acc.y = fmaf(f, y.y, acc.y);
            acc.z = fmaf(f, y.z, acc.z);
            acc.w = fmaf(f, y.w, acc.w);
          }
        }
        if (whole) {
          const float inv = ll == 0.f ? 0.f : 1.f / ll;
          store4<T>(static_cast<T*>(p.out) + (first_head + h) * D + d, make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv));
          if (p.lse && d == 0) p.lse[first_head + h] = (mm + log2f(ll)) * 0.6931471805599453f;
        } else {
          *reinterpret_cast<float4*>(state + h * D + d) = acc;
          if (d == 0) *reinterpret_cast<float2*>(state + state_heads * D + 2 * h) = make_float2(mm, ll);
        }
      }
      if (was_seg0 >= t0 && seg1 > t1) split = make_int4(block_of(seg1 - 1) - (int)blockIdx.x + 1, (int)first_head, heads, 0);
      worked = false;
    }
  }

  // sequences without rows
#pragma unroll 1
  for (int i = blockIdx.x; i < p.n_seqs; i += gridDim.x)
    if (pre[i] == pre[i + 1]) {
#pragma unroll 1
      for (int e = threadIdx.x; e < n_q_heads * D / 4; e += W * 32)
        store4<T>(static_cast<T*>(p.out) + (size_t)i * n_q_heads * D + e * 4, make_float4(0.f, 0.f, 0.f, 0.f));
      if (p.lse)
#pragma unroll 1
        for (int h = threadIdx.x; h < n_q_heads; h += W * 32) p.lse[(size_t)i * n_q_heads + h] = -INFINITY;
    }

  if (threadIdx.x == 0) p.split[blockIdx.x] = split;
}

// Joins the states of the segment that starts in block blockIdx.x of the launch above, for query head blockIdx.y of it.  Groups
// of D / 4 threads take every n-th state, four at a time in flight; their results are added in a fixed order.
constexpr int kAttJoinThreads = 128;

template <typename T, int D>
__global__ void __launch_bounds__(kAttJoinThreads)
join_attention_kernel(AttnParams p) {
  constexpr int kGroup = D / 4, kGroups = kAttJoinThreads / kGroup, kBatch = 4;
  __shared__ float4 s_o[kGroups][kGroup];
  __shared__ float2 s_ml[kGroups];
  begin_grid();
  const int4 split = p.split[blockIdx.x];
  const int parts = split.x, h = blockIdx.y;
  if (parts == 0 || h >= split.z) return;
  const int group = threadIdx.x / kGroup, d = threadIdx.x % kGroup;
  const int state_heads = gridDim.y, state_floats = attn_state_floats(state_heads, D);
  // the segment begins inside its first block (slot 1) and before all others (slot 0)
  auto state_of = [&](int z) { return p.partial + ((size_t)(blockIdx.x + z) * 2 + (z == 0)) * state_floats; };
  float mm = -INFINITY, ll = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  auto add = [&](float2 ml, float4 o) {
    const float mn = fmaxf(mm, ml.x), ref = mn == -INFINITY ? 0.f : mn;
    const float f0 = exp2_fast(mm - ref), f = exp2_fast(ml.x - ref);
    mm = mn;
    ll = fmaf(f, ml.y, ll * f0);
    acc.x = fmaf(f, o.x, acc.x * f0);
    acc.y = fmaf(f, o.y, acc.y * f0);
    acc.z = fmaf(f, o.z, acc.z * f0);
    acc.w = fmaf(f, o.w, acc.w * f0);
  };
#pragma unroll 1
  for (int z0 = group; z0 < parts; z0 += kGroups * kBatch) {
    float2 ml[kBatch];
    float4 o[kBatch];
#pragma unroll
    for (int y = 0; y < kBatch; ++y) {
      const float* st = state_of(min(z0 + y * kGroups, parts - 1));
      ml[y] = *reinterpret_cast<const float2*>(st + state_heads * D + 2 * h);
      o[y] = *reinterpret_cast<const float4*>(st + h * D + d * 4);
    }
#pragma unroll
    for (int y = 0; y < kBatch; ++y)
      if (z0 + y * kGroups < parts) add(ml[y], o[y]);
  }
  s_o[group][d] = acc;
  if (d == 0) s_ml[group] = make_float2(mm, ll);
  __syncthreads();
  if (group != 0) return;
#pragma unroll
  for (int y = 1; y < kGroups; ++y)
    if (y < parts) add(s_ml[y], s_o[y][d]);
  const float inv = ll == 0.f ? 0.f : 1.f / ll;
  store4<T>(static_cast<T*>(p.out) + ((size_t)split.y + h) * D + d * 4, make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv));
  if (p.lse && d == 0) p.lse[split.y + h] = (mm + log2f(ll)) * 0.6931471805599453f;
}

}  // namespace meda
