// Attention of one new token per sequence over quantised pages: the work split, the states and their joining are paged_attention.cuh's.
//
// A row's logit is the sum over its groups of step_g (q_g . codes_g) + low_g sum(q_g), an output the sum over the rows of
// (p step_g) codes_g + p low_g.  So the matrix instructions multiply by the codes themselves, and a code is its own fp16 operand: the whole
// number c in the lower bits of a half is the subnormal c 2^-24, exact, and needs no conversion, offset or scale, only a mask
// (and at 4 bits c << 4, a nibble further up, is 16 c 2^-24: the factor goes into the queries and out of the result).  Steps, lowest
// values, logits, maxima and sums are fp32.
//
// The matrix instructions cut off what a product's sum has below its largest term, and take a subnormal for as large as the smallest
// normal number: with codes as they are a logit is off by some 2^-20 of its products' sum.  In bf16 that is far below the output's own
// rounding; for fp32 outputs (2e-6 to 5e-6 over 30,000 rows) it is not.  There codes become normal numbers (one more instruction for two), the
// low parts of queries add up by themselves, and a run's values are added to the sums outside: 6.5e-7 to 1.0e-6, at 443 MB 111 -> 146 us then.
//
// Fragments, lane l: r = l / 4, c = l % 4.  Q K^T has A = codes of the keys (rows r and r + 8 of the tile), B = queries (column r: head r),
// group by group; sum(q) low is one instruction of bf16, the sums in three parts.  P V has A = codes of the values, transposed
// (rows are dimensions; a byte permute pairs the codes of neighbouring cache rows), B = (p step_g)^T, from the logits' layout by an 8 x 8
// transposition per group.  Columns are heads on both sides, so a lane's maxima, sums and results belong to the same two heads.
//
// Roundings.  Queries are scaled by a power of two per head, their largest element between 2^14 and 2^15 (fp32: 2^5 and 2^6).  fp16 then holds a bf16
// element exactly down to 2^-31 of the largest and cuts smaller ones off at 2^-39 of it (at 4 bits half of them carry the nibble's 1/16: 2^-27 and 2^-35); fp32
// ones go in two parts, 22 bits.  A weight p step is rounded to fp16, 2^-11 of itself, for fp32 outputs to two such parts, 2^-22; caches of 16 bits
// have theirs in two parts of bf16, which here costs 15 % (443 MB at 4 bits 86 -> 99 us).  The error goes with the codes' part of the sum, which lies within
// the values' range and averages out over the rows: the outputs' error against 64 bits is that of a computation in fp32, 0.0017 (the type's own), and
// one to three in a hundred come out as the neighbouring number.  Weights are scaled by a power of two for every head and group, which goes by the weights
// met (p step, not the step alone: a row with huge values and no weight takes nothing from the others): see settle().
// The reference of the exponentials is set 2^8 above the largest logit met (fp32: 2^6) and moves when one passes it: bringing the sums to a new one
// costs as much as a tile or two (with none at all in fp32 144 -> 155 us, at head_dim 256 151 -> 174).  No weight is ever above 1, so the sums reach no
// further than values times rows.
//
// Bound by issue slots beside memory: a 4-bit tile of 32 rows at head_dim 128 is 4.6 KB, 200 cycles of an SM's share of memory.  64 caches of 12,000
// rows, 28 / 4 heads of 128, 443 MB: 85 us, 79 % of a plain copy (the same copies without arithmetic 76.7); at 8 bits, 418 MB: 73 us, 87 %;
// ten of up to 32,768 rows, 32 heads, 765 MB: 122 to 134 us, 87 to 95 %; 192 of 36 to 18,944 rows, 342 MB: 73 to 82 us, 64 to 72 %; one of
// 129,072 rows, 74 MB: 26 us, 44 % (copies alone 22.5); one of 947 rows 8.9 us, more than the same rows in 16 bits take (8.2).
#pragma once

#include <cuda_fp16.h>

#include "page_codes.cuh"
#include "paged_attention.cuh"   // the walk's numbers, exp2_fast, store4, the states' layout
#include "sm100_primitives.cuh"

namespace meda {

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The first products of a sum: d is written, not added to.
__device__ __forceinline__ void mma_f16_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ void mma_bf16_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
// The transpose of the 8 x 8 matrix of halves whose row l / 4, columns 2 (l % 4) and + 1 lane l holds.
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint32_t halves(float lo, float hi) {           // two fp16, rounded to nearest
  uint32_t y;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(y) : "f"(hi), "f"(lo));
  return y;
}
__device__ __forceinline__ float half_low(uint32_t x) { return __half2float(__ushort_as_half((unsigned short)(x & 0xffffu))); }
__device__ __forceinline__ float half_high(uint32_t x) { return __half2float(__ushort_as_half((unsigned short)(x >> 16))); }
// (bf16(lo), bf16(hi)), and what is left of both
__device__ __forceinline__ uint32_t bf16_part(float& lo, float& hi) {
  const __nv_bfloat162 x = __floats2bfloat162_rn(lo, hi);
  lo -= __bfloat162float(x.x);
  hi -= __bfloat162float(x.y);
  uint32_t y;
  memcpy(&y, &x, 4);
  return y;
}
// (a c, b d) in one instruction, which may be put together with a sum behind it, into one rounding.
__device__ __forceinline__ void mul2(float& x, float& y, float a, float b, float c, float d) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(pair(a, b)), "l"(pair(c, d)));
  unpair(r, x, y);
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }    // -126 <= e <= 127

template <int N>
__device__ __forceinline__ void shared_words(uint32_t (&w)[N], const unsigned char* p) {
  static_assert(N == 1 || N == 2 || N == 4, "one load");
  if constexpr (N == 1) {
    w[0] = *reinterpret_cast<const uint32_t*>(p);
  } else if constexpr (N == 2) {
    const uint2 x = *reinterpret_cast<const uint2*>(p);
    w[0] = x.x;
    w[1] = x.y;
  } else {
    const uint4 x = *reinterpret_cast<const uint4*>(p);
    w[0] = x.x;
    w[1] = x.y;
    w[2] = x.z;
    w[3] = x.w;
  }
}
template <int N>
__device__ __forceinline__ void shared_piece(uint32_t (&w)[N], int i, const unsigned char* p) {
  const uint4 x = *reinterpret_cast<const uint4*>(p);
  w[i] = x.x;
  w[i + 1] = x.y;
  w[i + 2] = x.z;
  w[i + 3] = x.w;
}
// 16 bytes from global to shared memory behind the thread's back.
__device__ __forceinline__ void copy16(uint32_t to, const unsigned char* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
// In a branch that is hardly ever taken: it stays one (selects in its place would cost every tile).
__device__ __forceinline__ void keep_branch() { asm volatile(""); }

// T = type of queries and outputs, D = head_dim, NH = groups of eight query heads, SUB = runs of sixteen rows in a tile (each lies in one page).
template <typename TOUT, int D, int NH, int BITS, int SUBS>
struct AttnTileCoded {
  using T = TOUT;
  using Row = CodedRow<D, BITS>;
  static constexpr int SUB = SUBS;
  static constexpr int kHeads = 8 * NH;
  static constexpr int G = Row::kGroups, W = BITS / 4;           // groups, words per unit
  static constexpr int kRunCodes = 16 * Row::kCodes, kRunMore = 16 * Row::kMore;
  static constexpr int kHalf = kRunCodes + kRunMore;             // bytes of a run's keys or values
  static constexpr int kStage = 2 * SUB * kHalf;                 // of a tile: keys and values of every run
  static constexpr int PARTS = sizeof(T) == 4 ? 2 : 1;           // fp16 parts of a query element and of a weight
  static constexpr float kMostQuery = 1.2980742e33f;             // 2^110: `factor` and its inverse stay in fp32's range
  static constexpr int kMostScale = 126;
  static constexpr float kSlack = PARTS == 2 ? 6.f : 8.f;        // the reference is put this far (log2) above the maximum

  uint32_t q[NH][PARTS][2][G][4];        // unit 2c + i of group g: the four pairs that go with pair_of()
  uint32_t qsum[NH][2];                  // sums over the groups, in bf16 parts
  float factor[NH][2];                   // from products of codes and scaled queries to logits (log2), of the lane's two heads
  float o[G][4][NH][4];
  float low_sum[NH][2][G];               // sum of p low
  float l[NH][2];                        // sum of p = 2^(logit - reference)
  float ref[NH][2];                      // reference: no logit so far is above it (-inf: there is none yet)
  float scale[NH][2][G];                 // of the weights in o, a power of two: p step scale is 2^15 at most for the tile at hand

  // Two codes in the lower bits of a word's halves as an operand: as they are, c 2^-24, or for fp32 as normal numbers c 2^-14 ((1024 + c) 2^-14 - 2^-4).
  // A sum of products is multiplied by its step before `factor` takes the scale of queries and codes out again; the two keep it below fp32's end for
  // keys of up to 2^126: 4 groups of 64 products of 2^(kQueryTop + 1) with 3 2^126 (codes' part and lowest values) times kCodeScale.
  static constexpr float kCodeScale = PARTS == 2 ? 6.103515625e-5f : 5.9604644775390625e-8f;
  static constexpr int kQueryTop = PARTS == 2 ? 5 : 14;          // log2 of a head's largest query element as the operands have it, rounded down
  __device__ __forceinline__ static uint32_t operand(uint32_t codes) {
    if constexpr (PARTS == 1) return codes;
    const uint32_t x = codes | 0x64006400u;
    __half2 a;
    memcpy(&a, &x, 4);
    a = __hfma2(a, __float2half2_rn(kCodeScale), __float2half2_rn(-0.0625f));
    uint32_t y;
    memcpy(&y, &a, 4);
    return y;
  }
  // Pair j of a unit's eight codes, as the two halves of a word: elements (first, second).
  __device__ __forceinline__ static constexpr int pair_first(int j) { return BITS == 4 ? j : (j / 2) * 4 + j % 2; }
  __device__ __forceinline__ static constexpr int pair_second(int j) { return BITS == 4 ? j + 4 : (j / 2) * 4 + j % 2 + 2; }
  __device__ __forceinline__ static constexpr float pair_factor(int j) { return BITS == 4 && j % 2 == 1 ? 0.0625f : 1.f; }
  __device__ __forceinline__ static uint32_t pair_of(const uint32_t* unit, int j) {
    if constexpr (BITS == 4) return operand((j < 2 ? unit[0] : unit[0] >> 8) & (j % 2 ? 0x00f000f0u : 0x000f000fu));
    else return operand((j % 2 ? unit[j / 2] >> 8 : unit[j / 2]) & 0x00ff00ffu);
  }
  __device__ __forceinline__ static float step_of(const uint32_t (&w)[G], int g) {
    return __uint_as_float(g % 2 == 0 ? w[g / 2] << 16 : w[g / 2] & 0xffff0000u);
  }
  __device__ __forceinline__ static float low_of(const uint32_t (&w)[G], int g) {
    if constexpr (G == 1) return __uint_as_float(w[0] & 0xffff0000u);
    else return __uint_as_float(g % 2 == 0 ? w[G / 2 + g / 2] << 16 : w[G / 2 + g / 2] & 0xffff0000u);
  }

  __device__ __forceinline__ void load_q(const T* qh, int heads, float scale_log2, int lane) {     // qh: the segment's first query head
    const int r = lane / 4, c = lane % 4;
#pragma unroll
    for (int n = 0; n < NH; ++n) {
      const int h = r + 8 * n;
      float x[2][G][8], top = 0.f;
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int g = 0; g < G; ++g) {
          Eight<T> w;
          w.load(qh + (h < heads ? h : 0) * D + g * 64 + (2 * c + i) * 8);
          w.floats(x[i][g]);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            if (h >= heads) x[i][g][e] = 0.f;
            top = fmaxf(top, fabsf(x[i][g][e]));
          }
        }
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const int k2 = min(126, kQueryTop - ((int)(__float_as_uint(top) >> 23) - 127));
      const float scale = top < kMostQuery ? power_of_two(k2) : NAN;             // a query that is not finite, or huge, makes its logits NaN
      float sum[G];
#pragma unroll
      for (int g = 0; g < G; ++g) sum[g] = 0.f;
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float a = x[i][g][pair_first(j)] * scale, b = x[i][g][pair_second(j)] * scale;
            sum[g] += a + b;
            const float f = pair_factor(j);
            q[n][0][i][g][j] = halves(a * f, b * f);
            if constexpr (PARTS == 2)
              q[n][PARTS - 1][i][g][j] = halves(a * f - half_low(q[n][0][i][g][j]), b * f - half_high(q[n][0][i][g][j]));
          }
#pragma unroll
      for (int g = 0; g < G; ++g) {
        sum[g] += __shfl_xor_sync(0xffffffffu, sum[g], 1);
        sum[g] += __shfl_xor_sync(0xffffffffu, sum[g], 2);
        sum[g] *= kCodeScale;                                                    // as the products with codes have it
      }
      // A has the lowest values twice (G <= 2) or two pairs of them (G = 4) in every lane's columns; B the parts, one after the other
      if constexpr (G == 4) {
        float a = sum[0], b = sum[1], d = sum[G - 2], e = sum[G - 1];
        qsum[n][0] = bf16_part(a, b);
        qsum[n][1] = bf16_part(d, e);
        for (int part = 1; part < 4; ++part) {
          const uint32_t x0 = part < 3 ? bf16_part(a, b) : 0u, x1 = part < 3 ? bf16_part(d, e) : 0u;
          if (c == part) {
            qsum[n][0] = x0;
            qsum[n][1] = x1;
          }
        }
      } else {
        float a = G == 1 ? 0.f : sum[0], b = sum[G - 1];
        const uint32_t hi = bf16_part(a, b), mid = bf16_part(a, b), lo = bf16_part(a, b);
        qsum[n][0] = c == 0 ? hi : c == 1 ? lo : 0u;
        qsum[n][1] = c == 0 ? mid : 0u;
      }
      const float back = scale == scale ? power_of_two(-k2) * (scale_log2 / kCodeScale) : NAN;
      factor[n][0] = __shfl_sync(0xffffffffu, back, 8 * c);                      // head 2c is lane 4 * 2c's
      factor[n][1] = __shfl_sync(0xffffffffu, back, 8 * c + 4);
    }
  }
  __device__ __forceinline__ void reset() {
#pragma unroll
    for (int n = 0; n < NH; ++n)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        ref[n][x] = -INFINITY;
        l[n][x] = 0.f;
#pragma unroll
        for (int g = 0; g < G; ++g) {
          low_sum[n][x][g] = 0.f;
          scale[n][x][g] = power_of_two(kMostScale);
        }
      }
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int n = 0; n < NH; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[g][t][n][e] = 0.f;
  }
  // A run of rows in shared memory: 16-byte pieces of its codes, then its steps and lowest values.  The pieces are moved inside
  // a row, and the values' rows are sorted even ones first in each eight, so that the lanes that read together meet different banks.
  static constexpr int kPieces = Row::kCodes / 16;               // of a row
  static constexpr int kKeyBytes = 2 * G * BITS, kValueBytes = G * BITS;         // a lane reads of a row
  __device__ __forceinline__ static int key_piece(int row, int piece) {
    const int moved = kKeyBytes == 32 ? row & 1 : kKeyBytes == 64 ? (row & 1) << 1 | (piece >> 3 & 1) : 0;
    return row * kPieces + (piece ^ moved);
  }
  __device__ __forceinline__ static int value_piece(int row, int piece) {
    const int at = (row & 8) | (row & 1) << 2 | (row >> 1 & 3);
    const int moved = kValueBytes == 8 ? at & 2 : kValueBytes == 16 ? (at & 3) << 1 : kValueBytes == 32 ? (at & 1) | (at & 2) << 1 : 0;
    return at * kPieces + (piece ^ moved);
  }

  // Logits over `factor` of the run of keys at `stage`: s[n][0..1] row r, heads 2c, 2c + 1 (+ 8 n); s[n][2..3] row r + 8.
  __device__ __forceinline__ void logits(float (&s)[NH][4], const unsigned char* stage, int lane) {
    const int r = lane / 4, c = lane % 4;
    uint32_t k[2][2 * G * W], km[2][G];                        // rows r, r + 8: codes of units 2c, 2c + 1; steps and lowest values
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      if constexpr (kKeyBytes == 8) shared_words(k[t], stage + (r + 8 * t) * Row::kCodes + c * 8);
      else
#pragma unroll
        for (int x = 0; x < kKeyBytes / 16; ++x)
          shared_piece(k[t], 4 * x, stage + 8 * t * Row::kCodes + 16 * key_piece(r, c * (kKeyBytes / 16) + x));
      shared_words(km[t], stage + kRunCodes + (r + 8 * t) * Row::kMore);
    }
#pragma unroll
    for (int n = 0; n < NH; ++n) {
      constexpr int L0 = G / 2, L1 = G == 4 ? G / 2 + 1 : G / 2;                 // the words of the lowest values
      mma_bf16_first(s[n], km[0][L0], km[1][L0], km[0][L1], km[1][L1], qsum[n][0], qsum[n][1]);
    }
#pragma unroll
    for (int g = 0; g < G; ++g) {
      float acc[NH][4], low_parts[NH][4];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t *u0 = &k[0][(i * G + g) * W], *u1 = &k[1][(i * G + g) * W];
#pragma unroll
        for (int j = 0; j < 4; j += 2) {
          const uint32_t a0 = pair_of(u0, j), a1 = pair_of(u1, j), a2 = pair_of(u0, j + 1), a3 = pair_of(u1, j + 1);
          const bool first = i == 0 && j == 0;
#pragma unroll
          for (int n = 0; n < NH; ++n) {
            if (first) mma_f16_first(acc[n], a0, a1, a2, a3, q[n][0][i][g][j], q[n][0][i][g][j + 1]);
            else mma_f16(acc[n], a0, a1, a2, a3, q[n][0][i][g][j], q[n][0][i][g][j + 1]);
            if constexpr (PARTS == 2) {                        // a sum by itself
              if (first) mma_f16_first(low_parts[n], a0, a1, a2, a3, q[n][PARTS - 1][i][g][j], q[n][PARTS - 1][i][g][j + 1]);
              else mma_f16(low_parts[n], a0, a1, a2, a3, q[n][PARTS - 1][i][g][j], q[n][PARTS - 1][i][g][j + 1]);
            }
          }
        }
      }
      if constexpr (PARTS == 2)
#pragma unroll
        for (int n = 0; n < NH; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[n][e] += low_parts[n][e];
      const float s0 = step_of(km[0], g), s1 = step_of(km[1], g);
#pragma unroll
      for (int n = 0; n < NH; ++n) {
        s[n][0] = fmaf(s0, acc[n][0], s[n][0]);
        s[n][1] = fmaf(s0, acc[n][1], s[n][1]);
        s[n][2] = fmaf(s1, acc[n][2], s[n][2]);
        s[n][3] = fmaf(s1, acc[n][3], s[n][3]);
      }
    }
  }
  // The tile at `stage`; `rows`: how many rows of each run count, five bits each, the last run's lowest.
  static constexpr unsigned kFull = SUB == 2 ? 16 << 5 | 16 : 16;
  __device__ __forceinline__ void work(const unsigned char* stage, unsigned rows, int lane) {
    const int r = lane / 4;
    float s[SUB][NH][4];
#pragma unroll
    for (int u = 0; u < SUB; ++u) {
      logits(s[u], stage + 2 * u * kHalf, lane);
      // Rounded here, once: the reference goes by one of these numbers, and its own row's weight is what kSlack makes it.  (Were the product formed with the
      // exponential's subtraction, unrounded, that weight would be off by 2 to the power of what rounding had cut off: too large for fp16 from 5e7 on.)
#pragma unroll
      for (int n = 0; n < NH; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[u][n][e] = __fmul_rn(s[u][n][e], factor[n][e & 1]);
    }
    uint32_t vm[SUB][2][G];                                    // steps and lowest values of the values' rows r, r + 8
#pragma unroll
    for (int u = 0; u < SUB; ++u)
#pragma unroll
      for (int t = 0; t < 2; ++t) shared_words(vm[u][t], stage + (2 * u + 1) * kHalf + kRunCodes + (r + 8 * t) * Row::kMore);
    if (rows != kFull) {                                       // rows that do not count: logits of -inf, and 0 for the weight of 0 to meet
      keep_branch();
#pragma unroll
      for (int u = 0; u < SUB; ++u)
#pragma unroll
        for (int t = 0; t < 2; ++t)
          if (r + 8 * t >= (int)(rows >> 5 * (SUB - 1 - u) & 31)) {
#pragma unroll
            for (int n = 0; n < NH; ++n) s[u][n][2 * t] = s[u][n][2 * t + 1] = -INFINITY;
#pragma unroll
            for (int g = 0; g < G; ++g) vm[u][t][g] = 0u;
          }
    }
    bool unsettled = false;                                    // a logit above its reference, or a step whose row could weigh too much for fp16
#pragma unroll
    for (int n = 0; n < NH; ++n)
#pragma unroll
      for (int x = 0; x < 2; ++x) unsettled |= largest(s, n, x) > ref[n][x];
#pragma unroll
    for (int g = 0; g < G; ++g) {
      float most = scale[0][0][g];
#pragma unroll
      for (int n = 0; n < NH; ++n) most = fmaxf(most, fmaxf(scale[n][0][g], scale[n][1][g]));
      unsettled |= largest_step(vm, g) * most > 32768.f;
    }
    if (__any_sync(0xffffffffu, unsettled)) settle(s, vm);
#pragma unroll
    for (int u = 0; u < SUB; ++u)
#pragma unroll
      for (int n = 0; n < NH; ++n) {
        float (&p)[4] = s[u][n];
#pragma unroll
        for (int e = 0; e < 4; ++e) p[e] = exp2_fast(p[e] - ref[n][e & 1]);
        l[n][0] += p[0] + p[2];
        l[n][1] += p[1] + p[3];
#pragma unroll
        for (int g = 0; g < G; ++g) {
          const float low0 = low_of(vm[u][0], g), low1 = low_of(vm[u][1], g);
#pragma unroll
          for (int x = 0; x < 2; ++x) low_sum[n][x][g] = fmaf(p[2 + x], low1, fmaf(p[x], low0, low_sum[n][x][g]));
        }
      }
#pragma unroll
    for (int u = 0; u < SUB; ++u) attend(s[u], vm[u], stage + (2 * u + 1) * kHalf, lane);
  }
  __device__ __forceinline__ static float largest(const float (&s)[SUB][NH][4], int n, int x) {
    float most = fmaxf(s[0][n][x], s[0][n][2 + x]);
    if (SUB == 2) most = fmaxf(most, fmaxf(s[SUB - 1][n][x], s[SUB - 1][n][2 + x]));
    return most;
  }
  __device__ __forceinline__ static float largest_step(const uint32_t (&vm)[SUB][2][G], int g) {
    float most = fmaxf(step_of(vm[0][0], g), step_of(vm[0][1], g));
    if (SUB == 2) most = fmaxf(most, fmaxf(step_of(vm[SUB - 1][0], g), step_of(vm[SUB - 1][1], g)));
    return most;
  }
  __device__ __forceinline__ static int exponent(float x) { return (int)(__float_as_uint(x) >> 23) - 127; }       // of x >= 0
  __device__ __forceinline__ static float over_rows(float most) {
#pragma unroll
    for (int y = 4; y < 32; y <<= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, y));
    return most;
  }
  // References at or above the tile's logits `s`, the sums brought to them; and scales for the tile's weights p step, which then are at most 2^15.
  // Where a reference moves the scale is set anew: kRoom bits below what would fit the tile's largest step with a p of 1, so that the next tiles, whose steps
  // are much alike, need not be looked at this closely (with no room at all 443 MB 86 -> 106 us, in fp32 144 -> 165), but not so low that the tile's largest
  // weight p step would be below 2^kLeast, and no higher than leaves what o has where it is: weights that are too small for that are small beside it
  // for good.  Elsewhere it comes down only for a weight that is too large: a huge step alone, of a row that does not count, leaves it alone.
  static constexpr int kRoom = PARTS == 2 ? 3 : 6, kLeast = PARTS == 2 ? 0 : -6;
  __device__ __forceinline__ void settle(const float (&s)[SUB][NH][4], const uint32_t (&vm)[SUB][2][G]) {
#pragma unroll
    for (int n = 0; n < NH; ++n)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        // (which heads move differs among the lanes: no exchange below depends on it)
        const float most = over_rows(largest(s, n, x)), from = ref[n][x];
        const bool moved = most > from;                        // (with nothing but NaN so far there is no reference, and the sums become NaN)
        const float to = moved ? most + kSlack : from, f = exp2_fast(from - to);
        ref[n][x] = to;
        l[n][x] *= f;
        const int by = (int)fminf(to - from, 400.f);           // (more than fp32 has)
#pragma unroll
        for (int g = 0; g < G; ++g) {
          low_sum[n][x][g] *= f;
          float weight = 0.f;
#pragma unroll
          for (int u = 0; u < SUB; ++u)
#pragma unroll
            for (int t = 0; t < 2; ++t) weight = fmaxf(weight, exp2_fast(s[u][n][2 * t + x] - to) * step_of(vm[u][t], g));
          const int weight_exp = exponent(over_rows(weight)), step_exp = exponent(over_rows(largest_step(vm, g))), now = exponent(scale[n][x][g]);
          const int anew = min(max(14 - kRoom - step_exp, kLeast - weight_exp), moved ? now + by : now);
          const int e = max(moved || weight_exp + now >= 15 ? min(anew, kMostScale) : now, -126);
          scale[n][x][g] = power_of_two(e);
          const float change = e - now < -126 ? 0.f : f * power_of_two(min(e - now, 126));                       // (beyond 126 only where f is 0)
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            o[g][t][n][x] *= change;
            o[g][t][n][2 + x] *= change;
          }
        }
      }
  }
  // The values of a run, weighed.
  __device__ __forceinline__ void attend(const float (&p)[NH][4], const uint32_t (&vm)[2][G], const unsigned char* stage, int lane) {
    const int r = lane / 4, c = lane % 4;
    uint32_t v[4][G * W];                                      // rows 2c, 2c + 1, 2c + 8, 2c + 9: codes of unit r
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const unsigned char* rows = stage + ((t & 1) * 4 + (t >> 1) * 8) * Row::kCodes;            // as value_piece() has row 2c + (t & 1) + 8 (t >> 1)
      if constexpr (kValueBytes <= 8) shared_words(v[t], rows + 16 * value_piece(2 * c, r * kValueBytes / 16) + r * kValueBytes % 16);
      else
#pragma unroll
        for (int x = 0; x < kValueBytes / 16; ++x) shared_piece(v[t], 4 * x, rows + 16 * value_piece(2 * c, r * (kValueBytes / 16) + x));
    }
    uint32_t b[NH][PARTS][G][2];
#pragma unroll
    for (int n = 0; n < NH; ++n)
#pragma unroll
      for (int g = 0; g < G; ++g)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          // (p scale is at most 2^126: a weight of 0 stays 0 whatever its step)
          const float step = step_of(vm[t], g);
          float w0, w1;
          mul2(w0, w1, p[n][2 * t], p[n][2 * t + 1], scale[n][0][g], scale[n][1][g]);
          mul2(w0, w1, w0, w1, step, step);
          const uint32_t hi = halves(w0, w1);
          b[n][0][g][t] = transpose8(hi);
          if constexpr (PARTS == 2) b[n][PARTS - 1][g][t] = transpose8(halves(w0 - half_low(hi), w1 - half_high(hi)));
        }
    // dimensions of a unit: (0, 2), (1, 3), (4, 6), (5, 7) side by side; at 4 bits the odd ones come out sixteen times too large
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        uint32_t x0, x1, x2, x3;                               // dimensions 4y and on; rows (2c, 2c + 1) and (2c + 8, 2c + 9)
        uint32_t a[2][4];
        if constexpr (BITS == 4) {
          const uint32_t t0 = __byte_perm(v[0][g], v[1][g], y ? 0x7632 : 0x5410), t1 = __byte_perm(v[2][g], v[3][g], y ? 0x7632 : 0x5410);
          x0 = t0;
          x1 = t0 >> 8;
          x2 = t1;
          x3 = t1 >> 8;
          a[0][0] = operand(x0 & 0x000f000fu); a[0][1] = operand(x1 & 0x000f000fu); a[0][2] = operand(x2 & 0x000f000fu); a[0][3] = operand(x3 & 0x000f000fu);
          a[1][0] = operand(x0 & 0x00f000f0u); a[1][1] = operand(x1 & 0x00f000f0u); a[1][2] = operand(x2 & 0x00f000f0u); a[1][3] = operand(x3 & 0x00f000f0u);
        } else {
          const int w = g * W + (W - 1) * y;
          x0 = __byte_perm(v[0][w], v[1][w], 0x5410);
          x1 = __byte_perm(v[0][w], v[1][w], 0x7632);
          x2 = __byte_perm(v[2][w], v[3][w], 0x5410);
          x3 = __byte_perm(v[2][w], v[3][w], 0x7632);
          a[0][0] = operand(x0 & 0x00ff00ffu); a[0][1] = operand(x1 & 0x00ff00ffu); a[0][2] = operand(x2 & 0x00ff00ffu); a[0][3] = operand(x3 & 0x00ff00ffu);
          a[1][0] = operand(x0 >> 8 & 0x00ff00ffu); a[1][1] = operand(x1 >> 8 & 0x00ff00ffu);
          a[1][2] = operand(x2 >> 8 & 0x00ff00ffu); a[1][3] = operand(x3 >> 8 & 0x00ff00ffu);
        }
#pragma unroll
        for (int z = 0; z < 2; ++z)
#pragma unroll
          for (int n = 0; n < NH; ++n) {
            if constexpr (PARTS == 1) mma_f16(o[g][2 * y + z][n], a[z][0], a[z][1], a[z][2], a[z][3], b[n][0][g][0], b[n][0][g][1]);
            else {
              float part[4];
              mma_f16_first(part, a[z][0], a[z][1], a[z][2], a[z][3], b[n][0][g][0], b[n][0][g][1]);
              mma_f16(part, a[z][0], a[z][1], a[z][2], a[z][3], b[n][PARTS - 1][g][0], b[n][PARTS - 1][g][1]);
#pragma unroll
              for (int e = 0; e < 4; ++e) o[g][2 * y + z][n][e] += part[e];
            }
          }
      }
  }
  // The sums of every lane's two heads: l and the lowest values' share over all rows, then f(head, its l, its reference, values of unit r of
  // group g as 2^24 o + low) for heads below `heads`.  (A state without a reference has -inf.)
  template <typename F>
  __device__ __forceinline__ void finish(int heads, int lane, F f) {
    const int r = lane / 4, c = lane % 4;
    constexpr float a = 1.f / kCodeScale, odd = BITS == 4 ? 0.0625f * a : a;
#pragma unroll
    for (int n = 0; n < NH; ++n)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int h = 2 * c + x + 8 * n;
        float sum = l[n][x], low[G];
#pragma unroll
        for (int y = 4; y < 32; y <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, y);
#pragma unroll
        for (int g = 0; g < G; ++g) {
          low[g] = low_sum[n][x][g];
#pragma unroll
          for (int y = 4; y < 32; y <<= 1) low[g] += __shfl_xor_sync(0xffffffffu, low[g], y);
        }
        if (h < heads) {
          const float m = ref[n][x];
#pragma unroll
          for (int g = 0; g < G; ++g) {
            const float e = __uint_as_float((254u << 23) - __float_as_uint(scale[n][x][g]));     // 1 / scale
            float y[8] = {fmaf(o[g][0][n][x] * a, e, low[g]), fmaf(o[g][1][n][x] * odd, e, low[g]),
                          fmaf(o[g][0][n][2 + x] * a, e, low[g]), fmaf(o[g][1][n][2 + x] * odd, e, low[g]),
                          fmaf(o[g][2][n][x] * a, e, low[g]), fmaf(o[g][3][n][x] * odd, e, low[g]),
                          fmaf(o[g][2][n][2 + x] * a, e, low[g]), fmaf(o[g][3][n][2 + x] * odd, e, low[g])};
            f(h, sum, m, g, r, y);
          }
        }
      }
  }
};

// ---- the kernel ---------------------------------------------------------------------------------------------------
// Every warp takes an equal run of the tiles of its block, whose share is that of paged_attention_kernel, and goes through it by itself: its
// tiles come through a ring of its own in shared memory (cp.async, 16 bytes a lane: no register is left for tiles on their way.  A warp that
// loaded for the others with bulk copies, four a tile, took 390 cycles for each whatever its size), and segments (sequence, KV
// head) that lie in its run are finished by it alone.  Those that cross warps leave states in shared memory, which the block joins in the
// end, and those that cross blocks states in scratch, as there.  (With the tiles dealt round all warps and a joining at the end of every
// segment the 192 ragged caches took 167 us against 77 then.)
// Empty tiles counted with every segment, and tiles per block where the GPU has more blocks than that fills, as kAttSegment and
// kAttLeast but in rows.  Of 32, 64, 128 and 192 rows with a segment the 192 ragged caches take 84.5, 78.4, 73.2 and 73.6 us.  With blocks of 64, 128,
// 256, 384 and 512 rows at least one cache of 947 rows takes 8.9, 9.0, 9.4, 10.1 and 11.1 us, one of 4,000 10.5, 9.9, 9.8, 10.6 and 11.5, one of
// 16,000 13.7, 13.7, 13.7, 13.7 and 13.0, nine in fp32 of up to 1,024 9.5, 9.5, 9.6, 10.2 and 10.2; longer ones and larger batches fill all blocks
// with any of them.
constexpr int kCodedSegment = 128, kCodedLeast = 128;

template <int N>
__device__ __forceinline__ void copies_but() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Where a tile's runs of sixteen rows are: where their codes begin in the pools, in units of 64 bytes, and how far behind that their steps and lowest
// values do (20 bits; above those, with the first run, how many rows of each run count, 0: nothing to read, five bits each, the last run's lowest).
template <int SUB>
struct __align__(8 * SUB) CodedRuns {
  uint2 run[SUB];
};

// Where the tiles of a launch lie: all (sequence, KV head, tile) triples in one list, of which block b takes the b-th equal part.
// (All tile counts stay below 2^31: see meda_pages_create.)
template <typename Tile>
struct CodedWalk {
  using Row = typename Tile::Row;
  static constexpr int HP = Tile::kHeads, SUB = Tile::SUB, kRows = 16 * SUB;
  const AttnParams& p;
  const int* pre;                        // [n + 1] tiles before sequence i
  int chunks, H, gap, total, C, base, extra, t0, t1;

  __device__ __forceinline__ CodedWalk(const AttnParams& params, const int* prefix) : p(params), pre(prefix) {
    chunks = (p.group + HP - 1) / HP;
    H = p.n_heads * chunks;
    gap = p.n_seqs > 1 ? kCodedSegment / kRows : 0;
  }
  __device__ __forceinline__ int length(int i, bool& bad) const { return clamped_len(p.lens, p.lens_stride, i, p.width << p.page_shift, bad); }
  // Runs of sixteen rows of a sequence that are attended to.
  __device__ __forceinline__ int runs(int len) const {
    const int per_page = p.page_shift - 4, pages = (len + (1 << p.page_shift) - 1) >> p.page_shift;
    return p.sel ? min(p.keep, pages) << per_page : (len + 15) / 16;
  }
  __device__ __forceinline__ int block_start(int b) const { return base * b + div_small(extra * b, C); }
  __device__ __forceinline__ int block_of(int x) const {
    int b = min((int)((float)x * ((float)C / (float)total)), C - 1);
    while (block_start(b) > x) --b;
    while (b + 1 < C && block_start(b + 1) <= x) ++b;
    return b;
  }
  __device__ __forceinline__ void share() {                    // (see paged_attention_kernel)
    total = pre[p.n_seqs] * H;
    const int most = max(p.n_seqs * H, 1), each = most * (kCodedLeast / kRows);
    C = total == 0 ? 0 : min((int)gridDim.x, total <= (long long)each * gridDim.x ? most * (div_small(total - 1, each) + 1) : (int)gridDim.x);
    base = C == (int)gridDim.x ? p.grid_div.of(total) : (C > 0 ? div_small(total, C) : 0);
    extra = total - base * C;
    const bool has_work = (int)blockIdx.x < C;
    t0 = has_work ? block_start(blockIdx.x) : 0;
    t1 = has_work ? block_start(blockIdx.x + 1) : 0;
  }
  // The runs of tile x (nothing from `end` on) to `found`.
  __device__ __forceinline__ void lookup(int x, int end, CodedRuns<SUB>& found) const {
    unsigned rows = 0, at[SUB], more[SUB];
#pragma unroll
    for (int u = 0; u < SUB; ++u) at[u] = more[u] = 0;
    find(x, end, at, more, rows);
#pragma unroll
    for (int u = 0; u < SUB; ++u) found.run[u] = make_uint2(at[u], u == 0 ? more[u] | rows << 20 : more[u]);
  }
  __device__ __forceinline__ void find(int x, int end, unsigned (&at)[SUB], unsigned (&more)[SUB], unsigned& rows) const {
    if (x >= end) return;
    const int per_page = p.page_shift - 4, page_size = 1 << p.page_shift;
    const int i = ragged_find(pre, p.n_seqs, p.heads_div.of(x));
    const int tiles = pre[i + 1] - pre[i];
    const int local = x - pre[i] * H;
    const int sh = div_small(local, tiles), tile = local - sh * tiles, g = chunks == 1 ? sh : sh / chunks;
    if (tile >= tiles - gap) return;
    bool bad = false;
    const int len = length(i, bad);
#pragma unroll
    for (int u = 0; u < SUB; ++u) {
      const int run = tile * SUB + u;
      if (run >= runs(len)) break;
      int col = run >> per_page;
      const int r0 = (run & ((1 << per_page) - 1)) * 16;
      bool ok = true;
      if (p.sel) {
        col = p.sel[((size_t)i * p.n_heads + g) * p.keep + col];
        ok = col >= 0 && col < (len + page_size - 1) >> p.page_shift;
      }
      if (ok) {
        const int nv = min(16, max(0, len - ((col << p.page_shift) + r0)));
        if (nv > 0) {
          const int page = p.table[(size_t)i * p.width + col];
          ok = (unsigned)page < (unsigned)p.n_pages;
          if (ok) {
            at[u] = (unsigned)(((((long long)page * p.n_heads + g) << p.page_shift) * Row::kBytes + r0 * Row::kCodes) / 64);
            more[u] = (unsigned)(page_size * Row::kCodes - r0 * (Row::kCodes - Row::kMore));
            rows |= nv << 5 * (SUB - 1 - u);
          }
        }
      }
      if (!ok) set_status(p.status, MEDA_ERR_INVALID_ARG);
    }
  }
};

// S = tiles of a warp in the ring.
template <typename Tile, int D, int W, int S>
__global__ void __launch_bounds__(W * 32, 1)
coded_attention_kernel(AttnParams p) {
  using T = typename Tile::T;
  using Row = typename Tile::Row;
  constexpr int HP = Tile::kHeads, SUB = Tile::SUB;
  constexpr int LD = D + 4;
  begin_grid();
  extern __shared__ __align__(128) unsigned char coded_smem[];
  __shared__ int scratch[W + 1];
  __shared__ int4 part_of[2 * W];        // states, two per warp (the segment that ends in it, the one that goes on behind it): (first tile, one
                                         // past the last, first query head of [n_seqs][n_q_heads], query heads or 0: there is none)
  __shared__ CodedRuns<SUB> table[W][32];
  __shared__ int state_at[2 * W];        // where the states that are there lie, in floats
  __shared__ int2 chain_of[2 * W + 1];   // of every segment that has some the first in that list and its place in part_of; and the list's end
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  unsigned char* ring = coded_smem + warp * (S * Tile::kStage);                        // this warp's tiles
  constexpr int kState = attn_merge_floats(1, HP, D);                                  // a softmax state: [HP] maxima, [HP] sums, [HP][LD] values
  static_assert(kState * 4 <= S * Tile::kStage, "a warp's last state goes where its tiles were");
  float* heads_of = reinterpret_cast<float*>(coded_smem + W * S * Tile::kStage);       // [W] states of segments that end in a warp
  int* pre = reinterpret_cast<int*>(heads_of + W * kState);
  CodedWalk<Tile> walk(p, pre);
  ragged_prefix<W * 32>(p.n_seqs, pre, scratch, [&](int i) {
    bool bad = false;
    const int len = walk.length(i, bad);
    if (bad && blockIdx.x == 0) set_status(p.status, MEDA_ERR_INVALID_ARG);
    const int tiles = (walk.runs(len) + SUB - 1) / SUB;
    return tiles ? tiles + walk.gap : 0;
  });
  walk.share();
  const int n_q_heads = p.n_heads * p.group;
  const int state_heads = min(p.group, HP), state_floats = attn_state_floats(state_heads, D);
  const int H = walk.H, gap = walk.gap, t0 = walk.t0, t1 = walk.t1;
  const int each = (t1 - t0) / W, more = (t1 - t0) % W;        // tiles of a warp, and how many warps have one more
  const int w0 = t0 + each * warp + min(warp, more), w1 = w0 + each + (warp < more);

  // ---- copies.  Tile w0 + i goes to stage i % S; 32 tiles are looked up at a time, one by each lane, into `table`.  A copy of no rows is an
  // empty group, so that the groups count the tiles.
  int number = 32, into = 0, x_copy = w0 + lane;
  static_assert(5 * SUB * S <= 32, "`counts` has the rows of all tiles in the ring");
  unsigned counts = 0;                                         // rows of the tiles on their way, the last one's lowest
  const uint32_t ring_at = sm100::smem_u32(ring);
  constexpr int kMorePieces = Tile::kRunMore / 16;             // of a run of keys or values: side by side on the lanes, keys, values, the next run's
  const int more_half = lane / kMorePieces, more_run = SUB == 2 ? more_half >> 1 & 1 : 0;
  const unsigned char *k_lane = static_cast<const unsigned char*>(p.k) + lane * 16, *v_lane = static_cast<const unsigned char*>(p.v) + lane * 16;
  const unsigned char* more_lane = static_cast<const unsigned char*>(more_half & 1 ? p.v : p.k) + lane % kMorePieces * 16;
  auto copy_next = [&] {
    if (number == 32) {
      __syncwarp();
      walk.lookup(x_copy, w1, table[warp][lane]);
      __syncwarp();
      x_copy += 32;
      number = 0;
    }
    const uint32_t to = ring_at + into * Tile::kStage;
    const CodedRuns<SUB> found = table[warp][number];
    const uint2 mine = found.run[more_run];
    const unsigned rows = found.run[0].y >> 20;
    counts = counts << 5 * SUB | rows;
    auto copies = [&](auto live) {
#pragma unroll
      for (int u = 0; u < SUB; ++u) {
        const unsigned char *k = k_lane + (size_t)found.run[u].x * 64, *v = v_lane + (size_t)found.run[u].x * 64;
#pragma unroll
        for (int i = 0; i < Tile::kRunCodes / 512; ++i) {
          const int piece = lane + 32 * i, y = piece / Tile::kPieces, z = piece % Tile::kPieces;
          if (live(u, y)) {
            copy16(to + 2 * u * Tile::kHalf + 16 * Tile::key_piece(y, z), k + i * 512);
            copy16(to + (2 * u + 1) * Tile::kHalf + 16 * Tile::value_piece(y, z), v + i * 512);
          }
        }
      }
      // steps and lowest values: with 32 pieces or fewer one goes for each lane, else a turn for each run
      constexpr int kAll = 2 * SUB * kMorePieces;
#pragma unroll
      for (int i = 0; i < (kAll + 31) / 32; ++i) {
        const int u = kAll > 32 ? i : more_run;
        const uint2 run = kAll > 32 ? found.run[i] : mine;
        if ((kAll >= 32 || lane < kAll) && live(u, lane % kMorePieces * 16 / Row::kMore))
          copy16(to + (kAll > 32 ? 2 * i + (more_half & 1) : more_half) * Tile::kHalf + Tile::kRunCodes + lane % kMorePieces * 16,
                 more_lane + ((size_t)run.x * 64 + (run.y & 0xfffffu)));
      }
    };
    if (rows == Tile::kFull) copies([](int, int) { return true; });
    else copies([&](int u, int y) { return y < (int)(rows >> 5 * (SUB - 1 - u) & 31); });
    asm volatile("cp.async.commit_group;" ::: "memory");
    into = into + 1 == S ? 0 : into + 1;
    ++number;
  };

  // ---- the segments (sequence, KV head) of this warp
  int seq = 0, sh = 0, seg0 = w1, seg1 = w1;                   // tiles [seg0, seg1) count; w1: there is no segment
  auto next_segment = [&] {                                    // the next one with tiles
    seg0 += pre[seq + 1] - pre[seq];
    if (++sh == H) {
      sh = 0;
#pragma unroll 1
      do ++seq; while (seq < p.n_seqs && pre[seq] == pre[seq + 1]);
    }
    seg1 = seg0 < w1 ? seg0 + pre[seq + 1] - pre[seq] - gap : seg0;
  };
  if (w0 < w1) {
    seq = ragged_find(pre, p.n_seqs, p.heads_div.of(w0));
    const int tiles = pre[seq + 1] - pre[seq];
    sh = div_small(w0 - pre[seq] * H, tiles);
    seg0 = pre[seq] * H + sh * tiles;
    seg1 = seg0 + tiles - gap;
    if (w0 >= seg1) next_segment();                            // nothing but empty tiles of it here
  }
  Tile tile;
  int heads = 0;
  size_t first_head = 0;
  auto load_q = [&] {
    const int g = walk.chunks == 1 ? sh : sh / walk.chunks, h0 = (sh - g * walk.chunks) * HP;
    heads = min(HP, p.group - h0);
    first_head = (size_t)seq * n_q_heads + (size_t)g * p.group + h0;
    tile.load_q(static_cast<const T*>(p.q) + first_head * D, heads, p.scale_log2, lane);
    tile.reset();
  };
  auto finish = [&] {                                          // the segment ends in this warp, or the warp's run inside the segment
    const bool ends = seg1 <= w1, whole = ends && seg0 >= w0;
    float* state = ends ? heads_of + warp * kState : reinterpret_cast<float*>(ring);
    if (!ends) {                                               // (copies of nothing may still be on their way there)
      asm volatile("cp.async.wait_all;" ::: "memory");
      __syncwarp();
    }
    if (lane == 0 && !whole) part_of[2 * warp + (ends ? 0 : 1)] = make_int4(seg0, seg1, (int)first_head, heads);
    tile.finish(heads, lane, [&](int h, float sum, float m, int g, int r, float (&y)[8]) {
      if (whole) {
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] *= inv;
        Eight<T> w;
        w.round(y);
        w.store(static_cast<T*>(p.out) + (first_head + h) * D + g * 64 + r * 8);
        if (p.lse && g == 0 && r == 0) p.lse[first_head + h] = (m + log2f(sum)) * 0.6931471805599453f;
      } else {
        float4* d = reinterpret_cast<float4*>(state + 2 * HP + h * LD + g * 64 + r * 8);
        d[0] = make_float4(y[0], y[1], y[2], y[3]);
        d[1] = make_float4(y[4], y[5], y[6], y[7]);
        if (g == 0 && r == 0) {
          state[h] = m;
          state[HP + h] = sum;
        }
      }
    });
  };
  if (lane < 2) part_of[2 * warp + lane] = make_int4(0, 0, 0, 0);
  __syncwarp();
  int from = 0, x = w0 - (S - 1);
#pragma unroll 1
  while (seg0 < w1) {                                          // (a warp may have nothing but the last segment's empty tiles)
#pragma unroll 1
    for (; x < w0; ++x) copy_next();
    load_q();
    const int end = min(seg1, w1);
#pragma unroll 1
    for (; x < end; ++x) {
      __syncwarp();                                            // the stage about to be filled has been read by every lane
      copy_next();
      const unsigned rows = counts >> 5 * (S - 1) * SUB & ((1u << 5 * SUB) - 1);
      copies_but<S - 1>();
      __syncwarp();
      if (rows) tile.work(ring + from * Tile::kStage, rows, lane);
      from = from + 1 == S ? 0 : from + 1;
    }
    finish();
    next_segment();
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();

  // ---- states of segments that cross warps, joined in the warps' order: a list of the states that are there, and where in it a segment begins
  // (every warp writes the same)
  const int4 part = lane < 2 * W ? part_of[lane] : make_int4(0, 0, 0, 0);
  const unsigned there = __ballot_sync(0xffffffffu, part.w > 0), below = there & ((1u << lane) - 1);
  const int before = __shfl_sync(0xffffffffu, part.x, below ? 31 - __clz(below) : 0);
  const unsigned starts = __ballot_sync(0xffffffffu, part.w > 0 && (!below || before != part.x));
  const int chains = __popc(starts);
  if (part.w > 0)
    state_at[__popc(below)] = lane & 1 ? (lane >> 1) * (S * Tile::kStage / 4) : W * S * Tile::kStage / 4 + (lane >> 1) * kState;
  if (starts >> lane & 1) chain_of[__popc(starts & ((1u << lane) - 1))] = make_int2(__popc(below), lane);
  if (lane == 0) chain_of[chains] = make_int2(__popc(there), 0);
  __syncwarp();
  int4 split = make_int4(0, 0, 0, 0);
#pragma unroll 1
  for (int i = 0; i < chains; ++i) {
    const int begin = chain_of[i].x, end = chain_of[i + 1].x;
    const int4 part = part_of[chain_of[i].y];
#pragma unroll 1
    for (int e = threadIdx.x; e < part.w * (D / 4); e += W * 32) {
      const int h = e / (D / 4), d = e % (D / 4) * 4;
      const float* base = reinterpret_cast<const float*>(coded_smem) + h;
      constexpr int kBatch = 4;                                // states at a time; behind the last one that again, with a weight of 0
      float mm = -INFINITY;
#pragma unroll 1
      for (int z = begin; z < end; z += kBatch)
#pragma unroll
        for (int y = 0; y < kBatch; ++y) mm = fmaxf(mm, base[state_at[min(z + y, end - 1)]]);
      float ll = 0.f;
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
      for (int z = begin; z < end; z += kBatch) {
        float m[kBatch], l[kBatch];
        float4 o[kBatch];
#pragma unroll
        for (int y = 0; y < kBatch; ++y) {
          const int at = state_at[min(z + y, end - 1)];
          m[y] = base[at];
          l[y] = base[at + HP];
          o[y] = *reinterpret_cast<const float4*>(base + at + 2 * HP + h * (LD - 1) + d);
        }
#pragma unroll
        for (int y = 0; y < kBatch; ++y) {
          // (no state is -inf with a sum of 0; a sum that is NaN has a maximum of -inf when all logits are)
          const float f = z + y < end && (m[y] != -INFINITY || l[y] != 0.f) ? exp2_fast(m[y] - mm) : 0.f;
          ll = fmaf(f, l[y], ll);
          acc.x = fmaf(f, o[y].x, acc.x);
          acc.y = fmaf(f, o[y].y, acc.y);
          acc.z = fmaf(f, o[y].z, acc.z);
          acc.w = fmaf(f, o[y].w, acc.w);
        }
      }
      if (part.x >= t0 && part.y <= t1) {
        const float inv = ll == 0.f ? 0.f : 1.f / ll;
        store4<T>(static_cast<T*>(p.out) + ((size_t)part.z + h) * D + d, make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv));
        if (p.lse && d == 0) p.lse[part.z + h] = (mm + log2f(ll)) * 0.6931471805599453f;
      } else {
        float* state = p.partial + ((size_t)blockIdx.x * 2 + (part.x < t0 ? 0 : 1)) * state_floats;
        *reinterpret_cast<float4*>(state + h * D + d) = acc;
        if (d == 0) *reinterpret_cast<float2*>(state + state_heads * D + 2 * h) = make_float2(mm, ll);
      }
    }
    if (threadIdx.x == W * 32 - 1 && part.x >= t0 && part.y > t1)               // at most one goes on behind the block
      split = make_int4(walk.block_of(part.y - 1) - (int)blockIdx.x + 1, part.z, part.w, 0);
  }
  if (threadIdx.x == W * 32 - 1) p.split[blockIdx.x] = split;

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
}

}  // namespace meda
