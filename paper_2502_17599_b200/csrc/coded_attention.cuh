// The attention's tile over quantised pages (the walk over the pages is paged_attention.cuh's).
//
// A row's logit is the sum over its groups of step_g (q_g . codes_g) + low_g sum(q_g), an output the sum over the rows of
// (p step_g) codes_g + p low_g.  So the matrix instructions multiply by the codes themselves, and a code is its own fp16 operand: the whole
// number c in the lower bits of a half is the subnormal c 2^-24, exact, and needs no conversion, offset or scale, only a mask
// (and at 4 bits c << 4, a nibble further up, is 16 c 2^-24: the factor goes into the queries and out of the result).  Steps, lowest
// values, logits, maxima and sums are fp32; products of the queries with codes are exact and added in fp32.
//
// Fragments, lane l: r = l / 4, c = l % 4.  Q K^T has A = codes of the keys (rows r and r + 8 of the tile), B = queries (column r: head r),
// group by group; sum(q) low is one instruction of bf16, the sums in three parts.  P V has A = codes of the values, transposed
// (rows are dimensions; a byte permute pairs the codes of neighbouring cache rows), B = (p step_g)^T, from the logits' layout by an 8 x 8
// transposition per group.  Columns are heads on both sides, so a lane's maxima, sums and results belong to the same two heads.
//
// Roundings.  Queries are scaled by a power of two per head, their largest element between 2^14 and 2^15: fp16 then holds every bf16 element
// that matters exactly (the rest is below 2^-38 of the largest); fp32 ones go in two parts.  A weight p step is rounded to
// fp16 (2^-11 of itself: a quarter of the output's own rounding in bf16 at worst, and it averages out over the rows), for fp32 caches to two
// such parts; weights are scaled by a power of two that follows the largest step a warp has met, so that neither tiny nor huge values leave
// fp16's range.
#pragma once

#include "page_codes.cuh"
#include "paged_attention.cuh"   // exp2_fast
#include "pages_common.cuh"

namespace meda {

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_low(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
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
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }    // -126 <= e <= 127

template <int N>
__device__ __forceinline__ void load_words(uint32_t (&w)[N], const unsigned char* p) {
  if constexpr (N == 1) {
    asm volatile("ld.global.nc.L1::no_allocate.u32 %0, [%1];" : "=r"(w[0]) : "l"(p));
  } else if constexpr (N == 2) {
    asm volatile("ld.global.nc.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "l"(p));
  } else {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const uint4 x = load_stream(reinterpret_cast<const uint4*>(p + 4 * i));
      w[i] = x.x;
      w[i + 1] = x.y;
      w[i + 2] = x.z;
      w[i + 3] = x.w;
    }
  }
}

// T = type of queries and outputs, D = head_dim, NH = groups of eight query heads.
template <typename TOUT, int D, int NH, int BITS>
struct AttnTileCoded {
  using T = TOUT;
  using Row = CodedRow<D, BITS>;
  static constexpr bool kMma = false, kCoded = true;
  static constexpr int kHeads = 8 * NH;
  static constexpr int G = Row::kGroups, W = BITS / 4;           // groups, words per unit
  static constexpr int PARTS = sizeof(T) == 4 ? 2 : 1;           // fp16 parts of a query element and of a weight
  static constexpr int kScale = PARTS == 2 ? 13 : 5;             // weights reach 2^(kScale + 1) (times 2^kSlack)
  static constexpr float kSlack = PARTS == 2 ? 0.f : 8.f;        // the reference may stay this far (log2) behind the maximum

  uint32_t q[NH][PARTS][2][G][4];        // unit 2c + i of group g: the four pairs that go with pair_of()
  uint32_t qsum[NH][2];                  // sums over the groups, in bf16 parts
  float unscale[NH][2];                  // 2^-k of the scaled queries, of the lane's two heads
  uint32_t k[2][2 * G * W], km[2][G];    // rows r, r + 8: codes of units 2c, 2c + 1; steps and lowest values
  uint32_t v[4][G * W], vm[2][G];        // rows 2c, 2c + 1, 2c + 8, 2c + 9: codes of unit r; steps and lowest values of rows r, r + 8
  float o[G][4][NH][4];
  float low_sum[NH][2][G];               // sum of p low
  float m[NH][2], l[NH][2];
  float step_top;                        // steps below this fit the weights' scale
  int step_exp;                          // which is 2^(kScale - step_exp), 2^125 at most

  // Pair j of a unit's eight codes, as the two halves of a word: elements (first, second).
  __device__ __forceinline__ static constexpr int pair_first(int j) { return BITS == 4 ? j : (j / 2) * 4 + j % 2; }
  __device__ __forceinline__ static constexpr int pair_second(int j) { return BITS == 4 ? j + 4 : (j / 2) * 4 + j % 2 + 2; }
  __device__ __forceinline__ static constexpr float pair_factor(int j) { return BITS == 4 && j % 2 == 1 ? 0.0625f : 1.f; }
  __device__ __forceinline__ static uint32_t pair_of(const uint32_t* unit, int j) {
    if constexpr (BITS == 4) return (j < 2 ? unit[0] : unit[0] >> 8) & (j % 2 ? 0x00f000f0u : 0x000f000fu);
    else return (j % 2 ? unit[j / 2] >> 8 : unit[j / 2]) & 0x00ff00ffu;
  }
  __device__ __forceinline__ static float step_of(const uint32_t (&w)[G], int g) {
    return __uint_as_float(g % 2 == 0 ? w[g / 2] << 16 : w[g / 2] & 0xffff0000u);
  }
  __device__ __forceinline__ static float low_of(const uint32_t (&w)[G], int g) {
    if constexpr (G == 1) return __uint_as_float(w[0] & 0xffff0000u);
    else return __uint_as_float(g % 2 == 0 ? w[G / 2 + g / 2] << 16 : w[G / 2 + g / 2] & 0xffff0000u);
  }

  __device__ __forceinline__ void load_q(const T* qh, int heads, int lane) {     // qh: the segment's first query head
    const int r = lane / 4, c = lane % 4;
#pragma unroll
    for (int n = 0; n < NH; ++n) {
      const int h = r + 8 * n;
      float x[2][G][8], top = 0.f;
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            x[i][g][e] = h < heads ? to_f32<T>(qh[(size_t)h * D + g * 64 + (2 * c + i) * 8 + e]) : 0.f;
            top = fmaxf(top, fabsf(x[i][g][e]));
          }
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const int k2 = min(126, 14 - ((int)(__float_as_uint(top) >> 23) - 127));
      const float scale = top < INFINITY ? power_of_two(k2) : NAN;               // a query that is not finite makes its logits NaN
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
        sum[g] *= 5.9604644775390625e-8f;                                        // 2^-24, as the products with codes have it
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
      const float back = scale == scale ? power_of_two(-k2) : NAN;
      unscale[n][0] = __shfl_sync(0xffffffffu, back, 8 * c);                     // head 2c is lane 4 * 2c's
      unscale[n][1] = __shfl_sync(0xffffffffu, back, 8 * c + 4);
    }
  }
  __device__ __forceinline__ void reset() {
#pragma unroll
    for (int n = 0; n < NH; ++n)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        m[n][x] = -INFINITY;
        l[n][x] = 0.f;
#pragma unroll
        for (int g = 0; g < G; ++g) low_sum[n][x][g] = 0.f;
      }
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int n = 0; n < NH; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[g][t][n][e] = 0.f;
    step_top = 0.f;
    step_exp = kScale - 125;
  }
  // Rows behind the nv that count are not read: their lanes read the last one that does (see logits and attend).
  __device__ __forceinline__ void load_k(const void* pool, long long row, int page_size, int nv, int lane) {
    const int r = lane / 4, c = lane % 4, in = (int)row & (page_size - 1);
    const unsigned char* page = static_cast<const unsigned char*>(pool) + (row - in) * Row::kBytes;
    const unsigned char *codes = page + in * Row::kCodes + c * (2 * G * BITS), *more = page + page_size * Row::kCodes + in * Row::kMore;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int y = min(r + 8 * t, nv - 1);
      load_words(k[t], codes + y * Row::kCodes);
      load_words(km[t], more + y * Row::kMore);
    }
  }
  __device__ __forceinline__ void load_v(const void* pool, long long row, int page_size, int nv, int lane) {
    const int r = lane / 4, c = lane % 4, in = (int)row & (page_size - 1);
    const unsigned char* page = static_cast<const unsigned char*>(pool) + (row - in) * Row::kBytes;
    const unsigned char *codes = page + in * Row::kCodes + r * (G * BITS), *more = page + page_size * Row::kCodes + in * Row::kMore;
#pragma unroll
    for (int t = 0; t < 4; ++t) load_words(v[t], codes + min(2 * c + (t & 1) + (t >> 1) * 8, nv - 1) * Row::kCodes);
#pragma unroll
    for (int t = 0; t < 2; ++t) load_words(vm[t], more + min(r + 8 * t, nv - 1) * Row::kMore);
  }
  // Logits in the log2 domain: s[n][0..1] row r, heads 2c, 2c + 1 (+ 8 n); s[n][2..3] row r + 8.
  __device__ __forceinline__ void logits(float (&s)[NH][4], float scale_log2, int nv, int lane) {
    const int r = lane / 4;
#pragma unroll
    for (int n = 0; n < NH; ++n) {
#pragma unroll
      for (int e = 0; e < 4; ++e) s[n][e] = 0.f;
      constexpr int L0 = G / 2, L1 = G == 4 ? G / 2 + 1 : G / 2;                 // the words of the lowest values
      mma_low(s[n], km[0][L0], km[1][L0], km[0][L1], km[1][L1], qsum[n][0], qsum[n][1]);
    }
#pragma unroll
    for (int g = 0; g < G; ++g) {
      float acc[NH][4];
#pragma unroll
      for (int n = 0; n < NH; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[n][e] = 0.f;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t *u0 = &k[0][(i * G + g) * W], *u1 = &k[1][(i * G + g) * W];
#pragma unroll
        for (int j = 0; j < 4; j += 2) {
          const uint32_t a0 = pair_of(u0, j), a1 = pair_of(u1, j), a2 = pair_of(u0, j + 1), a3 = pair_of(u1, j + 1);
#pragma unroll
          for (int n = 0; n < NH; ++n)
#pragma unroll
            for (int x = 0; x < PARTS; ++x) mma_f16(acc[n], a0, a1, a2, a3, q[n][x][i][g][j], q[n][x][i][g][j + 1]);
        }
      }
      const float s0 = step_of(km[0], g), s1 = step_of(km[1], g);
#pragma unroll
      for (int n = 0; n < NH; ++n) {
        s[n][0] = fmaf(s0, acc[n][0], s[n][0]);
        s[n][1] = fmaf(s0, acc[n][1], s[n][1]);
        s[n][2] = fmaf(s1, acc[n][2], s[n][2]);
        s[n][3] = fmaf(s1, acc[n][3], s[n][3]);
      }
    }
    const float back = scale_log2 * 16777216.f;                                  // 2^24 (in two steps: 2^-k alone may fill fp32's range)
#pragma unroll
    for (int n = 0; n < NH; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[n][e] = s[n][e] * back * unscale[n][e & 1];
    if (nv < 16) {
#pragma unroll
      for (int n = 0; n < NH; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (r + (e >> 1) * 8 >= nv) s[n][e] = -INFINITY;
    }
  }
  __device__ __forceinline__ void attend(float (&s)[NH][4], int nv, int lane) {
    const int r = lane / 4;
    if (nv < 16) {                                             // a weight of 0 times whatever is there has to be 0
#pragma unroll
      for (int t = 0; t < 2; ++t)
        if (r + 8 * t >= nv)
#pragma unroll
          for (int g = 0; g < G; ++g) vm[t][g] = 0u;
    }
    float step[2][G], top = 0.f;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int g = 0; g < G; ++g) {
        step[t][g] = step_of(vm[t], g);
        top = fmaxf(top, step[t][g]);
      }
    bool moved = top >= step_top;
#pragma unroll
    for (int n = 0; n < NH; ++n)
#pragma unroll
      for (int x = 0; x < 2; ++x) moved |= fmaxf(s[n][x], s[n][2 + x]) > m[n][x] + kSlack;
    if (__any_sync(0xffffffffu, moved)) {                      // a new reference, or larger values than before: bring the sums to them
#pragma unroll
      for (int y = 1; y < 32; y <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, y));
      const int to = max(step_exp, (int)(__float_as_uint(top) >> 23) - 127);
      const float smaller = step_exp - to < -126 ? 0.f : power_of_two(step_exp - to);
      step_exp = to;
      step_top = to == 127 ? INFINITY : power_of_two(to + 1);
#pragma unroll
      for (int n = 0; n < NH; ++n)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          float mn = fmaxf(s[n][x], s[n][2 + x]);
#pragma unroll
          for (int y = 4; y < 32; y <<= 1) mn = fmaxf(mn, __shfl_xor_sync(0xffffffffu, mn, y));
          mn = fmaxf(mn, m[n][x]);
          const float f = exp2_fast(m[n][x] - (mn == -INFINITY ? 0.f : mn));
          m[n][x] = mn;
          l[n][x] *= f;
#pragma unroll
          for (int g = 0; g < G; ++g) {
            low_sum[n][x][g] *= f;
#pragma unroll
            for (int t = 0; t < 4; ++t) {
              o[g][t][n][x] *= f * smaller;
              o[g][t][n][2 + x] *= f * smaller;
            }
          }
        }
    }
    const float weight = power_of_two(kScale - step_exp);      // step_exp >= kScale - 125
    uint32_t b[NH][PARTS][G][2];
#pragma unroll
    for (int n = 0; n < NH; ++n) {
      float p[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) p[e] = exp2_fast(s[n][e] - (m[n][e & 1] == -INFINITY ? 0.f : m[n][e & 1]));
      l[n][0] += p[0] + p[2];
      l[n][1] += p[1] + p[3];
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const float low0 = low_of(vm[0], g), low1 = low_of(vm[1], g);
#pragma unroll
        for (int x = 0; x < 2; ++x) low_sum[n][x][g] = fmaf(p[2 + x], low1, fmaf(p[x], low0, low_sum[n][x][g]));
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const float f = step[t][g] * weight, w0 = p[2 * t] * f, w1 = p[2 * t + 1] * f;
          const uint32_t hi = halves(w0, w1);
          b[n][0][g][t] = transpose8(hi);
          if constexpr (PARTS == 2) b[n][PARTS - 1][g][t] = transpose8(halves(w0 - half_low(hi), w1 - half_high(hi)));
        }
      }
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
          a[0][0] = x0 & 0x000f000fu; a[0][1] = x1 & 0x000f000fu; a[0][2] = x2 & 0x000f000fu; a[0][3] = x3 & 0x000f000fu;
          a[1][0] = x0 & 0x00f000f0u; a[1][1] = x1 & 0x00f000f0u; a[1][2] = x2 & 0x00f000f0u; a[1][3] = x3 & 0x00f000f0u;
        } else {
          const int w = g * W + (W - 1) * y;
          x0 = __byte_perm(v[0][w], v[1][w], 0x5410);
          x1 = __byte_perm(v[0][w], v[1][w], 0x7632);
          x2 = __byte_perm(v[2][w], v[3][w], 0x5410);
          x3 = __byte_perm(v[2][w], v[3][w], 0x7632);
          a[0][0] = x0 & 0x00ff00ffu; a[0][1] = x1 & 0x00ff00ffu; a[0][2] = x2 & 0x00ff00ffu; a[0][3] = x3 & 0x00ff00ffu;
          a[1][0] = x0 >> 8 & 0x00ff00ffu; a[1][1] = x1 >> 8 & 0x00ff00ffu; a[1][2] = x2 >> 8 & 0x00ff00ffu; a[1][3] = x3 >> 8 & 0x00ff00ffu;
        }
#pragma unroll
        for (int z = 0; z < 2; ++z)
#pragma unroll
          for (int n = 0; n < NH; ++n)
#pragma unroll
            for (int x = 0; x < PARTS; ++x) mma_f16(o[g][2 * y + z][n], a[z][0], a[z][1], a[z][2], a[z][3], b[n][x][g][0], b[n][x][g][1]);
      }
  }
  // state to shared memory: sm [kHeads], sl [kHeads], so [kHeads][ld]
  __device__ __forceinline__ void put(float* sm, float* sl, float* so, int ld, int heads, int lane) {
    const int r = lane / 4, c = lane % 4;
    const float a = power_of_two(24 - kScale), e = power_of_two(step_exp), odd = BITS == 4 ? 0.0625f * a : a;
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
        if (r == 0) {
          sm[h] = m[n][x];
          sl[h] = sum;
        }
        if (h < heads) {
#pragma unroll
          for (int g = 0; g < G; ++g) {
            float4* d = reinterpret_cast<float4*>(so + h * ld + g * 64 + r * 8);
            d[0] = make_float4(fmaf(o[g][0][n][x] * a, e, low[g]), fmaf(o[g][1][n][x] * odd, e, low[g]),
                               fmaf(o[g][0][n][2 + x] * a, e, low[g]), fmaf(o[g][1][n][2 + x] * odd, e, low[g]));
            d[1] = make_float4(fmaf(o[g][2][n][x] * a, e, low[g]), fmaf(o[g][3][n][x] * odd, e, low[g]),
                               fmaf(o[g][2][n][2 + x] * a, e, low[g]), fmaf(o[g][3][n][2 + x] * odd, e, low[g]));
          }
        }
      }
  }
};

}  // namespace meda
