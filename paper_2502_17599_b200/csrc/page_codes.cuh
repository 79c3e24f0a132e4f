// Quantised pages: rows of 4- or 8-bit codes, written, read back and bounded.
//
// Every 64 dimensions of a row share a step and a lowest value, both bf16:
//   low = min x rounded down,  step = max(2^-126, (max x - low) * fl(1 / (2^BITS - 1)) rounded up),
//   code = rint(fl(fl(x - low) * fl(1 / step))),  read back as low + step * code.
// The step is rounded up, so the largest code is 2^BITS - 1 without a test; the product step * code is exact in fp32.  The
// operations are fp32 ones, each rounded by itself, so that every implementation of these lines writes the same bytes.  64
// dimensions: 4.5 bits per element at 4 bits, and groups that the eight lanes of a quarter warp hold as eight elements each.
//
// A page of one head is its rows' codes and then their (steps, lows).  The codes of a row lie in units of eight dimensions, unit i
// of group g at place i * groups + g: the lanes of the attention's fragments then find what they need of every group side by side.
//
// Work split as in page_rows.cuh: the pages of all sequences and heads form one list that the warps share out; a lane works on
// one unit of a row, so its dimensions never change and the bounds stay in registers.
//
// Bound by memory where the arithmetic lets it: some 60 instructions go into eight elements of bf16 with bounds, so it is fp32 pairs in one
// instruction (f32x2), extremes of two bf16 at once, sums with 2^23 in place of conversions, and one scale per lane for eight rows of a
// group, handed round, in place of eight equal ones.  28 layers of a 19K-token prompt (4 heads of 128, bf16, 4 bits): stored with
// their bounds, 330 MB, in 71 to 75 us, 67 to 71 % of a plain copy (without bounds 61 to 69), read back, 315 MB, in 54 us, 88 %; at 8 bits, 392 and 376
// MB, in 72 to 78 us, 77 to 83 %, and 63 us, 92 %; 64 caches read back from 8 bits, 629 MB, in 103 us, 93 %.  The same prompt in fp32 119 to 133 us and 98
// at 4 bits, 122 to 131 and 110 at 8.  Its keys' bounds alone: 33 to 40 us at 4 bits, 26 at 8 (arithmetic: 8 and 12 us of reading), in fp32 64 and 60; those of
// the last pages of 28 sequences 3.5 and 3.0 us.
#pragma once

#include "page_rows.cuh"

namespace meda {

constexpr int kCodeGroup = 64;                  // dimensions that share a step and a lowest value
constexpr float kCodeLeast = 1.17549435e-38f;   // 2^-126, the smallest step
constexpr float kCodeMost = 8.507059173e37f;    // 2^126: a group with an element this large or a NaN reads back as NaN

// Sizes of a row of D dimensions in a quantised page, in bytes.
template <int D, int BITS>
struct CodedRow {
  static constexpr int kGroups = D / kCodeGroup;
  static constexpr int kUnits = D / 8;           // lanes on a row
  static constexpr int kCodes = D * BITS / 8;
  static constexpr int kMore = 4 * kGroups;      // steps, then lowest values
  static constexpr int kBytes = kCodes + kMore;
  // where unit u of a row lies among the codes
  __device__ __forceinline__ static int place(int u) { return ((u % 8) * kGroups + u / 8) * BITS; }
};
__host__ __device__ constexpr int64_t coded_page_bytes(int d, int bits, int page_size) {
  return (int64_t)page_size * (d * bits / 8 + 4 * (d / kCodeGroup));
}

__device__ __forceinline__ float bf16_up(float x) {             // of x >= 0; NaN stays NaN
  const uint32_t b = __float_as_uint(x);
  return x != x ? x : __uint_as_float((b + 0xffffu) & 0xffff0000u);
}
__device__ __forceinline__ float bf16_down(float x) {           // of a finite x
  const uint32_t b = __float_as_uint(x);
  return __uint_as_float((b + (b >> 31 ? 0xffffu : 0u)) & 0xffff0000u);
}

// Eight elements of T: as they are loaded, and as floats.
template <typename T>
struct Eight;
template <>
struct Eight<__nv_bfloat16> {
  uint4 w;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { w = load_stream(reinterpret_cast<const uint4*>(p)); }
  __device__ __forceinline__ void floats(float (&x)[8]) const {
    const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[2 * e] = __uint_as_float(v[e] << 16);
      x[2 * e + 1] = __uint_as_float(v[e] & 0xffff0000u);
    }
  }
  __device__ __forceinline__ void round(const float (&x)[8]) {
    uint32_t v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * e], x[2 * e + 1]);
      memcpy(&v[e], &h, 4);
    }
    w = make_uint4(v[0], v[1], v[2], v[3]);
  }
  __device__ __forceinline__ void store(__nv_bfloat16* p) const { *reinterpret_cast<uint4*>(p) = w; }
  // The eight's extremes as (minimum, -maximum); a NaN wins.
  using Range = uint32_t;
  __device__ __forceinline__ Range range() const {
    const uint32_t v[4] = {w.x, w.y, w.z, w.w};
    __nv_bfloat162 x[4];
    memcpy(x, v, 16);
    const __nv_bfloat162 l = __hmin2_nan(__hmin2_nan(x[0], x[1]), __hmin2_nan(x[2], x[3]));
    const __nv_bfloat162 h = __hmax2_nan(__hmax2_nan(x[0], x[1]), __hmax2_nan(x[2], x[3]));
    uint32_t lw, hw;
    memcpy(&lw, &l, 4);
    memcpy(&hw, &h, 4);
    hw ^= 0x80008000u;
    return join(__byte_perm(lw, hw, 0x5410), __byte_perm(lw, hw, 0x7632));
  }
  __device__ __forceinline__ static Range join(Range a, Range b) {
    __nv_bfloat162 x, y;
    memcpy(&x, &a, 4);
    memcpy(&y, &b, 4);
    const __nv_bfloat162 m = __hmin2_nan(x, y);
    uint32_t r;
    memcpy(&r, &m, 4);
    return r;
  }
  __device__ __forceinline__ static Range other(Range a, int mask) { return __shfl_xor_sync(0xffffffffu, a, mask); }
  __device__ __forceinline__ static float low_of(Range a) { return __uint_as_float(a << 16); }
  __device__ __forceinline__ static float high_of(Range a) { return -__uint_as_float(a & 0xffff0000u); }
};
template <>
struct Eight<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    const uint4 x = load_stream(reinterpret_cast<const uint4*>(p)), y = load_stream(reinterpret_cast<const uint4*>(p) + 1);
    a = make_float4(__uint_as_float(x.x), __uint_as_float(x.y), __uint_as_float(x.z), __uint_as_float(x.w));
    b = make_float4(__uint_as_float(y.x), __uint_as_float(y.y), __uint_as_float(y.z), __uint_as_float(y.w));
  }
  __device__ __forceinline__ void floats(float (&x)[8]) const {
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  }
  __device__ __forceinline__ void round(const float (&x)[8]) {
    a = make_float4(x[0], x[1], x[2], x[3]);
    b = make_float4(x[4], x[5], x[6], x[7]);
  }
  __device__ __forceinline__ void store(float* p) const {
    reinterpret_cast<float4*>(p)[0] = a;
    reinterpret_cast<float4*>(p)[1] = b;
  }
  using Range = float2;
  __device__ __forceinline__ static float least(float a, float b) {
    float r;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
  }
  __device__ __forceinline__ Range range() const {
    const float2 x = make_float2(a.x, -a.x), y = make_float2(a.y, -a.y), z = make_float2(a.z, -a.z), w = make_float2(a.w, -a.w);
    const float2 p = make_float2(b.x, -b.x), q = make_float2(b.y, -b.y), r = make_float2(b.z, -b.z), t = make_float2(b.w, -b.w);
    return join(join(join(x, y), join(z, w)), join(join(p, q), join(r, t)));
  }
  __device__ __forceinline__ static Range join(Range a, Range b) { return make_float2(least(a.x, b.x), least(a.y, b.y)); }
  __device__ __forceinline__ static Range other(Range a, int mask) {
    return make_float2(__shfl_xor_sync(0xffffffffu, a.x, mask), __shfl_xor_sync(0xffffffffu, a.y, mask));
  }
  __device__ __forceinline__ static float low_of(Range a) { return a.x; }
  __device__ __forceinline__ static float high_of(Range a) { return -a.y; }
};

// Two fp32 operations in one instruction, each rounded as by itself.
__device__ __forceinline__ uint64_t pair(float x, float y) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
  return r;
}
__device__ __forceinline__ void unpair(uint64_t p, float& x, float& y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(p)); }
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

// What a group of 64 elements is quantised by.
struct CodeScale {
  uint32_t more;                 // step and lowest value, as a page has them: bf16, the step in the lower half
  float inverse;                 // 1 / step
  __device__ __forceinline__ float step() const { return __uint_as_float(more << 16); }
  __device__ __forceinline__ float low() const { return __uint_as_float(more & 0xffff0000u); }
  template <int BITS>
  __device__ __forceinline__ static CodeScale of(float lo, float hi) {
    const bool fine = lo > -kCodeMost && hi < kCodeMost;
    const float low = bf16_down(lo) + 0.f;       // (a zero counts as +0)
    const float step = fmaxf(bf16_up(__fmul_rn(__fsub_rn(hi, low), 1.f / ((1 << BITS) - 1))), kCodeLeast);
    CodeScale s;
    s.more = fine ? __float_as_uint(step) >> 16 | __float_as_uint(low) : 0x7fff7fffu;
    s.inverse = __frcp_rn(step);
    return s;
  }
};

// One unit of codes with its step and lowest value.
template <int BITS>
struct Unit {
  static constexpr int kWords = BITS / 4;
  uint32_t w[kWords];
  float step, low;

  // The eight lanes of a group call this together (and the other lanes of the warp at the same time).
  template <typename T>
  __device__ __forceinline__ CodeScale encode(const Eight<T>& v) {
    auto range = v.range();
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) range = Eight<T>::join(range, Eight<T>::other(range, o));
    const CodeScale by = CodeScale::of<BITS>(Eight<T>::low_of(range), Eight<T>::high_of(range));
    encode(v, by);
    return by;
  }
  template <typename T>
  __device__ __forceinline__ void encode(const Eight<T>& v, const CodeScale& by) {
    step = by.step();
    low = by.low();
    float x[8];
    v.floats(x);
    const uint64_t minus_low = pair(-by.low(), -by.low()), inverse = pair(by.inverse, by.inverse), magic = pair(8388608.f, 8388608.f);
    // The product is a sum with -0, which leaves it as it is, and in words that the compiler does not see through (the inverse is positive): a
    // plain mul.rn.f32x2 it puts together with the sum behind it, into one rounding.
    const float zero = __uint_as_float(~__float_as_uint(by.inverse) & 0x80000000u);
    const uint64_t minus_zero = pair(zero, zero);
    uint32_t u[8];
#pragma unroll
    for (int e = 0; e < 8; e += 2) {             // 2^23 + t: the sum's rounding is rint, its lower bits are the code
      float a, b;
      unpair(add2(fma2(add2(pair(x[e], x[e + 1]), minus_low), inverse, minus_zero), magic), a, b);
      u[e] = __float_as_uint(a);
      u[e + 1] = __float_as_uint(b);
    }
    if constexpr (BITS == 4) {
      // the exponents 0x4b000000 of the first two, shifted, come off again (the others' leave the word)
      w[0] = ((u[0] - 0xfb000000u + (u[1] << 4)) + ((u[2] << 8) + (u[3] << 12))) + (((u[4] << 16) + (u[5] << 20)) + ((u[6] << 24) + (u[7] << 28)));
    } else {
#pragma unroll
      for (int j = 0; j < kWords; ++j)
        w[j] = __byte_perm(__byte_perm(u[4 * j], u[4 * j + 1], 0x0040), __byte_perm(u[4 * j + 2], u[4 * j + 3], 0x0040), 0x5410);
    }
  }
  __device__ __forceinline__ void values(float (&x)[8]) const {
    const uint64_t steps = pair(step, step), lows = pair(low, low), magic = pair(-8388608.f, -8388608.f);
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      uint32_t c[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if constexpr (BITS == 4) c[i] = w[0] >> (4 * (e + i)) & 15u | 0x4b000000u;
        else c[i] = __byte_perm(w[e / 4], 0x4b000000u, 0x7440 | (e + i) % 4);
      }
      unpair(fma2(steps, add2(pair(__uint_as_float(c[0]), __uint_as_float(c[1])), magic), lows), x[e], x[e + 1]);
    }
  }
  // page: a page of one head; r: row in it; u: unit of the row
  template <int D>
  __device__ __forceinline__ void put_codes(unsigned char* page, int r, int u) const {
    using Row = CodedRow<D, BITS>;
    unsigned char* at = page + (size_t)r * Row::kCodes + Row::place(u);
    if constexpr (BITS == 4) *reinterpret_cast<uint32_t*>(at) = w[0];
    else *reinterpret_cast<uint2*>(at) = make_uint2(w[0], w[kWords - 1]);
  }
  template <int D>
  __device__ __forceinline__ static void put_more(unsigned char* page, int page_size, int r, int group, uint32_t value) {
    using Row = CodedRow<D, BITS>;
    unsigned char* more = page + (size_t)page_size * Row::kCodes + (size_t)r * Row::kMore + group * 2;
    *reinterpret_cast<uint16_t*>(more) = (uint16_t)value;
    *reinterpret_cast<uint16_t*>(more + 2 * Row::kGroups) = (uint16_t)(value >> 16);
  }
  template <int D>
  __device__ __forceinline__ void get_codes(const unsigned char* page, int r, int u) {
    using Row = CodedRow<D, BITS>;
    const unsigned char* at = page + (size_t)r * Row::kCodes + Row::place(u);
    if constexpr (BITS == 4) w[0] = __ldg(reinterpret_cast<const uint32_t*>(at));
    else {
      const uint2 x = __ldg(reinterpret_cast<const uint2*>(at));
      w[0] = x.x;
      w[kWords - 1] = x.y;
    }
  }
  template <int D>
  __device__ __forceinline__ static uint32_t get_more(const unsigned char* page, int page_size, int r, int group) {
    using Row = CodedRow<D, BITS>;
    const unsigned char* more = page + (size_t)page_size * Row::kCodes + (size_t)r * Row::kMore + group * 2;
    return (uint32_t)__ldg(reinterpret_cast<const uint16_t*>(more)) |
           (uint32_t)__ldg(reinterpret_cast<const uint16_t*>(more + 2 * Row::kGroups)) << 16;
  }
  __device__ __forceinline__ void scale(uint32_t more) {       // as CodeScale has it
    step = __uint_as_float(more << 16);
    low = __uint_as_float(more & 0xffff0000u);
  }
};

// Running bounds of a lane's unit.
template <typename T>
struct UnitBounds;
template <>
struct UnitBounds<__nv_bfloat16> {
  VecBounds<__nv_bfloat16> b;
  __device__ __forceinline__ void reset() { b.reset(); }
  __device__ __forceinline__ void add(const Eight<__nv_bfloat16>& v) { b.add(v.w); }
  __device__ __forceinline__ void join(int mask) { b.join(mask); }
  __device__ __forceinline__ void put_low(__nv_bfloat16* p) const { *reinterpret_cast<uint4*>(p) = b.low(); }
  __device__ __forceinline__ void put_high(__nv_bfloat16* p) const { *reinterpret_cast<uint4*>(p) = b.high(); }
};
template <>
struct UnitBounds<float> {
  VecBounds<float> b[2];
  __device__ __forceinline__ static uint4 word(const float4& x) {
    return make_uint4(__float_as_uint(x.x), __float_as_uint(x.y), __float_as_uint(x.z), __float_as_uint(x.w));
  }
  __device__ __forceinline__ void reset() { b[0].reset(); b[1].reset(); }
  __device__ __forceinline__ void add(const Eight<float>& v) { b[0].add(word(v.a)); b[1].add(word(v.b)); }
  __device__ __forceinline__ void join(int mask) { b[0].join(mask); b[1].join(mask); }
  __device__ __forceinline__ void put_low(float* p) const {
    reinterpret_cast<uint4*>(p)[0] = b[0].low();
    reinterpret_cast<uint4*>(p)[1] = b[1].low();
  }
  __device__ __forceinline__ void put_high(float* p) const {
    reinterpret_cast<uint4*>(p)[0] = b[0].high();
    reinterpret_cast<uint4*>(p)[1] = b[1].high();
  }
};

enum CodedPass { kCodedStore, kCodedBounds, kCodedLoad };

// kCodedStore: dense rows p.k, p.v into the pages, and the bounds of the keys as they will be read back if p.bounds is there.
// kCodedBounds: those bounds alone, from the pages p.k_pages, from the page of row lens_from on.
// kCodedLoad: rows [lens_from, lens) of the pages into dense rows p.k_rows, p.v_rows, the first of them to row 0.
struct CodedParams {
  const void* k;                 // dense rows to store
  const void* v;
  void* k_rows;                  // dense rows to load into
  void* v_rows;
  unsigned char* k_pages;
  unsigned char* v_pages;
  void* bounds;
  const int32_t* table;
  const int32_t* lens_from;
  const int32_t* lens;
  int* status;
  long long seq_stride, head_stride;     // in elements
  int lens_stride, n_seqs, n_heads, n_pages, width, page_shift, rows_capacity;
};

// Rows [from, rows) of sequence i that a load covers; a length that is no length or too many rows: none, and it is recorded.
__device__ __forceinline__ void load_span(const int32_t* lens_from, const int32_t* lens, int lens_stride, int i, int max_rows,
                                          int capacity, int* status, int& from, int& rows) {
  bool bad = false;
  rows = clamped_len(lens, lens_stride, i, max_rows, bad);
  from = lens_from ? clamped_len(lens_from, lens_stride, i, max_rows, bad) : 0;
  if (bad || rows - from > capacity) {
    if (blockIdx.x == 0) set_status(status, bad ? MEDA_ERR_INVALID_ARG : MEDA_ERR_WORKSPACE);
    rows = 0;
  }
  if (from >= rows) from = rows = 0;
}

// Blocks per SM that the registers are to leave room for.  Storing from bf16, four instead of the two of 104 registers: the 19K-token prompt 83.4 -> 72.8
// us (64 registers, with 24 bytes of spills at 4 bits and 32 at 8; five 81), from fp32 two (120 us, three 146); loading into fp32 three instead of four
// 116 -> 101.5 us, into bf16 no matter.
template <typename T, int BITS, CodedPass PASS>
constexpr int kCodedBlocks = PASS == kCodedStore ? (sizeof(T) == 2 ? 4 : 2) : sizeof(T) == 4 ? 3 : BITS == 4 ? 5 : 4;

// (Several warps to a page where there are fewer pages than warps: a prompt of 592 pages read back 17 -> 11.5 us by itself but 72.3 -> 71.1 behind its
// append, a step of 64 tokens with its reading back 8.5 -> 10.1: more code to fetch.)
template <typename T, int D, int BITS, CodedPass PASS>
__global__ void __launch_bounds__(kRowsThreads, kCodedBlocks<T, BITS, PASS>)
coded_rows_kernel(CodedParams p) {
  begin_grid();
  using Row = CodedRow<D, BITS>;
  constexpr int U = Row::kUnits, kRows = 32 / U;         // lanes on a row, rows a warp covers at once
  constexpr int kBatch = 4;                              // row steps in flight
  extern __shared__ __align__(16) int rows_smem[];
  __shared__ int scratch[kRowsThreads / 32 + 1];
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const int sub = lane / U, unit = lane % U;
  const int page_size = 1 << p.page_shift;
  const int max_rows = p.width << p.page_shift;
  const size_t page_bytes = (size_t)Row::kBytes << p.page_shift;

  auto span = [&](int i, int& from, int& rows) {         // rows [from, rows) of the sequence, from on a page's border unless loading
    if (PASS == kCodedLoad) {
      load_span(p.lens_from, p.lens, p.lens_stride, i, max_rows, p.rows_capacity, p.status, from, rows);
      return;
    }
    bool bad = false;
    rows = clamped_len(p.lens, p.lens_stride, i, max_rows, bad);
    from = 0;
    if (PASS == kCodedStore) {
      if (bad || rows > p.rows_capacity) {
        if (blockIdx.x == 0) set_status(p.status, bad ? MEDA_ERR_INVALID_ARG : MEDA_ERR_WORKSPACE);
        rows = 0;
      }
    } else {
      if (p.lens_from) from = clamped_len(p.lens_from, p.lens_stride, i, max_rows, bad);
      if (bad && blockIdx.x == 0) set_status(p.status, MEDA_ERR_INVALID_ARG);
      if (p.lens_from && p.lens_from[(size_t)i * p.lens_stride] >= rows) from = rows = 0;
      from = from >> p.page_shift << p.page_shift;
    }
  };
  ragged_prefix<kRowsThreads>(p.n_seqs, rows_smem, scratch, [&](int i) {
    int from, rows;
    span(i, from, rows);
    return ((rows + page_size - 1) >> p.page_shift) - (from >> p.page_shift);
  });
  const unsigned total = (unsigned)rows_smem[p.n_seqs] * p.n_heads;              // (below 2^31, as all sequences' tiles together)
  const int warps = gridDim.x * (kRowsThreads / 32);
#pragma unroll 1
  for (unsigned x = blockIdx.x * (kRowsThreads / 32) + warp; x < total; x += warps) {
    const int i = ragged_find(rows_smem, p.n_seqs, (int)(x / (unsigned)p.n_heads));
    const unsigned count = rows_smem[i + 1] - rows_smem[i], local = x - (unsigned)rows_smem[i] * p.n_heads;
    const int g = (int)(local / count);
    int from, rows;
    span(i, from, rows);
    const int col = (from >> p.page_shift) + (int)(local - g * count);
    const int page = p.table[(size_t)i * p.width + col];
    if ((unsigned)page >= (unsigned)p.n_pages) {
      if (lane == 0) set_status(p.status, MEDA_ERR_INVALID_ARG);
      continue;
    }
    const int row0 = col << p.page_shift;                // the page's first row in the sequence
    const int live = min(page_size, rows - row0), first = max(0, from - row0);
    const size_t cell = (size_t)page * p.n_heads + g;
    unsigned char* kpage = p.k_pages + cell * page_bytes;
    unsigned char* vpage = PASS == kCodedBounds ? nullptr : p.v_pages + cell * page_bytes;
    // element (row0 + r, unit) of the dense rows
    const long long dense = i * p.seq_stride + g * p.head_stride + (long long)(row0 - (PASS == kCodedLoad ? from : 0)) * D + unit * 8;
    UnitBounds<T> b;
    b.reset();
#pragma unroll 1
    for (int base = first; base < live; base += kRows * kBatch) {          // (all lanes together: encode() exchanges between them)
      if constexpr (PASS == kCodedStore) {
        static_assert(kBatch == 4, "a group's eight lanes, eight scales");
        Eight<T> x[2 * kBatch];                          // four rows of keys, four of values
        typename Eight<T>::Range range[2 * kBatch];
#pragma unroll
        for (int y = 0; y < kBatch; ++y) {
          const int r = min(base + y * kRows + sub, live - 1);             // behind the last row: that one again, not written
          x[y].load(static_cast<const T*>(p.k) + dense + (long long)r * D);
          x[kBatch + y].load(static_cast<const T*>(p.v) + dense + (long long)r * D);
        }
#pragma unroll
        for (int y = 0; y < 2 * kBatch; ++y) range[y] = x[y].range();
        // each of the group's eight lanes ends up with one of the eight scales, and works it out for all
        const int mine = lane & 7;
#pragma unroll
        for (int half = kBatch; half >= 1; half >>= 1)
#pragma unroll
          for (int y = 0; y < half; ++y) {
            const bool upper = (mine & half) != 0;
            const auto send = upper ? range[y] : range[y + half], keep = upper ? range[y + half] : range[y];
            range[y] = Eight<T>::join(keep, Eight<T>::other(send, half));
          }
        const CodeScale scale = CodeScale::of<BITS>(Eight<T>::low_of(range[0]), Eight<T>::high_of(range[0]));
        const int row = base + mine % kBatch * kRows + sub;
        if (row < live) Unit<BITS>::template put_more<D>(mine < kBatch ? kpage : vpage, page_size, row, unit / 8, scale.more);
#pragma unroll
        for (int y = 0; y < 2 * kBatch; ++y) {
          CodeScale by;
          by.more = __shfl_sync(0xffffffffu, scale.more, (lane & 24) | y);
          by.inverse = __shfl_sync(0xffffffffu, scale.inverse, (lane & 24) | y);
          const int r = base + y % kBatch * kRows + sub;
          Unit<BITS> c;
          c.encode(x[y], by);
          if (r < live) c.template put_codes<D>(y < kBatch ? kpage : vpage, r, unit);
          if (y < kBatch && p.bounds) {                  // (a row met twice changes no bound)
            float f[8];
            c.values(f);
            Eight<T> back;
            back.round(f);
            b.add(back);
          }
        }
      } else {
        constexpr int kItems = PASS == kCodedLoad ? 2 * kBatch : kBatch;           // four rows of keys, and of values if they are wanted
        Unit<BITS> c[kItems];
#pragma unroll
        for (int y = 0; y < kItems; ++y)
          c[y].template get_codes<D>(y < kBatch ? kpage : vpage, min(base + y % kBatch * kRows + sub, live - 1), unit);
        // the scales of a group's eight items, one by each of its lanes
        const int mine = lane & 7;
        const uint32_t more = Unit<BITS>::template get_more<D>(PASS == kCodedLoad && mine >= kBatch ? vpage : kpage, page_size,
                                                               min(base + mine % kBatch * kRows + sub, live - 1), unit / 8);
#pragma unroll
        for (int y = 0; y < kItems; ++y) {
          const int r = base + y % kBatch * kRows + sub;
          c[y].scale(__shfl_sync(0xffffffffu, more, (lane & 24) | y));
          float f[8];
          c[y].values(f);
          Eight<T> back;
          back.round(f);
          if (PASS == kCodedBounds) b.add(back);
          else if (r < live) back.store(static_cast<T*>(y < kBatch ? p.k_rows : p.v_rows) + dense + (long long)r * D);
        }
      }
    }
    if (PASS != kCodedLoad && p.bounds) {
#pragma unroll
      for (int o = U; o < 32; o <<= 1) b.join(o);
      T* bd = static_cast<T*>(p.bounds) + cell * 2 * D + unit * 8;
      if (sub == 0) b.put_low(bd);
      if (sub == kRows - 1) b.put_high(bd + D);
    }
  }
}

// ---- rows of pages that hold them as they are, read back ------------------------------------------------------------------
// VR = 16-byte vectors per row.  Bound by memory: 28 layers of a 19K-token prompt (4 heads of 128), 491 MB in bf16, in 79 us, 95 % of a plain copy, 983 MB
// in fp32 in 156 us, 96 %; the last 33 rows of each 3.9 and 5.3 us.
struct LoadParams {
  const uint4* k_pages;
  const uint4* v_pages;
  uint4* k;
  uint4* v;
  const int32_t* table;
  const int32_t* lens_from;
  const int32_t* lens;
  int* status;
  long long seq_stride, head_stride;     // in 16-byte vectors
  int lens_stride, n_seqs, n_heads, n_pages, width, page_shift, rows_capacity;
};

template <int VR>
__global__ void __launch_bounds__(kRowsThreads)
page_load_kernel(LoadParams p) {
  begin_grid();
  extern __shared__ __align__(16) int rows_smem[];
  __shared__ int scratch[kRowsThreads / 32 + 1];
  constexpr int kBatch = 4;
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const int page_size = 1 << p.page_shift, max_rows = p.width << p.page_shift;
  auto span = [&](int i, int& from, int& rows) {
    load_span(p.lens_from, p.lens, p.lens_stride, i, max_rows, p.rows_capacity, p.status, from, rows);
  };
  ragged_prefix<kRowsThreads>(p.n_seqs, rows_smem, scratch, [&](int i) {
    int from, rows;
    span(i, from, rows);
    return ((rows + page_size - 1) >> p.page_shift) - (from >> p.page_shift);
  });
  const unsigned total = (unsigned)rows_smem[p.n_seqs] * p.n_heads;              // (below 2^31, as all sequences' tiles together)
  const int warps = gridDim.x * (kRowsThreads / 32);
#pragma unroll 1
  for (unsigned x = blockIdx.x * (kRowsThreads / 32) + warp; x < total; x += warps) {
    const int i = ragged_find(rows_smem, p.n_seqs, (int)(x / (unsigned)p.n_heads));
    const unsigned count = rows_smem[i + 1] - rows_smem[i], local = x - (unsigned)rows_smem[i] * p.n_heads;
    const int g = (int)(local / count);
    int from, rows;
    span(i, from, rows);
    const int col = (from >> p.page_shift) + (int)(local - g * count);
    const int page = p.table[(size_t)i * p.width + col];
    if ((unsigned)page >= (unsigned)p.n_pages) {
      if (lane == 0) set_status(p.status, MEDA_ERR_INVALID_ARG);
      continue;
    }
    const int row0 = col << p.page_shift, first = max(0, from - row0);
    const int end = min(page_size, rows - row0) * VR;
    const size_t at = (((size_t)page * p.n_heads + g) << p.page_shift) * VR;
    const long long to = i * p.seq_stride + g * p.head_stride + (long long)(row0 - from) * VR;
    // a page's rows are one run of vectors on both sides
#pragma unroll 1
    for (int e0 = first * VR + lane; e0 < end; e0 += 32 * kBatch) {
      uint4 kx[kBatch], vx[kBatch];
#pragma unroll
      for (int y = 0; y < kBatch; ++y)
        if (e0 + y * 32 < end) {
          kx[y] = load_stream(p.k_pages + at + e0 + y * 32);
          vx[y] = load_stream(p.v_pages + at + e0 + y * 32);
        }
#pragma unroll
      for (int y = 0; y < kBatch; ++y)
        if (e0 + y * 32 < end) {
          p.k[to + e0 + y * 32] = kx[y];
          p.v[to + e0 + y * 32] = vx[y];
        }
    }
  }
}

}  // namespace meda
