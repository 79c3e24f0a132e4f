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
  __device__ __forceinline__ void extremes(float& lo, float& hi) const {         // a NaN wins
    VecBounds<__nv_bfloat16> b;
    b.reset();
    b.add(w);
    const __nv_bfloat162 l = __hmin2_nan(__hmin2_nan(b.lo[0], b.lo[1]), __hmin2_nan(b.lo[2], b.lo[3]));
    const __nv_bfloat162 h = __hmax2_nan(__hmax2_nan(b.hi[0], b.hi[1]), __hmax2_nan(b.hi[2], b.hi[3]));
    lo = __bfloat162float(__hmin_nan(l.x, l.y));
    hi = __bfloat162float(__hmax_nan(h.x, h.y));
  }
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
  __device__ __forceinline__ void extremes(float& lo, float& hi) const {
    float x[8];
    floats(x);
    lo = hi = x[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) {
      lo = min_nan(lo, x[e]);
      hi = max_nan(hi, x[e]);
    }
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
  __device__ __forceinline__ void encode(const Eight<T>& v) {
    float lo, hi;
    v.extremes(lo, hi);
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) {
      lo = min_nan(lo, __shfl_xor_sync(0xffffffffu, lo, o));
      hi = max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    }
    const bool fine = lo > -kCodeMost && hi < kCodeMost;
    low = fine ? bf16_down(lo) : NAN;
    step = fmaxf(bf16_up(__fmul_rn(__fsub_rn(hi, low), 1.f / ((1 << BITS) - 1))), kCodeLeast);
    if (!fine) step = NAN;
    const float inv = __frcp_rn(step);
    float x[8];
    v.floats(x);
    uint32_t u[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)                  // 2^23 + t: the sum's rounding is rint, its lower bits are the code
      u[e] = __float_as_uint(__fadd_rn(__fmul_rn(__fsub_rn(x[e], low), inv), 8388608.f));
    if constexpr (BITS == 4) {
      w[0] = 0u - 0xfb000000u;                   // the exponents 0x4b000000 of the first two, shifted (the others' leave the word)
#pragma unroll
      for (int e = 0; e < 8; ++e) w[0] += u[e] << (4 * e);
    } else {
#pragma unroll
      for (int j = 0; j < kWords; ++j) {
        w[j] = 0u - 0x4b000000u;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[j] += u[4 * j + e] << (8 * e);
      }
    }
  }
  __device__ __forceinline__ void values(float (&x)[8]) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t code = BITS == 4 ? w[0] >> (4 * e) & 15u : w[e / 4] >> (8 * (e % 4)) & 255u;
      x[e] = fmaf(step, __uint_as_float(0x4b000000u | code) - 8388608.f, low);
    }
  }
  // page: a page of one head; r: row in it; u: unit of the row
  template <int D>
  __device__ __forceinline__ void put(unsigned char* page, int page_size, int r, int u) const {
    using Row = CodedRow<D, BITS>;
    unsigned char* at = page + (size_t)r * Row::kCodes + Row::place(u);
    if constexpr (BITS == 4) *reinterpret_cast<uint32_t*>(at) = w[0];
    else *reinterpret_cast<uint2*>(at) = make_uint2(w[0], w[kWords - 1]);
    if (u % 8 == 0) {
      unsigned char* more = page + (size_t)page_size * Row::kCodes + (size_t)r * Row::kMore + (u / 8) * 2;
      *reinterpret_cast<uint16_t*>(more) = (uint16_t)(__float_as_uint(step) >> 16);
      *reinterpret_cast<uint16_t*>(more + 2 * Row::kGroups) = (uint16_t)(__float_as_uint(low) >> 16);
    }
  }
  template <int D>
  __device__ __forceinline__ void get(const unsigned char* page, int page_size, int r, int u) {
    using Row = CodedRow<D, BITS>;
    const unsigned char* at = page + (size_t)r * Row::kCodes + Row::place(u);
    if constexpr (BITS == 4) w[0] = __ldg(reinterpret_cast<const uint32_t*>(at));
    else {
      const uint2 x = __ldg(reinterpret_cast<const uint2*>(at));
      w[0] = x.x;
      w[kWords - 1] = x.y;
    }
    const unsigned char* more = page + (size_t)page_size * Row::kCodes + (size_t)r * Row::kMore + (u / 8) * 2;
    step = __uint_as_float((uint32_t)__ldg(reinterpret_cast<const uint16_t*>(more)) << 16);
    low = __uint_as_float((uint32_t)__ldg(reinterpret_cast<const uint16_t*>(more + 2 * Row::kGroups)) << 16);
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

template <typename T, int D, int BITS, CodedPass PASS>
__global__ void __launch_bounds__(kRowsThreads)
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
  const long long total = (long long)rows_smem[p.n_seqs] * p.n_heads;
  const int warps = gridDim.x * (kRowsThreads / 32);
#pragma unroll 1
  for (long long x = (long long)blockIdx.x * (kRowsThreads / 32) + warp; x < total; x += warps) {
    const int i = ragged_find(rows_smem, p.n_seqs, (int)(x / p.n_heads));
    const int count = rows_smem[i + 1] - rows_smem[i];
    const long long local = x - (long long)rows_smem[i] * p.n_heads;
    const int g = (int)(local / count);
    int from, rows;
    span(i, from, rows);
    const int col = (from >> p.page_shift) + (int)(local % count);
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
        Eight<T> kx[kBatch], vx[kBatch];
#pragma unroll
        for (int y = 0; y < kBatch; ++y) {
          const int r = min(base + y * kRows + sub, live - 1);             // behind the last row: that one again, not written
          kx[y].load(static_cast<const T*>(p.k) + dense + (long long)r * D);
          vx[y].load(static_cast<const T*>(p.v) + dense + (long long)r * D);
        }
#pragma unroll
        for (int y = 0; y < kBatch; ++y) {
          const int r = base + y * kRows + sub;
          if (base + y * kRows >= live) break;
          Unit<BITS> c;
          c.encode(kx[y]);
          if (r < live) c.template put<D>(kpage, page_size, r, unit);
          if (p.bounds) {                                // (a row met twice changes no bound)
            float f[8];
            c.values(f);
            Eight<T> back;
            back.round(f);
            b.add(back);
          }
          c.encode(vx[y]);
          if (r < live) c.template put<D>(vpage, page_size, r, unit);
        }
      } else {
        Unit<BITS> kc[kBatch], vc[kBatch];
#pragma unroll
        for (int y = 0; y < kBatch; ++y) {
          const int r = min(base + y * kRows + sub, live - 1);
          kc[y].template get<D>(kpage, page_size, r, unit);
          if (PASS == kCodedLoad) vc[y].template get<D>(vpage, page_size, r, unit);
        }
#pragma unroll
        for (int y = 0; y < kBatch; ++y) {
          const int r = base + y * kRows + sub;
          float f[8];
          Eight<T> back;
          kc[y].values(f);
          back.round(f);
          if (PASS == kCodedBounds) b.add(back);
          else if (r < live) {
            back.store(static_cast<T*>(p.k_rows) + dense + (long long)r * D);
            vc[y].values(f);
            back.round(f);
            back.store(static_cast<T*>(p.v_rows) + dense + (long long)r * D);
          }
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
// VR = 16-byte vectors per row.
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
  const long long total = (long long)rows_smem[p.n_seqs] * p.n_heads;
  const int warps = gridDim.x * (kRowsThreads / 32);
#pragma unroll 1
  for (long long x = (long long)blockIdx.x * (kRowsThreads / 32) + warp; x < total; x += warps) {
    const int i = ragged_find(rows_smem, p.n_seqs, (int)(x / p.n_heads));
    const int count = rows_smem[i + 1] - rows_smem[i];
    const long long local = x - (long long)rows_smem[i] * p.n_heads;
    const int g = (int)(local / count);
    int from, rows;
    span(i, from, rows);
    const int col = (from >> p.page_shift) + (int)(local % count);
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
