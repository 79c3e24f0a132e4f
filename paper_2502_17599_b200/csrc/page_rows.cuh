// Rows of dense caches into pages, and the key bounds of pages.
//
// A page of one head is contiguous on both sides (page_size rows of head_dim elements), so a warp moves it as
// 16-byte vectors, K and V together; lane l always meets the same dimensions, so the running minimum and maximum of
// the keys stay in its registers while they pass through and cost no second read.  The pages of all sequences
// and heads form one list (sequence, head, page) that the warps of a grid of fixed size share out.
// Bound by memory bandwidth: 2 reads and 2 writes per element, 2 / page_size of a row more for the bounds.  The 28 layers of a
// 19K-token prompt (506 MB) take 80.9 us, 6.3 TB/s or 97 % of a plain copy; the bounds of one step's pages 2.6 us.
#pragma once

#include "pages_common.cuh"

namespace meda {

constexpr int kRowsThreads = 256;

// Minimum and maximum that a NaN wins.
__device__ __forceinline__ float min_nan(float a, float b) { return a != a || b != b ? NAN : fminf(a, b); }
__device__ __forceinline__ float max_nan(float a, float b) { return a != a || b != b ? NAN : fmaxf(a, b); }

// Running elementwise (min, max) of 16-byte vectors of T.
template <typename T>
struct VecBounds;
template <>
struct VecBounds<float> {
  float lo[4], hi[4];
  __device__ __forceinline__ void reset() {
#pragma unroll
    for (int e = 0; e < 4; ++e) { lo[e] = INFINITY; hi[e] = -INFINITY; }
  }
  __device__ __forceinline__ void add(const uint4& x) {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float v = __uint_as_float(w[e]);
      lo[e] = min_nan(lo[e], v);
      hi[e] = max_nan(hi[e], v);
    }
  }
  __device__ __forceinline__ void join(int mask) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      lo[e] = min_nan(lo[e], __shfl_xor_sync(0xffffffffu, lo[e], mask));
      hi[e] = max_nan(hi[e], __shfl_xor_sync(0xffffffffu, hi[e], mask));
    }
  }
  __device__ __forceinline__ uint4 low() const {
    return make_uint4(__float_as_uint(lo[0]), __float_as_uint(lo[1]), __float_as_uint(lo[2]), __float_as_uint(lo[3]));
  }
  __device__ __forceinline__ uint4 high() const {
    return make_uint4(__float_as_uint(hi[0]), __float_as_uint(hi[1]), __float_as_uint(hi[2]), __float_as_uint(hi[3]));
  }
};
template <>
struct VecBounds<__nv_bfloat16> {
  __nv_bfloat162 lo[4], hi[4];
  __device__ __forceinline__ static __nv_bfloat162 pair(uint32_t w) {
    __nv_bfloat162 r;
    memcpy(&r, &w, 4);
    return r;
  }
  __device__ __forceinline__ static uint32_t word(__nv_bfloat162 v) {
    uint32_t r;
    memcpy(&r, &v, 4);
    return r;
  }
  __device__ __forceinline__ void reset() {
#pragma unroll
    for (int e = 0; e < 4; ++e) { lo[e] = pair(0x7f807f80u); hi[e] = pair(0xff80ff80u); }     // +inf, -inf
  }
  __device__ __forceinline__ void add(const uint4& x) {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      lo[e] = __hmin2_nan(lo[e], pair(w[e]));
      hi[e] = __hmax2_nan(hi[e], pair(w[e]));
    }
  }
  __device__ __forceinline__ void join(int mask) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      lo[e] = __hmin2_nan(lo[e], pair(__shfl_xor_sync(0xffffffffu, word(lo[e]), mask)));
      hi[e] = __hmax2_nan(hi[e], pair(__shfl_xor_sync(0xffffffffu, word(hi[e]), mask)));
    }
  }
  __device__ __forceinline__ uint4 low() const { return make_uint4(word(lo[0]), word(lo[1]), word(lo[2]), word(lo[3])); }
  __device__ __forceinline__ uint4 high() const { return make_uint4(word(hi[0]), word(hi[1]), word(hi[2]), word(hi[3])); }
};

__device__ __forceinline__ uint4 load_stream(const uint4* p) {       // read once: keep it out of the L1
  uint4 r;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p));
  return r;
}

struct RowsParams {
  const void* k;                 // store: dense caches; bounds: the key pool
  const void* v;
  void* k_pages;
  void* v_pages;
  void* bounds;
  const int32_t* table;
  const int32_t* lens_from;      // bounds only
  const int32_t* lens;
  int* status;
  long long seq_stride, head_stride;     // in 16-byte vectors
  int lens_stride, n_seqs, n_heads, n_pages, width, page_shift, rows_capacity;
};

// STORE: copies pages [0, pages of the sequence); otherwise bounds alone, from page lens_from / page_size on.
// VR = 16-byte vectors per row.
template <typename T, int VR, bool STORE>
__global__ void __launch_bounds__(kRowsThreads)
page_rows_kernel(RowsParams p) {
  begin_grid();
  extern __shared__ __align__(16) int rows_smem[];
  __shared__ int scratch[kRowsThreads / 32 + 1];
  constexpr int kCols = VR > 32 ? VR / 32 : 1;           // vectors of a row per lane
  constexpr int kLanes = VR > 32 ? 32 : VR;              // lanes side by side on a row
  constexpr int kRows = 32 / kLanes;                     // rows a warp covers at once
  constexpr int kBatch = 16 / kRows < 8 ? 16 / kRows : 8;        // row steps in flight (page_size >= 16 rows)
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const int sub = lane / kLanes, vec = lane % kLanes;
  const int page_size = 1 << p.page_shift;
  const int max_rows = p.width << p.page_shift;

  // first page and one past the last page of sequence i that this call covers
  auto span = [&](int i, int& from, int& rows) {
    bool bad = false;
    rows = clamped_len(p.lens, p.lens_stride, i, max_rows, bad);
    from = 0;
    if (STORE) {
      if (bad || rows > p.rows_capacity) {
        if (blockIdx.x == 0) set_status(p.status, bad ? MEDA_ERR_INVALID_ARG : MEDA_ERR_WORKSPACE);
        rows = 0;
      }
    } else {
      if (p.lens_from) from = min(clamped_len(p.lens_from, p.lens_stride, i, max_rows, bad), rows) >> p.page_shift;
      if (p.lens_from && p.lens_from[(size_t)i * p.lens_stride] >= rows) from = (rows + page_size - 1) >> p.page_shift;
      if (bad && blockIdx.x == 0) set_status(p.status, MEDA_ERR_INVALID_ARG);
    }
  };
  ragged_prefix<kRowsThreads>(p.n_seqs, rows_smem, scratch, [&](int i) {
    int from, rows;
    span(i, from, rows);
    return ((rows + page_size - 1) >> p.page_shift) - from;
  });
  const long long total = (long long)rows_smem[p.n_seqs] * p.n_heads;
  const int warps = gridDim.x * (kRowsThreads / 32);
#pragma unroll 1
  for (long long u = (long long)blockIdx.x * (kRowsThreads / 32) + warp; u < total; u += warps) {
    const int i = ragged_find(rows_smem, p.n_seqs, (int)(u / p.n_heads));
    const int count = rows_smem[i + 1] - rows_smem[i];
    const long long local = u - (long long)rows_smem[i] * p.n_heads;
    const int g = (int)(local / count);
    int from, rows;
    span(i, from, rows);
    const int col = from + (int)(local % count);
    const int page = p.table[(size_t)i * p.width + col];
    if ((unsigned)page >= (unsigned)p.n_pages) {
      if (lane == 0) set_status(p.status, MEDA_ERR_INVALID_ARG);
      continue;
    }
    const int live = min(page_size, rows - (col << p.page_shift));
    const size_t at = ((size_t)page * p.n_heads + g) << p.page_shift;             // first row of (page, head) in the pool
    const uint4* ks;
    const uint4* vs = nullptr;
    uint4* kd = nullptr;
    uint4* vd = nullptr;
    if (STORE) {
      const long long src = i * p.seq_stride + g * p.head_stride + ((long long)col << p.page_shift) * VR;
      ks = static_cast<const uint4*>(p.k) + src;
      vs = static_cast<const uint4*>(p.v) + src;
      kd = static_cast<uint4*>(p.k_pages) + at * VR;
      vd = static_cast<uint4*>(p.v_pages) + at * VR;
    } else {
      ks = static_cast<const uint4*>(p.k) + at * VR;
    }
#pragma unroll
    for (int c = 0; c < kCols; ++c) {
      VecBounds<T> b;
      b.reset();
      const int v0 = c * 32 + vec;
#pragma unroll 1
      for (int r0 = sub; r0 < live; r0 += kRows * kBatch) {
        uint4 kx[kBatch], vx[kBatch];
#pragma unroll
        for (int x = 0; x < kBatch; ++x) {
          const int r = r0 + x * kRows;
          if (r < live) {
            kx[x] = load_stream(ks + (size_t)r * VR + v0);
            if (STORE) vx[x] = load_stream(vs + (size_t)r * VR + v0);
          }
        }
#pragma unroll
        for (int x = 0; x < kBatch; ++x) {
          const int r = r0 + x * kRows;
          if (r < live) {
            b.add(kx[x]);
            if (STORE) {
              kd[(size_t)r * VR + v0] = kx[x];
              vd[(size_t)r * VR + v0] = vx[x];
            }
          }
        }
      }
      if (p.bounds) {
#pragma unroll
        for (int o = kLanes; o < 32; o <<= 1) b.join(o);
        uint4* bd = static_cast<uint4*>(p.bounds) + ((size_t)page * p.n_heads + g) * 2 * VR + v0;
        if (sub == 0) bd[0] = b.low();
        if (sub == kRows - 1) bd[VR] = b.high();
      }
    }
  }
}

}  // namespace meda
