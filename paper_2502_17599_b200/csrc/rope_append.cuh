// Rotary positions with three axes, fused with the write of the new rows into their pages.
//
// A frequency f_i = theta^(-i / half) / 2 pi, in turns per position, is below one turn: kept as a 64-bit fraction, its product
// with an int32 position wraps modulo one turn by itself, so the reduction of a far angle is one exact integer
// multiplication (an fp32 angle at position 100,000 would be off by 0.004; 64-bit floating point would cost a slow
// multiply and a conversion).  The signed fraction then goes through sincospi.  A block takes a few tokens, computes
// their sines and cosines once into shared memory (they serve all query and key heads), then its threads stream the heads
// as 16-byte vectors.  Bound by memory bandwidth for prompts (every element read and written once: 18,951 tokens of 28 + 4 + 4 heads,
// 350 MB, in 58.7 us, 92 % of a plain copy; 9,000 in fp32, 332 MB: 56 us), by latency for a step (64 tokens: 2.9 us; 2,000: 7.8 us,
// of which the bytes are 5.7).
#pragma once

#include "pages_common.cuh"
#include "page_rows.cuh"     // load_stream

namespace meda {

constexpr int kRopeThreads = 256;
constexpr int kRopeMaxTokens = 4;        // tokens per block

struct RopeParams {
  const void* q;
  const void* k;
  const void* v;
  const int32_t* positions;
  const int64_t* slots;
  void* q_out;
  void* k_pages;
  void* v_pages;
  const unsigned long long* freq;
  const int* axis;
  int* status;
  long long q_stride, k_stride, v_stride;      // in 16-byte vectors
  long long axis_stride;
  long long n_slots;
  int n_tokens, n_q_heads, n_kv_heads, half, page_shift, tokens_per_block;
};

template <typename T>
struct RopeVec;                          // a 16-byte vector as floats
template <>
struct RopeVec<float> {
  static constexpr int E = 4;
  __device__ __forceinline__ static void unpack(const uint4& x, float (&f)[4]) {
    f[0] = __uint_as_float(x.x); f[1] = __uint_as_float(x.y); f[2] = __uint_as_float(x.z); f[3] = __uint_as_float(x.w);
  }
  __device__ __forceinline__ static uint4 pack(const float (&f)[4]) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  }
};
template <>
struct RopeVec<__nv_bfloat16> {
  static constexpr int E = 8;
  __device__ __forceinline__ static void unpack(const uint4& x, float (&f)[8]) {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      f[2 * e] = __uint_as_float(w[e] << 16);
      f[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
    }
  }
  __device__ __forceinline__ static uint4 pack(const float (&f)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * e], f[2 * e + 1]);
      memcpy(&w[e], &h, 4);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};

// One work item is one vector (or, with paired halves, the two vectors of a pair) of one head of one token:
//   items [0, rot) of a head rotate, the next ones copy what is not rotated.
// D = head_dim.
template <typename T, int D, bool ADJACENT>
__global__ void __launch_bounds__(kRopeThreads)
rope_append_kernel(RopeParams p) {
  constexpr int E = RopeVec<T>::E;
  begin_grid();
  constexpr int VR = D / E;                                    // vectors per head
  // (cos, sin) of the block's tokens: the frequencies an item works on one after the other lie `items` apart, so that neighbouring
  // threads, which have neighbouring items, read neighbouring words (side by side in an item they met in two banks of 32)
  __shared__ float2 turn[kRopeMaxTokens][D / 2];
  constexpr int kPerItem = ADJACENT ? E / 2 : E;
  __shared__ int64_t slot_of[kRopeMaxTokens];
  const int t0 = blockIdx.x * p.tokens_per_block;
  const int n_tok = min(p.tokens_per_block, p.n_tokens - t0);
  const int half = p.positions ? p.half : 0;
  if ((int)threadIdx.x < n_tok) {
    int64_t s = p.slots[t0 + threadIdx.x];
    if (s >= p.n_slots || s < -1) {
      set_status(p.status, MEDA_ERR_INVALID_ARG);
      s = -1;
    }
    slot_of[threadIdx.x] = s;
  }
#pragma unroll 1
  for (int x = threadIdx.x; x < n_tok * half; x += kRopeThreads) {
    const int tok = x / half, i = x - tok * half;
    const long long pos = p.positions[p.axis[i] * p.axis_stride + t0 + tok];
    const long long frac = (long long)((unsigned long long)pos * p.freq[i]);          // turns, as a signed 64-bit fraction
    const float half_turns = (float)(int)(frac >> 32) * 4.656612873077393e-10f;       // 2^-31: twice the turns, for sincospi
    float s, c;
    sincospif(half_turns, &s, &c);
    turn[tok][(i % kPerItem) * (half / kPerItem) + i / kPerItem] = make_float2(c, s);
  }
  __syncthreads();

  // vectors of a head that one rotating item covers, and items per rotated head
  const int rot = ADJACENT ? 2 * half / E : half / E;
  const int per_head = rot + (VR - 2 * half / E);
  const int q_items = p.q ? p.n_q_heads * per_head : 0, k_items = p.n_kv_heads * per_head, v_items = p.n_kv_heads * VR;
  const int per_token = q_items + k_items + v_items;
  const int page_mask = (1 << p.page_shift) - 1;
  for (int x = threadIdx.x; x < n_tok * per_token; x += kRopeThreads) {
    const int tok = x / per_token;
    int item = x - tok * per_token;
    const int64_t slot = slot_of[tok];
    if (slot < 0) continue;
    const int token = t0 + tok;
    const uint4* src;
    uint4* dst;
    const int64_t page = slot >> p.page_shift;
    const int row = (int)(slot & page_mask);
    auto cell = [&](void* pool, int g) {                       // the head's row in its page
      return static_cast<uint4*>(pool) + ((((size_t)page * p.n_kv_heads + g) << p.page_shift) + row) * VR;
    };
    if (item >= q_items + k_items) {                           // a value: copied
      item -= q_items + k_items;
      const int g = item / VR, vec = item % VR;
      cell(p.v_pages, g)[vec] = load_stream(static_cast<const uint4*>(p.v) + token * p.v_stride + g * VR + vec);
      continue;
    }
    if (item < q_items) {
      const int h = item / per_head;
      item -= h * per_head;
      src = static_cast<const uint4*>(p.q) + token * p.q_stride + h * VR;
      dst = static_cast<uint4*>(p.q_out) + ((size_t)token * p.n_q_heads + h) * VR;
    } else {
      item -= q_items;
      const int g = item / per_head;
      item -= g * per_head;
      src = static_cast<const uint4*>(p.k) + token * p.k_stride + g * VR;
      dst = cell(p.k_pages, g);
    }
    if (item >= rot) {                                         // behind the rotated dimensions: copied
      const int vec = 2 * half / E + (item - rot);
      dst[vec] = src[vec];
      continue;
    }
    if (ADJACENT) {
      float f[E];
      RopeVec<T>::unpack(src[item], f);
#pragma unroll
      for (int e = 0; e < E / 2; ++e) {
        const float2 cs = turn[tok][e * rot + item];
        const float a = f[2 * e], b = f[2 * e + 1];
        f[2 * e] = a * cs.x - b * cs.y;
        f[2 * e + 1] = b * cs.x + a * cs.y;
      }
      dst[item] = RopeVec<T>::pack(f);
    } else {
      float a[E], b[E];
      const int other = item + half / E;
      const uint4 xa = src[item], xb = src[other];             // q_out may be q: both are read before either is written
      RopeVec<T>::unpack(xa, a);
      RopeVec<T>::unpack(xb, b);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float2 cs = turn[tok][e * rot + item];
        const float y = a[e] * cs.x - b[e] * cs.y;
        b[e] = b[e] * cs.x + a[e] * cs.y;
        a[e] = y;
      }
      dst[item] = RopeVec<T>::pack(a);
      dst[other] = RopeVec<T>::pack(b);
    }
  }
}

}  // namespace meda
