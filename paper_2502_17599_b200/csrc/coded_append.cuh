// Rotary positions with three axes (see rope_append.cuh), the new rows quantised into their pages.
//
// A key's codes hang on borders, so its rotation is stated step by step: a frequency is the 64-bit fraction of a turn that the handle was made
// with (from fp64: good to 2^-53 of itself), the angle is position times frequency modulo a turn, without rounding, its sine and
// cosine come from 64-bit arithmetic and are rounded to fp32, the two products and their sum are rounded one by one, and the key
// is rounded to the cache's type before it is quantised.  A prompt rotated elsewhere by the same steps gives the same pages, but for a sine or
// cosine so near the middle of two fp32 numbers that the last bits of the 64-bit one decide (one in 10^8).
// (64-bit sines cost 0.8 us of a prompt's 65: a block works each out once for all heads.)
//
// A block takes a few tokens.  Keys and values go by units of eight dimensions, eight neighbouring lanes to a group; a lane reads its
// unit and, with paired halves, the unit's partner (taking it from the other lane by shuffles measured the same).  Queries go by pairs of
// vectors (both read before either is written: q_out may be q).
//
// Bound by memory with its latency: 18,944 tokens of 28 + 4 + 4 heads of 128 at 4 bits, 322 MB, in 60 to 65 us, 76 to 82 % of a plain copy, at 8 bits, 331
// MB, 61 to 65; 9,000 tokens in fp32 at 8 bits, 305 MB, 51.5 us, 90 %; 64 tokens 3.5 us.
// What helps is warps, not loads ahead.  Keys first, and the 32 registers that eight blocks per SM leave: 64.6 -> 62.4 -> 59.8 us (9,000
// tokens in fp32 53.7 -> 50.7); the first units fetched before the sines 65.9, four tokens' units and queries on their way at once, their
// scales shared out among a group's lanes, 74 to 90.  It is the other way with neighbouring pairs in bf16 (40 registers 64.9 us, 32 66.5) and
// where keys and values outweigh the queries (9,000 tokens of 32 + 32 + 32 heads 92 -> 98 us).
#pragma once

#include "page_codes.cuh"
#include "rope_append.cuh"

namespace meda {

template <typename T, int D, int BITS, bool ADJACENT>
__global__ void __launch_bounds__(kRopeThreads, 8)
coded_append_kernel(RopeParams p) {
  constexpr int E = RopeVec<T>::E;
  begin_grid();
  constexpr int VR = D / E, U = D / 8;                         // vectors and units per head
  constexpr int kTurns = ADJACENT ? 4 : 8;                     // frequencies of a unit: they lie half / kTurns apart
  __shared__ float2 turn[kRopeMaxTokens][D / 2];               // (cos, sin) of the block's tokens
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
  const int apart = half / kTurns;
#pragma unroll 1
  for (int x = threadIdx.x; x < n_tok * half; x += kRopeThreads) {
    const int tok = x / half, i = x - tok * half;
    const long long pos = p.positions[p.axis[i] * p.axis_stride + t0 + tok];
    const long long frac = (long long)((unsigned long long)pos * p.freq[i]);          // turns, as a signed 64-bit fraction
    double s, c;
    sincospi((double)frac * 1.0842021724855044e-19, &s, &c);                          // 2^-63: twice the turns
    turn[tok][(i % kTurns) * apart + i / kTurns] = make_float2((float)c, (float)s);
  }
  __syncthreads();

  // ---- keys and values: a whole warp goes round together, its groups of eight lanes are all in or all out
  const int page_size = 1 << p.page_shift;
  const size_t page_bytes = (size_t)CodedRow<D, BITS>::kBytes << p.page_shift;
  const int u = threadIdx.x % U, heads = 2 * p.n_kv_heads;            // keys' heads, then values'
  int tok = 0;
#pragma unroll 1
  for (int head = threadIdx.x / U; ; head += kRopeThreads / U) {
    while (head >= heads && tok < n_tok) {
      head -= heads;
      ++tok;
    }
    const bool there = tok < n_tok;
    if (!__any_sync(0xffffffffu, there)) break;
    if (!there) {                                              // beside lanes that are: the last head again, not written
      tok = n_tok - 1;
      head = heads - 1;
    }
    const bool key = head < p.n_kv_heads;
    const int g = key ? head : head - p.n_kv_heads;
    const int64_t slot = slot_of[tok];
    const T* src = key ? static_cast<const T*>(p.k) + (t0 + tok) * p.k_stride * E : static_cast<const T*>(p.v) + (t0 + tok) * p.v_stride * E;
    src += (size_t)g * D;
    Eight<T> v;
    v.load(src + u * 8);
    if (key && u * 8 < 2 * half) {
      float f[8];
      v.floats(f);
      if (ADJACENT) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 cs = turn[tok][e * apart + u];
          const float a = f[2 * e], b = f[2 * e + 1];
          f[2 * e] = __fsub_rn(__fmul_rn(a, cs.x), __fmul_rn(b, cs.y));
          f[2 * e + 1] = __fadd_rn(__fmul_rn(b, cs.x), __fmul_rn(a, cs.y));
        }
      } else {
        const bool second = u * 8 >= half;
        const int at = second ? u - half / 8 : u;              // the pair's unit in the first half
        Eight<T> o;
        o.load(src + (second ? at : u + half / 8) * 8);
        float y[8];
        o.floats(y);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float2 cs = turn[tok][e * apart + at];
          const float mine = __fmul_rn(f[e], cs.x), other = __fmul_rn(y[e], cs.y);
          f[e] = second ? __fadd_rn(mine, other) : __fsub_rn(mine, other);
        }
      }
      v.round(f);
    }
    Unit<BITS> c;
    const CodeScale by = c.encode(v);
    if (!there) {
      tok = n_tok;
      head = heads;
      continue;
    }
    if (slot < 0) continue;
    unsigned char* pool = static_cast<unsigned char*>(key ? p.k_pages : p.v_pages);
    unsigned char* page = pool + ((size_t)(slot >> p.page_shift) * p.n_kv_heads + g) * page_bytes;
    const int row = (int)(slot & (page_size - 1));
    c.template put_codes<D>(page, row, u);
    if (u % 8 == 0) Unit<BITS>::template put_more<D>(page, page_size, row, u / 8, by.more);
  }
  // ---- queries
  const int rot = ADJACENT ? 2 * half / E : half / E;          // items of a head that rotate
  const int per_head = rot + (VR - 2 * half / E);
  // (indexes go up by what a turn of the block adds to them: divisions in every turn would cost more than the rotation)
  if (p.q) {
    const int turn_heads = kRopeThreads / per_head, turn_items = kRopeThreads % per_head;
    int h = threadIdx.x / per_head, item = threadIdx.x % per_head, tok = 0;
    for (;; h += turn_heads, item += turn_items) {
      if (item >= per_head) {
        item -= per_head;
        ++h;
      }
      while (h >= p.n_q_heads) {
        h -= p.n_q_heads;
        ++tok;
      }
      if (tok >= n_tok) break;
      if (slot_of[tok] < 0) continue;
      const uint4* src = static_cast<const uint4*>(p.q) + (t0 + tok) * p.q_stride + h * VR;
      uint4* dst = static_cast<uint4*>(p.q_out) + ((size_t)(t0 + tok) * p.n_q_heads + h) * VR;
      if (item >= rot) {
        const int vec = 2 * half / E + (item - rot);
        dst[vec] = src[vec];
        continue;
      }
      // the item's frequencies: in fp32 a vector has half a unit's
      const float2* turns = E == 8 ? turn[tok] + item : turn[tok] + (item & 1) * (kTurns / 2) * apart + (item >> 1);
      if (ADJACENT) {
        float f[E];
        RopeVec<T>::unpack(src[item], f);
#pragma unroll
        for (int e = 0; e < E / 2; ++e) {
          const float2 cs = turns[e * apart];
          const float a = f[2 * e], b = f[2 * e + 1];
          f[2 * e] = __fsub_rn(__fmul_rn(a, cs.x), __fmul_rn(b, cs.y));
          f[2 * e + 1] = __fadd_rn(__fmul_rn(b, cs.x), __fmul_rn(a, cs.y));
        }
        dst[item] = RopeVec<T>::pack(f);
      } else {
        float a[E], b[E];
        const int other = item + half / E;
        const uint4 xa = src[item], xb = src[other];
        RopeVec<T>::unpack(xa, a);
        RopeVec<T>::unpack(xb, b);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float2 cs = turns[e * apart];
          const float y = __fsub_rn(__fmul_rn(a[e], cs.x), __fmul_rn(b[e], cs.y));
          b[e] = __fadd_rn(__fmul_rn(b[e], cs.x), __fmul_rn(a[e], cs.y));
          a[e] = y;
        }
        dst[item] = RopeVec<T>::pack(a);
        dst[other] = RopeVec<T>::pack(b);
      }
    }
  }

}

}  // namespace meda
