// Host side of the paged caches: the handle and the launches behind meda_pages_* and the calls that take a meda_pages
// (declared in include/meda.h).  Included by meda.cu, which owns the entry points' visibility.
#pragma once

#include <math.h>
#include <stdint.h>
#include <string.h>

#include <algorithm>
#include <atomic>
#include <new>

#include "page_rows.cuh"
#include "page_tables.cuh"
#include "paged_attention.cuh"
#include "pages_common.cuh"
#include "rope_append.cuh"
#include "select_pages.cuh"

namespace {

using namespace meda;

// Makes the handle's device current for one call.
struct PagesDevice {
  int before = -1;
  bool ok = false, switched = false;
  explicit PagesDevice(const meda_pages* p) {
    if (cudaGetDevice(&before) != cudaSuccess) return;
    if (before != p->device) {
      if (cudaSetDevice(p->device) != cudaSuccess) return;
      switched = true;
    }
    ok = true;
  }
  ~PagesDevice() {
    if (switched) cudaSetDevice(before);
  }
};

// A launch that may be set up before the kernels ahead of it in the stream have finished (they and it start with begin_grid).
template <typename K, typename P>
meda_status launch_after(meda_pages* p, K kernel, dim3 grid, int block, size_t smem, cudaStream_t st, const P& params) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)block);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr = {};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  ++p->launches;
  if (cudaLaunchKernelEx(&cfg, kernel, params) == cudaSuccess) return MEDA_OK;
  cudaGetLastError();
  return MEDA_ERR_CUDA;
}

inline bool aligned16(const void* x) { return (reinterpret_cast<uintptr_t>(x) & 15u) == 0; }

// raise_dyn_smem, once for each kernel and device: a server makes handles while others are in use.
template <auto kernel>
meda_status raise_once() {
  static std::atomic<unsigned long long> done{0};              // a bit per device, up to 64 of them
  int device = 0;
  MEDA_CUDA_TRY(cudaGetDevice(&device));
  if (device < 64 && (done.load(std::memory_order_acquire) >> device & 1u)) return MEDA_OK;
  const meda_status r = raise_dyn_smem(kernel);
  if (r == MEDA_OK && device < 64) done.fetch_or(1ull << device, std::memory_order_release);
  return r;
}

int pages_element(const meda_pages* p) { return p->cfg.dtype == MEDA_F32 ? 4 : 2; }

// meda_* status of the arguments every call over sequences shares.
meda_status pages_batch_ok(const meda_pages* p, int32_t n_seqs, int32_t lens_stride) {
  if (n_seqs < 0 || lens_stride < 0) return MEDA_ERR_INVALID_ARG;
  return n_seqs > p->cfg.max_seqs ? MEDA_ERR_SHAPE : MEDA_OK;
}

// ---- attention ---------------------------------------------------------------------------------
template <typename Tile, int D, int W>
struct AttnKernel {
  static constexpr auto kernel = paged_attention_kernel<Tile, D, W>;
  static size_t smem(int n_seqs) { return (size_t)(attn_prefix_floats(n_seqs) + 2 * attn_merge_floats(W, Tile::kHeads, D)) * 4; }
  // One block per SM, with the shared memory of the largest batch.
  static meda_status prepare(meda_pages* p) {
    if (smem(p->cfg.max_seqs) > (size_t)kMaxDynSmem - 1024) return MEDA_ERR_SHAPE;
    // tiles of all segments, and as many again for the look-ahead, are counted in 32 bits
    const int64_t segments = (int64_t)p->cfg.n_kv_heads * ((p->group + Tile::kHeads - 1) / Tile::kHeads);
    if (segments * p->cfg.max_seqs * ((int64_t)p->cfg.max_seq_pages * (p->cfg.page_size / kAttTile) + kAttSegment) >= (int64_t(1) << 31) - 65536)
      return MEDA_ERR_SHAPE;
    p->attn_blocks = p->sm_count;
    return raise_once<kernel>();
  }
  static meda_status launch(meda_pages* p, AttnParams a, cudaStream_t st) {
    a.heads_div.set((unsigned)(a.n_heads * ((a.group + Tile::kHeads - 1) / Tile::kHeads)));
    a.grid_div.set((unsigned)p->attn_blocks);
    const meda_status r = launch_after(p, kernel, p->attn_blocks, W * 32, smem(a.n_seqs), st, a);
    if (r != MEDA_OK) return r;
    return launch_after(p, join_attention_kernel<typename Tile::T, D>, dim3(p->attn_blocks, std::min(a.group, Tile::kHeads)), kAttJoinThreads,
                        0, st, a);
  }
};

// Calls f with the AttnKernel for the handle's geometry.  Warps per block: what the registers of one block per SM allow.
// At head_dim 128, eight warps against twelve, replayed from a graph: 947 rows 7.1 and 7.6 us, 4,000 rows 8.0 and 8.5, 129,072 rows 50.5
// and 48.8, 64 sequences of 36 to 18,944 rows 76 and 71.4; twelve are taken for the long ones.
// At head_dim 256 a warp works on eight rows at a time: sixteen fill 224 registers before any temporary, and with the warps' states
// beside them what is in flight no longer fits the L1 (400 MB, 7 heads per KV head: sixteen 98.1 us, eight 78.6; 947 rows 10.4 and
// 9.0).  Elsewhere sixteen are better (head_dim 128: 67.8 and 80.2, the softmax's steps are per turn).
// (More than eight query heads per KV head at head_dim 256 take two segments: the accumulators of sixteen do not fit.)
template <typename F>
meda_status with_attn_kernel(const meda_pages* p, F f) {
  const int d = p->cfg.head_dim, g = p->group;
  if (p->cfg.dtype == MEDA_BF16) {
    if (d == 64) return g <= 8 ? f(AttnKernel<AttnTileBf16<64, 1>, 64, 16>()) : f(AttnKernel<AttnTileBf16<64, 2>, 64, 16>());
    if (d == 128) return g <= 8 ? f(AttnKernel<AttnTileBf16<128, 1>, 128, 12>()) : f(AttnKernel<AttnTileBf16<128, 2>, 128, 8>());
    return f(AttnKernel<AttnTileBf16<256, 1, 8>, 256, 8>());
  }
  if (d == 64)
    return g == 1 ? f(AttnKernel<AttnTileF32<64, 1>, 64, 16>()) : g == 2 ? f(AttnKernel<AttnTileF32<64, 2>, 64, 16>())
         : g <= 4 ? f(AttnKernel<AttnTileF32<64, 4>, 64, 16>()) : f(AttnKernel<AttnTileF32<64, 8>, 64, 16>());
  if (d == 128)
    return g == 1 ? f(AttnKernel<AttnTileF32<128, 1>, 128, 16>()) : g == 2 ? f(AttnKernel<AttnTileF32<128, 2>, 128, 16>())
         : g <= 4 ? f(AttnKernel<AttnTileF32<128, 4>, 128, 8>()) : f(AttnKernel<AttnTileF32<128, 8>, 128, 8>());
  return g == 1 ? f(AttnKernel<AttnTileF32<256, 1>, 256, 8>()) : g == 2 ? f(AttnKernel<AttnTileF32<256, 2>, 256, 8>())
                                                                       : f(AttnKernel<AttnTileF32<256, 4>, 256, 8>());
}

// ---- selection of pages ------------------------------------------------------------------------
template <typename T, int D, int GP>
struct SelectPagesKernels {
  static meda_status prepare() {
    meda_status r = raise_once<page_scores_kernel<T, D, GP>>();
    if (r == MEDA_OK) r = raise_once<choose_pages_kernel<T, D, 256>>();
    return r == MEDA_OK ? raise_once<choose_pages_kernel<T, D, 1024>>() : r;
  }
  static meda_status launch(meda_pages* p, const SelectPagesParams& a, cudaStream_t st) {
    // fp32 scores are bound by 64-bit arithmetic and want twice the warps (and no third block on an SM: see tables_smem)
    const int blocks = sizeof(T) == 4 ? 2 : 1;
    const size_t seqs = (size_t)(a.n_seqs + 1) * 4;
    const meda_status r = launch_after(p, page_scores_kernel<T, D, GP>, p->sm_count * blocks, kPscoreThreads,
                                       blocks == 2 ? std::max<size_t>(seqs, 77 * 1024) : seqs, st, a);
    if (r != MEDA_OK) return r;
    // a large block where it has an SM to itself, four small ones to an SM where there are more pairs than SMs
    const int pairs = a.n_seqs * a.n_heads;
    const size_t smem = choose_smem(a.width, a.group, D);
    return pairs <= p->sm_count ? launch_after(p, choose_pages_kernel<T, D, 1024>, pairs, 1024, smem, st, a)
                                : launch_after(p, choose_pages_kernel<T, D, 256>, pairs, 256, smem, st, a);
  }
};

template <typename T, int D, typename F>
meda_status with_select_group(const meda_pages* p, F f) {
  const int g = p->group;
  if constexpr (sizeof(T) == 2) {
    return g <= 8 ? f(SelectPagesKernels<T, D, 8>()) : f(SelectPagesKernels<T, D, 16>());
  } else {
    return g == 1 ? f(SelectPagesKernels<T, D, 1>()) : g <= 4 ? f(SelectPagesKernels<T, D, 4>())
         : g <= 8 ? f(SelectPagesKernels<T, D, 8>()) : f(SelectPagesKernels<T, D, 16>());
  }
}

template <typename F>
meda_status with_select_kernels(const meda_pages* p, F f) {
  const int d = p->cfg.head_dim;
  if (p->cfg.dtype == MEDA_BF16)
    return d == 64 ? with_select_group<__nv_bfloat16, 64>(p, f) : d == 128 ? with_select_group<__nv_bfloat16, 128>(p, f)
                                                                         : with_select_group<__nv_bfloat16, 256>(p, f);
  return d == 64 ? with_select_group<float, 64>(p, f) : d == 128 ? with_select_group<float, 128>(p, f)
                                                                 : with_select_group<float, 256>(p, f);
}

// Scratch of the selection: one sequence's scores and their bounds, in floats, and how many sequences it holds (at least
// one, more while that stays below 8 MB; a larger batch goes through it in several launches).
int64_t select_seq_floats(const meda_pages_config& c) {
  return (int64_t)c.n_kv_heads * ((c.max_seq_pages + 3) / 4 * 4 + 4 * pscore_units(c.max_seq_pages));
}
int select_scratch_seqs(const meda_pages_config& c) {
  return (int)std::max<int64_t>(1, std::min<int64_t>(c.max_seqs, (int64_t(8) << 20) / 4 / select_seq_floats(c)));
}

// ---- pages of rows -----------------------------------------------------------------------------
template <bool STORE>
meda_status launch_page_rows(meda_pages* p, const RowsParams& a, cudaStream_t st) {
  const int vr = p->cfg.head_dim * pages_element(p) / 16;
  // Copies want many blocks, which come and go (16 per SM: 80.8 us for the 506 MB of a 19K-token prompt's layers, 4: 86, 32: 80.4, but
  // then 8.7 instead of 5.3 us for a tiny one); the bounds of a step have little to do and want few.
  const int blocks = p->sm_count * (STORE ? 16 : 4);
  auto go = [&](auto kernel) { return launch_after(p, kernel, blocks, kRowsThreads, (size_t)(a.n_seqs + 1) * 4, st, a); };
  if (p->cfg.dtype == MEDA_F32)
    return vr == 16 ? go(page_rows_kernel<float, 16, STORE>) : vr == 32 ? go(page_rows_kernel<float, 32, STORE>)
                                                                        : go(page_rows_kernel<float, 64, STORE>);
  return vr == 8 ? go(page_rows_kernel<__nv_bfloat16, 8, STORE>) : vr == 16 ? go(page_rows_kernel<__nv_bfloat16, 16, STORE>)
                                                                           : go(page_rows_kernel<__nv_bfloat16, 32, STORE>);
}

// (32 KB of prefixes at most: below the limit every kernel starts with)
static_assert((kPagesMaxSeqs + 1) * 4 <= 48 * 1024, "page_rows_kernel would have to raise its shared memory");

template <typename T, bool ADJACENT>
meda_status launch_rope(meda_pages* p, const RopeParams& a, int grid, cudaStream_t st) {
  auto go = [&](auto kernel) { return launch_after(p, kernel, grid, kRopeThreads, 0, st, a); };
  const int d = p->cfg.head_dim;
  return d == 64 ? go(rope_append_kernel<T, 64, ADJACENT>) : d == 128 ? go(rope_append_kernel<T, 128, ADJACENT>)
                                                                    : go(rope_append_kernel<T, 256, ADJACENT>);
}

void pages_release(meda_pages* p) {
  cudaFree(p->slab);
  delete p;
}

}  // namespace

#pragma GCC visibility push(default)
extern "C" {

meda_status meda_pages_create(const meda_pages_config* config, meda_pages** out) {
  if (out) *out = nullptr;
  if (!config || !out) return MEDA_ERR_INVALID_ARG;
  const meda_pages_config& c = *config;
  if (c.dtype != MEDA_BF16 && c.dtype != MEDA_F32) return MEDA_ERR_INVALID_ARG;
  if (c.rope_order != MEDA_ROPE_RUNS && c.rope_order != MEDA_ROPE_DEALT) return MEDA_ERR_INVALID_ARG;
  if (c.rope_pairing != MEDA_ROPE_HALVES && c.rope_pairing != MEDA_ROPE_ADJACENT) return MEDA_ERR_INVALID_ARG;
  if (!(c.rope_theta > 1.0) || !(c.rope_theta < 1e300)) return MEDA_ERR_INVALID_ARG;
  if (c.n_q_heads < 1 || c.n_kv_heads < 1 || c.n_q_heads % c.n_kv_heads != 0 || c.n_q_heads / c.n_kv_heads > 16 ||
      c.n_kv_heads > 1024)
    return MEDA_ERR_SHAPE;
  if (c.head_dim != 64 && c.head_dim != 128 && c.head_dim != 256) return MEDA_ERR_SHAPE;
  if (c.page_size < 16 || c.page_size > 256 || (c.page_size & (c.page_size - 1)) != 0) return MEDA_ERR_SHAPE;
  if (c.n_pages < 1 || c.max_seqs < 1 || c.max_seqs > kPagesMaxSeqs || c.max_seq_pages < 1 || c.max_seq_pages > kPagesMaxSeqPages)
    return MEDA_ERR_SHAPE;
  if ((int64_t)c.max_seqs * c.max_seq_pages * (c.page_size / 16) * c.n_kv_heads >= (int64_t(1) << 31) ||
      (int64_t)c.n_pages * c.n_kv_heads * c.page_size >= (int64_t(1) << 40))
    return MEDA_ERR_SHAPE;
  int64_t half = 0;
  for (int a = 0; a < 3; ++a) {
    if (c.rope_sections[a] < 0 || c.rope_sections[a] > c.head_dim / 2) return MEDA_ERR_SHAPE;
    half += c.rope_sections[a];
  }
  if (half < 8 || half % 8 != 0 || half > c.head_dim / 2) return MEDA_ERR_SHAPE;
  int axis[128];
  for (int i = 0; i < (int)half; ++i) {
    if (c.rope_order == MEDA_ROPE_RUNS)
      axis[i] = i < c.rope_sections[0] ? 0 : (i < c.rope_sections[0] + c.rope_sections[1] ? 1 : 2);
    else
      axis[i] = i % 3 == 1 && i < 3 * c.rope_sections[1] ? 1 : (i % 3 == 2 && i < 3 * c.rope_sections[2] ? 2 : 0);
  }
  for (int a = 1; a < 3; ++a)                                  // dealt out: every section must find its places
    if (std::count(axis, axis + half, a) != c.rope_sections[a]) return MEDA_ERR_SHAPE;
  unsigned long long freq[128];
  for (int i = 0; i < (int)half; ++i)                          // below one turn per position: 2^64 / 2 pi at most
    freq[i] = (unsigned long long)(pow(c.rope_theta, -(double)i / (double)half) / 6.283185307179586476925 * 18446744073709551616.0);

  meda_pages* p = new (std::nothrow) meda_pages();
  if (!p) return MEDA_ERR_CUDA;
  p->cfg = c;
  p->group = c.n_q_heads / c.n_kv_heads;
  p->page_shift = 4;
  while ((1 << p->page_shift) < c.page_size) ++p->page_shift;
  meda_status st = MEDA_OK;
  if (cudaGetDevice(&p->device) != cudaSuccess ||
      cudaDeviceGetAttribute(&p->sm_count, cudaDevAttrMultiProcessorCount, p->device) != cudaSuccess)
    st = MEDA_ERR_CUDA;
  if (st == MEDA_OK) st = with_attn_kernel(p, [&](auto k) { return k.prepare(p); });
  if (st == MEDA_OK) st = with_select_kernels(p, [](auto k) { return k.prepare(); });
  if (st == MEDA_OK) st = raise_once<page_tables_kernel>();
  if (st == MEDA_OK) {
    // one allocation: [status | frequencies | axes | splits | states | scores]; the first three from the host, the others need no start
    const auto up = [](int64_t x) { return (x + 255) / 256 * 256; };
    const int64_t freq_at = 256, axis_at = freq_at + up(half * 8), split_at = axis_at + up(half * 4);
    const int64_t partial_at = split_at + up((int64_t)p->attn_blocks * (int64_t)sizeof(int4));
    const int64_t scores_at = partial_at + up((int64_t)p->attn_blocks * 2 * attn_state_floats(p->group, c.head_dim) * 4);
    const int64_t bytes = scores_at + up(select_seq_floats(c) * select_scratch_seqs(c) * 4);
    alignas(8) unsigned char host[256 + 1024 + 512] = {0};
    memcpy(host + freq_at, freq, (size_t)half * 8);
    memcpy(host + axis_at, axis, (size_t)half * 4);
    char* slab = nullptr;
    if (cudaMalloc(reinterpret_cast<void**>(&slab), (size_t)bytes) != cudaSuccess) st = MEDA_ERR_CUDA;
    else {
      p->slab = slab;
      p->bytes = bytes;
      p->status = reinterpret_cast<int*>(slab);
      p->rope_freq = reinterpret_cast<unsigned long long*>(slab + freq_at);
      p->rope_axis = reinterpret_cast<int*>(slab + axis_at);
      p->attn_split = reinterpret_cast<int4*>(slab + split_at);
      p->attn_partial = reinterpret_cast<float*>(slab + partial_at);
      p->select_scratch = reinterpret_cast<float*>(slab + scores_at);
      if (cudaMemcpy(slab, host, (size_t)split_at, cudaMemcpyHostToDevice) != cudaSuccess || cudaStreamSynchronize(nullptr) != cudaSuccess)
        st = MEDA_ERR_CUDA;
    }
  }
  if (st != MEDA_OK) {
    pages_release(p);
    cudaGetLastError();
    return st;
  }
  *out = p;
  return MEDA_OK;
}

void meda_pages_destroy(meda_pages* pages) {
  if (pages) pages_release(pages);
}

int64_t meda_pages_workspace_bytes(const meda_pages* pages) { return pages ? pages->bytes : 0; }

int64_t meda_pages_launch_count(const meda_pages* pages) { return pages ? pages->launches : 0; }

meda_status meda_pages_poll_status(meda_pages* pages, void* stream) {
  if (!pages) return MEDA_ERR_INVALID_ARG;
  PagesDevice dev(pages);
  if (!dev.ok) return MEDA_ERR_CUDA;
  // on `stream` alone: work on the default stream would wait for other streams, and a clearing still under way there could
  // take the error of the next call with it
  int code = 0;
  MEDA_CUDA_TRY(cudaMemcpyAsync(&code, pages->status, sizeof(int), cudaMemcpyDeviceToHost, as_stream(stream)));
  MEDA_CUDA_TRY(cudaStreamSynchronize(as_stream(stream)));
  if (code != 0) {
    MEDA_CUDA_TRY(cudaMemsetAsync(pages->status, 0, sizeof(int), as_stream(stream)));
    MEDA_CUDA_TRY(cudaStreamSynchronize(as_stream(stream)));
  }
  return (meda_status)code;
}

meda_status meda_page_tables(meda_pages* pages, const int32_t* lens, int32_t lens_stride, const int32_t* new_lens,
                             int32_t new_stride, int32_t n_seqs, int32_t* free_pages, const int32_t* free_top,
                             int32_t* free_top_out, int32_t* table, int32_t* cu_new, int64_t* slots,
                             int64_t slots_capacity, void* stream) {
  if (!pages || !free_pages || !free_top || !free_top_out || !cu_new) return MEDA_ERR_INVALID_ARG;
  if (free_top == free_top_out || slots_capacity < 0 || new_stride < 0) return MEDA_ERR_INVALID_ARG;
  if (slots_capacity > INT32_MAX) return MEDA_ERR_SHAPE;
  const meda_status r = pages_batch_ok(pages, n_seqs, lens_stride);
  if (r != MEDA_OK) return r;
  if ((n_seqs > 0 && (!new_lens || !table)) || (slots_capacity > 0 && !slots)) return MEDA_ERR_INVALID_ARG;
  if (slots_capacity == 0) slots = nullptr;
  PagesDevice dev(pages);
  if (!dev.ok) return MEDA_ERR_CUDA;
  const meda_pages_config& c = pages->cfg;
  TablesParams a = {lens, new_lens, free_pages, free_top, free_top_out, table, cu_new, slots, pages->status,
                    lens_stride, new_stride, n_seqs, c.n_pages, c.max_seq_pages, pages->page_shift, (int)slots_capacity};
  // every page that gets rows is a lane's; the warps that hold them are spread over blocks, two to each, one block per SM at most
  // (each block repeats the scans)
  const int64_t units = slots_capacity ? (slots_capacity >> pages->page_shift) + 2 * (int64_t)n_seqs
                                       : std::min<int64_t>(c.n_pages, (int64_t)n_seqs * c.max_seq_pages);
  const int grid = (int)std::min<int64_t>(pages->sm_count, std::max<int64_t>(1, (units + 63) / 64));
  return launch_after(pages, page_tables_kernel, grid, kTabThreads, tables_smem(n_seqs), as_stream(stream), a);
}

meda_status meda_page_store(meda_pages* pages, const void* k, const void* v, int64_t seq_stride, int64_t head_stride,
                            int32_t rows_capacity, const int32_t* lens, int32_t lens_stride, int32_t n_seqs,
                            const int32_t* table, void* k_pages, void* v_pages, void* bounds, void* stream) {
  if (!pages || rows_capacity < 0 || seq_stride < 0 || head_stride < 0) return MEDA_ERR_INVALID_ARG;
  const meda_status r = pages_batch_ok(pages, n_seqs, lens_stride);
  if (r != MEDA_OK || n_seqs == 0) return r;
  if ((rows_capacity > 0 && (!k || !v)) || !lens || !table || !k_pages || !v_pages) return MEDA_ERR_INVALID_ARG;
  const meda_pages_config& c = pages->cfg;
  const int e = 16 / pages_element(pages);
  if (!aligned16(k) || !aligned16(v) || !aligned16(k_pages) || !aligned16(v_pages) || !aligned16(bounds) || seq_stride % e != 0 ||
      head_stride % e != 0)
    return MEDA_ERR_SHAPE;
  PagesDevice dev(pages);
  if (!dev.ok) return MEDA_ERR_CUDA;
  RowsParams a = {k, v, k_pages, v_pages, bounds, table, nullptr, lens, pages->status, seq_stride / e, head_stride / e,
                  lens_stride, n_seqs, c.n_kv_heads, c.n_pages, c.max_seq_pages, pages->page_shift, rows_capacity};
  return launch_page_rows<true>(pages, a, as_stream(stream));
}

meda_status meda_page_bounds(meda_pages* pages, const void* k_pages, const int32_t* table, const int32_t* lens_from,
                             const int32_t* lens, int32_t lens_stride, int32_t n_seqs, void* bounds, void* stream) {
  if (!pages) return MEDA_ERR_INVALID_ARG;
  const meda_status r = pages_batch_ok(pages, n_seqs, lens_stride);
  if (r != MEDA_OK || n_seqs == 0) return r;
  if (!k_pages || !table || !lens || !bounds) return MEDA_ERR_INVALID_ARG;
  if (!aligned16(k_pages) || !aligned16(bounds)) return MEDA_ERR_SHAPE;
  PagesDevice dev(pages);
  if (!dev.ok) return MEDA_ERR_CUDA;
  const meda_pages_config& c = pages->cfg;
  RowsParams a = {k_pages, nullptr, nullptr, nullptr, bounds, table, lens_from, lens, pages->status, 0, 0,
                  lens_stride, n_seqs, c.n_kv_heads, c.n_pages, c.max_seq_pages, pages->page_shift, 0};
  return launch_page_rows<false>(pages, a, as_stream(stream));
}

meda_status meda_rope_append(meda_pages* pages, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                             const void* v, int64_t v_stride, const int32_t* positions, int64_t axis_stride,
                             const int64_t* slots, int32_t n_tokens, void* q_out, void* k_pages, void* v_pages,
                             void* stream) {
  if (!pages || n_tokens < 0 || q_stride < 0 || k_stride < 0 || v_stride < 0 || axis_stride < 0) return MEDA_ERR_INVALID_ARG;
  if (n_tokens == 0) return MEDA_OK;
  if (!k || !v || !slots || !k_pages || !v_pages || (q == nullptr) != (q_out == nullptr)) return MEDA_ERR_INVALID_ARG;
  const meda_pages_config& c = pages->cfg;
  const int e = 16 / pages_element(pages);
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(q_out) || !aligned16(k_pages) || !aligned16(v_pages) ||
      q_stride % e != 0 || k_stride % e != 0 || v_stride % e != 0)
    return MEDA_ERR_SHAPE;
  if (q && q == q_out && n_tokens > 1 && q_stride != (int64_t)c.n_q_heads * c.head_dim) return MEDA_ERR_INVALID_ARG;
  PagesDevice dev(pages);
  if (!dev.ok) return MEDA_ERR_CUDA;
  const int half = c.rope_sections[0] + c.rope_sections[1] + c.rope_sections[2];
  // one token per block while there are fewer tokens than the GPU holds blocks, else enough of them to
  // share the block's start
  const int tokens = (int)std::min<int64_t>(kRopeMaxTokens, std::max<int64_t>(1, n_tokens / (pages->sm_count * 8)));
  RopeParams a = {q, k, v, positions, slots, q_out, k_pages, v_pages, pages->rope_freq, pages->rope_axis, pages->status,
                  q_stride / e, k_stride / e, v_stride / e, axis_stride, (long long)c.n_pages << pages->page_shift,
                  n_tokens, c.n_q_heads, c.n_kv_heads, half, pages->page_shift, tokens};
  const int grid = (int)(((int64_t)n_tokens + tokens - 1) / tokens);
  cudaStream_t st = as_stream(stream);
  const bool adjacent = c.rope_pairing == MEDA_ROPE_ADJACENT;
  if (c.dtype == MEDA_F32) return adjacent ? launch_rope<float, true>(pages, a, grid, st) : launch_rope<float, false>(pages, a, grid, st);
  return adjacent ? launch_rope<__nv_bfloat16, true>(pages, a, grid, st) : launch_rope<__nv_bfloat16, false>(pages, a, grid, st);
}

meda_status meda_select_pages(meda_pages* pages, const void* q, const void* bounds, const int32_t* table,
                              const int32_t* lens, int32_t lens_stride, int32_t n_seqs, int32_t n_first, int32_t n_last,
                              int32_t keep, int32_t* sel, void* stream) {
  if (!pages || keep < 1 || n_first < 0 || n_last < 0 || (int64_t)n_first + n_last > keep) return MEDA_ERR_INVALID_ARG;
  const meda_status r = pages_batch_ok(pages, n_seqs, lens_stride);
  if (r != MEDA_OK || n_seqs == 0) return r;
  if (!q || !bounds || !table || !lens || !sel) return MEDA_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(bounds)) return MEDA_ERR_SHAPE;
  PagesDevice dev(pages);
  if (!dev.ok) return MEDA_ERR_CUDA;
  const meda_pages_config& c = pages->cfg;
  const int some = select_scratch_seqs(c), e = pages_element(pages);
  for (int i = 0; i < n_seqs; i += some) {
    const int count = std::min(some, n_seqs - i);
    float* scores = pages->select_scratch;
    SelectPagesParams a = {static_cast<const char*>(q) + (size_t)i * c.n_q_heads * c.head_dim * e, bounds,
                           table + (size_t)i * c.max_seq_pages, lens + (size_t)i * lens_stride, sel + (size_t)i * c.n_kv_heads * keep,
                           scores, reinterpret_cast<float4*>(scores + (int64_t)some * c.n_kv_heads * ((c.max_seq_pages + 3) / 4 * 4)), pages->status, lens_stride, count,
                           c.n_kv_heads, pages->group, c.n_pages, c.max_seq_pages, pages->page_shift, keep, n_first, n_last, {}};
    a.heads_div.set((unsigned)c.n_kv_heads);
    const meda_status done = with_select_kernels(pages, [&](auto kern) { return kern.launch(pages, a, as_stream(stream)); });
    if (done != MEDA_OK) return done;
  }
  return MEDA_OK;
}

meda_status meda_paged_attention(meda_pages* pages, const void* q, const void* k_pages, const void* v_pages,
                                 const int32_t* table, const int32_t* lens, int32_t lens_stride, int32_t n_seqs,
                                 const int32_t* sel, int32_t keep, void* out, float* lse, void* stream) {
  if (!pages || (sel && keep < 1)) return MEDA_ERR_INVALID_ARG;
  const meda_status r = pages_batch_ok(pages, n_seqs, lens_stride);
  if (r != MEDA_OK || n_seqs == 0) return r;
  if (!q || !k_pages || !v_pages || !table || !lens || !out) return MEDA_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(k_pages) || !aligned16(v_pages) || !aligned16(out)) return MEDA_ERR_SHAPE;
  PagesDevice dev(pages);
  if (!dev.ok) return MEDA_ERR_CUDA;
  const meda_pages_config& c = pages->cfg;
  AttnParams a = {q, k_pages, v_pages, table, lens, sel, out, lse, pages->attn_partial, pages->attn_split, pages->status,
                  lens_stride, n_seqs, c.n_kv_heads, pages->group, c.n_pages, c.max_seq_pages, pages->page_shift, keep,
                  1.4426950408889634f / sqrtf((float)c.head_dim), {}, {}};
  return with_attn_kernel(pages, [&](auto kern) { return kern.launch(pages, a, as_stream(stream)); });
}

}  // extern "C"
#pragma GCC visibility pop
