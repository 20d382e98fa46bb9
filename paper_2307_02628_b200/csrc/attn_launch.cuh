// The cache object, and the launches of attention over it: kernel choice and how the keys are split.  Part of skipdecode.cu and attn_scores.cu, each of which
// has its own copy of what is in the unnamed namespace.
#pragma once
#include <algorithm>
#include <cmath>
#include <mutex>
#include <type_traits>

#include "../../include/skipdecode.h"
#include "attn_chunk.cuh"
#include "attn_four.cuh"
#include "attn_paged.cuh"
#include "paged.cuh"

struct sd_cache {
  std::mutex busy;           // held while a call enqueues: the launches of one call share a workspace and stay together
  sd_cache_config cfg;
  int row_bytes, page_shift, group, device, sm_count;            // row_bytes: of a (token, head) in the pool
  bool scaled, four;
  char* arena;
  cudaStream_t stream;
  size_t layer_bytes, v_off, ks_off, vs_off, kb_off, vb_off;   // K pool, V pool, K and V scales, K and V block scales: offsets within a layer
  size_t minus_pos, last_row, part_acc, part_ml, part_used, counters, status_off, total;
  size_t plan, claim, copy_from, copy_to, place, totals;         // workspace of the calls on pages
  sd::EncodeTiledFn encode = nullptr;
  int tile_blocks[2][18] = {};          // blocks per SM of each form of the kernel for few rows, without and with changed scores
  int64_t launches = 0;      // kernels launched
  bool copy_ready = false;   // the same for the kernel that copies pages
  bool test_expire = false;  // test hook: the next launch for chunks makes a wait run out (one shot)
  unsigned long long tile_ready[2] = {};   // bit per kernel whose shared-memory size has been allowed on this device
  char* layer(int l) const { return arena + (size_t)l * layer_bytes; }
  template <typename T> T* at(size_t off) const { return reinterpret_cast<T*>(arena + off); }
  int* status() const { return at<int>(status_off); }
};

namespace {

using bf16 = __nv_bfloat16;

constexpr int kPartSlots = 32768;      // 17 MB of head size 128
// Positions that a table may reach.  Key numbers are 32-bit in the kernels, which round them up to whole tiles and look table entries
// up some thousands of keys ahead: sums of a position below this and of such distances, or of two positions, do not wrap.
constexpr int64_t kMostPositions = 1 << 30;

bool wide(const sd_heads* t) {                                  // 16-byte accesses to eight elements at a time
  const int64_t e = t->dtype == SD_DTYPE_FP32 ? 4 : 2;
  return reinterpret_cast<uintptr_t>(t->data) % 16 == 0 && t->row_stride * e % 16 == 0 && t->head_stride * e % 16 == 0;
}

sd::Rows rows_of(const sd_heads* t) { return sd::Rows{t->data, t->row_stride, t->head_stride, t->dtype}; }

sd::BatchView view_of(const sd_cache* c, const sd_batch* b) {
  return sd::BatchView{b->pages, b->first, b->len, b->n_seqs, b->pages_per_seq, b->n_tokens, b->max_new,
                       c->cfg.n_pages, c->cfg.page_len, c->page_shift, c->cfg.n_kv_heads, c->status()};
}

template <typename TC> struct LayerPools { TC *k, *v; float *ks, *vs; uint8_t *kb, *vb; };
template <typename TC>
LayerPools<TC> pools(const sd_cache* c, int l) {
  char* p = c->layer(l);
  return {reinterpret_cast<TC*>(p), reinterpret_cast<TC*>(p + c->v_off), c->scaled ? reinterpret_cast<float*>(p + c->ks_off) : nullptr,
          c->scaled ? reinterpret_cast<float*>(p + c->vs_off) : nullptr,
          c->four ? reinterpret_cast<uint8_t*>(p + c->kb_off) : nullptr, c->four ? reinterpret_cast<uint8_t*>(p + c->vb_off) : nullptr};
}

// Calls f with a value of the cache's element type, resp. the rows' element type, resp. the head size as a constant.
template <typename F> int with_cache_type(int dtype, F f) {
  switch (dtype) {
    case SD_DTYPE_FP32: return f(float{});
    case SD_DTYPE_BF16: return f(bf16{});
    case SD_DTYPE_INT8: return f(int8_t{});
    case SD_DTYPE_E2M1: return f(sd::e2m1{});
    default: return f(sd::e4m3{});
  }
}
template <typename F> int with_row_type(int dtype, F f) {
  return dtype == SD_DTYPE_FP32 ? f(float{}) : dtype == SD_DTYPE_BF16 ? f(bf16{}) : f(__half{});
}
template <typename F> int with_head_dim(int hd, F f) {
  return hd == 128 ? f(std::integral_constant<int, 128>{}) : hd == 64 ? f(std::integral_constant<int, 64>{}) : f(std::integral_constant<int, 32>{});
}

int launched(sd_cache* c, int n = 1) {
  c->launches += n;
  return cudaGetLastError() == cudaSuccess ? SD_OK : SD_ERR_CUDA;
}

// Keys per split for `units` blocks over up to max_len keys each, `rows` rows of partial results in all, `slots` blocks at a time on the device.
// All of them should have work, and the last wave should not be long: three single tokens over 50 000..61 000 positions in
// bf16 take 120 us with 12 splits (288 blocks, 296 slots), 135 with 18, 149 with 32; splitting stops at 256 keys, below which
// a block's start and end outweigh its walk.
int pick_split(long slots, long units, long rows, int64_t max_len) {
  int best = 1;
  double best_cost = 1e30;
  for (int splits = 1; splits <= 512; splits = splits < 4 ? splits + 1 : splits + splits / 4) {
    const int64_t chunk = (max_len + splits * 64 - 1) / (splits * 64) * 64;
    if (splits > 1 && (chunk < 256 || rows * splits > kPartSlots || units > kPartSlots)) break;
    const double waves = (double)((units * splits + slots - 1) / slots);
    const double cost = waves * (chunk + 160);
    if (cost < best_cost * 0.999) { best_cost = cost; best = splits; }
  }
  return (int)std::min<int64_t>((max_len + best * 64 - 1) / (best * 64) * 64, 0x7fffffc0);
}

// The tensor core's additions truncate, so that a sum over many keys comes out smaller; joining splits rounds to nearest.  Where results are fp32 a split has
// no more than this many keys, as far as there is room for the partial results: 1000 single rows of 5 heads over 65 536 positions in bf16 were 1.5e-5 off in one.
constexpr int64_t kSumKeys = 8192;
int split_sums(int chunk, long units, long rows, int64_t max_len) {
  if (chunk <= kSumKeys || units > kPartSlots) return chunk;
  const int64_t splits = std::min<int64_t>((max_len + kSumKeys - 1) / kSumKeys, kPartSlots / rows);
  return splits < 2 ? chunk : (int)std::min<int64_t>(chunk, (max_len + splits * 64 - 1) / (splits * 64) * 64);
}

// Bound on the keys that a block of `rows` query rows goes over.  A window leaves, beside its own length, a token for each row (tokens of one head) and
// the rounding of the first key to a tile.
int most_keys(const sd_cache* c, const sd_batch* b, const sd::Scores& sc, int rows) {
  const int64_t len = b->max_len > 0 ? b->max_len : (int64_t)b->pages_per_seq * c->cfg.page_len;
  return (int)(sc.window > 0 && !sc.hi ? std::min(len, (int64_t)sc.window + rows + 128) : len);
}

// Sequences of rows_below query rows per key head or more are left out (another kernel takes them).
template <typename TC> constexpr int kTypeIndex = std::is_same<TC, bf16>::value ? 0 : std::is_same<TC, int8_t>::value ? 1 : std::is_same<TC, sd::e4m3>::value ? 2 : 4;

template <typename TC, int HD, bool THIRD, bool SC>
int attention_tiles(sd_cache* c, int l, const sd_batch* b, const sd_heads* q, float scale_log2, const sd_heads* out, const sd::Scores& sc, int64_t rows_below, bool early = false) {
  using S = sd::ap::Shape<TC, HD>;
  constexpr int index = (HD == 128 ? 0 : HD == 64 ? 1 : 2) + 3 * (THIRD ? 3 : kTypeIndex<TC>);
  constexpr unsigned long long bit = 1ull << index;
  auto kernel = sd::paged_attn_tile_kernel<TC, HD, THIRD, SC>;
  if (!(c->tile_ready[SC] & bit)) {
    int per_sm = 0;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM) != cudaSuccess ||
        cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout, 100) != cudaSuccess ||
        cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, sd::ap::THREADS, S::SMEM) != cudaSuccess) { cudaGetLastError(); return SD_ERR_CUDA; }
    c->tile_blocks[SC][index] = std::max(per_sm, 1);
    c->tile_ready[SC] |= bit;
  }
  const auto P = pools<TC>(c, l);
  const int64_t most = std::min((int64_t)b->max_new * c->group, rows_below - 1);       // rows of a sequence that this launch takes
  const int tiles = (int)((most + sd::ap::ROWS - 1) / sd::ap::ROWS), slot_rows = (int)std::min<int64_t>(most, sd::ap::ROWS);
  const int64_t units = (int64_t)tiles * c->cfg.n_kv_heads * b->n_seqs;
  if (units > 0x7fffffff) return SD_ERR_ARG;
  const int max_len = most_keys(c, b, sc, sd::ap::ROWS);
  int chunk = pick_split((long)c->tile_blocks[SC][index] * c->sm_count, (long)units, (long)units * slot_rows, max_len);
  if (out->dtype == SD_DTYPE_FP32) chunk = split_sums(chunk, (long)units, (long)units * slot_rows, max_len);
  const int splits = (int)(((int64_t)max_len + chunk - 1) / chunk);
  sd::launch_kernel(early, c->stream, kernel, dim3((unsigned)units, splits), dim3(sd::ap::THREADS), S::SMEM,
      view_of(c, b), rows_of(q), rows_of(out), (const TC*)P.k, (const TC*)P.v, (const float*)P.ks, (const float*)P.vs, c->group, scale_log2, wide(q),
      tiles, (int)std::min<int64_t>(rows_below, 0x7fffffff), chunk, slot_rows, c->at<float>(c->part_acc), c->at<float>(c->part_ml), c->at<int>(c->counters), early, sc);
  return launched(c);
}

// The same over a cache in 4 bits.  A weight enters as one fp16 where queries and results are bf16, else as two.
template <int HD, bool FINE, bool SC>
int attention_four(sd_cache* c, int l, const sd_batch* b, const sd_heads* q, float scale_log2, const sd_heads* out, const sd::Scores& sc, int64_t rows_below, bool early) {
  using S = sd::a4::Shape<HD>;
  constexpr int index = 12 + (HD == 128 ? 0 : HD == 64 ? 1 : 2) + (FINE ? 3 : 0);
  auto kernel = sd::paged_attn_four_kernel<HD, FINE, SC>;
  if (!(c->tile_ready[SC] >> index & 1u)) {
    int per_sm = 0;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM) != cudaSuccess ||
        cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout, 100) != cudaSuccess ||
        cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, sd::a4::THREADS, S::SMEM) != cudaSuccess) { cudaGetLastError(); return SD_ERR_CUDA; }
    c->tile_blocks[SC][index] = std::max(per_sm, 1);
    c->tile_ready[SC] |= 1ull << index;
  }
  const auto P = pools<sd::e2m1>(c, l);
  const int64_t most = std::min((int64_t)b->max_new * c->group, rows_below - 1);       // rows of a sequence that this launch takes
  const int tiles = (int)((most + sd::a4::ROWS - 1) / sd::a4::ROWS), slot_rows = (int)std::min<int64_t>(most, sd::a4::ROWS);
  const int64_t units = (int64_t)tiles * c->cfg.n_kv_heads * b->n_seqs;
  if (units > 0x7fffffff) return SD_ERR_ARG;
  const int max_len = most_keys(c, b, sc, sd::a4::ROWS);
  int chunk = pick_split((long)c->tile_blocks[SC][index] * c->sm_count, (long)units, (long)units * slot_rows, max_len);
  if (out->dtype == SD_DTYPE_FP32) chunk = split_sums(chunk, (long)units, (long)units * slot_rows, max_len);
  const int splits = (int)(((int64_t)max_len + chunk - 1) / chunk);
  sd::launch_kernel(early, c->stream, kernel, dim3((unsigned)units, splits), dim3(sd::a4::THREADS), S::SMEM,
      view_of(c, b), rows_of(q), rows_of(out), (const sd::e2m1*)P.k, (const sd::e2m1*)P.v, (const float*)P.ks, (const float*)P.vs, (const uint8_t*)P.kb, (const uint8_t*)P.vb, c->group,
      scale_log2, wide(q), tiles, (int)std::min<int64_t>(rows_below, 0x7fffffff), chunk, slot_rows, c->at<float>(c->part_acc), c->at<float>(c->part_ml), c->at<int>(c->counters),
      early, sc);
  return launched(c);
}

// The kernel for few rows that a call's types take.
template <typename TC, int HD, bool SC>
int attention_few(sd_cache* c, int l, const sd_batch* b, const sd_heads* q, float scale_log2, const sd_heads* out, const sd::Scores& sc, int64_t rows_below, bool early = false) {
  if constexpr (sd::kFour<TC>) {
    return q->dtype == SD_DTYPE_BF16 && out->dtype == SD_DTYPE_BF16 ? attention_four<HD, false, SC>(c, l, b, q, scale_log2, out, sc, rows_below, early)
                                                                    : attention_four<HD, true, SC>(c, l, b, q, scale_log2, out, sc, rows_below, early);
  } else {
    if constexpr (std::is_same<TC, bf16>::value) {
      if (out->dtype == SD_DTYPE_FP32) return attention_tiles<TC, HD, true, SC>(c, l, b, q, scale_log2, out, sc, rows_below, early);
    }
    return attention_tiles<TC, HD, false, SC>(c, l, b, q, scale_log2, out, sc, rows_below, early);
  }
}

// A bf16 pool as [n_pages * n_kv_heads][page_len][HD], boxes of one page by 64 elements (128 bytes, swizzled).
template <int HD>
bool pool_map(const sd_cache* c, void* pool, CUtensorMap* out) {
  const int64_t planes = (int64_t)c->cfg.n_pages * c->cfg.n_kv_heads;
  if (!c->encode || planes > 0x7fffffff) return false;          // coordinates are 32-bit
  const cuuint64_t dims[3] = {HD, (cuuint64_t)c->cfg.page_len, (cuuint64_t)planes};
  const cuuint64_t strides[2] = {HD * 2, (cuuint64_t)c->cfg.page_len * HD * 2};
  const cuuint32_t box[3] = {64, (cuuint32_t)c->cfg.page_len, 1}, estr[3] = {1, 1, 1};
  return c->encode(out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, pool, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                   CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The same for the kernel for chunks, one block per SM, in units of what a key costs it (17 ns for 256 rows).  A block's start and
// end cost as much as 450 keys, 800 where it leaves a share of its rows, and the joining launch 480 (8 us).  Measured, unsplit and as
// chosen: 64 new tokens of 32 heads over 8 key heads at position 60 000 in bf16 902 and 83 us (16 splits); 512 at 30 000 467 and
// 257 (2); 256 tokens of 32 heads at 4096 in int8 82 and 36 (4); 300 of 32 heads at 1500 33 us whole, 35 in 2.
// No more than 32 splits, one per lane of the warp that joins them.
constexpr int64_t kNoSplit = 0x7fffff80;
int64_t pick_chunk_split(int64_t slots, int64_t units, int64_t rows, int64_t max_len) {
  int64_t best = kNoSplit, best_cost = (units + slots - 1) / slots * (max_len + 450);
  for (int splits = 2; splits <= 32 && rows * splits <= kPartSlots; ++splits) {
    const int64_t chunk = (max_len + splits * 128 - 1) / (splits * 128) * 128;
    const int64_t cost = (units * splits + slots - 1) / slots * (chunk + 800) + 480;
    if (cost < best_cost) { best_cost = cost; best = chunk; }
  }
  return best;
}

template <typename TC, int HD, bool PAIRS, bool SC>
int attention_chunks(sd_cache* c, int l, const sd_batch* b, const sd_heads* q, float scale_log2, const sd_heads* out, const sd::Scores& sc, int rows_from, bool* split) {
  using L = sd::ac::Layout<HD, PAIRS>;
  constexpr unsigned long long bit = 1ull << (32 + (HD == 128 ? 0 : 1) + 2 * (kTypeIndex<TC> == 4 ? 3 : kTypeIndex<TC>) + (PAIRS ? 8 : 0));
  auto kernel = sd::paged_attn_chunk_kernel<TC, HD, PAIRS, SC>;
  if (!(c->tile_ready[SC] & bit)) {
    cudaFuncAttributes attr;                 // the warpgroups redistribute what the block is launched with: it must be that much
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, L::SMEM) != cudaSuccess ||
        cudaFuncGetAttributes(&attr, kernel) != cudaSuccess || attr.numRegs != sd::ac::LAUNCH_REGS) { cudaGetLastError(); return SD_ERR_CUDA; }
    c->tile_ready[SC] |= bit;
  }
  const auto P = pools<TC>(c, l);
  CUtensorMap mk = {}, mv = {};
  const int use_maps = std::is_same<TC, bf16>::value && pool_map<HD>(c, P.k, &mk) && pool_map<HD>(c, P.v, &mv);
  const int blocks = (int)(((int64_t)b->max_new * c->group + L::ROWS - 1) / L::ROWS);
  const int64_t grid = (int64_t)blocks * c->cfg.n_kv_heads * b->n_seqs;
  if (grid > 0x7fffffff) return SD_ERR_ARG;
  // blocks that can have rows: max_new is a bound for every sequence, n_tokens one for all of them
  const int64_t units = std::min(grid, ((int64_t)b->n_tokens * c->group / L::ROWS + b->n_seqs) * c->cfg.n_kv_heads);
  const int64_t rows = (int64_t)b->n_tokens * c->cfg.n_heads;
  const int64_t max_len = most_keys(c, b, sc, L::ROWS);
  const int64_t chunk = pick_chunk_split(c->sm_count, units, rows, max_len);
  const int splits = chunk == kNoSplit ? 1 : (int)((max_len + chunk - 1) / chunk);
  kernel<<<dim3((unsigned)grid, splits), sd::ac::THREADS, L::SMEM, c->stream>>>(
      mk, mv, use_maps, view_of(c, b), rows_of(q), rows_of(out), (const TC*)P.k, (const TC*)P.v, (const float*)P.ks, (const float*)P.vs, (const uint8_t*)P.kb, (const uint8_t*)P.vb, c->group, scale_log2, wide(q), wide(out),
      blocks, rows_from, (int)chunk, c->at<float>(c->part_acc), c->at<float>(c->part_ml), c->test_expire ? 1 : 0, sc, SC ? c->at<int>(c->part_used) : nullptr);
  c->test_expire = false;
  if (splits > 1)
    sd::paged_attn_join_kernel<HD><<<dim3(b->n_tokens, (c->cfg.n_heads + 7) / 8), 256, 0, c->stream>>>(
        view_of(c, b), rows_of(out), c->group, rows_from, L::ROWS, (int)chunk, splits, c->at<float>(c->part_acc), c->at<float>(c->part_ml),
        SC ? (const int*)c->at<int>(c->part_used) : nullptr);
  *split = splits > 1;
  return launched(c, splits > 1 ? 2 : 1);
}

// Query rows per key head from which a sequence goes to the kernel for chunks, whose time hardly depends on them up to 256; the kernel for few
// rows reads the keys again for every 8.  Measured, chunks against few rows: bf16, 16 sequences of 1024 positions, 32 heads of 128, 12 rows
// 70 and 131 us, 32 rows 71 and 133; 2 of 4096, 8 heads, 12 rows 18 and 28; one of 30 000, one key head, 12 rows 26 and 151; 8 of 300,
// 12 heads of 64, 12 rows 10 and 8.  In 8 bits, where the few rows' kernel has less to read and this one codes to convert: int8,
// 64 of 4096 over 2 key heads of 128, 16 rows 111 and 82, 32 rows 111 and 140; e4m3, 16 of 1024, 32 heads of 64, 24 rows 75 and 66,
// 32 rows 75 and 116.  With pairs (results in fp16, few rows' time beside it): bf16, 16 of 1024, 32 heads of 64, 32 rows 133 and 74, 64 rows 135
// and 133; 2 of 4096, 8 heads of 128, 32 rows 41 and 33, 48 rows 41 and 41; one of 30 000, one head, 32 rows 49 and 96; e4m3, 16 of 1024,
// 8 heads of 128, 25 rows 49 and 67; 2 of 4096 41 and 45; 8 of 300, 12 heads of 64, 22 and 14.  In 4 bits, where both kernels convert and the few rows' has a
// half to read: bf16, 16 of 1024, 32 heads of 128, 40 rows 120 and 102, 56 rows 120 and 135; 64 of 4096 over 2 key heads, 32 rows 99 and 90, 48 rows 99 and 127; 2
// of 4096, 8 heads, 40 and 37, 64 rows 40 and 39; 8 of 300, 12 heads of 64, 48 rows 22 and 14, 64 rows 22 and 21; fp32, 16 of 1024, 40 rows 149 and 135, 56 rows 150
// and 179 (158 since sums are in parts, the few rows' kernel 159 at 48).  In 8 bits with pairs and changed scores, e4m3, results written in fp32 by both, the same, 40 rows 234 and 201, 56 rows 236 and 272; 2 of 4096 58 and 49, 58 and 64.
template <typename TC, bool SC> constexpr int kChunkRows(bool pairs) {
  constexpr bool scaled = sd::CacheType<TC>::TOP > 0.f;
  return sd::kFour<TC> || (scaled && SC && pairs) ? 49 : scaled ? 25 : pairs ? 41 : 9;
}

template <bool SC>
int cache_attention(sd_cache* c, int l, const sd_batch* b, const sd_heads* q, float scale, const sd_heads* out, const sd::Scores& sc) {
  if (scale == 0.f) scale = 1.f / sqrtf((float)c->cfg.head_dim);
  const float scale_log2 = scale * 1.4426950408889634f;
  return with_cache_type(c->cfg.dtype, [&](auto tc) {
    using TC = decltype(tc);
    return with_head_dim(c->cfg.head_dim, [&](auto hd) {
      constexpr int HD = decltype(hd)::value;
      if constexpr (std::is_same<TC, float>::value) {
        const auto P = pools<TC>(c, l);
        sd::paged_attn_row_kernel<TC, HD, SC><<<dim3(b->n_tokens, c->cfg.n_heads), 128, 0, c->stream>>>(
            view_of(c, b), rows_of(q), rows_of(out), (const TC*)P.k, (const TC*)P.v, (const float*)P.ks, (const float*)P.vs, c->group, scale_log2, sc);
        return launched(c);
      } else {
        const int64_t most = (int64_t)b->max_new * c->group;
        if (most > 0x7fffff00) return (int)SD_ERR_ARG;
        if constexpr (HD >= 64) {
          // one bf16 for a query or a weight only where the queries have no more and the results keep no more
          const bool pairs = q->dtype != SD_DTYPE_BF16 || out->dtype != SD_DTYPE_BF16;
          const int enough = kChunkRows<TC, SC>(pairs);
          if (most >= enough && (sd::kFour<TC> || out->dtype != SD_DTYPE_FP32)) {       // over 4 bits pairs are fp16 there too, 22 bits
            // max_new is only a bound: which kernel takes a sequence is decided on the device, by its own rows
            bool split = false;
            const int rows_from = b->n_seqs == 1 ? 1 : enough;
            const int rc = pairs ? attention_chunks<TC, HD, true, SC>(c, l, b, q, scale_log2, out, sc, rows_from, &split)
                                 : attention_chunks<TC, HD, false, SC>(c, l, b, q, scale_log2, out, sc, rows_from, &split);
            if (rc != SD_OK || b->n_seqs == 1) return rc;
            // it may begin early where the two do not share the workspace for split keys
            return attention_few<TC, HD, SC>(c, l, b, q, scale_log2, out, sc, enough, !split);
          }
        }
        return attention_few<TC, HD, SC>(c, l, b, q, scale_log2, out, sc, most + 1);
      }
    });
  });
}

}  // namespace

namespace sd {
// attn_scores.cu: cache_attention<true>
int attention_with_scores(sd_cache* c, int l, const sd_batch* b, const sd_heads* q, float scale, const sd_heads* out, const Scores& sc);
}  // namespace sd
