// Host side of the paged cache and of sd_extend: argument checks, arena carving, kernel choice.  Part of skipdecode.cu.
#pragma once
#include <mutex>

struct sd_cache {
  std::mutex busy;           // held while a call enqueues: the launches of one call share a workspace and stay together
  sd_cache_config cfg;
  int row_bytes, page_shift, group, device, sm_count;            // row_bytes: of a (token, head) in the pool
  bool scaled, four;
  char* arena;
  cudaStream_t stream;
  size_t layer_bytes, v_off, ks_off, vs_off, kb_off, vb_off;   // K pool, V pool, K and V scales, K and V block scales: offsets within a layer
  size_t minus_pos, last_row, part_acc, part_ml, counters, status_off, total;
  size_t plan, claim, copy_from, copy_to, place, totals;         // workspace of the calls on pages
  sd::EncodeTiledFn encode = nullptr;
  int tile_blocks[15] = {};   // blocks per SM of each form of the kernel for few rows
  int64_t launches = 0;      // kernels launched
  bool test_expire = false;  // test hook: the next launch for chunks makes a wait run out (one shot)
  unsigned long long tile_ready = 0;    // bit per kernel whose shared-memory size has been allowed on this device
  char* layer(int l) const { return arena + (size_t)l * layer_bytes; }
  template <typename T> T* at(size_t off) const { return reinterpret_cast<T*>(arena + off); }
  int* status() const { return at<int>(status_off); }
};

namespace {

constexpr int kPartSlots = 32768;      // 17 MB of head size 128
// Positions that a table may reach.  Key numbers are 32-bit in the kernels, which round them up to whole tiles and look table entries
// up some thousands of keys ahead: sums of a position below this and of such distances, or of two positions, do not wrap.
constexpr int64_t kMostPositions = 1 << 30;

// Makes `device` current for the length of a call.
struct DeviceGuard {
  int before = -1;
  bool ok = true;
  explicit DeviceGuard(int device) {
    if (cudaGetDevice(&before) != cudaSuccess) { cudaGetLastError(); ok = false; return; }
    if (before == device) { before = -1; return; }
    if (cudaSetDevice(device) != cudaSuccess) { cudaGetLastError(); ok = false; }
  }
  ~DeviceGuard() { if (before >= 0) cudaSetDevice(before); }
};

int device_of(const void* p, int* device) {
  cudaPointerAttributes attr;
  if (cudaPointerGetAttributes(&attr, p) != cudaSuccess) { cudaGetLastError(); return SD_ERR_CUDA; }
  if (attr.type != cudaMemoryTypeDevice && attr.type != cudaMemoryTypeManaged) return SD_ERR_ARG;
  *device = attr.device;
  return SD_OK;
}

bool valid_cache_config(const sd_cache_config* c) {
  if (!c) return false;
  if (c->n_layers < 1 || c->n_heads < 1 || c->n_kv_heads < 1 || c->n_pages < 1 || c->max_seqs < 1 || c->max_tokens < 1) return false;
  if (c->n_heads % c->n_kv_heads || c->n_heads > 65535) return false;                // heads are a grid dimension
  if (c->head_dim != 32 && c->head_dim != 64 && c->head_dim != 128) return false;
  if (c->page_len < 8 || c->page_len > 128 || (c->page_len & (c->page_len - 1))) return false;
  return c->dtype == SD_DTYPE_FP32 || c->dtype == SD_DTYPE_BF16 || c->dtype == SD_DTYPE_INT8 || c->dtype == SD_DTYPE_E4M3 || c->dtype == SD_DTYPE_E2M1;
}

// Lays the arena out; false when a size does not fit 62 bits.
bool carve_cache(const sd_cache_config& c, sd_cache& A) {
  A.cfg = c;
  A.four = c.dtype == SD_DTYPE_E2M1;
  A.scaled = c.dtype == SD_DTYPE_INT8 || c.dtype == SD_DTYPE_E4M3 || A.four;
  A.row_bytes = A.four ? c.head_dim / 2 : c.head_dim * (c.dtype == SD_DTYPE_FP32 ? 4 : c.dtype == SD_DTYPE_BF16 ? 2 : 1);
  A.page_shift = 0;
  while ((1 << A.page_shift) < c.page_len) ++A.page_shift;
  A.group = c.n_heads / c.n_kv_heads;
  const unsigned __int128 entries = (unsigned __int128)c.n_pages * c.n_kv_heads * c.page_len;
  const int blocks = A.four ? c.head_dim / sd::kBlock : 0;
  const unsigned __int128 per_layer = 2 * entries * (A.row_bytes + (A.scaled ? 4 : 0) + blocks) + 6 * kAlign;
  if (per_layer * c.n_layers > ((unsigned __int128)1 << 61)) return false;
  size_t off = 0;
  auto take = [&](size_t bytes) { size_t o = off; off = align_up(off + bytes); return o; };
  const size_t values = (size_t)entries * A.row_bytes, scales = A.scaled ? (size_t)entries * 4 : 0;
  take(values);
  A.v_off = take(values);
  A.ks_off = take(scales);
  A.vs_off = take(scales);
  A.kb_off = take((size_t)entries * blocks);
  A.vb_off = take((size_t)entries * blocks);
  A.layer_bytes = off;
  off *= c.n_layers;
  A.minus_pos = take((size_t)c.max_tokens * 4);
  A.last_row = take((size_t)c.max_seqs * 4);
  // partial results of attention over split keys: a fixed number of (row, split) slots, which bounds the splits of a call
  A.part_acc = take((size_t)kPartSlots * c.head_dim * 4);
  A.part_ml = take((size_t)kPartSlots * 8);
  A.counters = take((size_t)kPartSlots * 4);
  A.plan = take((size_t)c.max_seqs * 16);
  A.claim = take((size_t)c.max_seqs * 4);
  A.copy_from = take((size_t)c.n_pages * 4);
  A.copy_to = take((size_t)c.n_pages * 4);
  A.place = take((size_t)c.n_pages * 4);
  A.totals = take(256);
  A.status_off = take(256);
  A.total = off;
  return true;
}

int check_batch(const sd_cache* c, const sd_batch* b) {
  if (!b || !b->pages || !b->first || !b->len) return SD_ERR_ARG;
  if (b->n_seqs < 1 || b->pages_per_seq < 1 || b->n_tokens < 0 || b->max_len < 0) return SD_ERR_ARG;
  if ((int64_t)b->pages_per_seq * c->cfg.page_len > kMostPositions) return SD_ERR_ARG;
  if (b->n_seqs > c->cfg.max_seqs || b->n_tokens > c->cfg.max_tokens) return SD_ERR_CAPACITY;
  if (b->n_tokens > 0 && (b->max_new < 1 || b->max_new > b->n_tokens)) return SD_ERR_ARG;
  return SD_OK;
}

int check_rows(const sd_cache* c, const sd_batch* b, const sd_heads* t, int heads, bool output) {
  if (!t) return SD_ERR_ARG;
  if (t->dtype != SD_DTYPE_FP32 && t->dtype != SD_DTYPE_BF16 && t->dtype != SD_DTYPE_FP16) return SD_ERR_ARG;
  if (b->n_tokens == 0) return SD_OK;
  if (!t->data || t->row_stride < 0 || t->head_stride < 0) return SD_ERR_ARG;
  const int e = t->dtype == SD_DTYPE_FP32 ? 4 : 2;
  if (reinterpret_cast<uintptr_t>(t->data) % e) return SD_ERR_ARG;
  const int64_t far = (int64_t)1 << 50;                         // extents stay inside 64-bit byte offsets
  if (t->row_stride > far / b->n_tokens || t->head_stride > far / heads) return SD_ERR_ARG;
  if (output) {                                                 // rows of heads, or heads of rows, without overlap
    const int64_t hd = c->cfg.head_dim, R = b->n_tokens, H = heads;
    const bool by_row = (H == 1 || t->head_stride >= hd) && (R == 1 || t->row_stride >= (H - 1) * t->head_stride + hd);
    const bool by_head = (R == 1 || t->row_stride >= hd) && (H == 1 || t->head_stride >= (R - 1) * t->row_stride + hd);
    if (!by_row && !by_head) return SD_ERR_ARG;
  }
  return SD_OK;
}

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

// Rows of a block of the copying kernels, as a power of two: two, so that neighbouring rows' codes and scales are touched together,
// where eight blocks per SM are left (24 sequences of 900..1500 positions read in int8: 140 us with one, 131 with two, 128 with
// four; 4005 rows appended from fp32: 50, 51, 52 us; read into fp32: 38, 37, 40 us).
int row_shift(const sd_cache* c, const sd_batch* b) { return b->n_tokens >= 16 * c->sm_count ? 1 : 0; }
static_assert(sd::MOST_ROWS == 2, "rows of a block");

int cache_append(sd_cache* c, int l, const sd_batch* b, const sd_heads* k, const sd_heads* v) {
  const bool vec = wide(k) && wide(v);
  return with_cache_type(c->cfg.dtype, [&](auto tc) {
    using TC = decltype(tc);
    const auto P = pools<TC>(c, l);
    return with_row_type(k->dtype, [&](auto ts) {
      using TS = decltype(ts);
      return with_head_dim(c->cfg.head_dim, [&](auto hd) {
        constexpr int HD = decltype(hd)::value;
        auto kernel = vec ? sd::cache_append_kernel<TS, TC, HD, true> : sd::cache_append_kernel<TS, TC, HD, false>;
        const int shift = row_shift(c, b);
        kernel<<<((b->n_tokens - 1) >> shift) + 1, 256, 0, c->stream>>>(view_of(c, b), shift, rows_of(k), rows_of(v), P.k, P.v, P.ks, P.vs, P.kb, P.vb);
        return launched(c);
      });
    });
  });
}

int cache_read(sd_cache* c, int l, const sd_batch* b, const sd_heads* k, const sd_heads* v) {
  const bool vec = wide(k) && wide(v);
  return with_cache_type(c->cfg.dtype, [&](auto tc) {
    using TC = decltype(tc);
    const auto P = pools<TC>(c, l);
    return with_row_type(k->dtype, [&](auto to) {
      using TO = decltype(to);
      return with_head_dim(c->cfg.head_dim, [&](auto hd) {
        constexpr int HD = decltype(hd)::value;
        auto kernel = vec ? sd::cache_read_kernel<TO, TC, HD, true> : sd::cache_read_kernel<TO, TC, HD, false>;
        const int shift = row_shift(c, b);
        kernel<<<((b->n_tokens - 1) >> shift) + 1, 256, 0, c->stream>>>(view_of(c, b), shift, rows_of(k), rows_of(v), (const TC*)P.k, (const TC*)P.v,
                                                   (const float*)P.ks, (const float*)P.vs, (const uint8_t*)P.kb, (const uint8_t*)P.vb);
        return launched(c);
      });
    });
  });
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

// Sequences of rows_below query rows per key head or more are left out (another kernel takes them).
template <typename TC> constexpr int kTypeIndex = std::is_same<TC, bf16>::value ? 0 : std::is_same<TC, int8_t>::value ? 1 : std::is_same<TC, sd::e4m3>::value ? 2 : 4;

template <typename TC, int HD, bool THIRD>
int attention_tiles(sd_cache* c, int l, const sd_batch* b, const sd_heads* q, float scale_log2, const sd_heads* out, int64_t rows_below, bool early = false) {
  using S = sd::ap::Shape<TC, HD>;
  constexpr int index = (HD == 128 ? 0 : HD == 64 ? 1 : 2) + 3 * (THIRD ? 3 : kTypeIndex<TC>);
  constexpr unsigned long long bit = 1ull << index;
  auto kernel = sd::paged_attn_tile_kernel<TC, HD, THIRD>;
  if (!(c->tile_ready & bit)) {
    int per_sm = 0;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM) != cudaSuccess ||
        cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout, 100) != cudaSuccess ||
        cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, sd::ap::THREADS, S::SMEM) != cudaSuccess) { cudaGetLastError(); return SD_ERR_CUDA; }
    c->tile_blocks[index] = std::max(per_sm, 1);
    c->tile_ready |= bit;
  }
  const auto P = pools<TC>(c, l);
  const int64_t most = std::min((int64_t)b->max_new * c->group, rows_below - 1);       // rows of a sequence that this launch takes
  const int tiles = (int)((most + sd::ap::ROWS - 1) / sd::ap::ROWS), slot_rows = (int)std::min<int64_t>(most, sd::ap::ROWS);
  const int64_t units = (int64_t)tiles * c->cfg.n_kv_heads * b->n_seqs;
  if (units > 0x7fffffff) return SD_ERR_ARG;
  const int max_len = b->max_len > 0 ? b->max_len : b->pages_per_seq * c->cfg.page_len;
  const int chunk = pick_split((long)c->tile_blocks[index] * c->sm_count, (long)units, (long)units * slot_rows, max_len);
  const int splits = (int)(((int64_t)max_len + chunk - 1) / chunk);
  sd::launch_kernel(early, c->stream, kernel, dim3((unsigned)units, splits), dim3(sd::ap::THREADS), S::SMEM,
      view_of(c, b), rows_of(q), rows_of(out), (const TC*)P.k, (const TC*)P.v, (const float*)P.ks, (const float*)P.vs, (const uint8_t*)P.kb, (const uint8_t*)P.vb, c->group, scale_log2, wide(q),
      tiles, (int)std::min<int64_t>(rows_below, 0x7fffffff), chunk, slot_rows, c->at<float>(c->part_acc), c->at<float>(c->part_ml), c->at<int>(c->counters), early);
  return launched(c);
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

template <typename TC, int HD, bool PAIRS>
int attention_chunks(sd_cache* c, int l, const sd_batch* b, const sd_heads* q, float scale_log2, const sd_heads* out, int rows_from, bool* split) {
  using L = sd::ac::Layout<HD, PAIRS>;
  constexpr unsigned long long bit = 1ull << (32 + (HD == 128 ? 0 : 1) + 2 * (kTypeIndex<TC> == 4 ? 3 : kTypeIndex<TC>) + (PAIRS ? 8 : 0));
  auto kernel = sd::paged_attn_chunk_kernel<TC, HD, PAIRS>;
  if (!(c->tile_ready & bit)) {
    cudaFuncAttributes attr;                 // the warpgroups redistribute what the block is launched with: it must be that much
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, L::SMEM) != cudaSuccess ||
        cudaFuncGetAttributes(&attr, kernel) != cudaSuccess || attr.numRegs != sd::ac::LAUNCH_REGS) { cudaGetLastError(); return SD_ERR_CUDA; }
    c->tile_ready |= bit;
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
  const int64_t max_len = b->max_len > 0 ? b->max_len : (int64_t)b->pages_per_seq * c->cfg.page_len;
  const int64_t chunk = pick_chunk_split(c->sm_count, units, rows, max_len);
  const int splits = chunk == kNoSplit ? 1 : (int)((max_len + chunk - 1) / chunk);
  kernel<<<dim3((unsigned)grid, splits), sd::ac::THREADS, L::SMEM, c->stream>>>(
      mk, mv, use_maps, view_of(c, b), rows_of(q), rows_of(out), (const TC*)P.k, (const TC*)P.v, (const float*)P.ks, (const float*)P.vs, (const uint8_t*)P.kb, (const uint8_t*)P.vb, c->group, scale_log2, wide(q), wide(out),
      blocks, rows_from, (int)chunk, c->at<float>(c->part_acc), c->at<float>(c->part_ml), c->test_expire ? 1 : 0);
  c->test_expire = false;
  if (splits > 1)
    sd::paged_attn_join_kernel<HD><<<dim3(b->n_tokens, (c->cfg.n_heads + 7) / 8), 256, 0, c->stream>>>(
        view_of(c, b), rows_of(out), c->group, rows_from, L::ROWS, (int)chunk, splits, c->at<float>(c->part_acc), c->at<float>(c->part_ml));
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
// 8 heads of 128, 25 rows 49 and 67; 2 of 4096 41 and 45; 8 of 300, 12 heads of 64, 22 and 14.
template <typename TC> constexpr int kChunkRows(bool pairs) { return sd::CacheType<TC>::TOP > 0.f ? 25 : pairs ? 41 : 9; }

int cache_attention(sd_cache* c, int l, const sd_batch* b, const sd_heads* q, float scale, const sd_heads* out) {
  if (scale == 0.f) scale = 1.f / sqrtf((float)c->cfg.head_dim);
  const float scale_log2 = scale * 1.4426950408889634f;
  return with_cache_type(c->cfg.dtype, [&](auto tc) {
    using TC = decltype(tc);
    return with_head_dim(c->cfg.head_dim, [&](auto hd) {
      constexpr int HD = decltype(hd)::value;
      if constexpr (std::is_same<TC, float>::value) {
        const auto P = pools<TC>(c, l);
        sd::paged_attn_row_kernel<TC, HD><<<dim3(b->n_tokens, c->cfg.n_heads), 128, 0, c->stream>>>(
            view_of(c, b), rows_of(q), rows_of(out), (const TC*)P.k, (const TC*)P.v, (const float*)P.ks, (const float*)P.vs, c->group, scale_log2);
        return launched(c);
      } else {
        const int64_t most = (int64_t)b->max_new * c->group;
        if (most > 0x7fffff00) return (int)SD_ERR_ARG;
        if constexpr (HD >= 64) {
          // one bf16 for a query or a weight only where the queries have no more and the results keep no more
          const bool pairs = q->dtype != SD_DTYPE_BF16 || out->dtype != SD_DTYPE_BF16;
          const int enough = kChunkRows<TC>(pairs);
          if (most >= enough && out->dtype != SD_DTYPE_FP32) {
            // max_new is only a bound: which kernel takes a sequence is decided on the device, by its own rows
            bool split = false;
            const int rows_from = b->n_seqs == 1 ? 1 : enough;
            const int rc = pairs ? attention_chunks<TC, HD, true>(c, l, b, q, scale_log2, out, rows_from, &split)
                                 : attention_chunks<TC, HD, false>(c, l, b, q, scale_log2, out, rows_from, &split);
            if (rc != SD_OK || b->n_seqs == 1) return rc;
            // it may begin early where the two do not share the workspace for split keys
            return attention_tiles<TC, HD, false>(c, l, b, q, scale_log2, out, enough, !split);
          }
        }
        if constexpr (std::is_same<TC, bf16>::value) {
          if (out->dtype == SD_DTYPE_FP32) return attention_tiles<TC, HD, true>(c, l, b, q, scale_log2, out, most + 1);
        }
        return attention_tiles<TC, HD, false>(c, l, b, q, scale_log2, out, most + 1);
      }
    });
  });
}

// The layers of sd_extend.  The GEMM, LayerNorm and embedding launches are the decode step's; the K and V columns of the QKV
// product go to the paged cache and the attention reads them from there.
template <typename T>
int extend_layers(sd_handle* h, sd_cache* c, const sd_batch* b, const int32_t* d_tokens, int n_active, int warmup, float* d_logits) {
  Launcher Lc{h, false, h->at<float>(h->A.part_acc), h->at<float>(h->A.part_ml)};
  const sd_config& m = h->cfg;
  const int d = m.d_model, f = m.d_ffn, rows = b->n_tokens, top = m.n_layers - (n_active - warmup);
  float* x = h->at<float>(h->A.x);
  T* u = h->at<T>(h->A.u);
  float* qkv = h->at<float>(h->A.qkv);
  T* o = h->at<T>(h->A.o);
  T* y = h->at<T>(h->A.y);
  const int64_t before = c->launches;
  sd::cache_rows_kernel<<<rows, 128, 0, h->stream>>>(view_of(c, b), c->at<int>(c->minus_pos), c->at<int>(c->last_row));
  Lc.end();
  const sd::RowMap map{1, 0, 0, nullptr, nullptr, c->at<int>(c->minus_pos)};
  enqueue_embed<T>(Lc, d_tokens, rows, map);
  const sd_heads q{qkv, 3 * d, h->hd, SD_DTYPE_FP32}, k{qkv + d, 3 * d, h->hd, SD_DTYPE_FP32}, v{qkv + 2 * d, 3 * d, h->hd, SD_DTYPE_FP32};
  // the out-projection's operand: fp32, or fp16 values (see Operand)
  const sd_heads out{o, d, h->hd, std::is_same<T, float>::value ? SD_DTYPE_FP32 : SD_DTYPE_FP16};
  auto norm = [&](const void* g, const void* be) {
    sd::launch_kernel(pdl_for(h, SD_K_LAYERNORM), h->stream, sd::layernorm_kernel<T>, dim3(rows), dim3(ln_threads(d)), 0, x, (const T*)g, (const T*)be, u, d, m.ln_eps, nullptr);
    Lc.end();
  };
  for (int l = 0; l < m.n_layers && !Lc.err; ++l) {
    if (!(l < warmup || l >= top)) continue;
    norm(h->ln1_g[l], h->ln1_b[l]);
    launch_gemm<T>(Lc, SD_K_GEMM_QKV, u, (const T*)h->w_qkv[l], h->A.wp_qkv[l], (const T*)h->b_qkv[l], rows, 3 * d, d, qkv, 3 * d, sd::EPI_STORE_F32);
    if (cache_append(c, l, b, &k, &v) != SD_OK || cache_attention(c, l, b, &q, 0.f, &out) != SD_OK) return SD_ERR_CUDA;
    launch_gemm<T>(Lc, SD_K_GEMM_OUT, o, (const T*)h->w_o[l], h->A.wp_o[l], (const T*)h->b_o[l], rows, d, d, x, d, sd::EPI_RESIDUAL_F32);
    norm(h->ln2_g[l], h->ln2_b[l]);
    launch_gemm<T>(Lc, SD_K_GEMM_FC1, u, (const T*)h->w_fc1[l], h->A.wp_fc1[l], (const T*)h->b_fc1[l], rows, f, d, y, f * sd::Operand<T>::PARTS, sd::EPI_RELU_T);
    launch_gemm<T>(Lc, SD_K_GEMM_FC2, y, (const T*)h->w_fc2[l], h->A.wp_fc2[l], (const T*)h->b_fc2[l], rows, d, f, x, d, sd::EPI_RESIDUAL_F32);
  }
  enqueue_head<T>(Lc, b->n_seqs, c->at<int>(c->last_row), d_logits);
  h->launches += Lc.count + (c->launches - before);
  return Lc.err;
}

// ---- pages

int check_tables(const sd_cache* c, const sd_tables* t) {
  if (!t || !t->pages || !t->len || !t->refs || t->n_seqs < 1 || t->pages_per_seq < 1) return SD_ERR_ARG;
  if ((int64_t)t->pages_per_seq * c->cfg.page_len > kMostPositions) return SD_ERR_ARG;
  return t->n_seqs > c->cfg.max_seqs ? SD_ERR_CAPACITY : SD_OK;
}

sd::Books books_of(const sd_cache* c, const sd_tables* t) {
  return sd::Books{t ? t->pages : nullptr, t ? t->len : nullptr, t ? t->refs : nullptr, t ? t->n_seqs : 0, t ? t->pages_per_seq : 0, c->cfg.n_pages, c->page_shift, c->status()};
}

sd::PageWork page_work(const sd_cache* c) {
  return sd::PageWork{c->at<int4>(c->plan), c->at<int>(c->claim), c->at<int>(c->copy_from), c->at<int>(c->copy_to), c->at<int>(c->place), c->at<int>(c->totals)};
}

// The second launch of a call on pages.  n_copies NULL: n copies of the caller's lists.  planned: behind a first launch, beside whose end it may begin.
int copy_pages(sd_cache* c, const sd_tables* t, const int* from, const int* to, const int* n_copies, int n, bool remap, bool planned) {
  sd::PageRuns runs = {};
  const int64_t entries = (int64_t)c->cfg.n_kv_heads * c->cfg.page_len;
  auto run = [&](int64_t offset, int64_t bytes) {
    if (bytes == 0) return;
    runs.offset[runs.n] = offset;
    runs.words[runs.n] = (int)(bytes / 16);
    runs.pieces[runs.n] = (int)((bytes / 16 + sd::PIECE - 1) / sd::PIECE);
    runs.all_pieces += runs.pieces[runs.n++];
  };
  const int64_t scales = c->scaled ? entries * 4 : 0, blocks = c->four ? entries * (c->cfg.head_dim / sd::kBlock) : 0;
  run(0, entries * c->row_bytes);
  run((int64_t)c->v_off, entries * c->row_bytes);
  run((int64_t)c->ks_off, scales);
  run((int64_t)c->vs_off, scales);
  run((int64_t)c->kb_off, blocks);
  run((int64_t)c->vb_off, blocks);
  const int64_t most = (int64_t)(n_copies ? c->cfg.n_pages : n) * c->cfg.n_layers * runs.all_pieces;
  const int grid = (int)std::min<int64_t>(most, (int64_t)c->sm_count * 4);
  sd::launch_kernel(planned, c->stream, sd::pages_copy_kernel, dim3(grid), dim3(256), 0, books_of(c, t), c->arena, (long long)c->layer_bytes, (int)c->cfg.n_layers, runs, from, to,
                    n_copies, n, (const int*)c->at<int>(c->place), remap ? 1 : 0);
  return launched(c);
}

}  // namespace

extern "C" {

int sd_cache_bytes(const sd_cache_config* cfg, size_t* out) {
  if (!valid_cache_config(cfg) || !out) return SD_ERR_ARG;
  sd_cache A;
  if (!carve_cache(*cfg, A)) return SD_ERR_ARG;
  *out = A.total;
  return SD_OK;
}

int sd_cache_create(const sd_cache_config* cfg, void* arena, size_t arena_bytes, void* stream, sd_cache** out) {
  if (!valid_cache_config(cfg) || !out || !arena || reinterpret_cast<uintptr_t>(arena) % kAlign) return SD_ERR_ARG;
  sd_cache* c = new (std::nothrow) sd_cache();
  if (!c) return SD_ERR_ARG;
  if (!carve_cache(*cfg, *c)) { delete c; return SD_ERR_ARG; }
  if (c->total > arena_bytes) { delete c; return SD_ERR_CAPACITY; }
  c->arena = static_cast<char*>(arena);
  c->stream = static_cast<cudaStream_t>(stream);
  int rc = device_of(arena, &c->device);
  if (rc != SD_OK) { delete c; return rc; }
  DeviceGuard guard(c->device);
  c->sm_count = 0;
  if (!guard.ok || cudaDeviceGetAttribute(&c->sm_count, cudaDevAttrMultiProcessorCount, c->device) != cudaSuccess ||
      cudaMemsetAsync(c->status(), 0, 256, c->stream) != cudaSuccess ||
      cudaMemsetAsync(c->at<int>(c->counters), 0, (size_t)kPartSlots * 4, c->stream) != cudaSuccess) {
    cudaGetLastError();
    delete c;
    return SD_ERR_CUDA;
  }
  void* fn = nullptr;
  cudaDriverEntryPointQueryResult found;
  if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &found) == cudaSuccess && found == cudaDriverEntryPointSuccess)
    c->encode = reinterpret_cast<sd::EncodeTiledFn>(fn);
  else cudaGetLastError();                                      // without it keys and values come by plain asynchronous copies
  *out = c;
  return SD_OK;
}

int sd_cache_layer(sd_cache* c, int layer, void** k, void** v, float** ks, float** vs) {
  if (!c || layer < 0 || layer >= c->cfg.n_layers) return SD_ERR_ARG;
  const auto P = pools<char>(c, layer);
  if (k) *k = P.k;
  if (v) *v = P.v;
  if (ks) *ks = P.ks;
  if (vs) *vs = P.vs;
  return SD_OK;
}

int sd_cache_layer_blocks(sd_cache* c, int layer, uint8_t** kb, uint8_t** vb) {
  if (!c || layer < 0 || layer >= c->cfg.n_layers) return SD_ERR_ARG;
  const auto P = pools<char>(c, layer);
  if (kb) *kb = P.kb;
  if (vb) *vb = P.vb;
  return SD_OK;
}

int sd_cache_append(sd_cache* c, int layer, const sd_batch* b, const sd_heads* k, const sd_heads* v) {
  if (!c || layer < 0 || layer >= c->cfg.n_layers) return SD_ERR_ARG;
  int rc = check_batch(c, b);
  if (rc == SD_OK) rc = check_rows(c, b, k, c->cfg.n_kv_heads, false);
  if (rc == SD_OK) rc = check_rows(c, b, v, c->cfg.n_kv_heads, false);
  if (rc != SD_OK) return rc;
  if (k->dtype != v->dtype) return SD_ERR_ARG;
  if (b->n_tokens == 0) return SD_OK;
  DeviceGuard guard(c->device);
  if (!guard.ok) return SD_ERR_CUDA;
  std::lock_guard<std::mutex> lock(c->busy);
  return cache_append(c, layer, b, k, v);
}

int sd_cache_read(sd_cache* c, int layer, const sd_batch* b, const sd_heads* k, const sd_heads* v) {
  if (!c || layer < 0 || layer >= c->cfg.n_layers) return SD_ERR_ARG;
  int rc = check_batch(c, b);
  if (rc == SD_OK) rc = check_rows(c, b, k, c->cfg.n_kv_heads, true);
  if (rc == SD_OK) rc = check_rows(c, b, v, c->cfg.n_kv_heads, true);
  if (rc != SD_OK) return rc;
  if (k->dtype != v->dtype) return SD_ERR_ARG;
  if (b->n_tokens == 0) return SD_OK;
  DeviceGuard guard(c->device);
  if (!guard.ok) return SD_ERR_CUDA;
  std::lock_guard<std::mutex> lock(c->busy);
  return cache_read(c, layer, b, k, v);
}

int sd_cache_attention(sd_cache* c, int layer, const sd_batch* b, const sd_heads* q, float scale, const sd_heads* out) {
  if (!c || layer < 0 || layer >= c->cfg.n_layers || !(fabsf(scale) <= 2e38f)) return SD_ERR_ARG;   // its product with log2 e is finite too
  int rc = check_batch(c, b);
  if (rc == SD_OK) rc = check_rows(c, b, q, c->cfg.n_heads, false);
  if (rc == SD_OK) rc = check_rows(c, b, out, c->cfg.n_heads, true);
  if (rc != SD_OK) return rc;
  if (b->n_tokens == 0) return SD_OK;
  DeviceGuard guard(c->device);
  if (!guard.ok) return SD_ERR_CUDA;
  std::lock_guard<std::mutex> lock(c->busy);
  return cache_attention(c, layer, b, q, scale, out);
}

int sd_cache_fork(sd_cache* c, const sd_tables* t, const int32_t* src, const int32_t* dst, int n) {
  if (!c || n < 0) return SD_ERR_ARG;
  const int rc = check_tables(c, t);
  if (rc != SD_OK) return rc;
  if (n == 0) return SD_OK;
  if (!src || !dst || n > t->n_seqs) return SD_ERR_ARG;
  DeviceGuard guard(c->device);
  if (!guard.ok) return SD_ERR_CUDA;
  std::lock_guard<std::mutex> lock(c->busy);
  const sd::PageWork w = page_work(c);
  sd::pages_fork_kernel<<<1, sd::pg::THREADS, 0, c->stream>>>(books_of(c, t), src, dst, n, w);
  const int err = launched(c);
  return err != SD_OK ? err : copy_pages(c, t, w.from, w.to, w.totals, 0, false, true);
}

int sd_cache_resize(sd_cache* c, const sd_tables* t, const int32_t* len) {
  if (!c || !len) return SD_ERR_ARG;
  const int rc = check_tables(c, t);
  if (rc != SD_OK) return rc;
  DeviceGuard guard(c->device);
  if (!guard.ok) return SD_ERR_CUDA;
  std::lock_guard<std::mutex> lock(c->busy);
  const sd::PageWork w = page_work(c);
  sd::pages_resize_kernel<<<1, sd::pg::THREADS, 0, c->stream>>>(books_of(c, t), len, w);
  const int err = launched(c);
  return err != SD_OK ? err : copy_pages(c, t, w.from, w.to, w.totals, 0, false, true);
}

int sd_cache_compact(sd_cache* c, const sd_tables* t, int32_t* n_used) {
  if (!c) return SD_ERR_ARG;
  const int rc = check_tables(c, t);
  if (rc != SD_OK) return rc;
  DeviceGuard guard(c->device);
  if (!guard.ok) return SD_ERR_CUDA;
  std::lock_guard<std::mutex> lock(c->busy);
  const sd::PageWork w = page_work(c);
  sd::pages_compact_kernel<<<1, sd::pg::THREADS, 0, c->stream>>>(books_of(c, t), n_used, w);
  const int err = launched(c);
  return err != SD_OK ? err : copy_pages(c, t, w.from, w.to, w.totals, 0, true, true);
}

int sd_cache_copy(sd_cache* c, const int32_t* src, const int32_t* dst, int n) {
  if (!c || n < 0) return SD_ERR_ARG;
  if (n == 0) return SD_OK;
  if (!src || !dst) return SD_ERR_ARG;
  DeviceGuard guard(c->device);
  if (!guard.ok) return SD_ERR_CUDA;
  std::lock_guard<std::mutex> lock(c->busy);
  return copy_pages(c, nullptr, src, dst, nullptr, n, false, false);
}

int sd_cache_status(sd_cache* c, int32_t* device_status) {
  if (!c) return SD_ERR_ARG;
  DeviceGuard guard(c->device);
  int32_t v = 0;
  if (!guard.ok) return SD_ERR_CUDA;
  std::lock_guard<std::mutex> lock(c->busy);                    // reading and clearing stay together
  if (cudaMemcpyAsync(&v, c->status(), 4, cudaMemcpyDeviceToHost, c->stream) != cudaSuccess ||
      cudaMemsetAsync(c->status(), 0, 4, c->stream) != cudaSuccess || cudaStreamSynchronize(c->stream) != cudaSuccess) {
    cudaGetLastError();
    return SD_ERR_CUDA;
  }
  if (device_status) *device_status = v;
  return v ? SD_ERR_DEVICE : SD_OK;
}

int sd_cache_set_option(sd_cache* c, int option, int value) {
  if (!c || option != SD_CACHE_OPT_TEST_WAIT_EXPIRY || value < 0 || value > 1) return SD_ERR_ARG;
  std::lock_guard<std::mutex> lock(c->busy);
  c->test_expire = value != 0;
  return SD_OK;
}

void sd_cache_destroy(sd_cache* c) { delete c; }

int sd_extend(sd_handle* h, sd_cache* c, const sd_batch* b, const int32_t* d_tokens, int n_active, int warmup, float* d_logits) {
  if (!h || !c || !d_tokens || !d_logits) return SD_ERR_ARG;
  const sd_config& m = h->cfg;
  if (c->cfg.n_layers != m.n_layers || c->cfg.n_heads != m.n_heads || c->cfg.n_kv_heads != m.n_heads || c->cfg.head_dim != h->hd) return SD_ERR_ARG;
  if (c->stream != h->stream || warmup < 0 || n_active <= warmup || n_active > m.n_layers) return SD_ERR_ARG;
  const int rc = check_batch(c, b);
  if (rc != SD_OK) return rc;
  if (b->n_tokens > h->A.rows_max || b->n_seqs > m.max_batch) return SD_ERR_CAPACITY;
  if (b->n_tokens == 0) return SD_OK;
  int device = 0;                                               // the default stream is a stream of every device
  const int found = device_of(h->arena, &device);
  if (found != SD_OK) return found;
  if (device != c->device) return SD_ERR_ARG;
  DeviceGuard guard(c->device);
  if (!guard.ok) return SD_ERR_CUDA;
  std::lock_guard<std::mutex> lock(c->busy);
  return m.dtype == SD_DTYPE_BF16 ? extend_layers<bf16>(h, c, b, d_tokens, n_active, warmup, d_logits)
                                  : extend_layers<float>(h, c, b, d_tokens, n_active, warmup, d_logits);
}

int sd_sample(sd_handle* h, const float* d_logits, int B, const sd_sampling* s, const float* d_uniforms, int32_t* d_next) {
  if (!h || !d_logits || B < 1 || !s || !d_uniforms || !d_next) return SD_ERR_ARG;
  int device = 0;
  const int rc = device_of(h->arena, &device);
  if (rc != SD_OK) return rc;
  DeviceGuard guard(device);
  if (!guard.ok) return SD_ERR_CUDA;
  const int vocab = h->cfg.vocab;
  // Blocks per row: as many as leave each SM at most one block and each block 6000 logits.  Measured at 50 272 logits, 1, 2, 4, 8
  // blocks: one row 31, 25, 19, 18 us; 32 rows 35, 29, 24, 28 us; 148 rows 38, 45, 65, 110 us; 64 rows of 8000: 16, 17, 20, 45 us.
  int C = 8;
  while (C > 1 && ((int64_t)B * C > h->tc.sm_count || vocab < 6000 * C)) C >>= 1;
  if ((int64_t)B * C > 0x7fffffff) return SD_ERR_ARG;
  const int part = (vocab + 8 * C - 1) / (8 * C) * 8;          // a multiple of 8: parts keep the row's 16-byte alignment
  int bits = 0;                                                // sums of vocab weights of at most 2^fraction stay below 2^63
  while ((1ll << bits) < vocab) ++bits;
  const int fraction = std::min(52, 63 - bits);
  const size_t with_slices = sizeof(sd::sr::Shared) + (size_t)part * 2;
  const bool slices = with_slices <= (size_t)sd::sr::MAX_SMEM;
  const size_t smem = slices ? with_slices : sizeof(sd::sr::Shared);
  auto kernel = C == 1 ? (slices ? sd::sample_rows_kernel<1024, true, true> : sd::sample_rows_kernel<1024, true, false>)
                       : (slices ? sd::sample_rows_kernel<512, false, true> : sd::sample_rows_kernel<512, false, false>);
  const unsigned bit = (C == 1 ? 1u : 4u) << (slices ? 0 : 1);
  if (!(h->sample_rows_ready & bit)) {       // per handle: the attributes belong to the handle's device
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, sd::sr::MAX_SMEM) != cudaSuccess ||
        cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout, 100) != cudaSuccess) {
      cudaGetLastError();
      return SD_ERR_CUDA;
    }
    h->sample_rows_ready |= bit;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(B * C); cfg.blockDim = dim3(C == 1 ? 1024 : 512); cfg.dynamicSmemBytes = smem; cfg.stream = h->stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = C; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr; cfg.numAttrs = 1;
  if (cudaLaunchKernelEx(&cfg, kernel, d_logits, vocab, part, fraction, d_uniforms, s->temperature, s->top_k, s->top_p, s->min_p, d_next, h->status()) != cudaSuccess) {
    cudaGetLastError();
    return SD_ERR_CUDA;
  }
  h->launches += 1;
  return SD_OK;
}

}  // extern "C"
