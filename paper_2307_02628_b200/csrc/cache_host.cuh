// Host side of the paged cache and of sd_extend: argument checks, arena carving, the copying kernels.  Part of skipdecode.cu.
#pragma once
#include "attn_launch.cuh"

namespace {

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
  if (A.four && entries > 0xffffffffu) return false;            // beyond the device's memory; the kernels number its keys in 32 bits
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
  A.part_used = take((size_t)kPartSlots * 4);
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
    if (cache_append(c, l, b, &k, &v) != SD_OK || cache_attention<false>(c, l, b, &q, 0.f, &out, sd::Scores{}) != SD_OK) return SD_ERR_CUDA;
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

// Whether a small block is enough for the books: a round of its threads for the rows, a few for the pages.
bool little(const sd_cache* c, const sd_tables* t) { return t->n_seqs <= sd::pg::SMALL && c->cfg.n_pages <= 4 * sd::pg::SPAN<sd::pg::SMALL>; }

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
  const int grid = (int)std::min<int64_t>(most, (int64_t)c->sm_count);
  if (!c->copy_ready) {
    if (cudaFuncSetAttribute(sd::pages_copy_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, sd::COPY_SMEM) != cudaSuccess) { cudaGetLastError(); return SD_ERR_CUDA; }
    c->copy_ready = true;
  }
  sd::launch_kernel(planned, c->stream, sd::pages_copy_kernel, dim3(grid), dim3(256), sd::COPY_SMEM, books_of(c, t), c->arena, (long long)c->layer_bytes, (int)c->cfg.n_layers, runs, from, to,
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

// The checks that both calls of attention share; 1: there is nothing to do.
static int check_attention(const sd_cache* c, int layer, const sd_batch* b, const sd_heads* q, float scale, const sd_heads* out) {
  if (!c || layer < 0 || layer >= c->cfg.n_layers || !(fabsf(scale) <= 2e38f)) return SD_ERR_ARG;   // its product with log2 e is finite too
  int rc = check_batch(c, b);
  if (rc == SD_OK) rc = check_rows(c, b, q, c->cfg.n_heads, false);
  if (rc == SD_OK) rc = check_rows(c, b, out, c->cfg.n_heads, true);
  return rc != SD_OK ? rc : b->n_tokens == 0 ? 1 : SD_OK;
}

int sd_cache_attention(sd_cache* c, int layer, const sd_batch* b, const sd_heads* q, float scale, const sd_heads* out) {
  const int rc = check_attention(c, layer, b, q, scale, out);
  if (rc != SD_OK) return rc < 0 ? rc : SD_OK;
  DeviceGuard guard(c->device);
  if (!guard.ok) return SD_ERR_CUDA;
  std::lock_guard<std::mutex> lock(c->busy);
  return cache_attention<false>(c, layer, b, q, scale, out, sd::Scores{});
}

int sd_cache_attention_scores(sd_cache* c, int layer, const sd_batch* b, const sd_heads* q, float scale, const sd_scores* s, const sd_heads* out) {
  const int rc = check_attention(c, layer, b, q, scale, out);
  if (rc < 0) return rc;
  // the cap and its inverse, in base-2 units, are normal numbers
  if (!s || s->window < 0 || !(s->cap == 0.f || (s->cap >= 1e-30f && s->cap <= 1e30f))) return SD_ERR_ARG;
  if (rc != SD_OK) return SD_OK;
  DeviceGuard guard(c->device);
  if (!guard.ok) return SD_ERR_CUDA;
  std::lock_guard<std::mutex> lock(c->busy);
  const sd::Scores sc{s->cap, s->slopes, s->window, s->lo, s->hi};
  return sd::attention_with_scores(c, layer, b, q, scale, out, sc);
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
  if (little(c, t)) sd::pages_fork_kernel<sd::pg::SMALL><<<1, sd::pg::SMALL, 0, c->stream>>>(books_of(c, t), src, dst, n, w);
  else sd::pages_fork_kernel<sd::pg::LARGE><<<1, sd::pg::LARGE, 0, c->stream>>>(books_of(c, t), src, dst, n, w);
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
  if (little(c, t)) sd::pages_resize_kernel<sd::pg::SMALL><<<1, sd::pg::SMALL, 0, c->stream>>>(books_of(c, t), len, w);
  else sd::pages_resize_kernel<sd::pg::LARGE><<<1, sd::pg::LARGE, 0, c->stream>>>(books_of(c, t), len, w);
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
  if (little(c, t)) sd::pages_compact_kernel<sd::pg::SMALL><<<1, sd::pg::SMALL, 0, c->stream>>>(books_of(c, t), n_used, w);
  else sd::pages_compact_kernel<sd::pg::LARGE><<<1, sd::pg::LARGE, 0, c->stream>>>(books_of(c, t), n_used, w);
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
