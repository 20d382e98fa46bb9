// Work on the pages of a paged cache: forking sequences, growing, cutting and ending them, compacting the pool, copying pages.  The
// books are the caller's device arrays: a table of page numbers per sequence, lengths, and for every page how many tables hold it (0: free).
//
// A call is two launches.  The first, one block, works on the books: which pages are given back, taken or moved.  Everything is decided by order,
// not by arrival: new pages are the lowest free ones, row by row.  It leaves a list of (source, destination) pages.  The second copies those pages in all
// layers with all SMs; the number of copies stays on the device, so that neither launch waits for the host and both can be captured.
#pragma once
#include "paged.cuh"

namespace sd {

enum : int { STATUS_NO_PAGES = 128 };

struct Books {
  int *pages, *len, *refs;
  int n_seqs, columns, n_pages, page_shift;
  int* status;
  __host__ __device__ __forceinline__ void say(int bit) const {
#ifdef __CUDA_ARCH__
    atomicOr(status, bit);
#else
    *status |= bit;                             // the index arithmetic is tested on the host
#endif
  }
  __host__ __device__ __forceinline__ bool is_page(int p) const { return (unsigned)p < (unsigned)n_pages; }
  __host__ __device__ __forceinline__ bool is_length(int l) const { return l >= 0 && (long long)l <= (long long)columns << page_shift; }
  // Columns of the table that a sequence of l positions uses; l is a length.
  __host__ __device__ __forceinline__ int columns_of(int l) const { return (int)(((long long)l + (1 << page_shift) - 1) >> page_shift); }
  __host__ __device__ __forceinline__ int* row(int s) const { return pages + (size_t)s * columns; }
};

// What a resize does to a row: how many columns it has and shall have, and the column of the page that it keeps in part (-1: none).
struct Resize {
  int have, want, part;
  bool ok;
};
__host__ __device__ __forceinline__ Resize resize_of(const Books& b, int length, int target) {
  Resize r{0, 0, -1, b.is_length(length) && b.is_length(target)};
  if (!r.ok) return r;
  r.have = b.columns_of(length);
  r.want = b.columns_of(target);
  const int kept = length < target ? length : target;
  if (kept & ((1 << b.page_shift) - 1)) r.part = kept >> b.page_shift;     // below have and want, so a column of the row
  return r;
}

// Workspace of a call, in the cache's arena.
struct PageWork {
  int4* plan;          // [max_seqs] of a row (resize) or a fork
  int* claim;          // [max_seqs] the fork that a row is for
  int *from, *to;      // [n_pages] the copies
  int* place;          // [n_pages] new numbers of pages that a compaction moves, -1: none (from the first number that is not kept on)
  int* totals;         // number of copies, pages in use
};

namespace pg {

// A block has 1024 threads, or 256 where there is little to look at, whose barriers take less: one request forked three times and resized, 12 heads of 64, two
// layers, 18.5 and 16.5 us with the calls queued ahead, five small sequences compacted 12.3 and 10.3.
constexpr int LARGE = 1024, SMALL = 256, ROUNDS = 8;
template <int T> constexpr int WARPS = T / 32;
template <int T> constexpr int SPAN = T * ROUNDS;

// Exclusive prefix sum of one number per thread, and the block's total.
template <int THREADS, typename T> __device__ __forceinline__ T block_scan(T v, T& total, T* sm) {          // sm: [32]
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  T x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const T y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) sm[warp] = x;
  __syncthreads();
  if (warp == 0) {
    T w = lane < WARPS<THREADS> ? sm[lane] : T(0);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const T y = __shfl_up_sync(0xffffffffu, w, o);
      if (lane >= o) w += y;
    }
    sm[lane] = w;
  }
  __syncthreads();
  total = sm[WARPS<THREADS> - 1];
  const T before = warp ? sm[warp - 1] : T(0);
  __syncthreads();                              // sm may be written again
  return before + x - v;
}

// One span of pages from number p0 on: a warp's 256, of which its lanes see 32 in each round.  yes(p) says which count, at(p, k) is called
// for each of them with its rank k.  Returns the rank after the span.
template <int THREADS, typename Yes, typename At>
__device__ __forceinline__ int rank_span(int p0, int n_pages, int rank, int* sm, Yes yes, At at) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, first = p0 + warp * (ROUNDS * 32) + lane;
  unsigned mask[ROUNDS];
  bool on[ROUNDS];
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) on[r] = first + r * 32 < n_pages && yes(first + r * 32);
  int count = 0;
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) {
    mask[r] = __ballot_sync(0xffffffffu, on[r]);
    count += __popc(mask[r]);
  }
  int total;
  int k = rank + block_scan<THREADS>(lane == 0 ? count : 0, total, sm);
  k = __shfl_sync(0xffffffffu, k, 0);
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) {
    if (on[r]) at(first + r * 32, k + __popc(mask[r] & ((1u << lane) - 1)));
    k += __popc(mask[r]);
  }
  return rank + total;
}

// The lowest `need` free pages to list[0..need), as far as there are so many; returns how many there are (up to the end of a span).
template <int THREADS> __device__ __forceinline__ int find_free(const Books& b, int need, int* list, int* sm) {
  int found = 0;
  for (int p0 = 0; p0 < b.n_pages && found < need; p0 += SPAN<THREADS>)
    found = rank_span<THREADS>(p0, b.n_pages, found, sm, [&](int p) { return __ldcg(b.refs + p) == 0; }, [&](int p, int k) { if (k < need) list[k] = p; });
  __syncthreads();
  return found;
}

// Goes over the pieces of 32 rows, a lane's row having `count` of them: f(lane of the row, piece, a and b of that lane), one piece to a lane at a time, so
// that many rows with a piece or two take no longer than one with many.
template <typename F>
__device__ __forceinline__ void spread(int count, int a, int b, F f) {
  const int lane = threadIdx.x & 31;
  long long upto = count;                       // pieces of the rows up to this one
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += y;
  }
  const long long total = __shfl_sync(0xffffffffu, upto, 31), before = upto - count;
  for (long long k = 0; k < total; k += 32) {
    const long long i = k + lane;
    int of = 0;                                 // the first row whose pieces reach past i
#pragma unroll
    for (int step = 16; step > 0; step >>= 1)
      if (__shfl_sync(0xffffffffu, upto, of + step - 1) <= i) of += step;
    const int e = (int)(i - __shfl_sync(0xffffffffu, before, of)), a_of = __shfl_sync(0xffffffffu, a, of), b_of = __shfl_sync(0xffffffffu, b, of);
    if (i < total) f(of, e, a_of, b_of);
  }
}

__device__ __forceinline__ void add_copy(const PageWork& w, int from, int to) {
  const int m = atomicAdd(&w.totals[0], 1);     // at most one copy per row: fewer than there are pages
  w.from[m] = from;
  w.to[m] = to;
}

}  // namespace pg

// Fork i makes row dst[i], which has to be empty, a copy of row src[i]: whole pages are shared, the last one, where it is not full, is copied to a
// new page.  A row that two forks are for goes to the first of them.
template <int THREADS>
__global__ void __launch_bounds__(THREADS)
pages_fork_kernel(const Books b, const int* __restrict__ src, const int* __restrict__ dst, int n, const PageWork w) {
  using namespace pg;
  __shared__ int sm[32];
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (threadIdx.x == 0) w.totals[0] = 0;
  for (int s = threadIdx.x; s < b.n_seqs; s += THREADS) w.claim[s] = 0x7fffffff;
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += THREADS)
    if ((unsigned)dst[i] < (unsigned)b.n_seqs) atomicMin(&w.claim[dst[i]], i);
  __syncthreads();
  int need = 0;                                 // of all forks so far
  for (int i0 = 0; i0 < n; i0 += THREADS) {
    const int i = i0 + threadIdx.x;
    int length = -1, part = 0;
    if (i < n) {
      const int from = src[i], to = dst[i];
      if ((unsigned)from < (unsigned)b.n_seqs && (unsigned)to < (unsigned)b.n_seqs && from != to && __ldcg(w.claim + to) == i && b.len[to] == 0 && b.is_length(b.len[from])) {
        length = b.len[from];
        const int column = length >> b.page_shift;
        part = (length & ((1 << b.page_shift) - 1)) && b.is_page(b.row(from)[column]);
      } else {
        b.say(STATUS_BAD_BATCH);
      }
    }
    int total;
    const int before = block_scan<THREADS>(part, total, sm);
    if (i < n) w.plan[i] = make_int4(need + before, part, length, 0);
    need += total;
  }
  const int found = find_free<THREADS>(b, need, w.to, sm);
  // the list of free pages is the copies' destinations too: copies are numbered by rank, and what is not served comes last
  const int served = min(found, need);
  if (threadIdx.x == 0) w.totals[0] = served;
  for (int i0 = warp * 32; i0 < n; i0 += THREADS) {
    const int i = i0 + lane;
    const int4 plan = i < n ? w.plan[i] : make_int4(0, 0, -1, 0);
    const int length = plan.z, row_from = length >= 0 ? src[i] : 0, row_to = length >= 0 ? dst[i] : 0;
    const bool short_of = length >= 0 && plan.y && plan.x >= served, on = length >= 0 && !short_of;
    if (short_of) b.say(STATUS_NO_PAGES);
    const int whole = on ? length >> b.page_shift : 0;
    spread(whole, row_from, row_to, [&](int, int e, int from, int to) {
      const int p = b.row(from)[e];
      if (b.is_page(p)) atomicAdd(&b.refs[p], 1);
      else b.say(STATUS_BAD_BATCH);
      b.row(to)[e] = b.is_page(p) ? p : -1;
    });
    if (!on) continue;                          // no shuffle follows for these rows
    if (plan.y) {
      const int p = w.to[plan.x];
      b.row(row_to)[whole] = p;
      b.refs[p] = 1;
      w.from[plan.x] = b.row(row_from)[whole];
    } else if (b.columns_of(length) > whole) {
      b.row(row_to)[whole] = -1;
      b.say(STATUS_BAD_BATCH);
    }
    b.len[row_to] = length;
  }
}

// Row s takes the length target[s].  All rows first give back the pages past their new ends.  Then a page that a row keeps in part and others hold too is
// replaced by a copy, and missing pages are added: the lowest free ones, row by row, a row's copy first.  From the first row on for which there are
// not enough, rows that need any stay as they are (cut, but still sharing their last page, if they were to be cut).
template <int THREADS>
__global__ void __launch_bounds__(THREADS)
pages_resize_kernel(const Books b, const int* __restrict__ target, const PageWork w) {
  using namespace pg;
  __shared__ int sm[32];
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (threadIdx.x == 0) w.totals[0] = 0;
  for (int s0 = warp * 32; s0 < b.n_seqs; s0 += THREADS) {
    const int s = s0 + lane;
    Resize r{0, 0, -1, true};
    if (s < b.n_seqs) r = resize_of(b, b.len[s], target[s]);
    if (!r.ok) b.say(STATUS_BAD_BATCH);
    spread(max(r.have - r.want, 0), r.want, 0, [&](int of, int e, int want, int) {
      int* entry = b.row(s0 + of) + want + e;
      const int p = *entry;
      *entry = -1;
      if (!b.is_page(p)) b.say(STATUS_BAD_BATCH);
      else if (atomicSub(&b.refs[p], 1) <= 0) {                  // nobody was said to hold it
        atomicAdd(&b.refs[p], 1);
        b.say(STATUS_BAD_BATCH);
      }
    });
  }
  __syncthreads();
  __shared__ long long sums[32];
  long long need = 0;                           // rows may ask for more than there can be
  for (int s0 = 0; s0 < b.n_seqs; s0 += THREADS) {
    const int s = s0 + threadIdx.x;
    long long copy = 0, more = 0;
    if (s < b.n_seqs) {
      const Resize r = resize_of(b, b.len[s], target[s]);
      more = r.want > r.have ? r.want - r.have : 0;
      if (r.part >= 0) {
        const int p = b.row(s)[r.part];
        copy = b.is_page(p) && __ldcg(b.refs + p) > 1;
      }
    }
    long long total;
    const long long before = need + block_scan<THREADS>(copy + more, total, sums);
    if (s < b.n_seqs) w.plan[s] = make_int4((int)min(before, 0x7fffffffll), (int)copy, (int)more, 0);
    need += total;
  }
  int* list = w.place;
  const int found = find_free<THREADS>(b, (int)min(need, (long long)b.n_pages), list, sm);
  for (int s0 = warp * 32; s0 < b.n_seqs; s0 += THREADS) {
    const int s = s0 + lane;
    Resize r{0, 0, -1, false};
    int length = 0, length_new = 0;
    int4 plan = make_int4(0, 0, 0, 0);
    if (s < b.n_seqs) {
      length = b.len[s];
      length_new = target[s];
      r = resize_of(b, length, length_new);
      plan = w.plan[s];
    }
    const bool served = r.ok && (plan.y + plan.z == 0 || (plan.x <= found && plan.y + plan.z <= found - plan.x));
    if (r.ok && !served) b.say(STATUS_NO_PAGES);
    spread(served ? plan.z : 0, r.have, plan.x + plan.y, [&](int of, int e, int have, int at) {
      const int p = list[at + e];
      b.row(s0 + of)[have + e] = p;
      b.refs[p] = 1;
    });
    if (served && plan.y) {
      int* entry = b.row(s) + r.part;
      const int p = list[plan.x], old = *entry;
      *entry = p;
      b.refs[p] = 1;
      atomicSub(&b.refs[old], 1);
      add_copy(w, old, p);
    }
    if (served || (r.ok && length_new < length)) b.len[s] = length_new;
  }
}

// The pages in use get the numbers from 0 on: those beyond move, in order, to the free ones below, in order.
template <int THREADS>
__global__ void __launch_bounds__(THREADS)
pages_compact_kernel(const Books b, int* __restrict__ n_used, const PageWork w) {
  using namespace pg;
  __shared__ int sm[32];
  pdl_launch_dependents();
  int used = 0;
  for (int p = threadIdx.x; p < b.n_pages; p += THREADS) used += b.refs[p] != 0;
  int total;
  block_scan<THREADS>(used, total, sm);
  used = total;
  int holes = 0, moves = 0;
  for (int p0 = 0; p0 < b.n_pages; p0 += SPAN<THREADS>) {
    if (p0 < used)
      holes = rank_span<THREADS>(p0, used, holes, sm, [&](int p) { return b.refs[p] == 0; }, [&](int p, int k) { w.to[k] = p; });
    __syncthreads();
    if (p0 + SPAN<THREADS> > used) {
      for (int p = max(p0, used) + threadIdx.x; p < min(p0 + SPAN<THREADS>, b.n_pages); p += THREADS) w.place[p] = -1;
      __syncthreads();
      moves = rank_span<THREADS>(p0, b.n_pages, moves, sm, [&](int p) { return p >= used && b.refs[p] != 0; },
                        [&](int p, int k) { w.from[k] = p; w.place[p] = w.to[k]; });
    }
  }
  __syncthreads();
  for (int k = threadIdx.x; k < moves; k += THREADS) {
    b.refs[w.to[k]] = b.refs[w.from[k]];
    b.refs[w.from[k]] = 0;
  }
  if (threadIdx.x == 0) {
    w.totals[0] = moves;
    w.totals[1] = used;
    if (n_used) *n_used = used;
  }
}

// What a layer holds of a page: up to six runs of bytes (K, V, their scales, their block scales).
struct PageRuns {
  long long offset[6];     // of the pool within a layer
  int words[6];            // 16-byte words of a page in it
  int pieces[6];           // of PIECE words, the last one shorter
  int n, all_pieces;
};
constexpr int PIECE = 2048, COPY_STAGES = 6, COPY_AHEAD = 3, COPY_SMEM = COPY_STAGES * PIECE * 16;      // 192 KB: a block to an SM
struct CopySpan { char* to; const char* from; uint32_t bytes; };                                         // bytes 0: nothing to copy

// Copies the listed pages in all layers, and gives the tables the new numbers where a compaction moved pages (remap).  One thread of a block streams pieces of 32 KB
// through shared memory by bulk copies, three on their way in while others leave, so that both directions of the memory are busy all the time.  What
// bounds it is memory: 150 pages of 2.1 MB 108 us, 5.8 TB/s (117 us by 16-byte loads and stores of 1024 threads to an SM, eight each on their way).
__global__ void __launch_bounds__(256)
pages_copy_kernel(const Books b, char* __restrict__ arena, long long layer_bytes, int layers, const PageRuns runs, const int* __restrict__ from, const int* __restrict__ to,
                  const int* __restrict__ n_copies, int n, const int* __restrict__ place, int remap) {
  extern __shared__ __align__(128) unsigned char copy_smem[];
  __shared__ uint64_t full[COPY_STAGES];
  __shared__ CopySpan spans[COPY_STAGES];
  pdl_wait();
  if (remap) {
    const int used = n_copies[1];
    for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < (long long)b.n_seqs * b.columns; i += (long long)gridDim.x * blockDim.x) {
      const int s = (int)(i / b.columns), e = (int)(i % b.columns);
      const int l = b.len[s];
      if (!b.is_length(l) || e >= b.columns_of(l)) continue;
      const int p = b.pages[i];
      if (b.is_page(p) && p < used) continue;
      const int q = b.is_page(p) ? place[p] : -1;
      if (q < 0) b.say(STATUS_BAD_BATCH);                        // no page, or one that nobody was said to hold
      else b.pages[i] = q;
    }
  }
  if (threadIdx.x != 0) return;
  const long long pieces = (long long)(n_copies ? *n_copies : n) * layers * runs.all_pieces;
  const long long mine = blockIdx.x < pieces ? (pieces - 1 - blockIdx.x) / gridDim.x + 1 : 0;            // this block's: every gridDim.x-th
  if (mine == 0) return;
  auto span_of = [&](long long k) {
    const long long i = blockIdx.x + k * gridDim.x;
    int piece = (int)(i % runs.all_pieces);
    const long long rest = i / runs.all_pieces;
    const int layer = (int)(rest % layers), m = (int)(rest / layers);
    int run = 0;
    while (piece >= runs.pieces[run]) piece -= runs.pieces[run++];
    const int f = from[m], t = to[m];
    CopySpan c{nullptr, nullptr, 0u};
    if (!b.is_page(f) || !b.is_page(t)) {
      b.say(STATUS_BAD_BATCH);
    } else if (f != t) {
      char* pool = arena + layer * layer_bytes + runs.offset[run];
      c.from = pool + ((long long)f * runs.words[run] + (long long)piece * PIECE) * 16;
      c.to = pool + ((long long)t * runs.words[run] + (long long)piece * PIECE) * 16;
      c.bytes = (uint32_t)min(PIECE, runs.words[run] - piece * PIECE) * 16;
    }
    return c;
  };
  const uint32_t smem = (uint32_t)__cvta_generic_to_shared(copy_smem), bar = (uint32_t)__cvta_generic_to_shared(full);
  for (int s = 0; s < COPY_STAGES; ++s) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bar + 8 * s) : "memory");
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  unsigned phases = 0u, asked = 0u;              // a bit per stage: the phase to wait for next; copies in that have not been waited for
  auto landed = [&](int s) {                     // bounded: false when a copy did not land in two seconds, which has no reason to happen
    const long long t0 = clock64();
    const uint32_t parity = phases >> s & 1u;
    for (;;) {
      uint32_t done;
      asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.b32 %0, 1, 0, p;\n}\n" : "=r"(done) : "r"(bar + 8 * s), "r"(parity) : "memory");
      if (done) break;
      if (clock64() - t0 > 4000000000ll) return false;
    }
    phases ^= 1u << s;
    asked &= ~(1u << s);
    return true;
  };
  bool ok = true;
  for (long long k = 0; k < mine + COPY_AHEAD && ok; ++k) {
    if (k < mine) {
      const int s = (int)(k % COPY_STAGES);
      // the piece that was here before has left: all but the last STAGES - AHEAD - 1 groups
      asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(COPY_STAGES - COPY_AHEAD - 1) : "memory");
      const CopySpan c = span_of(k);
      spans[s] = c;
      if (c.bytes) {
        asked |= 1u << s;
        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar + 8 * s), "r"(c.bytes) : "memory");
        asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                     ::"r"(smem + s * PIECE * 16), "l"(c.from), "r"(c.bytes), "r"(bar + 8 * s) : "memory");
      }
    }
    if (k >= COPY_AHEAD) {
      const int s = (int)((k - COPY_AHEAD) % COPY_STAGES);
      const CopySpan c = spans[s];
      if (c.bytes) {
        ok = landed(s);
        if (ok) asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(c.to), "r"(smem + s * PIECE * 16), "r"(c.bytes) : "memory");
      }
      asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
  }
  if (!ok) {                                     // giving up: copies that are still on their way must land before the block's memory goes
    b.say(STATUS_WAIT_EXPIRED);
    for (int s = 0; s < COPY_STAGES; ++s)
      if (asked >> s & 1u) landed(s);
  }
  asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
}

}  // namespace sd
