// Token selection with each row's own temperature, top-k, top-p and min-p.
//
// A cluster of C blocks shares one row: block c holds the c-th contiguous part of it in shared memory.  Weights are
// w = 2^F exp((x - max) / T) rounded to integers (computed in double precision; F as large as 63-bit sums over the
// vocabulary allow, 47 for 50 272 tokens), so that every sum is exact and independent of the order in which threads add, and a
// comparison at a border comes out as in 64-bit floating point.
//
//   1. The row's maximum and smallest finite value, across the cluster.
//   2. A histogram of weight (and of counts, if top-k asks for them) over 1024 slices of equal width in (x - max) / T,
//      which cut the order "largest logit first" into consecutive pieces.  Shared memory has no native 64-bit atomic
//      addition, so a weight is added to two 32-bit counters, the carry of the lower going to the upper.
//   3. Up to three searches for the element at which a running sum (or count) passes a target: rank top_k - 1, then top_p of
//      the mass found, then the draw.  Block 0 finds the slice; all blocks send it the slice's elements; it ranks them by
//      comparing all pairs.  A slice with more than LIST elements is first cut again, into 1024 pieces of the elements' bit
//      patterns, until it is small enough or all its elements are equal; equal ones are told apart by counting.
// min-p is a threshold on w: the mass above it is a plain sum of step 2.  All three cut a prefix of the same order, so the kept
// mass is the smallest of the three, and the draw needs no list of kept tokens.
#pragma once
#include <cooperative_groups.h>
#include <cstdint>
#include <cuda_runtime.h>

#include "sample.cuh"
#include "paged.cuh"

namespace sd {
namespace sr {

namespace cg = cooperative_groups;

constexpr int THREADS = 512;
constexpr int BINS = 1024;
constexpr int LIST = 1024;
constexpr int MAX_SMEM = 227 * 1024;
typedef unsigned long long u64;

struct Shared {
  u64 mass[BINS];                       // block 0: the row's totals per slice
  uint32_t count[BINS];
  uint32_t lo[BINS], hi[BINS], num[BINS];   // this block's counters
  union {                               // block 0; a finer cut is made only after a list has proved too short
    struct { u64 list_w[LIST]; uint32_t list_key[LIST]; int list_id[LIST]; };
    struct { u64 sub_mass[BINS]; uint32_t sub_count[BINS]; };
  };
  double exp_table[64];
  u64 red[32];
  float redf[32], redf2[32];
  int redi[32];
  // broadcast by block 0, read by the others through the cluster
  float m, lowest;
  u64 z, z_min_p;
  int list_n;
  uint32_t key_lo, key_hi;              // bit patterns the search is confined to
  uint32_t seen_lo, seen_hi;            // smallest and largest among the slice's elements
  int slice;
  u64 before;                           // mass (rank) of everything ahead of the confined elements
  uint32_t before_n;
  u64 found_before, found_w;            // the element: mass ahead of it and its weight
  uint32_t found_key;
  int found_id;                         // -1: one of several equal elements, number found_j of them in token order
  u64 found_j;
  int part_n[16];                       // equal elements per block
};

// exp in double precision, the table method (Tang 1989): 2^y = 2^(k / 64) * 2^f with |f| <= 1/128 and a Taylor polynomial whose
// first left-out term is below 4e-17.  Returns round(2^fraction * 2^y) for -(fraction + 1) <= y <= 0.
__device__ __forceinline__ u64 weight_of(double y, const double* table, int fraction) {
  const double magic = 6755399441055744.0 / 64.0;              // 1.5 * 2^52 / 64: adding it leaves multiples of 1/64
  const double t = y + magic;
  const int k = __double2loint(t);                             // round(64 y), two's complement
  const double f = (y - (t - magic)) * 0.6931471805599453094;
  const double p = fma(fma(fma(fma(fma(f, 1.0 / 120.0, 1.0 / 24.0), f, 1.0 / 6.0), f, 0.5), f, 1.0), f, 1.0);
  const double v = p * table[k & 63];
  const double scaled = __hiloint2double(__double2hiint(v) + (((k >> 6) + fraction) << 20), __double2loint(v));
  return (u64)__double2ll_rn(scaled);
}

struct Row {
  const float* src;                     // this block's part (shared or global memory)
  int n, id0;
  double m, c;                          // maximum; log2(e) / T
  double reach;                         // weights vanish below 2^-reach of the maximum's
  float slice_scale;
  __device__ __forceinline__ double exponent(float x) const { return ((double)x - m) * c; }
  // slice of an exponent, -1 where the weight vanishes
  __device__ __forceinline__ int slice(double y) const {
    if (!(y >= -reach)) return -1;                           // NaN and -inf too
    const int s = (int)((float)-y * slice_scale);
    return s < BINS ? s : BINS - 1;
  }
};

static_assert(sizeof(Shared) % 16 == 0, "the staged row follows at a 16-byte boundary");

__device__ __forceinline__ void add64(uint32_t* lo, uint32_t* hi, u64 w) {
  const uint32_t l = (uint32_t)w;
  const uint32_t h = (uint32_t)(w >> 32) + (atomicAdd(lo, l) > ~l ? 1u : 0u);
  if (h) atomicAdd(hi, h);
}

__device__ __forceinline__ u64 block_sum64(u64 v, u64* red) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if (lane == 0) red[warp] = v;
  __syncthreads();
  v = lane < THREADS / 32 ? red[lane] : 0ull;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Block 0, warp 0: the bin at which the running value, bins 0.. in order, first exceeds target, and what is ahead of it.
template <typename T>
__device__ __forceinline__ void find_bin(const T* bins, u64 base, u64 target, int lane, int& bin, u64& ahead) {
  constexpr int PER = BINS / 32;
  u64 mine = 0ull;
  for (int j = 0; j < PER; ++j) mine += bins[lane * PER + ((j + lane) & (PER - 1))];      // rotated: no bank conflicts
  u64 incl = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const u64 v = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += v;
  }
  const unsigned ballot = __ballot_sync(0xffffffffu, base + incl > target);
  const int owner = ballot ? __ffs(ballot) - 1 : 31;
  // the owner's bins one per lane: a second scan
  const u64 start = __shfl_sync(0xffffffffu, incl - mine, owner);
  const u64 v0 = bins[owner * PER + lane];
  u64 run = v0;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const u64 v = __shfl_up_sync(0xffffffffu, run, o);
    if (lane >= o) run += v;
  }
  const unsigned hit = __ballot_sync(0xffffffffu, base + start + run > target);
  const int at = hit ? __ffs(hit) - 1 : 31;
  bin = owner * PER + at;
  ahead = base + start + __shfl_sync(0xffffffffu, run - v0, at);
}

// Sum of bins[first .. bin) of the counters (warp 0): ranks ahead of a bin found by mass, or masses ahead of one found by rank.
template <typename T>
__device__ __forceinline__ u64 sum_before(const T* bins, int bin, int lane) {
  u64 s = 0ull;
  for (int j = lane; j < bin; j += 32) s += bins[j];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  return s;
}

}  // namespace sr

// grid (C * rows), cluster (C): block c of a cluster holds elements [c * part, ...) of its row.
template <bool ROW_IN_SMEM>
__global__ void __launch_bounds__(sr::THREADS)
sample_rows_kernel(const float* __restrict__ logits, int vocab, int part, int fraction, const float* __restrict__ uniforms,
                   const float* __restrict__ temperatures, const int32_t* __restrict__ top_ks, const float* __restrict__ top_ps,
                   const float* __restrict__ min_ps, int32_t* __restrict__ next, int* __restrict__ status) {
  using namespace sr;
  extern __shared__ __align__(16) unsigned char sr_smem[];
  Shared& sh = *reinterpret_cast<Shared*>(sr_smem);
  cg::cluster_group cluster = cg::this_cluster();
  const int C = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int row_id = blockIdx.x / C;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  Shared* lead = cluster.map_shared_rank(&sh, 0);

  const float* row = logits + (size_t)row_id * vocab;
  Row R;
  R.id0 = min(rank * part, vocab);
  R.n = min(vocab - R.id0, part);
  const float* src = row + R.id0;

  // the settings; one that is no setting makes the row greedy
  const float T = temperatures ? temperatures[row_id] : 1.f;
  const int top_k = top_ks ? top_ks[row_id] : 0;
  const float top_p = top_ps ? top_ps[row_id] : 1.f;
  const float min_p = min_ps ? min_ps[row_id] : 0.f;
  const bool bad = !(T >= 0.f) || T == INFINITY || top_p != top_p || min_p != min_p;
  const bool greedy = bad || T == 0.f;
  if (bad && tid == 0 && rank == 0) atomicOr(status, STATUS_BAD_SETTING);

  // 1. stage the part, maximum and smallest finite value
  float* staged = reinterpret_cast<float*>(sr_smem + sizeof(Shared));
  float m = -INFINITY, low = INFINITY;
  if (ROW_IN_SMEM && (reinterpret_cast<uintptr_t>(src) & 15) == 0) {
    const int n4 = R.n >> 2;
#pragma unroll 4
    for (int i = tid; i < n4; i += THREADS) {
      const float4 v = reinterpret_cast<const float4*>(src)[i];
      reinterpret_cast<float4*>(staged)[i] = v;
      m = fmaxf(fmaxf(fmaxf(m, v.x), fmaxf(v.y, v.z)), v.w);
      low = fminf(low, fminf(fminf(v.x > -INFINITY ? v.x : low, v.y > -INFINITY ? v.y : low), fminf(v.z > -INFINITY ? v.z : low, v.w > -INFINITY ? v.w : low)));
    }
    for (int i = 4 * n4 + tid; i < R.n; i += THREADS) {
      const float x = src[i];
      staged[i] = x;
      m = fmaxf(m, x);
      if (x > -INFINITY) low = fminf(low, x);
    }
  } else {
    for (int i = tid; i < R.n; i += THREADS) {
      const float x = src[i];
      if (ROW_IN_SMEM) staged[i] = x;
      m = fmaxf(m, x);                                           // NaN is dropped
      if (x > -INFINITY) low = fminf(low, x);
    }
  }
  R.src = ROW_IN_SMEM ? staged : src;
  for (int i = tid; i < BINS; i += THREADS) { sh.lo[i] = 0u; sh.hi[i] = 0u; sh.num[i] = 0u; }
  if (tid < 64) sh.exp_table[tid] = exp2((double)tid / 64.0);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    low = fminf(low, __shfl_xor_sync(0xffffffffu, low, o));
  }
  if (lane == 0) { sh.redf[warp] = m; sh.redf2[warp] = low; }
  __syncthreads();
  if (warp == 0) {
    m = lane < THREADS / 32 ? sh.redf[lane] : -INFINITY;
    low = lane < THREADS / 32 ? sh.redf2[lane] : INFINITY;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
      low = fminf(low, __shfl_xor_sync(0xffffffffu, low, o));
    }
    if (lane == 0) { sh.m = m; sh.lowest = low; }
  }
  cluster.sync();
  {
    const int c = lane < C ? lane : 0;
    const Shared* other = cluster.map_shared_rank(&sh, c);
    m = other->m;
    low = other->lowest;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
      low = fminf(low, __shfl_xor_sync(0xffffffffu, low, o));
    }
  }

  if (greedy || !(m > -INFINITY) || m == INFINITY) {
    // the lowest index of the maximum; uniform over the cluster
    int best = 0x7fffffff;
    for (int i = tid; i < R.n; i += THREADS)
      if (R.src[i] == m) { best = R.id0 + i; break; }
    best = __reduce_min_sync(0xffffffffu, best);
    if (lane == 0) sh.redi[warp] = best;
    __syncthreads();
    if (warp == 0) {
      best = __reduce_min_sync(0xffffffffu, lane < THREADS / 32 ? sh.redi[lane] : 0x7fffffff);
      if (lane == 0) sh.found_id = best;
    }
    cluster.sync();
    if (rank == 0 && tid == 0) {
      for (int c = 0; c < C; ++c) best = min(best, cluster.map_shared_rank(&sh, c)->found_id);
      next[row_id] = best == 0x7fffffff ? 0 : best;
    }
    cluster.sync();                                              // nobody leaves while its memory may be read
    return;
  }

  R.m = (double)m;
  R.c = 1.4426950408889634074 / (double)T;
  {
    R.reach = (double)(fraction + 1);
    const double reach = fmin(-R.exponent(low), R.reach);        // the slices cover what the row has
    R.slice_scale = (float)((double)BINS / fmax(reach, 1e-30));
    if (!(R.slice_scale < 1e30f)) R.slice_scale = 0.f;           // all equal: one slice
  }

  // 2. the histogram
  const bool want_counts = top_k > 0 && top_k < vocab;
  const double min_w = min_p > 0.f ? log2((double)min_p) : -INFINITY;   // w >= min_p, as a bound on the exponent
  u64 z = 0ull, zm = 0ull;
  for (int i = tid; i < R.n; i += THREADS) {
    const double y = R.exponent(R.src[i]);
    const int s = R.slice(y);
    if (s < 0) continue;
    const u64 w = weight_of(y, sh.exp_table, fraction);
    z += w;
    if (y >= min_w) zm += w;
    add64(&sh.lo[s], &sh.hi[s], w);
    if (want_counts) atomicAdd(&sh.num[s], 1u);
  }
  z = block_sum64(z, sh.red);
  zm = block_sum64(zm, sh.red);
  if (tid == 0) { sh.z = z; sh.z_min_p = zm; }
  cluster.sync();
  // every block adds up its share of the slices over the cluster and leaves it with block 0
  const int share = (BINS + C - 1) / C;
  for (int i = rank * share + tid; i < min((rank + 1) * share, BINS); i += THREADS) {
    u64 t = 0ull;
    uint32_t n = 0u;
    for (int c = 0; c < C; ++c) {
      const Shared* other = cluster.map_shared_rank(&sh, c);
      t += (u64)other->lo[i] + ((u64)other->hi[i] << 32);
      n += other->num[i];
    }
    lead->mass[i] = t;
    lead->count[i] = n;
  }
  z = 0ull; zm = 0ull;
  for (int c = 0; c < C; ++c) {
    const Shared* other = cluster.map_shared_rank(&sh, c);
    z += other->z;
    zm += other->z_min_p;
  }
  cluster.sync();

  // 3. the searches.  All blocks run the same control flow on values that block 0 publishes.
  u64 kept = min_p > 0.f ? (zm > 0ull ? zm : (1ull << fraction)) : z;   // min_p > 1 keeps the maximum alone
  u64 base_mass = z;                                              // mass of the top-k set
  for (int stage = 0; stage < 3; ++stage) {
    u64 target;
    bool by_rank = false;
    if (stage == 0) {
      if (!want_counts) continue;
      by_rank = true;
      target = (u64)(top_k - 1);
    } else if (stage == 1) {
      if (!(top_p < 1.f)) continue;
      const u64 want = __double2ull_ru((double)top_p * (double)base_mass);     // a negative top_p gives 0
      target = want > 0ull ? min(want, base_mass) - 1ull : 0ull;
    } else {
      float u = uniforms[row_id];
      u = u >= 0.f ? fminf(u, 1.f) : 0.f;
      target = __double2ull_rd((double)u * (double)kept);
      if (target >= kept) target = kept - 1ull;
    }
    // which slice; everything ahead of it
    if (rank == 0 && warp == 0) {
      int bin;
      u64 ahead, other;
      if (by_rank) { find_bin(sh.count, 0ull, target, lane, bin, ahead); other = sum_before(sh.mass, bin, lane); }
      else { find_bin(sh.mass, 0ull, target, lane, bin, ahead); other = 0ull; }
      if (lane == 0) {
        sh.slice = bin;
        sh.before = by_rank ? other : ahead;
        sh.before_n = by_rank ? (uint32_t)ahead : 0u;
        sh.key_lo = 0u; sh.key_hi = 0xffffffffu;
        sh.list_n = 0; sh.seen_lo = 0xffffffffu; sh.seen_hi = 0u;
      }
    }
    cluster.sync();
    if (by_rank) {
      // fewer than top_k elements weigh anything: the set is the whole row
      bool short_row;
      {
        u64 n = 0ull;
        for (int i = tid; i < BINS; i += THREADS) n += lead->count[i];
        n = block_sum64(n, sh.red);
        short_row = n <= target;
      }
      if (short_row) { cluster.sync(); continue; }
    }
    const int slice = lead->slice;
    while (true) {
      const uint32_t key_lo = lead->key_lo, key_hi = lead->key_hi;
      // the confined elements go to block 0's list
      for (int i0 = 0; i0 < part; i0 += THREADS) {
        const int i = i0 + tid;
        bool in = i < R.n;
        uint32_t key = 0u;
        double y = 0.0;
        if (in) {
          const float x = R.src[i];
          y = R.exponent(x);
          in = R.slice(y) == slice;
          key = sample_key(x);
          in = in && key >= key_lo && key <= key_hi;
        }
        const unsigned who = __ballot_sync(0xffffffffu, in);
        if (who == 0u) continue;
        int at = 0;
        if (lane == __ffs(who) - 1) at = atomicAdd(&lead->list_n, __popc(who));
        at = __shfl_sync(0xffffffffu, at, __ffs(who) - 1) + __popc(who & ((1u << lane) - 1u));
        if (in) {
          if (at < LIST) {
            lead->list_key[at] = key;
            lead->list_id[at] = R.id0 + i;
            lead->list_w[at] = weight_of(y, sh.exp_table, fraction);
          }
          atomicMin(&lead->seen_lo, key);
          atomicMax(&lead->seen_hi, key);
        }
      }
      cluster.sync();
      const int n = lead->list_n;
      const uint32_t seen_lo = lead->seen_lo, seen_hi = lead->seen_hi;
      if (n <= LIST) {
        if (rank == 0) {
          // each element's place: everything ahead of it, by comparing all pairs
          for (int e = tid; e < n; e += THREADS) {
            const uint32_t k = sh.list_key[e];
            const int id = sh.list_id[e];
            const u64 w = sh.list_w[e];
            u64 ahead = sh.before;
            uint32_t ahead_n = sh.before_n;
            for (int o = 0; o < n; ++o) {
              const uint32_t k2 = sh.list_key[o];
              if (k2 > k || (k2 == k && sh.list_id[o] < id)) { ahead += sh.list_w[o]; ++ahead_n; }
            }
            const bool hit = by_rank ? ahead_n == (uint32_t)target : (ahead <= target && target < ahead + w);
            if (hit) { sh.found_before = ahead; sh.found_w = w; sh.found_key = k; sh.found_id = id; }
          }
        }
        break;
      }
      if (seen_lo == seen_hi) {                                  // all equal: the place follows by division
        if (rank == 0 && tid == 0) {
          const u64 w = sh.list_w[0];
          const u64 j = by_rank ? target - sh.before_n : (target - sh.before) / w;
          sh.found_before = sh.before + j * w;
          sh.found_w = w;
          sh.found_key = seen_lo;
          sh.found_id = -1;
          sh.found_j = j;
        }
        break;
      }
      // cut the confined bit patterns into at most BINS pieces, largest first
      const uint32_t width = (uint32_t)(((u64)(seen_hi - seen_lo) + BINS) / BINS);
      for (int i = tid; i < BINS; i += THREADS) { sh.lo[i] = 0u; sh.hi[i] = 0u; sh.num[i] = 0u; }
      __syncthreads();
      for (int i = tid; i < R.n; i += THREADS) {
        const float x = R.src[i];
        const double y = R.exponent(x);
        const uint32_t key = sample_key(x);
        if (R.slice(y) != slice || key < key_lo || key > key_hi) continue;
        const uint32_t p = (seen_hi - key) / width;
        add64(&sh.lo[p], &sh.hi[p], weight_of(y, sh.exp_table, fraction));
        atomicAdd(&sh.num[p], 1u);
      }
      cluster.sync();
      for (int i = rank * share + tid; i < min((rank + 1) * share, BINS); i += THREADS) {
        u64 t = 0ull;
        uint32_t k = 0u;
        for (int c = 0; c < C; ++c) {
          const Shared* other = cluster.map_shared_rank(&sh, c);
          t += (u64)other->lo[i] + ((u64)other->hi[i] << 32);
          k += other->num[i];
        }
        lead->sub_mass[i] = t;
        lead->sub_count[i] = k;
      }
      cluster.sync();
      if (rank == 0 && warp == 0) {
        int bin;
        u64 ahead;
        u64 mass_before;
        uint32_t n_before;
        if (by_rank) {
          find_bin(sh.sub_count, (u64)sh.before_n, target, lane, bin, ahead);
          mass_before = sh.before + sum_before(sh.sub_mass, bin, lane);
          n_before = (uint32_t)ahead;
        } else {
          find_bin(sh.sub_mass, sh.before, target, lane, bin, ahead);
          mass_before = ahead;
          n_before = 0u;
        }
        __syncwarp();
        if (lane == 0) {
          sh.before = mass_before;
          sh.before_n = n_before;
          const uint32_t top = seen_hi - (uint32_t)bin * width;  // bin * width <= seen_hi - seen_lo for a bin with elements
          sh.key_hi = top;
          sh.key_lo = top - seen_lo >= width ? top - width + 1u : seen_lo;
          sh.list_n = 0; sh.seen_lo = 0xffffffffu; sh.seen_hi = 0u;
        }
      }
      cluster.sync();
    }
    cluster.sync();
    const u64 through = lead->found_before + lead->found_w;
    if (stage == 0) { base_mass = through; kept = min(kept, through); }
    if (stage == 1) kept = min(kept, through);
    if (stage == 2) {
      const int id = lead->found_id;
      if (id >= 0) {
        if (rank == 0 && tid == 0) next[row_id] = id;
      } else {
        // number found_j of the elements with this bit pattern, in token order: block by block, then round by round
        const uint32_t key = lead->found_key;
        int mine = 0;
        for (int i0 = 0; i0 < part; i0 += THREADS) {
          const int i = i0 + tid;
          mine += __syncthreads_count(i < R.n && sample_key(R.src[i]) == key);
        }
        if (tid == 0) lead->part_n[rank] = mine;
        cluster.sync();
        long long want = (long long)lead->found_j;
        for (int c = 0; c < rank; ++c) want -= lead->part_n[c];
        if (want >= 0 && want < mine) {                          // uniform over the block
          int before = 0;
          for (int i0 = 0; i0 < part; i0 += THREADS) {
            const int i = i0 + tid;
            const bool match = i < R.n && sample_key(R.src[i]) == key;
            const int cnt = __syncthreads_count(match);
            if (want < before + cnt) {
              const unsigned ballot = __ballot_sync(0xffffffffu, match);
              if (lane == 0) sh.redi[warp] = __popc(ballot);
              __syncthreads();
              int place = before + __popc(ballot & ((1u << lane) - 1u));
              for (int wI = 0; wI < warp; ++wI) place += sh.redi[wI];
              if (match && place == (int)want) next[row_id] = R.id0 + i;
              break;
            }
            before += cnt;
          }
        }
      }
    }
    cluster.sync();                                              // block 0's memory stays until everybody has read it
  }
}

}  // namespace sd
