// Token selection with each row's own temperature, top-k, top-p and min-p.
//
// A cluster of C blocks shares one row, block c its c-th contiguous part.  Weights are w = 2^F exp((x - max) / T) rounded to
// integers (computed in double precision; F as large as 63-bit sums over the vocabulary allow, 47 for 50 272 tokens), so that every
// sum is exact and independent of the order in which threads add, and a comparison at a border comes out as in 64-bit floating
// point.
//
//   1. The row's maximum and smallest finite value, across the cluster.
//   2. A histogram of weight (and of counts, if top-k asks for them) over 1024 slices of equal width in max - x, which cut the
//      order "largest logit first" into consecutive pieces; each element's slice is remembered in 16 bits.  Shared memory
//      has no native 64-bit atomic addition, so a weight is added to two 32-bit counters, the carry of the lower going to the
//      upper.  Every block ends up with the whole row's totals.
//   3. Up to three searches for the element at which a running sum (or count) passes a target: rank top_k - 1, then top_p of
//      the mass found, then the draw.  Every block finds the slice, sends its elements of that slice to all blocks of the cluster, and
//      after one cluster barrier each ranks the same list by comparing all pairs.  A slice with more than LIST elements is first cut
//      again, into 1024 pieces of the elements' bit patterns, until it is small enough or all its elements are equal; equal ones
//      are told apart by counting.
// min-p is a threshold on w: the mass above it is a plain sum of step 2.  All three cut a prefix of the same order, so the kept
// mass is the smallest of the three, and the draw needs no list of kept tokens.
//
// What bounds it: 256 rows of 50 272 logits take 66 us, two rounds of blocks; the bytes would take 8.  Half of a block's 62 000 clocks is
// step 2, bound by instruction issue: some forty per logit, a third of them in double precision at half rate (sums in fp32 would not
// place a border as 64-bit floating point does).  33 rows of 1021: 11 us, one row of 50 272 in 8 blocks: 18 us, a chain of
// barriers and searches.
#pragma once
#include <cooperative_groups.h>
#include <cstdint>
#include <cuda_runtime.h>

#include "sample.cuh"
#include "paged.cuh"

namespace sd {
namespace sr {

namespace cg = cooperative_groups;

constexpr int BINS = 1024;
constexpr int LIST = 384;
constexpr int MAX_SMEM = 227 * 1024;
typedef unsigned long long u64;

struct alignas(16) Shared {
  u64 mass[BINS];                       // the row's totals per slice, summed up: everything in this slice and ahead of it
  uint32_t count[BINS];
  union {
    struct { uint32_t lo[BINS + 32], hi[BINS + 32], num[BINS + 32]; };         // this block's counters; the last 32 are never read
    struct { u64 mine_w[2][LIST], mine_key[2][LIST]; };                        // this block's elements of a slice, for the others to read
  };
  union {                               // a finer cut is made only when a list would be too short
    struct { u64 list_w[LIST], list_key[LIST]; };                              // the row's elements of a slice
    struct { u64 sub_mass[BINS]; uint32_t sub_count[BINS]; };
  };
  int mine_n[3];
  uint32_t seen_lo[3], seen_hi[3];      // smallest and largest bit pattern among this block's elements of each search
  double exp_table[32];
  u64 red[32], red2[32];
  float redf[32], redf2[32];
  int redi[32];
  float m, lowest;                      // this block's, then read by the others
  double c, reach, min_y, min_dx;       // of the settings: log2(e) / T; how far below the maximum weights reach; min-p as an exponent and a distance
  u64 z, z_min_p;
  int best;                             // greedy: lowest index of the maximum in this block
  int bin;                              // of the latest search
  u64 ahead, ahead_other;
  u64 found_before, found_w;            // the element: mass ahead of it and its weight
  u64 found_key;                        // bit pattern above, inverted token id below
  u64 found_j;
  int found_equal;                      // 1: one of several equal elements, number found_j of them in token order
  int part_n;                           // equal elements in this block
};

// exp in double precision, the table method (Tang 1989): 2^y = 2^(k / 32) * 2^f with |f| <= 1/64 and a Taylor polynomial
// (coefficients ln2^i / i!) whose first left-out term is below 4e-18.  Returns round(2^fraction * 2^y) for
// -(fraction + 2) < y <= 0; fraction <= 52.  Integers are taken from the low bits of sums with large constants: the conversion
// instructions run at a quarter of the rate of the double-precision ones.  The table has one entry per lane so that the
// histogram's loop can keep it in registers and look it up by shuffles: look-ups in shared memory, at 32 different places, had more
// bank conflicts than the histogram's own additions.
struct Exponent {
  double p;                              // 2^f
  int k;
};
__device__ __forceinline__ Exponent reduce(double y) {
  constexpr double L = 0.6931471805599453094;
  const double magic = 6755399441055744.0 / 32.0;              // 1.5 * 2^52 / 32: adding it leaves multiples of 1/32
  const double t = y + magic;
  const double f = y - (t - magic);
  double p = fma(f, L * L * L * L * L * L / 720.0, L * L * L * L * L / 120.0);
  p = fma(p, f, L * L * L * L / 24.0);
  p = fma(p, f, L * L * L / 6.0);
  p = fma(p, f, L * L / 2.0);
  p = fma(p, f, L);
  return {fma(p, f, 1.0), __double2loint(t)};                    // k = round(32 y), two's complement
}
__device__ __forceinline__ u64 weight_of(const Exponent& e, double entry, int fraction) {
  const double v = e.p * entry;
  const double scaled = __hiloint2double(__double2hiint(v) + (((e.k >> 5) + fraction) << 20), __double2loint(v));
  return (u64)(__double_as_longlong(scaled + 4503599627370496.0) - 0x4330000000000000ll);      // 2^52, whose last place is 1
}
__device__ __forceinline__ u64 weight_of(double y, const double* table, int fraction) {
  const Exponent e = reduce(y);
  return weight_of(e, table[e.k & 31], fraction);
}
// A float as a double, by its bits: exact for normal numbers; zero and subnormal ones become other numbers below 2^-125.
__device__ __forceinline__ double widen_bits(float x) {
  const uint32_t b = __float_as_uint(x);
  return __hiloint2double((int)((((b >> 3) & 0x0fffffffu) + 0x38000000u) | (b & 0x80000000u)), (int)(b << 29));
}

struct Row {
  const float* src;                     // this block's part of the row
  int n, id0;
  double m, c;                          // maximum; log2(e) / T
  float floor;                          // logits at or below it (minus infinity among them) and NaN weigh nothing: less than 2^-1.4 units
  float mf, slice_scale;
  __device__ __forceinline__ double exponent(float x) const { return (widen_bits(x) - m) * c; }
  __device__ __forceinline__ bool weighs(float x) const { return x > floor; }
  // slice of a logit that weighs something: a monotone function of it, rounded to an integer by a sum with 2^23
  __device__ __forceinline__ int slice(float x) const {
    return (int)(__float_as_uint(fminf((mf - x) * slice_scale, (float)(BINS - 1)) + 8388608.f) & (BINS - 1));
  }
};
__device__ __forceinline__ void add64(uint32_t* lo, uint32_t* hi, u64 w) {
  const uint32_t l = (uint32_t)w;
  const uint32_t h = (uint32_t)(w >> 32) + (atomicAdd(lo, l) > ~l ? 1u : 0u);
  if (h) atomicAdd(hi, h);
}

// Two sums over the block at once; every thread gets both.
template <int THREADS>
__device__ __forceinline__ void block_sums(u64& a, u64& b, Shared& sh) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) { a += __shfl_xor_sync(0xffffffffu, a, o); b += __shfl_xor_sync(0xffffffffu, b, o); }
  if (lane == 0) { sh.red[warp] = a; sh.red2[warp] = b; }
  __syncthreads();
  a = lane < THREADS / 32 ? sh.red[lane] : 0ull;
  b = lane < THREADS / 32 ? sh.red2[lane] : 0ull;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) { a += __shfl_xor_sync(0xffffffffu, a, o); b += __shfl_xor_sync(0xffffffffu, b, o); }
}

// Inclusive sums of the BINS values in place, over the block.
template <int THREADS, typename T>
__device__ __forceinline__ void block_scan(T* v, Shared& sh) {
  constexpr int PER = BINS / THREADS;
  static_assert(PER == 1 || PER == 2, "one or two values per thread");
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const T last = v[PER * threadIdx.x + PER - 1];
  u64 run = (u64)last + (PER == 2 ? v[PER * threadIdx.x] : (T)0);
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const u64 x = __shfl_up_sync(0xffffffffu, run, o);
    if (lane >= o) run += x;
  }
  if (lane == 31) sh.red[warp] = run;
  __syncthreads();
  u64 w = lane < warp ? sh.red[lane] : 0ull;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) w += __shfl_xor_sync(0xffffffffu, w, o);
  run += w;
  if (PER == 2) v[PER * threadIdx.x] = (T)(run - last);
  v[PER * threadIdx.x + PER - 1] = (T)run;
  __syncthreads();
}

// The bin at which the summed-up values first exceed target (base included in them): sh.bin, and what is ahead of it in these
// values (sh.ahead) and in the other ones (sh.ahead_other).  sh.bin = BINS when they never do.
template <int THREADS, typename T, typename U>
__device__ __forceinline__ void find_bin(const T* sums, const U* others, u64 base, u64 target, Shared& sh) {
  if (threadIdx.x == 0) sh.bin = BINS;
  __syncthreads();
#pragma unroll
  for (int i = threadIdx.x; i < BINS; i += THREADS) {
    const u64 ahead = base + (i ? (u64)sums[i - 1] : 0ull);
    if (ahead <= target && target < base + (u64)sums[i]) {
      sh.bin = i;
      sh.ahead = ahead;
      sh.ahead_other = i ? (u64)others[i - 1] : 0ull;
    }
  }
  __syncthreads();
}

}  // namespace sr

// ONE: a row per block (C = 1), without the cluster's barriers, which cost about a thousand clocks each even then.
// grid (C * rows), cluster (C): block c of a cluster holds elements [c * part, ...) of its row.  SLICES: the elements' slices fit
// in shared memory (16 bits each); otherwise they are worked out again when they are asked for.
template <int THREADS, bool ONE, bool SLICES>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS)
sample_rows_kernel(const float* __restrict__ logits, int vocab, int part, int fraction, const float* __restrict__ uniforms,
                   const float* __restrict__ temperatures, const int32_t* __restrict__ top_ks, const float* __restrict__ top_ps,
                   const float* __restrict__ min_ps, int32_t* __restrict__ next, int* __restrict__ status) {
  using namespace sr;
  extern __shared__ __align__(16) unsigned char sr_smem[];
  Shared& sh = *reinterpret_cast<Shared*>(sr_smem);
  uint16_t* slices = reinterpret_cast<uint16_t*>(sr_smem + sizeof(Shared));
  cg::cluster_group cluster = cg::this_cluster();
  const int C = ONE ? 1 : (int)cluster.num_blocks(), rank = ONE ? 0 : (int)cluster.block_rank();
  const int row_id = blockIdx.x / C;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  auto block = [&](int c) -> Shared* { return ONE ? &sh : cluster.map_shared_rank(&sh, c); };
  auto at_block = [&](auto* p, int c) { return ONE ? p : cluster.map_shared_rank(p, c); };
  auto sync_row = [&] { if (ONE) __syncthreads(); else cluster.sync(); };

  Row R;
  R.id0 = min(rank * part, vocab);
  R.n = min(vocab - R.id0, part);
  R.src = logits + (size_t)row_id * vocab + R.id0;

  // the row's random number and settings; a setting that is none makes the row greedy
  float u = uniforms[row_id];
  u = u >= 0.f ? fminf(u, 1.f) : 0.f;
  const float T = temperatures ? temperatures[row_id] : 1.f;
  const int top_k = top_ks ? top_ks[row_id] : 0;
  const float top_p = top_ps ? top_ps[row_id] : 1.f;
  const float min_p = min_ps ? min_ps[row_id] : 0.f;
  const bool bad = !(T >= 0.f) || T == INFINITY || top_p != top_p || min_p != min_p;
  const bool greedy = bad || T == 0.f;
  if (bad && tid == 0 && rank == 0) atomicOr(status, STATUS_BAD_SETTING);

  for (int i = tid; i < BINS; i += THREADS) { sh.lo[i] = 0u; sh.hi[i] = 0u; sh.num[i] = 0u; }
  if (tid == 32) {                                               // one thread for the long operations, while the loads are on their way
    sh.c = 1.4426950408889634074 / (double)T;
    sh.reach = ((double)fraction + 1.4) * 0.6931471805599453094 * (double)T;
    sh.min_y = min_p > 0.f && min_p <= 1.f ? log2((double)min_p) - 8e-17 : 0.0;   // log2(1 - 2^-54): what rounds to 1 in 64 bits counts as 1
    sh.min_dx = sh.min_y * 0.6931471805599453094 * (double)T;
  }
  if (tid < 32) sh.exp_table[tid] = exp2((double)tid / 32.0);
  if (tid < 3) { sh.mine_n[tid] = 0; sh.seen_lo[tid] = 0xffffffffu; sh.seen_hi[tid] = 0u; }

  // 1. maximum and smallest finite value
  const bool wide = (reinterpret_cast<uintptr_t>(R.src) & 15) == 0;
  const int n4 = wide ? R.n >> 2 : 0;
  float m = -INFINITY, low = INFINITY;
#pragma unroll 4
  for (int i = tid; i < n4; i += THREADS) {
    const float4 v = __ldg(reinterpret_cast<const float4*>(R.src) + i);
    m = fmaxf(fmaxf(fmaxf(m, v.x), fmaxf(v.y, v.z)), v.w);       // NaN is dropped
    const float l = fminf(fminf(v.x, v.y), fminf(v.z, v.w));
    if (l > -INFINITY) low = fminf(low, l);
    else {                                                       // masked logits among the four
      if (v.x > -INFINITY) low = fminf(low, v.x);
      if (v.y > -INFINITY) low = fminf(low, v.y);
      if (v.z > -INFINITY) low = fminf(low, v.z);
      if (v.w > -INFINITY) low = fminf(low, v.w);
    }
  }
  for (int i = 4 * n4 + tid; i < R.n; i += THREADS) {
    const float x = __ldg(R.src + i);
    m = fmaxf(m, x);
    if (x > -INFINITY) low = fminf(low, x);
  }
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
  sync_row();
  {
    const Shared* other = block(lane < C ? lane : 0);
    m = other->m;
    low = other->lowest;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
      low = fminf(low, __shfl_xor_sync(0xffffffffu, low, o));
    }
  }

  if (greedy || !(m > -INFINITY) || m == INFINITY) {
    // the lowest index of the maximum; uniform over the cluster.  Where that is minus infinity every logit is one, NaN among them
    const bool any = !(m > -INFINITY);
    int best = 0x7fffffff;
    for (int i = tid; i < R.n; i += THREADS)
      if (any || __ldg(R.src + i) == m) { best = R.id0 + i; break; }
    best = __reduce_min_sync(0xffffffffu, best);
    if (lane == 0) sh.redi[warp] = best;
    __syncthreads();
    if (warp == 0) {
      best = __reduce_min_sync(0xffffffffu, lane < THREADS / 32 ? sh.redi[lane] : 0x7fffffff);
      if (lane == 0) sh.best = best;
    }
    sync_row();
    if (rank == 0 && tid == 0) {
      for (int c = 0; c < C; ++c) best = min(best, block(c)->best);
      next[row_id] = best == 0x7fffffff ? 0 : best;
    }
    sync_row();                                              // nobody leaves while its memory may be read
    return;
  }

  R.mf = m;
  R.m = widen_bits(m);
  R.c = sh.c;
  const double reach = sh.reach;
  // rounded down, and below the maximum: the next float above the floor is in reach, the maximum always is
  R.floor = fminf(__double2float_rd((double)m - reach), nextafterf(m, -INFINITY));
  {
    const float span = (float)fmin((double)m - (double)low, reach);   // the slices cover what the row has, or what weighs anything
    R.slice_scale = (float)(BINS - 1) / fmaxf(span, 1e-30f);
    if (!(R.slice_scale < 1e30f)) R.slice_scale = 0.f;           // all equal: one slice
  }

  // 2. the histogram
  const bool want_counts = top_k > 0 && top_k < vocab;
  // w >= min_p, as a bound on the logit: the smallest float whose exponent is at least log2 min_p
  float min_x = INFINITY;
  if (min_p > 0.f && min_p <= 1.f) {
    min_x = fminf((float)(R.m + sh.min_dx), m);
    if (R.exponent(min_x) < sh.min_y) min_x = fminf(nextafterf(min_x, INFINITY), m);
  }
  u64 z = 0ull, zm = 0ull;
  const int entry_lo = __double2loint(sh.exp_table[lane]), entry_hi = __double2hiint(sh.exp_table[lane]);
  // Four logits at a time, so that their chains of double-precision operations overlap; returns their slices.  For whole warps.
  auto enter = [&](const float (&x)[4], uint32_t (&s)[4]) {
    u64 w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const bool in = R.weighs(x[k]);
      const Exponent e = reduce(R.exponent(x[k]));
      w[k] = weight_of(e, __hiloint2double(__shfl_sync(0xffffffffu, entry_hi, e.k & 31), __shfl_sync(0xffffffffu, entry_lo, e.k & 31)), fraction);
      if (!in) w[k] = 0ull;                                      // out of weight_of's range
      s[k] = in ? (uint32_t)R.slice(x[k]) : (uint32_t)(BINS + lane);     // beyond the slices, without bank conflicts
      z += w[k];
      if (x[k] >= min_x) zm += w[k];
    }
    uint32_t h[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t l = (uint32_t)w[k];
      h[k] = (uint32_t)(w[k] >> 32);
      h[k] += atomicAdd(&sh.lo[s[k]], l) > ~l ? 1u : 0u;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (h[k]) atomicAdd(&sh.hi[s[k]], h[k]);
    if (want_counts) {
#pragma unroll
      for (int k = 0; k < 4; ++k) atomicAdd(&sh.num[s[k]], 1u);
    }
  };
  const float4 none = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
  auto fetch = [&](int i) { return i < n4 ? __ldg(reinterpret_cast<const float4*>(R.src) + i) : none; };
  float4 ahead = fetch(tid);
  for (int i = tid; i - tid < n4; i += THREADS) {
    const float x[4] = {ahead.x, ahead.y, ahead.z, ahead.w};
    ahead = fetch(i + THREADS);
    uint32_t s[4];
    enter(x, s);
    if (SLICES && i < n4) reinterpret_cast<uint2*>(slices)[i] = make_uint2(s[0] | s[1] << 16, s[2] | s[3] << 16);
  }
  for (int i0 = 4 * n4; i0 < R.n; i0 += 4 * THREADS) {           // rows that are not 16-byte aligned, and the last elements of others
    float x[4];
    uint32_t s[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = i0 + k * THREADS + tid < R.n ? __ldg(R.src + i0 + k * THREADS + tid) : -INFINITY;   // weighs nothing
    enter(x, s);
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (SLICES && i0 + k * THREADS + tid < R.n) slices[i0 + k * THREADS + tid] = (uint16_t)s[k];
  }
  block_sums<THREADS>(z, zm, sh);
  if (tid == 0) { sh.z = z; sh.z_min_p = zm; }
  sync_row();
  // every block adds up its share of the slices over the cluster and gives it to all
  const int share = BINS / C;
  auto total = [&](u64* mass, uint32_t* count, bool counts) {
    // C / 2 neighbouring threads share a slice, each with two of the blocks: one round of remote accesses (C is a power of two)
    const int subs = max(C / 2, 1), sub = tid & (subs - 1);
    for (int i = rank * share + tid / subs; i < (rank + 1) * share; i += THREADS / subs) {
      u64 t = 0ull;
      uint32_t n = 0u;
      const int c0 = sub, c1 = sub + subs;
      const Shared *one = block(c0), *two = block(c1 < C ? c1 : c0);
      t = (u64)one->lo[i] + ((u64)one->hi[i] << 32);
      if (counts) n = one->num[i];
      if (c1 < C) {
        t += (u64)two->lo[i] + ((u64)two->hi[i] << 32);
        if (counts) n += two->num[i];
      }
      for (int o = 1; o < subs; o <<= 1) { t += __shfl_xor_sync(0xffffffffu, t, o); n += __shfl_xor_sync(0xffffffffu, n, o); }
      at_block(mass, c0)[i] = t;
      if (counts) at_block(count, c0)[i] = n;
      if (c1 < C) {
        at_block(mass, c1)[i] = t;
        if (counts) at_block(count, c1)[i] = n;
      }
    }
  };
  total(sh.mass, sh.count, want_counts);
  z = 0ull; zm = 0ull;
#pragma unroll 4
  for (int c = 0; c < C; ++c) {
    const Shared* other = block(c);
    z += other->z;
    zm += other->z_min_p;
  }
  sync_row();
  block_scan<THREADS>(sh.mass, sh);
  if (want_counts) block_scan<THREADS>(sh.count, sh);

  // 3. the searches.  All blocks run the same control flow on equal values.
  u64 kept = min_p > 0.f ? (zm > 0ull ? zm : (1ull << fraction)) : z;   // min_p > 1 keeps the maximum alone
  u64 base_mass = z;                                              // mass of the top-k set
  int buf = 0;                                                    // list buffers take turns, so a search needs one cluster barrier
  for (int stage = 0; stage < 3; ++stage) {
    u64 target;
    const bool by_rank = stage == 0;
    if (stage == 0) {
      if (!want_counts) continue;
      target = (u64)(top_k - 1);
    } else if (stage == 1) {
      if (!(top_p < 1.f)) continue;
      const u64 want = __double2ull_ru((double)top_p * (double)base_mass);     // a negative top_p gives 0
      target = want > 0ull ? min(want, base_mass) - 1ull : 0ull;
    } else {
      target = __double2ull_rd((double)u * (double)kept);
      if (target >= kept) target = kept - 1ull;
    }
    // which slice; everything ahead of it (mass and, for a rank, number)
    if (by_rank) find_bin<THREADS>(sh.count, sh.mass, 0ull, target, sh);
    else find_bin<THREADS>(sh.mass, sh.mass, 0ull, target, sh);
    const int slice = sh.bin;
    if (slice == BINS) { __syncthreads(); continue; }            // fewer than top_k elements weigh anything: the whole row
    u64 before = by_rank ? sh.ahead_other : sh.ahead;
    u64 before_n = by_rank ? sh.ahead : 0ull;
    uint32_t key_lo = 0u, key_hi = 0xffffffffu;
    while (true) {
      // this block's confined elements
      if (tid == 0) { sh.mine_n[stage] = 0; sh.seen_lo[stage] = 0xffffffffu; sh.seen_hi[stage] = 0u; }
      __syncthreads();
      auto look = [&](int i, bool in) {
        float x = 0.f;
        uint32_t key = 0u;
        if (in) {
          x = __ldg(R.src + i);
          key = sample_key(x);
          if (!SLICES) in = R.weighs(x) && R.slice(x) == slice;
          in = in && key >= key_lo && key <= key_hi;
        }
        if (in) {
          const int at = atomicAdd(&sh.mine_n[stage], 1);
          if (at < LIST) {
            sh.mine_key[buf][at] = (u64)key << 32 | (uint32_t)~(R.id0 + i);
            sh.mine_w[buf][at] = weight_of(R.exponent(x), sh.exp_table, fraction);
          }
          atomicMin(&sh.seen_lo[stage], key);
          atomicMax(&sh.seen_hi[stage], key);
        }
      };
      if (SLICES) {
        const uint32_t want = (uint32_t)slice * 0x10001u;
        for (int i = 8 * tid; i < R.n; i += 8 * THREADS) {        // 8 slices per thread and round
          const uint4 v = *reinterpret_cast<const uint4*>(slices + i);
          const uint32_t w[4] = {v.x ^ want, v.y ^ want, v.z ^ want, v.w ^ want};      // a half that is zero: this slice
          auto zeros = [](uint32_t t) { return (t - 0x00010001u) & ~t & 0x80008000u; };    // may name an upper half of 1 above a zero
          if ((zeros(w[0]) | zeros(w[1]) | zeros(w[2]) | zeros(w[3])) == 0u) continue;
#pragma unroll
          for (int k = 0; k < 8; ++k)
            if (i + k < R.n && ((w[k >> 1] >> (16 * (k & 1))) & 0xffffu) == 0u) look(i + k, true);
        }
      } else {
        for (int i = tid; i < R.n; i += THREADS) look(i, true);
      }
      sync_row();
      // everybody's: lane c asks block c
      const Shared* other = block(lane < C ? lane : 0);
      const int their_n = lane < C ? other->mine_n[stage] : 0;
      const uint32_t seen_lo = __reduce_min_sync(0xffffffffu, other->seen_lo[stage]);
      const uint32_t seen_hi = __reduce_max_sync(0xffffffffu, other->seen_hi[stage]);
      const int n = __reduce_add_sync(0xffffffffu, their_n);
      if (n <= LIST) {
        // one list of all (a warp per block); then each element's place: everything ahead of it
        int at = their_n;                                        // lane c: where block c's elements go
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int v = __shfl_up_sync(0xffffffffu, at, o);
          if (lane >= o) at += v;
        }
        at -= their_n;
        for (int c = warp; c < C; c += THREADS / 32) {
          const int m_c = __shfl_sync(0xffffffffu, their_n, c), at_c = __shfl_sync(0xffffffffu, at, c);
          const Shared* from = block(c);
          for (int e = lane; e < m_c; e += 32) { sh.list_key[at_c + e] = from->mine_key[buf][e]; sh.list_w[at_c + e] = from->mine_w[buf][e]; }
        }
        __syncthreads();
        constexpr int LANES = 8;                                 // threads that share an element's comparisons
        for (int e0 = 0; e0 < n; e0 += THREADS / LANES) {
          const int e = e0 + tid / LANES;
          const u64 k = e < n ? sh.list_key[e] : ~0ull;
          u64 ahead = 0ull;
          uint32_t ahead_n = 0u;
#pragma unroll 4
          for (int o = tid % LANES; o < n; o += LANES) {
            const bool earlier = sh.list_key[o] > k;
            ahead += earlier ? sh.list_w[o] : 0ull;
            ahead_n += earlier ? 1u : 0u;
          }
#pragma unroll
          for (int o = LANES / 2; o > 0; o >>= 1) {
            ahead += __shfl_xor_sync(0xffffffffu, ahead, o);
            ahead_n += __shfl_xor_sync(0xffffffffu, ahead_n, o);
          }
          if (e < n && tid % LANES == 0) {
            const u64 w = sh.list_w[e];
            ahead += before;
            const bool hit = by_rank ? before_n + ahead_n == target : (ahead <= target && target < ahead + w);
            if (hit) { sh.found_before = ahead; sh.found_w = w; sh.found_key = k; sh.found_equal = 0; }
          }
        }
        break;
      }
      if (seen_lo == seen_hi) {                                  // all equal: the place follows by division
        if (tid == 0) {
          const u64 w = weight_of(R.exponent(sample_unkey(seen_lo)), sh.exp_table, fraction);
          const u64 j = by_rank ? target - before_n : (target - before) / w;
          sh.found_before = before + j * w;
          sh.found_w = w;
          sh.found_key = (u64)seen_lo << 32;
          sh.found_equal = 1;
          sh.found_j = j;
        }
        break;
      }
      // cut the confined bit patterns into at most BINS pieces, largest first
      const uint32_t width = (uint32_t)(((u64)(seen_hi - seen_lo) + BINS) / BINS);
      for (int i = tid; i < BINS; i += THREADS) { sh.lo[i] = 0u; sh.hi[i] = 0u; sh.num[i] = 0u; }
      __syncthreads();
      for (int i = tid; i < R.n; i += THREADS) {
        if (SLICES && slices[i] != slice) continue;
        const float x = __ldg(R.src + i);
        const uint32_t key = sample_key(x);
        if (!SLICES && (!R.weighs(x) || R.slice(x) != slice)) continue;
        if (key < key_lo || key > key_hi) continue;
        const uint32_t p = (seen_hi - key) / width;
        add64(&sh.lo[p], &sh.hi[p], weight_of(R.exponent(x), sh.exp_table, fraction));
        atomicAdd(&sh.num[p], 1u);
      }
      sync_row();
      total(sh.sub_mass, sh.sub_count, true);
      sync_row();
      block_scan<THREADS>(sh.sub_mass, sh);
      block_scan<THREADS>(sh.sub_count, sh);
      if (by_rank) {
        find_bin<THREADS>(sh.sub_count, sh.sub_mass, before_n, target, sh);
        before += sh.ahead_other;
        before_n = sh.ahead;
      } else {
        find_bin<THREADS>(sh.sub_mass, sh.sub_mass, before, target, sh);
        before = sh.ahead;
      }
      const uint32_t top = seen_hi - (uint32_t)min(sh.bin, BINS - 1) * width;   // bin * width <= seen_hi - seen_lo for a bin with elements
      key_hi = top;
      key_lo = top - seen_lo >= width ? top - width + 1u : seen_lo;
      __syncthreads();                                           // the counters become lists again
    }
    __syncthreads();
    const u64 through = sh.found_before + sh.found_w;
    if (stage == 0) { base_mass = through; kept = min(kept, through); }
    if (stage == 1) kept = min(kept, through);
    if (stage == 2) {
      if (!sh.found_equal) {
        if (rank == 0 && tid == 0) next[row_id] = (int32_t)~(uint32_t)sh.found_key;
      } else {
        // number found_j of the elements with this bit pattern, in token order: block by block, then round by round
        const uint32_t key = (uint32_t)(sh.found_key >> 32);
        int mine = 0;
        for (int i0 = 0; i0 < part; i0 += THREADS) {
          const int i = i0 + tid;
          mine += __syncthreads_count(i < R.n && sample_key(__ldg(R.src + i)) == key);
        }
        if (tid == 0) sh.part_n = mine;
        sync_row();
        long long want = (long long)sh.found_j;
        for (int c = 0; c < rank; ++c) want -= block(c)->part_n;
        if (want >= 0 && want < mine) {                          // uniform over the block
          int ahead = 0;
          for (int i0 = 0; i0 < part; i0 += THREADS) {
            const int i = i0 + tid;
            const bool match = i < R.n && sample_key(__ldg(R.src + i)) == key;
            const int cnt = __syncthreads_count(match);
            if (want < ahead + cnt) {
              const unsigned ballot = __ballot_sync(0xffffffffu, match);
              if (lane == 0) sh.redi[warp] = __popc(ballot);
              __syncthreads();
              int place = ahead + __popc(ballot & ((1u << lane) - 1u));
              for (int wI = 0; wI < warp; ++wI) place += sh.redi[wI];
              if (match && place == (int)want) next[row_id] = R.id0 + i;
              break;
            }
            ahead += cnt;
          }
        }
      }
    }
    buf ^= 1;                                                    // read last before a barrier that everybody has passed by its next turn
  }
  sync_row();                                                // nobody leaves while its memory may be read
}

}  // namespace sd
