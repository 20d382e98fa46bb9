// Attention of few query rows over a paged cache in bf16 or 8 bits: single tokens, and chunks whose results are wanted in
// fp32.  One block per (sequence, key head, tile of 8 query rows, split of the keys); a query row is a (token, head of the group)
// pair, so grouped heads share the keys they read.
//
// What bounds it is the cache's bytes.  Three single tokens of 32 heads over 8 key heads of 128 at 20 000..65 521 positions in bf16: 120 us,
// 5.9 TB/s of 6.4 that a plain copy reaches.  64 single tokens of 32 heads of 128 at 1024..1536 positions in int8: 138 us,
// 4.8 TB/s; there the conversion of codes and the four products per piece of a key keep the issue slots half busy, and registers leave three
// blocks per SM (with the queries in shared memory and four blocks: 153 us; two warps per block: 147..174 us).
//
// The products run on the tensor cores (m16n8k16, fp32 accumulation) because the CUDA
// cores could not convert and multiply 8-bit elements at the rate at which the memory delivers them (23 per clock and SM).  The
// 16 rows of a tile are the 8 query rows twice: once the upper and once the lower half of each query element (and of
// each softmax weight), two 16-bit numbers that together keep 16 bits in bf16 and 22 in fp16, so the operands' rounding stays
// near fp32 at no cost: with 8 rows or fewer the other half of the tile would be empty.  8-bit codes are fp16 numbers exactly.
// bf16 caches multiply in bf16, and where results are fp32 with a third part of each operand, 24 bits, in products of their own (the form
// THIRD): relative to 64-bit arithmetic 4.8e-7 instead of 3e-6.  64 single tokens at 1280, 32 heads of 128: 221 us (211 without the third
// part), 3 of 32 heads over 8 at 65 000: 164 (156); 4 x 512 tokens at 2048, where the products are what it does, 975 (700).
//
// Each of the block's four warps walks its own 16-key tiles with a ring of its own in shared memory, filled by 16-byte asynchronous copies: no
// block-wide synchronisation until the end, and every warp keeps STAGES - 1 tiles in flight.  The fragments are read in the order
// in which the bytes lie: the sum over the head's elements may run in any order, so a thread takes whole 16-byte pieces of a key
// and the queries are laid out to match; for the values, a thread takes a run of elements of four keys, and the
// accumulator's columns stand for the elements that order implies.  Pieces are XOR-swizzled against bank conflicts.
//
// 8-bit scales.  A key's scale multiplies its score.  A value's scale joins its weight, relative to a power of two that no scale
// seen so far exceeds (ve) and times 2^7.  That power and the running maximum (m) are raised only when a scale passes the one or a
// score the other by 2^8, so most tiles need no reduction across lanes and no rescaling: weights stay below 2^15, inside fp16, whose
// grid ends at 2^-24: a weight is exact to 2^-32 of the largest |value| of the sequence.
#pragma once
#include "attn_prefill.cuh"
#include "paged.cuh"

namespace sd {
namespace ap {

constexpr int NW = 4, THREADS = 32 * NW, ROWS = 8, KEYS = 16;

template <typename TC, int HD> struct Shape {
  static constexpr bool SCALED = CacheType<TC>::TOP > 0.f;
  static constexpr int E = sizeof(TC);
  static constexpr int ROW = HD * E;                         // bytes of a key
  static constexpr int PIECES = ROW / 16;
  static constexpr int SWZ = PIECES < 8 ? PIECES - 1 : 7;
  static constexpr int EC = 16 / E < HD / 4 ? 16 / E : HD / 4;   // elements a thread reads at a time for the scores
  static constexpr int NCH = HD / (4 * EC);
  static constexpr int KS = HD / 16, NT = HD / 8;
  static constexpr int STAGE = 2 * KEYS * ROW + (SCALED ? 2 * KEYS * 4 : 0);
  // two blocks of 98 KB per SM (bf16, 128 elements), else three or four of 50 to 66 KB, as registers allow
  static constexpr int STAGES = STAGE >= 8192 ? 3 : STAGE >= 4096 ? 4 : 6;
  static constexpr int MERGE = NW * ROWS * (HD + 2) * 4;
  static constexpr int SMEM = NW * STAGES * STAGE > MERGE ? NW * STAGES * STAGE : MERGE;
};

__device__ __forceinline__ int swz(int key) { return ((key & 1) << 2) | ((key >> 1) & 3); }

__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, __nv_bfloat16) { pf_mma(c, a, b0, b1); }
template <typename T>
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, T) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// two floats as packed 16-bit pairs: the values rounded, and what the rounding left
__device__ __forceinline__ void split(float x, float y, uint32_t& hi, uint32_t& lo, __nv_bfloat16) { pf_split(x, y, hi, lo); }
template <typename T> __device__ __forceinline__ void split(float x, float y, uint32_t& hi, uint32_t& lo, T) {
  const __half hx = __float2half_rn(x), hy = __float2half_rn(y);
  hi = (uint32_t)__half_as_ushort(hx) | ((uint32_t)__half_as_ushort(hy) << 16);
  lo = pack_f16(x - __half2float(hx), y - __half2float(hy));
}

// what the two parts of split() leave of a bf16 operand, rounded: a third part, 24 bits in all
__device__ __forceinline__ uint32_t third_of(float x, float y, uint32_t hi, uint32_t lo) {
  const float hx = __uint_as_float(hi << 16), hy = __uint_as_float(hi & 0xffff0000u), lx = __uint_as_float(lo << 16), ly = __uint_as_float(lo & 0xffff0000u);
  return pack_bf16((x - hx) - lx, (y - hy) - ly);
}

// Codes to fp16 pairs.  flip() prepares a word of four codes; lower(), upper() give its first and last two as fp16.  An int8
// with its sign bit flipped is the code plus 128, and 0x64 above a byte makes it the fp16 number 1024 + byte.
__device__ __forceinline__ uint32_t flip(uint32_t w, int8_t) { return w ^ 0x80808080u; }
__device__ __forceinline__ uint32_t flip(uint32_t w, e4m3) { return w; }
__device__ __forceinline__ uint32_t minus_1152(uint32_t v) {
  const uint32_t c = 0x64806480u;
  const __half2 d = __hsub2(*reinterpret_cast<const __half2*>(&v), *reinterpret_cast<const __half2*>(&c));
  return *reinterpret_cast<const uint32_t*>(&d);
}
__device__ __forceinline__ uint32_t lower(uint32_t w, int8_t) { return minus_1152(__byte_perm(w, 0x64646464u, 0x4140)); }
__device__ __forceinline__ uint32_t upper(uint32_t w, int8_t) { return minus_1152(__byte_perm(w, 0x64646464u, 0x4342)); }
__device__ __forceinline__ uint32_t widen(uint32_t w) {
  const __half2_raw r = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)w, __NV_E4M3);
  return (uint32_t)r.x | ((uint32_t)r.y << 16);
}
__device__ __forceinline__ uint32_t lower(uint32_t w, e4m3) { return widen(w & 0xffffu); }
__device__ __forceinline__ uint32_t upper(uint32_t w, e4m3) { return widen(w >> 16); }

template <int B> __device__ __forceinline__ void lds(uint32_t addr, uint32_t (&r)[(B + 3) / 4]) {
  if constexpr (B == 16) asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
  else if constexpr (B == 8) asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(r[0]), "=r"(r[1]) : "r"(addr));
  else if constexpr (B == 2) asm volatile("ld.shared.u16 %0, [%1];" : "=r"(r[0]) : "r"(addr));
  else asm volatile("ld.shared.u32 %0, [%1];" : "=r"(r[0]) : "r"(addr));
}
__device__ __forceinline__ float2 lds_f32x2(uint32_t addr) {
  float2 v;
  asm volatile("ld.shared.v2.f32 {%0,%1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr));
  return v;
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Keeps a block, on every way out, until the kernel before has ended.  A launch that was allowed to begin early must not end first:
// what follows it in the stream waits for it alone.
struct UntilPredecessorEnds {
  bool on;
  __device__ __forceinline__ ~UntilPredecessorEnds() { if (on) pdl_wait(); }
};

// Splits that have keys, of `keys` keys; chunk may come from a length that the caller only guessed, up to 2^31.
__device__ __forceinline__ int splits_of(int keys, int chunk, int splits) { return min(splits, (int)(((long long)keys + chunk - 1) / chunk)); }

// N consecutive elements of a row, any type; vec: 16-byte accesses are allowed
template <int N> __device__ __forceinline__ void load_run(const Rows& t, long long at, bool vec, float (&o)[N]) {
  if (vec) {
#pragma unroll
    for (int i = 0; i < N; i += 8) {
      float x[8];
      if (t.dtype == DT_FP32) load8<true>(static_cast<const float*>(t.data) + at + i, x);
      else if (t.dtype == DT_BF16) load8<true>(static_cast<const __nv_bfloat16*>(t.data) + at + i, x);
      else load8<true>(static_cast<const __half*>(t.data) + at + i, x);
#pragma unroll
      for (int j = 0; j < 8; ++j) o[i + j] = x[j];
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = load_elem(t, at + i);
  }
}

}  // namespace ap

// grid (tiles_per_seq * n_kv_heads * n_seqs, splits).  Sequences with rows_below query rows or more are another kernel's.  Split z takes keys
// [z * chunk, (z + 1) * chunk), the last one all that follow.
// Several splits leave partial results (accumulator, maximum, sum) of the rows they see, slot_rows (the most rows that a tile can have) to a
// unit, and the block that arrives last at a unit's counter adds them in split order, so the result does not depend on who came when.
// early: launched to begin once the kernel for chunks of the same call has no block left to start, whose last blocks it runs beside
// (33 sequences of 11..329 new tokens in e4m3: 213 us a call, 221 one after the other).
// THIRD: queries and weights are sums of three parts (bf16 caches, results in fp32), the third in products of its own.
// SC: scores are changed and keys masked as `sc` says; split z counts from the first key that a row of the tile sees.
template <typename TC, int HD, bool THIRD, bool SC>
__global__ void __launch_bounds__(ap::THREADS)
paged_attn_tile_kernel(const BatchView b, const Rows q, const Rows out, const TC* __restrict__ Kp, const TC* __restrict__ Vp,
                       const float* __restrict__ Ksc, const float* __restrict__ Vsc, int group, float scale_log2, bool q_vec,
                       int tiles_per_seq, int rows_below, int chunk, int slot_rows, float* part_acc, float* part_ml, int* __restrict__ counters, bool early, const Scores sc) {
  using namespace ap;
  using S = Shape<TC, HD>;
  extern __shared__ __align__(128) unsigned char ap_smem[];
  __shared__ int sm_last;
  const UntilPredecessorEnds hold{early && blockIdx.x == 0 && blockIdx.y == 0};

  const int unit = blockIdx.x, tile = unit % tiles_per_seq, g_head = (unit / tiles_per_seq) % b.n_kv_heads, seq = unit / tiles_per_seq / b.n_kv_heads;
  const int splits = gridDim.y, z = blockIdx.y;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;

  // the sequence's rows; whatever does not fit the tensors is reported and left out
  const int f0 = b.first[seq], f1 = b.first[seq + 1], len = b.seq_len(seq);
  int n_new = f1 - f0;
  if (f0 < 0 || n_new < 0 || f1 > b.n_tokens || n_new > b.max_new) {
    if (threadIdx.x == 0) b.bad();
    if (f0 < 0 || n_new < 0) return;
    n_new = min(n_new, min(b.max_new, b.n_tokens - f0));
  }
  const int n_rows = min(ROWS, n_new * group - tile * ROWS);
  if (n_rows <= 0 || n_new * group >= rows_below) return;
  const long long pos_first = (long long)b.len[seq] - (f1 - f0);            // position of the first new token, negative without a place
  const int last_token = (tile * ROWS + n_rows - 1) / group;
  // this thread's query row (rows past the tile repeat the last one and are not stored) and the last key it sees
  const int row = tile * ROWS + min(g, n_rows - 1);
  const int token = row / group, head = g_head * group + row % group;
  int key_end = (int)min(max(pos_first + last_token + 1, 0ll), (long long)len);            // keys that any row of the tile sees
  int row_last = (int)max(min(pos_first + token, (long long)len - 1), -1ll);               // -1: none
  int all_see = (int)max(min(pos_first + (tile * ROWS) / group, (long long)len - 1), -1ll);   // the last key that every row sees
  int row_first = 0, all_from = 0, key_begin = 0, base = 0;                                 // the first ones; where the splits begin
  if constexpr (SC) {
    const Span v = visible(sc, f0 + token, pos_first + token, len);
    row_first = v.lo;
    row_last = v.hi;
    int from = v.lo <= v.hi ? v.lo : 0x7fffffff, to = v.hi;
    all_from = v.lo; all_see = v.hi;
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) {
      from = min(from, __shfl_xor_sync(0xffffffffu, from, o));
      to = max(to, __shfl_xor_sync(0xffffffffu, to, o));
      all_from = max(all_from, __shfl_xor_sync(0xffffffffu, all_from, o));
      all_see = min(all_see, __shfl_xor_sync(0xffffffffu, all_see, o));
    }
    key_end = to + 1;
    key_begin = key_end > 0 ? from : 0;
    base = key_begin & ~63;                                                                 // chunks are multiples of 64
  }
  const int used_splits = max(1, splits_of(key_end - base, chunk, splits));
  if (z >= used_splits) return;
  const int k0 = base + z * chunk, k1 = z == splits - 1 ? key_end : (int)min((long long)k0 + chunk, (long long)key_end);
  const float cap = SC ? sc.cap * 1.4426950408889634f : 0.f, inv_cap = SC && sc.cap > 0.f ? 1.f / cap : 0.f;
  const float slope = SC && sc.slopes ? sc.slopes[head] * 1.4426950408889634f : 0.f;
  const int row_pos = (int)min(max(pos_first + token, 0ll), 1ll << 30);
  const int nearest = abs(row_pos - min(max(row_pos, row_first), row_last));                // distance of the nearest visible key, which bias is relative to

  float acc[S::NT][4];
#pragma unroll
  for (int n = 0; n < S::NT; ++n) { acc[n][0] = acc[n][1] = acc[n][2] = acc[n][3] = 0.f; }
  float m = -INFINITY, l = 0.f;                    // the maximum is a row's, the sum is this thread's share
  float ve = 0.f, inv_ve = 0.f;                    // 2^7 over it; 0: no value has had a scale yet

  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(ap_smem) + warp * (S::STAGES * S::STAGE);
  const int tile0 = k0 / KEYS + warp, n_tiles = (k1 + KEYS - 1) / KEYS;      // this warp's tiles: tile0, tile0 + NW, ...
  const int* table = b.pages + (size_t)seq * b.pages_per_seq;
  uint32_t valid = 0u;                             // two bits per stage: the halves of the tile whose page exists
  const bool split_tile = b.page_len < KEYS;       // else one page holds a tile
  // Table entries of this warp's next 32 tiles (from number win on), one per lane and half: one round of loads instead of one per tile.
  int window[2] = {0, 0}, win = -32;
  auto look_up = [&](int n) {                      // n: the warp's n-th tile, in order
    if (n < win + 32) return;
    win = n;
    const int key = (tile0 + (n + lane) * NW) * KEYS;
    window[0] = key < k1 ? table[key >> b.page_shift] : 0;
    window[1] = !split_tile ? window[0] : key + 8 < k1 ? table[(key + 8) >> b.page_shift] : 0;
  };
  // this lane's piece of the first keys of a tile: the others follow at fixed distances
  const int lane_key = lane / S::PIECES, lane_piece = lane % S::PIECES;
  constexpr int STEPS = KEYS * S::PIECES / 32, STEP_KEYS = 32 / S::PIECES;
  static_assert(KEYS * S::PIECES % 32 == 0, "whole warps of copies");
  // Keys ahead of key_begin are seen by no row: they may be anything, and their pages need not exist.
  auto issue = [&](int n, int stage) {
    look_up(n);
    const int kt = tile0 + n * NW;
    const int page[2] = {__shfl_sync(0xffffffffu, window[0], n - win), __shfl_sync(0xffffffffu, window[1], n - win)};
    const uint32_t dst = ring + stage * S::STAGE;
    const int key0 = kt * KEYS;
    if (!split_tile && key0 + KEYS <= k1 && !(SC && key0 < key_begin) && (unsigned)page[0] < (unsigned)b.n_pages) {
      // a whole tile inside one page
      const size_t e = b.entry(page[0], g_head, key0);
      const TC* ks = Kp + e * HD + lane * (16 / S::E);
      const TC* vs = Vp + e * HD + lane * (16 / S::E);
#pragma unroll
      for (int i = 0; i < STEPS; ++i) {
        const int key = lane_key + i * STEP_KEYS;
        const uint32_t at = dst + key * S::ROW + ((lane_piece ^ (swz(key) & S::SWZ)) << 4);
        pf_cp16(at, ks + i * 32 * (16 / S::E), 16);
        pf_cp16(at + KEYS * S::ROW, vs + i * 32 * (16 / S::E), 16);
      }
      if constexpr (S::SCALED) {
        if (lane < 8) pf_cp16(dst + 2 * KEYS * S::ROW + lane * 16, (lane < 4 ? Ksc : Vsc) + e + (lane & 3) * 4, 16);
      }
      valid |= 3u << (2 * stage);
      return;
    }
    size_t e[2];
    uint32_t ok = 0u;
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      const int key = key0 + 8 * hf;
      const bool there = (unsigned)page[hf] < (unsigned)b.n_pages;
      if (!there && key < k1 && !(SC && key + 7 < key_begin) && lane == 0) b.bad();
      e[hf] = there ? b.entry(page[hf], g_head, key) : 0;
      ok |= there ? 1u << hf : 0u;
    }
    valid = (valid & ~(3u << (2 * stage))) | (ok << (2 * stage));
#pragma unroll 1
    for (int i = 0; i < STEPS; ++i) {
      const int key = lane_key + i * STEP_KEYS, hf = key >> 3;
      const bool on = key0 + key < k1 && !(SC && key0 + key < key_begin) && ((ok >> hf) & 1u);                  // off: zeros, nothing is read
      const size_t src = on ? ((hf ? e[1] : e[0]) + (key & 7)) * HD + lane_piece * (16 / S::E) : 0;
      const uint32_t at = dst + key * S::ROW + ((lane_piece ^ (swz(key) & S::SWZ)) << 4);
      pf_cp16(at, Kp + src, on ? 16 : 0);
      pf_cp16(at + KEYS * S::ROW, Vp + src, on ? 16 : 0);
    }
    if constexpr (S::SCALED) {
      if (lane < 8) {                              // 16 scales of each: four pieces of four
        const int key = (lane & 3) * 4, hf = key >> 3;
        const bool on = key0 + key < k1 && !(SC && key0 + key + 3 < key_begin) && ((ok >> hf) & 1u);
        const float* src = (lane < 4 ? Ksc : Vsc) + (on ? (hf ? e[1] : e[0]) + (key & 7) : 0);
        pf_cp16(dst + 2 * KEYS * S::ROW + lane * 16, src, on ? 16 : 0);
      }
    }
  };

  // the query row is asked for, then the first keys, and both are on their way together
  constexpr int PER = S::EC;
  float q_raw[S::NCH][PER];
  {
    const long long at = (long long)(f0 + token) * q.row_stride + head * q.head_stride;
#pragma unroll
    for (int c = 0; c < S::NCH; ++c) load_run<PER>(q, at + (t + 4 * c) * PER, q_vec, q_raw[c]);
  }
  const int mine = tile0 < n_tiles ? (n_tiles - tile0 + NW - 1) / NW : 0;     // this warp's tiles
  look_up(0);
#pragma unroll
  for (int s = 0; s < S::STAGES - 1; ++s) {
    if (s < mine) issue(s, s);
    pf_commit();
  }
  uint32_t qf[S::KS][4], q3[THIRD ? S::KS : 1][2];
  float row_scale = scale_log2;
  {
    float top = 0.f;
#pragma unroll
    for (int c = 0; c < S::NCH; ++c)
#pragma unroll
      for (int i = 0; i < PER; ++i) top = fmaxf(top, fabsf(q_raw[c][i]));
    float down = 1.f;
    if constexpr (S::SCALED) {                     // queries enter as fp16: brought near 1 by a power of two
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const int e = min(max((int)((__float_as_uint(top) >> 23) & 0xff), 2), 252);
      down = __uint_as_float((uint32_t)(254 - e) << 23);           // 2^(127 - e)
      row_scale *= __uint_as_float((uint32_t)e << 23);             // 2^(e - 127)
    }
#pragma unroll
    for (int ks = 0; ks < S::KS; ++ks) {
      const float* v = q_raw[ks / (PER / 4)] + 4 * (ks % (PER / 4));
      split(v[0] * down, v[1] * down, qf[ks][0], qf[ks][1], TC{});
      split(v[2] * down, v[3] * down, qf[ks][2], qf[ks][3], TC{});
      if constexpr (THIRD) {
        q3[ks][0] = third_of(v[0], v[1], qf[ks][0], qf[ks][1]);
        q3[ks][1] = third_of(v[2], v[3], qf[ks][2], qf[ks][3]);
      }
    }
  }

  int stage = 0, fill = S::STAGES - 1;
  for (int n = 0; n < mine; ++n) {
    const int kt = tile0 + n * NW;
    if (n + S::STAGES - 1 < mine) issue(n + S::STAGES - 1, fill);
    pf_commit();
    fill = fill + 1 == S::STAGES ? 0 : fill + 1;
    pf_wait<S::STAGES - 1>();
    __syncwarp();
    const uint32_t ks_base = ring + stage * S::STAGE, vs_base = ks_base + KEYS * S::ROW, sc_base = vs_base + KEYS * S::ROW;

    // scores: 8 query rows (twice) x 16 keys
    float s[2][4], s3[2][4];                        // s3: of the third parts, a chain of its own
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.f;
      s3[n][0] = s3[n][1] = s3[n][2] = s3[n][3] = 0.f;
      const int key = n * 8 + g;
#pragma unroll
      for (int c = 0; c < S::NCH; ++c) {
        constexpr int B = S::EC * S::E;                                       // 16 bytes, or 8
        uint32_t w[B / 4];
        const int off = (t + 4 * c) * B;
        lds<B>(ks_base + key * S::ROW + (((off >> 4) ^ (swz(key) & S::SWZ)) << 4) + (off & 15), w);
#pragma unroll
        for (int k = 0; k < S::EC / 4; ++k) {
          if constexpr (S::SCALED) {
            const uint32_t f = flip(w[k], TC{});
            mma(s[n], qf[c * (S::EC / 4) + k], lower(f, TC{}), upper(f, TC{}), TC{});
          } else {
            mma(s[n], qf[c * (S::EC / 4) + k], w[2 * k], w[2 * k + 1], TC{});
            if constexpr (THIRD) {
              const uint32_t a[4] = {q3[c * (S::EC / 4) + k][0], 0u, q3[c * (S::EC / 4) + k][1], 0u};
              mma(s3[n], a, w[2 * k], w[2 * k + 1], TC{});
            }
          }
        }
      }
    }
    // this thread's four: keys n * 8 + 2 t + {0, 1}
    float sc_[2][2], vsc[2][2];
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      sc_[n][0] = s[n][0] + (THIRD ? s[n][2] + s3[n][0] : s[n][2]);
      sc_[n][1] = s[n][1] + (THIRD ? s[n][3] + s3[n][1] : s[n][3]);
      if constexpr (S::SCALED) {
        const float2 k = lds_f32x2(sc_base + (n * 8 + 2 * t) * 4), v = lds_f32x2(sc_base + (KEYS + n * 8 + 2 * t) * 4);
        sc_[n][0] *= k.x; sc_[n][1] *= k.y;
        vsc[n][0] = v.x; vsc[n][1] = v.y;
      }
    }
    if constexpr (SC) {
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float y = sc_[n][i] * row_scale;
          if (sc.cap > 0.f) y = capped(y, cap, inv_cap);
          if (sc.slopes) y -= slope * (float)(abs(row_pos - (kt * KEYS + n * 8 + 2 * t + i)) - nearest);
          sc_[n][i] = y;
        }
    }
    const uint32_t ok = valid >> (2 * stage);
    uint32_t hidden = 0u;                           // of the four: keys that the row does not see
    if (kt * KEYS + KEYS - 1 > all_see || kt * KEYS + KEYS > k1 || (ok & 3u) != 3u || (SC && kt * KEYS < all_from)) {
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int at = kt * KEYS + n * 8 + 2 * t + i;
          const bool there = at < k1 && !(SC && at < key_begin) && ((ok >> n) & 1u);
          if (!there || at > row_last || (SC && at < row_first)) hidden |= 1u << (2 * n + i);
          if (!there) vsc[n][i] = 0.f;              // outside what the rows see or on a page that does not exist: it may be anything
        }
    }
    float mb = m == -INFINITY ? 0.f : m;
    float x[2][2];                                  // scores relative to the maximum, base 2
    auto relative = [&] {
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          x[n][i] = SC ? sc_[n][i] - mb : fmaf(sc_[n][i], row_scale, -mb);
          if (hidden && ((hidden >> (2 * n + i)) & 1u)) x[n][i] = -INFINITY;
        }
    };
    relative();
    const float mx = fmaxf(fmaxf(x[0][0], x[0][1]), fmaxf(x[1][0], x[1][1]));
    bool raise = mx > 8.f || m == -INFINITY;
    if constexpr (S::SCALED) raise = raise || fmaxf(fmaxf(vsc[0][0], vsc[0][1]), fmaxf(vsc[1][0], vsc[1][1])) > ve;
    if (__any_sync(0xffffffffu, raise)) {
      float top = mx;
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const float m_new = fmaxf(m, top + mb);
      float a = exp2_safe(m, m_new);
      l *= a;
      m = m_new;
      if constexpr (S::SCALED) {
        float v = fmaxf(fmaxf(vsc[0][0], vsc[0][1]), fmaxf(vsc[1][0], vsc[1][1]));
        v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 1));
        v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 2));       // the four lanes of a row see all 16 keys
        if (v > ve) {
          // the next power of two, kept where 2^7 over it is a normal number too
          const int e = min(max((int)((__float_as_uint(v) >> 23) & 0xff) + 1, 14), 254);
          const float ve_new = __uint_as_float((uint32_t)e << 23);
          a *= ve / ve_new;
          ve = ve_new;
          inv_ve = __uint_as_float((uint32_t)(254 - e + 7) << 23);
        }
      }
#pragma unroll
      for (int n = 0; n < S::NT; ++n) { acc[n][0] *= a; acc[n][1] *= a; acc[n][2] *= a; acc[n][3] *= a; }
      mb = m == -INFINITY ? 0.f : m;
      relative();
    }
    // weights: the sum's, and the ones that multiply the values
    uint32_t pf[4], p3[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      float p[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        p[i] = ex2(x[n][i]);
        l += p[i];
        if constexpr (S::SCALED) p[i] *= vsc[n][i] * inv_ve;
      }
      split(p[0], p[1], pf[2 * n], pf[2 * n + 1], TC{});
      if constexpr (THIRD) p3[2 * n] = third_of(p[0], p[1], pf[2 * n], pf[2 * n + 1]);
    }

    // values
    if constexpr (S::SCALED) {
      constexpr int B = HD / 8;                                               // bytes of a thread's run: elements [run * B, +B)
      const int run = ((g & 1) << 2) | (g >> 1);
      uint32_t w[4][B / 4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int key = 2 * t + (i & 1) + (i >> 1) * 8, off = run * B;
        lds<B>(vs_base + key * S::ROW + (((off >> 4) ^ (swz(key) & S::SWZ)) << 4) + (off & 15), w[i]);
      }
#pragma unroll
      for (int k = 0; k < B / 4; ++k) {
        // bytes of keys 0 and 1 (2 and 3) side by side, element by element
        const uint32_t a0 = flip(__byte_perm(w[0][k], w[1][k], 0x5140), TC{}), a1 = flip(__byte_perm(w[0][k], w[1][k], 0x7362), TC{});
        const uint32_t b0 = flip(__byte_perm(w[2][k], w[3][k], 0x5140), TC{}), b1 = flip(__byte_perm(w[2][k], w[3][k], 0x7362), TC{});
        mma(acc[4 * k + 0], pf, lower(a0, TC{}), lower(b0, TC{}), TC{});
        mma(acc[4 * k + 1], pf, upper(a0, TC{}), upper(b0, TC{}), TC{});
        mma(acc[4 * k + 2], pf, lower(a1, TC{}), lower(b1, TC{}), TC{});
        mma(acc[4 * k + 3], pf, upper(a1, TC{}), upper(b1, TC{}), TC{});
      }
    } else {
      const int mi = lane >> 3, mr = lane & 7, key = ((mi & 1) << 3) + mr;
#pragma unroll
      for (int n = 0; n < S::NT; n += 2) {
        uint32_t v[4];
        pf_ldmatrix_t(v, vs_base + key * S::ROW + (((n + (mi >> 1)) ^ (swz(key) & S::SWZ)) << 4));
        mma(acc[n], pf, v[0], v[1], TC{});
        mma(acc[n + 1], pf, v[2], v[3], TC{});
        if constexpr (THIRD) {
          mma(acc[n], p3, v[0], v[1], TC{});
          mma(acc[n + 1], p3, v[2], v[3], TC{});
        }
      }
    }
    __syncwarp();                                                             // the stage is refilled in the next round
    stage = stage + 1 == S::STAGES ? 0 : stage + 1;
  }
  pf_wait<0>();

  // this warp's rows: accumulators and sums in units of 2^m, sums over the quad
  l += __shfl_xor_sync(0xffffffffu, l, 1);
  l += __shfl_xor_sync(0xffffffffu, l, 2);
  const float back = S::SCALED ? ve * 0.0078125f : 1.f;                       // the unit of the values' weights
  __syncthreads();                                                            // every warp is done with its ring
  float* sm_acc = reinterpret_cast<float*>(ap_smem);                          // [NW][ROWS][HD]
  float* sm_m = sm_acc + NW * ROWS * HD;                                      // [NW][ROWS]
  float* sm_l = sm_m + NW * ROWS;
#pragma unroll
  for (int n = 0; n < S::NT; ++n)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int col = 2 * t + i;
      const int d = S::SCALED ? (((col & 1) << 2) | (col >> 1)) * (HD / 8) + n : n * 8 + col;
      sm_acc[(warp * ROWS + g) * HD + d] = (acc[n][i] + acc[n][2 + i]) * back;
    }
  if (t == 0) { sm_m[warp * ROWS + g] = m; sm_l[warp * ROWS + g] = l; }
  __syncthreads();

  auto place = [&](int r, int& tok, int& hd) {
    const int rr = tile * ROWS + r;
    tok = f0 + rr / group;
    hd = g_head * group + rr % group;
  };
  for (int i = threadIdx.x; i < n_rows * HD; i += THREADS) {
    const int r = i / HD, c = i % HD;
    float M = -INFINITY, L = 0.f, a = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) M = fmaxf(M, sm_m[w * ROWS + r]);
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float f = exp2_safe(sm_m[w * ROWS + r], M);
      L += sm_l[w * ROWS + r] * f;
      a += sm_acc[(w * ROWS + r) * HD + c] * f;
    }
    int tok, hd;
    place(r, tok, hd);
    if (used_splits == 1) {
      store_elem(out, (long long)tok * out.row_stride + hd * out.head_stride + c, normalised(a, L));
    } else {
      const size_t slot = ((size_t)unit * slot_rows + r) * splits + z;
      __stcg(part_acc + slot * HD + c, a);
      if (c == 0) { __stcg(part_ml + slot * 2, M); __stcg(part_ml + slot * 2 + 1, L); }
    }
  }
  if (used_splits == 1) return;
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) {
    const int done = atomicAdd(&counters[unit], 1);
    sm_last = done == used_splits - 1;
    if (sm_last) counters[unit] = 0;                                          // ready for the next launch
  }
  __syncthreads();
  if (!sm_last) return;
  __threadfence();
  for (int i = threadIdx.x; i < n_rows * HD; i += THREADS) {
    const int r = i / HD, c = i % HD;
    int tok, hd;
    place(r, tok, hd);
    const size_t slot0 = ((size_t)unit * slot_rows + r) * splits;
    float M = -INFINITY, L = 0.f, a = 0.f;
    for (int s = 0; s < used_splits; ++s) M = fmaxf(M, __ldcg(part_ml + (slot0 + s) * 2));
    for (int s = 0; s < used_splits; ++s) {
      const float f = exp2_safe(__ldcg(part_ml + (slot0 + s) * 2), M);
      L += __ldcg(part_ml + (slot0 + s) * 2 + 1) * f;
      a += __ldcg(part_acc + (slot0 + s) * HD + c) * f;
    }
    store_elem(out, (long long)tok * out.row_stride + hd * out.head_stride + c, normalised(a, L));
  }
}

}  // namespace sd
