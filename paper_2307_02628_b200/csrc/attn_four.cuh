// Attention of few query rows over a paged cache in 4 bits: the same division of the work as attn_paged.cuh (a block per sequence, key head, tile of 8
// query rows and split of the keys, a ring of asynchronous copies per warp, partial results joined by the block that arrives last), with products
// laid out for codes of which two make a byte.
//
// value = code * block scale * scale.  Code times block scale is an fp16 number exactly: one conversion and one multiplication for a pair.  A key's scale multiplies
// its score, a value's scale its weight, relative to a power of two above all scales so far and times 2^7, as in 8 bits.
//
// At 152 bytes a key and head of 128 the memory could deliver a key every 8 clocks to an SM, which four schedulers have 32 slots for, and conversion alone
// takes 13 (a warp's instruction for 32 lanes: 256 values in pairs, two instructions each, plus the values' interleaving).  Nothing is full (64 single tokens at
// 1024..1536: issue and ALU 53 %, memory 48 %): 15 warps to an SM, each a chain of copies, products, maxima and exponentials, do not cover one another's
// waits, and a block's start and end are a fifth of it.  So instructions and steps are kept few:
//  - 32 keys of a warp go through the loop at a time, so that copies, waits and maxima are paid once for them;
//  - scores are S^T = K Q^T with the keys as the 16-row operand, and O^T = V^T P^T has the values there: the 8 query rows fill the other side of both, so that
//    either takes half the products, and half the accumulators, that it would take with the rows' operand padded.  A thread holds scores of two
//    query rows, the rows of its accumulators; the weights' fragment is their transpose, one instruction for 8 keys;
//  - a values' operand pairs two keys: nibbles of the two are interleaved by masks, four words at a time, before they are converted, and not after;
//  - queries and results in bf16 have weights of one fp16 (11 bits), others (FINE) of two.
#pragma once
#include "attn_paged.cuh"

namespace sd {
namespace a4 {

// Warps of a block: fewer wait for one another where a block begins and ends, more have fewer shares of split keys to join.  Measured, 2, 3 and 5 warps (15 to an SM as
// the ring of 14.6 KB a warp allows): 64 single tokens at 1280 positions, 32 heads of 128: 98, 96, 102 us; at 640: 59, 60, 67; 3 of 32 heads over 8 at
// 20 000..65 521: 76, 75, 65; 200 at 100..600: 110, 116, 142.
constexpr int NW = 3, THREADS = 32 * NW, ROWS = 8, KEYS = 32, STAGES = 3, PER_SM = 5;

template <int HD> struct Shape {
  static constexpr int ROW = HD / 2, PIECES = ROW / 16, SWZ = PIECES - 1;                  // bytes and 16-byte pieces of a key
  static constexpr int EC = HD / 4, KS = HD / 16, MT = HD / 16;                            // elements of a key that a thread has; products for 8 keys, for 16 keys
  static constexpr int BLOCKS = HD / kBlock;                                               // block scales of a key, a byte each
  static constexpr int V = KEYS * ROW, SCALES = 2 * V, BLOCK = SCALES + 2 * KEYS * 4, STAGE = BLOCK + 2 * KEYS * BLOCKS;
  static constexpr int MERGE = NW * ROWS * (HD + 2) * 4;
  static constexpr int SMEM = NW * STAGES * STAGE > MERGE ? NW * STAGES * STAGE : MERGE;   // five blocks of 44 KB to an SM at HD = 128
};
__device__ __forceinline__ int swz(int key) { return key >> 1; }

__device__ __forceinline__ float lds_f32(uint32_t addr) {
  float v;
  asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(addr));
  return v;
}
__device__ __forceinline__ uint32_t transpose(uint32_t pair) {             // 8 x 8 of 16 bits
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(pair));
  return r;
}
// c = a b
__device__ __forceinline__ void mma_first(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};\n"
               : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
// a byte by its number, as two fp16
__device__ __forceinline__ uint32_t widen(uint32_t w, int byte) {          // byte is a constant after unrolling
  return byte == 0 ? e2m1_widen<0>(w) : byte == 1 ? e2m1_widen<1>(w) : byte == 2 ? e2m1_widen<2>(w) : e2m1_widen<3>(w);
}

}  // namespace a4

// Arguments as those of paged_attn_tile_kernel.  FINE: weights of two fp16, and queries of two where they have more bits than one.
template <int HD, bool FINE, bool SC>
__global__ void __launch_bounds__(a4::THREADS, a4::PER_SM)
paged_attn_four_kernel(const BatchView b, const Rows q, const Rows out, const e2m1* __restrict__ Kp, const e2m1* __restrict__ Vp, const float* __restrict__ Ksc,
                       const float* __restrict__ Vsc, const uint8_t* __restrict__ Kb, const uint8_t* __restrict__ Vb, int group, float scale_log2, bool q_vec, int tiles_per_seq,
                       int rows_below, int chunk, int slot_rows, float* part_acc, float* part_ml, int* __restrict__ counters, bool early, const Scores sc) {
  using namespace a4;
  using S = Shape<HD>;
  extern __shared__ __align__(128) unsigned char a4_smem[];
  __shared__ int sm_last;
  const ap::UntilPredecessorEnds hold{early && blockIdx.x == 0 && blockIdx.y == 0};

  const int unit = blockIdx.x, tile = unit % tiles_per_seq, g_head = (unit / tiles_per_seq) % b.n_kv_heads, seq = unit / tiles_per_seq / b.n_kv_heads;
  const int splits = gridDim.y, z = blockIdx.y;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;

  // the sequence's rows; whatever does not fit the tensors is reported and left out
  const int f0 = b.first[seq], f1 = b.first[seq + 1], raw_len = b.len[seq], len = b.held_len(raw_len);
  int n_new = f1 - f0;
  if (f0 < 0 || n_new < 0 || f1 > b.n_tokens || n_new > b.max_new) {
    if (threadIdx.x == 0) b.bad();
    if (f0 < 0 || n_new < 0) return;
    n_new = min(n_new, min(b.max_new, b.n_tokens - f0));
  }
  const int n_rows = min(ROWS, n_new * group - tile * ROWS);
  if (n_rows <= 0 || n_new * group >= rows_below) return;
  const long long pos_first = (long long)raw_len - (f1 - f0);               // position of the first new token, negative without a place
  // Token and head (of the group) of the tile's rows: the first one's, and what lies r < 8 rows on, a quotient below 2^17 that fp32 divides rightly.
  const int token0 = tile * ROWS / group, member0 = tile * ROWS - token0 * group;
  const float per_group = 1.f / (float)group;
  auto place = [&](int r, int& tok, int& hd) {
    const int member = member0 + r, more = (int)(((float)member + 0.5f) * per_group);
    tok = token0 + more;
    hd = g_head * group + member - more * group;
  };

  // This thread's two query rows (rows past the tile repeat the last one and are not stored), the keys they see, and those that any and every row of the
  // tile sees.
  const float cap = SC ? sc.cap * 1.4426950408889634f : 0.f, inv_cap = SC && sc.cap > 0.f ? 1.f / cap : 0.f;
  Span seen[2];
  int row_pos[2], nearest[2];                      // position, and the distance of the nearest visible key, which bias is relative to
  float slope[2];
  int key_begin = 0x7fffffff, key_end = 0, all_from = 0, all_see = 0x7fffffff;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int token, head;
    place(min(2 * t + i, n_rows - 1), token, head);
    const Span v = visible(sc, f0 + token, pos_first + token, len);
    seen[i] = v;
    if (v.lo <= v.hi) key_begin = min(key_begin, v.lo);
    key_end = max(key_end, v.hi + 1);
    all_from = max(all_from, v.lo);
    all_see = min(all_see, v.hi);
    if constexpr (SC) {
      row_pos[i] = (int)min(max(pos_first + token, 0ll), 1ll << 30);
      nearest[i] = abs(row_pos[i] - min(max(row_pos[i], v.lo), v.hi));
      slope[i] = sc.slopes ? sc.slopes[head] * 1.4426950408889634f : 0.f;
    }
  }
#pragma unroll
  for (int o = 1; o < 4; o <<= 1) {
    key_end = max(key_end, __shfl_xor_sync(0xffffffffu, key_end, o));
    all_see = min(all_see, __shfl_xor_sync(0xffffffffu, all_see, o));
    if constexpr (SC) {
      key_begin = min(key_begin, __shfl_xor_sync(0xffffffffu, key_begin, o));
      all_from = max(all_from, __shfl_xor_sync(0xffffffffu, all_from, o));
    }
  }
  if (!SC || key_end == 0) key_begin = 0;
  const int base = key_begin & ~63;                                         // chunks are multiples of 64
  const int used_splits = max(1, ap::splits_of(key_end - base, chunk, splits));
  if (z >= used_splits) return;
  const int k0 = base + z * chunk, k1 = z == splits - 1 ? key_end : (int)min((long long)k0 + chunk, (long long)key_end);

  float acc[S::MT][4];                             // element 2 i (c0, c1) and 2 i + 1 (c2, c3) of run g, query rows 2 t and 2 t + 1
#pragma unroll
  for (int i = 0; i < S::MT; ++i) { acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.f; }
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};   // of the two rows: the maximum is a row's, the sum is this thread's share
  // Values' weights are relative to ve, times 2^7: 2^lift within the exponential, and what a lift of 60 does not reach, `rest`, by itself.
  float ve = 0.f, lift = 0.f, rest = 1.f;          // 0: no value has had a scale yet

  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(a4_smem) + warp * (STAGES * S::STAGE);
  const int tile0 = k0 / KEYS + warp, n_tiles = (k1 + KEYS - 1) / KEYS;     // this warp's tiles: tile0, tile0 + NW, ...
  const int* table = b.pages + (size_t)seq * b.pages_per_seq;
  uint32_t valid = 0u;                             // four bits per stage: the groups of 8 keys whose page exists
  // Table entries of this warp's next tiles (from number win on), 32 / parts of them: one round of loads instead of one per tile.
  const int part_shift = min(b.page_shift, 5), parts_log = 5 - part_shift;  // a tile is 1, 2 or 4 pages or parts of one
  int window = 0, win = 0, win_end = 0;
  auto look_up = [&](int n) {                      // n: the warp's n-th tile, in order
    if (n < win_end) return;
    win = n;
    win_end = n + (32 >> parts_log);
    const long long key = ((long long)tile0 + (long long)(n + (lane >> parts_log)) * NW) * KEYS + ((lane & ((1 << parts_log) - 1)) << part_shift);
    window = key < k1 ? table[key >> b.page_shift] : 0;
  };
  // copies: this lane's piece of the first keys of a tile, the others follow at fixed distances; scales, four keys a piece; block scales
  const int lane_key = lane / S::PIECES, lane_piece = lane % S::PIECES;
  constexpr int STEPS = KEYS * S::PIECES / 32, STEP_KEYS = 32 / S::PIECES, BP = KEYS * S::BLOCKS / 16, BKEYS = 16 / S::BLOCKS;   // pieces of block scales, keys of one
  const int b_key = (lane % BP) * BKEYS, s_key = (lane & 7) * 4;
  static_assert(STEP_KEYS / 2 % (S::SWZ + 1) == 0, "a lane's pieces are swizzled alike");
  // a whole tile inside one page: this lane's sources, of the pool's first key (a pool has fewer than 2^32 keys)
  const e2m1 *k_src = Kp + lane * 16, *v_src = Vp + lane * 16;
  const float* s_src = (lane < 8 ? Ksc : Vsc) + s_key;
  const uint8_t* b_src = (lane < BP ? Kb : Vb) + (lane % BP) * 16;
  const uint32_t lane_at = lane_key * S::ROW + ((lane_piece ^ (swz(lane_key) & S::SWZ)) << 4);
  // Keys ahead of key_begin are seen by no row: they may be anything, and their pages need not exist.
  auto issue = [&](int n, int stage) {
    look_up(n);
    const int key0 = (tile0 + n * NW) * KEYS, slot = (n - win) << parts_log;
    const uint32_t dst = ring + stage * S::STAGE;
    const int page0 = __shfl_sync(0xffffffffu, window, slot);
    if (parts_log == 0 && key0 + KEYS <= k1 && !(SC && key0 < key_begin) && (unsigned)page0 < (unsigned)b.n_pages) {
      const uint32_t e = (((uint32_t)page0 * b.n_kv_heads + g_head) << b.page_shift) + (key0 & (b.page_len - 1));
      const e2m1 *ks = k_src + (size_t)e * S::ROW, *vs = v_src + (size_t)e * S::ROW;
#pragma unroll
      for (int i = 0; i < STEPS; ++i) {
        pf_cp16(dst + lane_at + i * 512, ks + i * 512, 16);
        pf_cp16(dst + lane_at + i * 512 + S::V, vs + i * 512, 16);
      }
      if (lane < 16) pf_cp16(dst + S::SCALES + lane * 16, s_src + e, 16);
      if (lane < 2 * BP) pf_cp16(dst + S::BLOCK + lane * 16, b_src + (size_t)e * S::BLOCKS, 16);
      valid |= 15u << (4 * stage);
      return;
    }
    // The page of `some` keys from one on, of one part, -1: none, or no row sees them.  What is not copied is what an earlier tile left: its keys are
    // hidden, its values' weights and scales zero.
    auto page_of = [&](int key, int some) {
      const int page = __shfl_sync(0xffffffffu, window, slot + (key >> part_shift));
      return key0 + key < k1 && !(SC && key0 + key + some - 1 < key_begin) && (unsigned)page < (unsigned)b.n_pages ? page : -1;
    };
    const int eight = (lane & 3) * 8, mine = page_of(eight, 8);
    const uint32_t ok = __ballot_sync(0xffffffffu, mine >= 0 || key0 + eight >= k1 || (SC && key0 + eight + 7 < key_begin)) & 15u;
    if (ok != 15u && lane == 0) b.bad();
    valid = (valid & ~(15u << (4 * stage))) | (ok << (4 * stage));
#pragma unroll 1
    for (int i = 0; i < STEPS; ++i) {
      const int key = lane_key + i * STEP_KEYS, page = page_of(key, 1);
      if (page < 0) continue;                                               // no shuffle follows in this round
      const size_t from = b.entry(page, g_head, key0 + key) * S::ROW + lane_piece * 16;
      pf_cp16(dst + lane_at + i * 512, Kp + from, 16);
      pf_cp16(dst + lane_at + i * 512 + S::V, Vp + from, 16);
    }
    __syncwarp();
    const int ps = page_of(s_key, 4), pb = page_of(b_key, BKEYS);
    if (lane < 16 && ps >= 0) pf_cp16(dst + S::SCALES + lane * 16, (lane < 8 ? Ksc : Vsc) + b.entry(ps, g_head, key0 + s_key), 16);
    if (lane < 2 * BP && pb >= 0) pf_cp16(dst + S::BLOCK + lane * 16, (lane < BP ? Kb : Vb) + b.entry(pb, g_head, key0 + b_key) * S::BLOCKS, 16);
  };

  // the query row is asked for, then the first keys, and both are on their way together
  float q_raw[S::EC];                              // of row g: the products want another division than the softmax
  {
    int token, head;
    place(min(g, n_rows - 1), token, head);
    ap::load_run<S::EC>(q, (long long)(f0 + token) * q.row_stride + head * q.head_stride + t * S::EC, q_vec, q_raw);
  }
  const int mine = tile0 < n_tiles ? (n_tiles - tile0 + NW - 1) / NW : 0;   // this warp's tiles
#pragma unroll
  for (int s = 0; s < STAGES - 1; ++s) {
    if (s < mine) issue(s, s);
    pf_commit();
  }
  uint32_t qf[S::KS][2], ql[FINE ? S::KS : 1][2];
  float row_scale[2];
  {
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < S::EC; ++i) top = fmaxf(top, fabsf(q_raw[i]));
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const int e = min(max((int)((__float_as_uint(top) >> 23) & 0xff), 2), 252);
    const float down = __uint_as_float((uint32_t)(254 - e) << 23);          // 2^(127 - e): queries enter as fp16, brought near 1
#pragma unroll
    for (int i = 0; i < 2; ++i) row_scale[i] = scale_log2 * __uint_as_float((uint32_t)__shfl_sync(0xffffffffu, e, 8 * t + 4 * i) << 23);   // 2^(e - 127)
#pragma unroll
    for (int k = 0; k < S::KS; ++k) {
      const float* v = q_raw + 4 * k;
      if constexpr (FINE) {
        ap::split(v[0] * down, v[1] * down, qf[k][0], ql[k][0], __half{});
        ap::split(v[2] * down, v[3] * down, qf[k][1], ql[k][1], __half{});
      } else {
        qf[k][0] = pack_f16(v[0] * down, v[1] * down);
        qf[k][1] = pack_f16(v[2] * down, v[3] * down);
      }
    }
  }

  // Where this thread's pieces lie within a stage, the others at fixed distances.  Keys: key g, EC elements from t on.  Values: key 2 t, run g.
  constexpr int KB = S::EC / 2, VB = HD / 16, VW = VB < 4 ? 4 : VB;          // bytes of either; a run of two is cut out of its word
  const int k_blk = t * S::EC / kBlock, v_blk = g * (HD / 8) / kBlock;
  const uint32_t k_at = g * S::ROW + ((((t * KB) >> 4) ^ (swz(g) & S::SWZ)) << 4) + (t * KB & 15);
  const uint32_t v_at = S::V + 2 * t * S::ROW + ((((g * VB) >> 4) ^ (t & S::SWZ)) << 4) + (g * VB & (16 - VW));
  const uint32_t kb_at = S::BLOCK + g * S::BLOCKS + (k_blk & ~1), vb_at = S::BLOCK + (KEYS + 2 * t) * S::BLOCKS + (v_blk & ~1);
  const uint32_t s_at = S::SCALES + 4 * g;
  const int k_sel = k_blk & 1 ? 0x3232 : 0x1010, v_sel = v_blk & 1 ? 0x0051 : 0x0040;
  static_assert(4 % (S::SWZ + 1) == 0, "keys 8 apart are swizzled alike");

  const int all_end = min(all_see + 1, k1);        // tiles up to here need no mask
  int stage = 0, fill = STAGES - 1;
  for (int n = 0; n < mine; ++n) {
    const int key0 = (tile0 + n * NW) * KEYS;
    if (n + STAGES - 1 < mine) issue(n + STAGES - 1, fill);
    pf_commit();
    fill = fill + 1 == STAGES ? 0 : fill + 1;
    pf_wait<STAGES - 1>();
    __syncwarp();
    const uint32_t at = ring + stage * S::STAGE;

    // scores: 32 keys x 8 query rows; this thread's eight: keys 8 j + g, rows 2 t and 2 t + 1
    float x[4][2], vsc[4];
#pragma unroll
    for (int jj = 0; jj < 2; ++jj) {
      uint32_t w[2][KB / 4], unit[2][2];                                    // block scales of the first and the last 16 elements, twice each
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        uint32_t two[1];
        ap::lds<KB>(at + k_at + (jj * 16 + r * 8) * S::ROW, w[r]);
        ap::lds<2>(at + kb_at + (jj * 16 + r * 8) * S::BLOCKS, two);
        const uint32_t u = blocks_widen(two[0]);
        unit[r][0] = __byte_perm(u, 0u, HD == 128 ? 0x1010 : k_sel);
        unit[r][1] = __byte_perm(u, 0u, 0x3232);                            // HD = 128
      }
      float c[4];
#pragma unroll
      for (int k = 0; k < S::KS; ++k) {                                     // two bytes of two keys: four elements of each
        const uint32_t a[4] = {hmul2(widen(w[0][k >> 1], 2 * (k & 1)), unit[0][k >> 2]), hmul2(widen(w[1][k >> 1], 2 * (k & 1)), unit[1][k >> 2]),
                               hmul2(widen(w[0][k >> 1], 2 * (k & 1) + 1), unit[0][k >> 2]), hmul2(widen(w[1][k >> 1], 2 * (k & 1) + 1), unit[1][k >> 2])};
        if (k == 0) mma_first(c, a, qf[k][0], qf[k][1]);
        else ap::mma(c, a, qf[k][0], qf[k][1], __half{});
        if constexpr (FINE) ap::mma(c, a, ql[k][0], ql[k][1], __half{});
      }
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const float ks = lds_f32(at + s_at + (jj * 16 + r * 8) * 4);
        vsc[2 * jj + r] = lds_f32(at + s_at + KEYS * 4 + (jj * 16 + r * 8) * 4);
        x[2 * jj + r][0] = c[2 * r] * ks;
        x[2 * jj + r][1] = c[2 * r + 1] * ks;
      }
    }
    const bool changed = SC && (sc.cap > 0.f || sc.slopes);
    if constexpr (SC) {
      if (changed) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            float y = x[j][i] * row_scale[i];
            if (sc.cap > 0.f) y = capped(y, cap, inv_cap);
            if (sc.slopes) y -= slope[i] * (float)(abs(row_pos[i] - (key0 + j * 8 + g)) - nearest[i]);
            x[j][i] = y;
          }
      }
    }
    const uint32_t ok = valid >> (4 * stage) & 15u;
    uint32_t hidden = 0u, gone = 0u;               // of the eight: keys that a row does not see; of the eight whose values this thread takes: keys that are not there
    if (key0 + KEYS > all_end || ok != 15u || (SC && key0 < all_from)) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int key = key0 + j * 8 + g;
        const bool there = key < k1 && !(SC && key < key_begin) && ((ok >> j) & 1u);
        if (!there) vsc[j] = 0.f;                  // outside what the rows see or on a page that does not exist: it may be anything
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          if (!there || key > seen[i].hi || (SC && key < seen[i].lo)) hidden |= 1u << (2 * j + i);
          const int of = key0 + j * 8 + 2 * t + i;
          if (of >= k1 || (SC && of < key_begin) || !((ok >> j) & 1u)) gone |= 1u << (2 * j + i);
        }
      }
    }
    // scores relative to the maximum, base 2, and the lift
    float top[2], mb[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      mb[i] = (m[i] == -INFINITY ? 0.f : m[i]) - lift;
      const float unit_x = changed ? 1.f : row_scale[i];
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j][i] = fmaf(x[j][i], unit_x, -mb[i]);
    }
    if (hidden) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 2; ++i)
          if ((hidden >> (2 * j + i)) & 1u) x[j][i] = -INFINITY;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) top[i] = fmaxf(fmaxf(x[0][i], x[1][i]), fmaxf(x[2][i], x[3][i]));
    float most = fmaxf(fmaxf(vsc[0], vsc[1]), fmaxf(vsc[2], vsc[3]));
    if (__any_sync(0xffffffffu, fmaxf(top[0], top[1]) > 8.f + lift || fminf(m[0], m[1]) == -INFINITY || most > ve)) {
      float a[2], shift[2];
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) {                                    // the eight lanes of a pair of rows see all 32 keys
        top[0] = fmaxf(top[0], __shfl_xor_sync(0xffffffffu, top[0], o));
        top[1] = fmaxf(top[1], __shfl_xor_sync(0xffffffffu, top[1], o));
        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float m_new = fmaxf(m[i], top[i] + mb[i]);
        a[i] = exp2_safe(m[i], m_new);
        l[i] *= a[i];
        m[i] = m_new;
      }
      if (most > ve) {
        // the next power of two, kept where 2^7 over it is a normal number too
        const int e = min(max((int)((__float_as_uint(most) >> 23) & 0xff) + 1, 14), 254), up = 134 - e, lift_new = min(max(up, -60), 60);
        const float ve_new = __uint_as_float((uint32_t)e << 23), more = exp2f((float)lift_new - lift);
        a[0] *= ve / ve_new;
        a[1] *= ve / ve_new;
        ve = ve_new;
        l[0] *= more;
        l[1] *= more;
        lift = (float)lift_new;
        rest = __uint_as_float((uint32_t)(127 + up - lift_new) << 23);      // up - lift_new: 60 at most either way
      }
#pragma unroll
      for (int i = 0; i < S::MT; ++i) { acc[i][0] *= a[0]; acc[i][1] *= a[1]; acc[i][2] *= a[0]; acc[i][3] *= a[1]; }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        shift[i] = mb[i] - ((m[i] == -INFINITY ? 0.f : m[i]) - lift);
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j][i] += shift[i];
      }
    }
    if (rest != 1.f) {
#pragma unroll
      for (int j = 0; j < 4; ++j) vsc[j] *= rest;
    }
    // weights: the sum's, and the ones that multiply the values
    uint32_t pf[4], pl[FINE ? 4 : 1];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float p0 = ap::ex2(x[j][0]), p1 = ap::ex2(x[j][1]);
      l[0] += p0;
      l[1] += p1;
      if constexpr (FINE) {
        uint32_t hi, lo;
        ap::split(p0 * vsc[j], p1 * vsc[j], hi, lo, __half{});
        pf[j] = transpose(hi);
        pl[j] = transpose(lo);
      } else {
        pf[j] = transpose(pack_f16(p0 * vsc[j], p1 * vsc[j]));
      }
    }

    // values, 16 keys at a time: this thread's four are 2 t, 2 t + 1, 2 t + 8, 2 t + 9, its elements run g of HD / 8
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32_t w[4][VW / 4], blk[4][1];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int step = h * 16 + (i & 1) + (i >> 1) * 8;                   // keys from 2 t on
        ap::lds<VW>(at + v_at + step * S::ROW, w[i]);
        if constexpr (VB < 4) w[i][0] >>= (g * VB & 2) * 8;
        ap::lds<2>(at + vb_at + step * S::BLOCKS, blk[i]);
      }
      if (gone >> (4 * h) & 15u) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if ((gone >> (4 * h + i)) & 1u) blk[i][0] = 0u;
      }
      const uint32_t ua = blocks_widen(__byte_perm(blk[0][0], blk[1][0], v_sel)), ub = blocks_widen(__byte_perm(blk[2][0], blk[3][0], v_sel));   // this block's byte of the two
#pragma unroll
      for (int k = 0; k < VW / 4; ++k) {
        constexpr uint32_t LOW = 0x0f0f0f0fu;
        const uint32_t a_even = (w[0][k] & LOW) | (w[1][k] << 4 & ~LOW), a_odd = (w[0][k] >> 4 & LOW) | (w[1][k] & ~LOW);
        const uint32_t b_even = (w[2][k] & LOW) | (w[3][k] << 4 & ~LOW), b_odd = (w[2][k] >> 4 & LOW) | (w[3][k] & ~LOW);
#pragma unroll
        for (int i = 0; i < (VB < 4 ? VB : 4); ++i) {                         // elements 8 k + 2 i and 8 k + 2 i + 1
          const uint32_t v[4] = {hmul2(widen(a_even, i), ua), hmul2(widen(a_odd, i), ua), hmul2(widen(b_even, i), ub), hmul2(widen(b_odd, i), ub)};
          ap::mma(acc[4 * k + i], v, pf[2 * h], pf[2 * h + 1], __half{});
          if constexpr (FINE) ap::mma(acc[4 * k + i], v, pl[2 * h], pl[2 * h + 1], __half{});
        }
      }
    }
    __syncwarp();                                                           // the stage is refilled in the next round
    stage = stage + 1 == STAGES ? 0 : stage + 1;
  }
  pf_wait<0>();

  // this warp's rows: accumulators and sums in units of 2^m, sums over the eight lanes of a pair of rows
  const float down = exp2f(-lift);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], o);
    l[i] *= down;
  }
  const float back = ve * 0.0078125f;                                       // the unit of the values' weights
  __syncthreads();                                                          // every warp is done with its ring
  auto store4 = [&](int r, int c, float4 a, float L) {
    int tok, hd;
    place(r, tok, hd);
    const long long to = (long long)(f0 + tok) * out.row_stride + hd * out.head_stride + c;
    store_elem(out, to, normalised(a.x, L));
    store_elem(out, to + 1, normalised(a.y, L));
    store_elem(out, to + 2, normalised(a.z, L));
    store_elem(out, to + 3, normalised(a.w, L));
  };
  float* sm_acc = reinterpret_cast<float*>(a4_smem);                        // [NW][ROWS][HD]
  float* sm_m = sm_acc + NW * ROWS * HD;                                    // [NW][ROWS]
  float* sm_l = sm_m + NW * ROWS;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (2 * t + i >= n_rows) continue;
#pragma unroll
    for (int k = 0; k < S::MT; ++k)
      *reinterpret_cast<float2*>(sm_acc + (warp * ROWS + 2 * t + i) * HD + g * (HD / 8) + 2 * k) = make_float2(acc[k][i] * back, acc[k][2 + i] * back);
    if (g == 0) { sm_m[warp * ROWS + 2 * t + i] = m[i]; sm_l[warp * ROWS + 2 * t + i] = l[i]; }
  }
  __syncthreads();

  for (int i = threadIdx.x; i < n_rows * (HD / 4); i += THREADS) {          // four columns at a time
    const int r = i / (HD / 4), c = i % (HD / 4) * 4;
    float M = -INFINITY, L = 0.f;
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < NW; ++w) M = fmaxf(M, sm_m[w * ROWS + r]);
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float f = exp2_safe(sm_m[w * ROWS + r], M);
      const float4 v = *reinterpret_cast<const float4*>(sm_acc + (w * ROWS + r) * HD + c);
      L += sm_l[w * ROWS + r] * f;
      a.x += v.x * f; a.y += v.y * f; a.z += v.z * f; a.w += v.w * f;
    }
    if (used_splits == 1) {
      store4(r, c, a, L);
    } else {
      const size_t slot = ((size_t)unit * slot_rows + r) * splits + z;
      __stcg(reinterpret_cast<float4*>(part_acc + slot * HD + c), a);
      if (c == 0) __stcg(reinterpret_cast<float2*>(part_ml + slot * 2), make_float2(M, L));
    }
  }
  if (used_splits == 1) return;
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) {
    const int done = atomicAdd(&counters[unit], 1);
    sm_last = done == used_splits - 1;
    if (sm_last) counters[unit] = 0;                                        // ready for the next launch
  }
  __syncthreads();
  if (!sm_last) return;
  __threadfence();
  // The shares are added in split order, sixteen splits' loads on their way together; a warp for each row finds its maximum and sum before.
  float* sm_M = sm_m;
  float* sm_L = sm_l;
  for (int r = warp; r < n_rows; r += NW) {
    const float2* ml = reinterpret_cast<const float2*>(part_ml) + ((size_t)unit * slot_rows + r) * splits;
    float M = -INFINITY, L = 0.f;
    for (int s = lane; s < used_splits; s += 32) {
      const float2 v = __ldcg(ml + s);
      const float top = fmaxf(M, v.x);
      L = L * exp2_safe(M, top) + v.y * exp2_safe(v.x, top);
      M = top;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const float M2 = __shfl_xor_sync(0xffffffffu, M, o), L2 = __shfl_xor_sync(0xffffffffu, L, o), top = fmaxf(M, M2);
      L = L * exp2_safe(M, top) + L2 * exp2_safe(M2, top);
      M = top;
    }
    if (lane == 0) { sm_M[r] = M; sm_L[r] = L; }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < n_rows * (HD / 4); i += THREADS) {
    const int r = i / (HD / 4), c = i % (HD / 4) * 4;
    const size_t slot0 = ((size_t)unit * slot_rows + r) * splits;
    const float M = sm_M[r];
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 16
    for (int s = 0; s < used_splits; ++s) {
      const float f = exp2_safe(__ldcg(part_ml + (slot0 + s) * 2), M);
      const float4 v = __ldcg(reinterpret_cast<const float4*>(part_acc + (slot0 + s) * HD + c));
      a.x += v.x * f; a.y += v.y * f; a.z += v.z * f; a.w += v.w * f;
    }
    store4(r, c, a, sm_L[r]);
  }
}

}  // namespace sd
