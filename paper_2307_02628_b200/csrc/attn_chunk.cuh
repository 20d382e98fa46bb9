// Attention of chunks of new tokens over a paged cache in bf16 or 8 bits, on the fifth-generation tensor cores.
//
// One block per (sequence, key head, 256 query rows, or 128: see PAIRS below); a query row is a (token, head of the group) pair, so grouped heads share
// the keys they read.  The 256 rows are two tiles of 128.  Keys come in tiles of 128; for every half i of one (64 keys) and each tile t:
//     S_t,i = Q_t K_i^T    (both operands in shared memory, result in tensor memory)
//     P_t,i = 2^(S - m)    (one thread per row: maximum, exponentials, sum; P in bf16 over S's own columns)
//     O_t += P_t,i V_i     (P from tensor memory, V from shared memory as it lies: keys are the product's inner axis)
// Tensor memory holds for each tile S of two halves (64 columns each) and O (HD columns).  S of half i + 2 takes the columns of half i
// once the product that reads P there has completed, so the scores of the next half are there when a softmax is done with one, and the
// tensor core works through both tiles' softmax.  (Scores of 128 keys at a time leave no columns for a second set: every
// softmax then waited for its two products, 1500 of 3700 clocks.)
//
// Operands are bf16, the type of a bf16 cache; codes of 8-bit caches are bf16 numbers exactly.  Over 4-bit caches they are fp16: codes times their block's scale
// are fp16 numbers exactly, two instructions a pair (six to bf16), and queries are brought near 1 by a power of two for each row.  A value's scale joins
// its weight, relative to a power of two above all scales so far, times 2^7 (the weights stay below 2^15); where queries and results are bf16 it joins
// the value instead, whose block scale times scale is then rounded to 11 bits, and once more times a code of 1.5, 3 or 6 (2^-10 of a value at most, both), and the
// weight, of 11 bits too, is times 2^7 by itself: half as many scales to read and multiply by in the softmax.  Where queries and results are bf16 too, the only
// rounding is that of the weights, once to 8 bits of significand: relative to 64-bit arithmetic results are 2.3e-3 off, of which their own
// rounding is 1.7e-3.  Queries or results with more bits (fp32, fp16) take the form PAIRS: queries and weights are sums of two
// bf16, 16 bits, in two products each; the weights' lower halves take the other 32 columns of their scores.  Twice the
// products, and at HD = 128 one tile of rows instead of two: 4 chunks of 512 tokens at 2048, 32 heads of 128, bf16: 230 us from and to fp16, 90
// from and to bf16; 2 x 1024 tokens, 32 heads of 64: 66 and 37.  fp32 results take 22 bits: over 4 bits, whose pairs are fp16, they
// come here too (8 chunks of 3-1024 tokens at 1024-4096, 32 heads of 128, from and to fp32: 694 us, 2091 in the kernel for few rows), else they go to the
// kernel for few rows, which has three bf16, or two fp16, for them.  A key's scale (8-bit caches) multiplies its score in the softmax, a value's scale its weight, before the rounding.
//
// The running maximum is raised only when it would be passed by 2^8 (weights then reach 256, well inside bf16 and the fp32
// sums): O_t is rescaled in tensor memory in the first tiles and hardly ever after.
//
// Where there are fewer blocks than SMs the keys are split over several, each of which leaves its rows' shares to a second kernel.
//
// What bounds it: for 128 keys the 2 x 128 x 128 weights take 2048 clocks on the unit that computes exponentials, and the products
// 2 x (768 + 512) clocks of the tensor core at HD = 128 (64 x 128 x 16 reads its operands for 48 clocks, not 32).  A half takes about
// 1750 clocks, exponentials 1024 of them; the rest is reading scores, maxima, packing and the hand-over between warps, and a block's
// start and end cost as much as 450 keys.  Eight chunks of 1000..1024 tokens of 32 heads of 128 at 1024..4096 positions in bf16:
// 255 us, 0.83 PFLOP/s.  33 sequences of 11..329 new tokens at 364..1471 positions, 32 heads of 64 in e4m3: 197 us; a block
// has 129 of 256 rows on average, half of the blocks one tile only, whose products and softmax do not overlap, and 1050 keys, so that its start and
// end are 30 % of it; the two scales add 2 x 32 packed products per row and half.
// Exponentials by polynomial on the other units for an eighth to a half of the weights changed nothing (250..260 us).
//
// Warps: 0-3 and 4-7 softmax of tile 0 and 1 (one thread per row, which is a lane of tensor memory), 8-11 loaders (page
// look-up, copies into the swizzled layout the tensor core reads, conversion of codes), 12 and 13 issue the products of tile 0 and 1.
// Every wait is bounded; on expiry the block records it, waits (bounded) for the products in flight and frees its tensor memory.
#pragma once
#include "attn_paged.cuh"
#include "gemm_tc.cuh"

namespace sd {
namespace ac {

constexpr int THREADS = 512, KEYS = 128, TILE_ROWS = 128, STAGES = 2, SIDE = 4, HALF = 64;
constexpr float SLACK = 8.f;
constexpr int SUM_HALVES = 4;            // halves after which O joins a sum of its own, where results are fp32: a power of two
// Registers per thread of the softmax, the loader and the product warpgroups; the block is launched with 128 for each of its
// 512 threads, and the shares add up to no more: 2 x 128 x 168 + 128 x 120 + 128 x 40 = 63 488.
constexpr int LAUNCH_REGS = 128, SOFTMAX_REGS = 168, LOADER_REGS = 120, PRODUCT_REGS = 40;
static_assert(2 * 128 * SOFTMAX_REGS + 128 * LOADER_REGS + 128 * PRODUCT_REGS <= THREADS * LAUNCH_REGS, "a larger share would wait forever");
static_assert(SOFTMAX_REGS >= LAUNCH_REGS && LOADER_REGS <= LAUNCH_REGS && PRODUCT_REGS <= LAUNCH_REGS, "the first is raised, the others are lowered");

template <int HD, bool PAIRS> struct Layout {
  static constexpr int TILE = 128 * HD * 2;                    // a tile of Q, K or V: blocks of 64 elements, 128 rows of 128 bytes each
  // tiles of query rows of a block; the lower halves of pairs lie behind the upper ones.  At HD = 128 two tiles of pairs leave no room for two
  // stages of keys and values
  static constexpr int TILES = PAIRS && HD == 128 ? 1 : 2, ROWS = TILES * TILE_ROWS, Q_LOW = TILES * TILE;
  static constexpr int Q = 0, K = TILES * (PAIRS ? 2 : 1) * TILE, V = K + STAGES * TILE, END = V + STAGES * TILE;
  static constexpr int SIDE_OFF = END;                         // per key tile: 128 key scales, 128 value scales, mask of existing pages
  static constexpr int SIDE_BYTES = 2 * KEYS * 4 + 16;
  static constexpr int NEED = END + SIDE * SIDE_BYTES + 1024;  // + alignment
  static constexpr int SMEM = NEED > 116 * 1024 ? NEED : 116 * 1024;   // one block per SM: each takes all of the tensor memory
  static constexpr int O_COL = 256;                            // tensor memory: S_0 at 0 and 64, S_1 at 128 and 192, O_0, O_1 from 256,
  static constexpr int SUM_COL = O_COL + 128;                  // and with pairs sums of O_0, O_1
};

// bf16 x bf16 (half: fp16 x fp16) -> fp32, 128 rows; b_mn: B is stored with its output axis contiguous
__host__ __device__ constexpr uint32_t idesc(int n, bool b_mn, bool half) {
  return (1u << 4) | (half ? 0u : (1u << 7) | (1u << 10)) | (b_mn ? 1u << 16 : 0u) | ((uint32_t)(n >> 3) << 17) | (8u << 24);
}
// V as it lies: 64-element blocks `lead` bytes apart, groups of 8 keys 1024 bytes apart, 128-byte swizzle
__device__ __forceinline__ uint64_t v_desc(uint32_t addr, uint32_t lead) {
  return (uint64_t)((addr >> 4) & 0x3FFF) | ((uint64_t)(lead >> 4) << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}
// One lane of a warp, chosen so that the compiler knows it to be one: what it issues takes its operands from uniform registers, and
// a product goes out every 64 clocks (128 x 128 x 16).  Under a branch on the lane's number, with operands that the compiler cannot
// show to be uniform, it took 130.
__device__ __forceinline__ bool elect() {
  uint32_t p;
  asm volatile("{\n .reg .pred q;\n elect.sync _|q, 0xffffffff;\n selp.b32 %0, 1, 0, q;\n}\n" : "=r"(p));
  return p != 0;
}
template <typename T> __device__ __forceinline__ T uniform(T v) { return __shfl_sync(0xffffffffu, v, 0); }
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t id, uint32_t acc) { tc::umma(d, a, b, id, acc); }
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t id, uint32_t acc) {
  asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n"
               ::"r"(d), "r"(a), "l"(b), "r"(id), "r"(acc) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t (&r)[16]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
               ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
                 "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t addr, const uint32_t (&r)[32]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
               "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
               ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
                 "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
                 "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
                 "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]) : "memory");
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void sts16(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
               ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
// two floats at a time
struct F2 { unsigned long long v; };
__device__ __forceinline__ F2 f2(float a, float b) { F2 r; asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ void un2(F2 x, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x.v)); }
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) { F2 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v)); return r; }
__device__ __forceinline__ F2 add2(F2 a, F2 b) { F2 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v)); return r; }
__device__ __forceinline__ F2 mul2(F2 a, F2 b) { F2 r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v)); return r; }
__device__ __forceinline__ uint32_t pack(float a, float b, __nv_bfloat16) { return pack_bf16(a, b); }
__device__ __forceinline__ uint32_t pack(float a, float b, __half) { return pack_f16(a, b); }
// Query row of row r of the block's tile t, whose first row is row0 and whose tiles have n_rows: rows past the tile's end are its last one, and a tile without
// rows has the block's first one, so that what is looked up for a row is always that of one of the caller's.
__host__ __device__ __forceinline__ int tile_row(int row0, int t, int n_rows, int r) {
  return n_rows > 0 ? row0 + t * TILE_ROWS + (r < n_rows ? r : n_rows - 1) : row0;
}
// Number i (0..255) of the tokens that a tile of rows > 0 rows from `first_row` on belongs to (up to 129 of them), -1: there is none.
__host__ __device__ __forceinline__ int tile_token(int first_row, int rows, int group, int i) {
  const int token = first_row / group + i;
  return rows > 0 && token <= (first_row + rows - 1) / group ? token : -1;
}
// byte offset of 16-byte piece c (8 elements) of row r in a tile
__device__ __forceinline__ uint32_t piece(int r, int c) { return (uint32_t)((c >> 3) * (128 * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4)); }

// Four codes (a word) to two bf16 pairs.  int8: the lower seven bits under the exponent of 128 are 128 + those bits; the sign bit
// lands in the exponent of the subtrahend and makes 128 of it 256.
__device__ __forceinline__ uint32_t int8_pair(uint32_t two) {              // two codes in the lower bytes of the halves
  const uint32_t a = (two & 0x007f007fu) | 0x43004300u, s = (two & 0x00800080u) | 0xc300c300u;
  const __nv_bfloat162 d = __hadd2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&s));
  return *reinterpret_cast<const uint32_t*>(&d);
}
__device__ __forceinline__ void to_bf16(uint32_t w, uint32_t& lo, uint32_t& hi, int8_t) {
  lo = int8_pair(__byte_perm(w, 0u, 0x4140));
  hi = int8_pair(__byte_perm(w, 0u, 0x4342));
}
__device__ __forceinline__ void to_bf16(uint32_t w, uint32_t& lo, uint32_t& hi, e4m3) {
  const float2 a = e4m3_widen(w & 0xffffu), b = e4m3_widen(w >> 16);
  lo = pack_bf16(a.x, a.y);
  hi = pack_bf16(b.x, b.y);
}
// Which of 32 columns are within [right, left], a bit each.
__device__ __forceinline__ uint32_t columns(int right, int left) {
  const uint32_t below = left >= 31 ? 0xffffffffu : left < 0 ? 0u : (2u << left) - 1u;
  return right <= 0 ? below : right > 31 ? 0u : below & (0xffffffffu << right);
}
// Four bits to the four bytes of a word.
__device__ __forceinline__ uint32_t bytes_of(uint32_t four) { return (((four & 15u) * 0x00204081u) & 0x01010101u) * 0xffu; }

// as TANH0.. of paged.cuh, of degree 3 for [0, 0.45] and of degree 4 for [0, 0.7]: off by 2.5e-7 and 3.1e-7, with fp32's roundings 4.0e-7 and 4.7e-7
constexpr float CLOSE0 = 0x1.fffff8p-1f, CLOSE1 = -0x1.554b32p-2f, CLOSE2 = 0x1.0f14b2p-3f, CLOSE3 = -0x1.79101ep-5f;
constexpr float NEAR0 = 0x1.fffff6p-1f, NEAR1 = -0x1.554d28p-2f, NEAR2 = 0x1.0fff48p-3f, NEAR3 = -0x1.a07350p-5f, NEAR4 = 0x1.c35640p-7f;
// A half's 64 scores of a row, in place, to base-2 units: scale (8 and 4 bits: done), cap, distance.  pos: the row's position, counted from the first
// column; ahead: there may be visible keys behind the row's position.
template <bool SCALED>
__device__ __forceinline__ void change_scores(uint32_t (&s)[2][32], float scale, bool cap_on, float cap, float inv_cap, bool slope_on, float slope, int pos, int nearest, bool ahead) {
  const F2 scale2 = f2(scale, scale);
  auto get = [&](int k) { return f2(__uint_as_float(s[k >> 4][2 * k & 31]), __uint_as_float(s[k >> 4][(2 * k & 31) + 1])); };
  auto put = [&](int k, F2 y) {
    float a, b;
    un2(y, a, b);
    s[k >> 4][2 * k & 31] = __float_as_uint(a);
    s[k >> 4][(2 * k & 31) + 1] = __float_as_uint(b);
  };
  if (cap_on) {
    float top = 0.f;
#pragma unroll
    for (int k = 0; k < 64; k += 2) top = fmaxf(top, fmaxf(fabsf(__uint_as_float(s[k >> 5][k & 31])), fabsf(__uint_as_float(s[k >> 5][(k & 31) + 1]))));
    const float to_u = SCALED ? inv_cap : scale * inv_cap;
    top = top * (SCALED ? 1.f : scale) * inv_cap;
    // y = x (C0 + C1 x^2 + ..) with the cap and the unit within the numbers: five instructions a pair up to 0.45 of the cap, six up to 0.7.  Where
    // the numbers would leave fp32's range, and up to the cap, u is a product of its own: nine.
    const float k2 = to_u * to_u, first = SCALED ? 1.f : scale;
    // Which form it is goes by the whole warp: the unit may be a row's own (4 bits), so it is part of the votes, which all lanes take.
    const bool near_one = first > 0x1p-19f && first < 0x1p19f;
    const bool linear = !__any_sync(0xffffffffu, top > 0x1p-12f);    // a third of the square is below a rounding
    const bool close = !__any_sync(0xffffffffu, !(top <= 0.45f && near_one && to_u > 0x1p-15f && to_u < 0x1p15f));
    const bool near = !__any_sync(0xffffffffu, !(top <= 0.7f && near_one && to_u > 0x1p-12f && to_u < 0x1p12f));
    const bool below = !__any_sync(0xffffffffu, !(top <= 1.f && to_u < 1e38f));
    const F2 to_u2 = f2(to_u, to_u), cap2 = f2(cap, cap);
    auto polynomial = [&](auto... terms) {                           // the highest first
      constexpr int N = sizeof...(terms);
      const float number[N] = {terms...};
      F2 c[N];
      float power = first;
#pragma unroll
      for (int i = N - 1; i >= 0; --i) { c[i] = f2(number[i] * power, number[i] * power); power *= k2; }
#pragma unroll
      for (int k = 0; k < 32; ++k) {
        const F2 x = get(k), v = mul2(x, x);
        F2 p = c[0];
#pragma unroll
        for (int i = 1; i < N; ++i) p = fma2(v, p, c[i]);
        put(k, mul2(x, p));
      }
    };
    if (linear) {
#pragma unroll
      for (int k = 0; k < 32; ++k) put(k, mul2(get(k), f2(first, first)));
    } else if (close) {
      polynomial(CLOSE3, CLOSE2, CLOSE1, CLOSE0);
    } else if (near) {
      polynomial(NEAR4, NEAR3, NEAR2, NEAR1, NEAR0);
    } else if (below) {
#pragma unroll
      for (int k = 0; k < 32; ++k) {
        const F2 u = mul2(get(k), to_u2), v = mul2(u, u);
        F2 p = fma2(v, f2(TANH6, TANH6), f2(TANH5, TANH5));
        p = fma2(v, p, f2(TANH4, TANH4));
        p = fma2(v, p, f2(TANH3, TANH3));
        p = fma2(v, p, f2(TANH2, TANH2));
        p = fma2(v, p, f2(TANH1, TANH1));
        p = fma2(v, p, f2(TANH0, TANH0));
        put(k, mul2(mul2(u, cap2), p));
      }
    } else {                                                       // 1 - 2 / (1 + e^(2 u)): off by 2^-21 of the cap at most, small scores too
      const float to_e = inv_cap * 2.8853901f, twice = -2.f * cap;
#pragma unroll
      for (int k = 0; k < 64; ++k) {
        float e, d;
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(__uint_as_float(s[k >> 5][k & 31]) * (SCALED ? 1.f : scale) * to_e));
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(d) : "f"(1.f + e));
        s[k >> 5][k & 31] = __float_as_uint(fmaf(twice, d, cap));
      }
    }
  }
  if (slope_on) {
    if (!ahead || __all_sync(0xffffffffu, pos >= 63)) {            // -slope (pos - c - nearest) = slope away, away = c - (pos - nearest)
      // The distances are whole numbers, counted on two at a time: a bias is rounded once, with its sum where that is one instruction.  (Sums of slopes in
      // their place save a product where there is neither scale nor cap, and were off by roundings of the largest bias in the half.)
      const float begin = (float)(nearest - pos);
      const F2 slope2 = f2(slope, slope), two = f2(2.f, 2.f);
#pragma unroll
      for (int k8 = 0; k8 < 4; ++k8) {
        F2 away = add2(f2(begin, begin), f2(16.f * k8, 16.f * k8 + 1.f));
#pragma unroll
        for (int k = 8 * k8; k < 8 * k8 + 8; ++k) {
          put(k, SCALED || cap_on ? fma2(away, slope2, get(k)) : fma2(get(k), scale2, mul2(away, slope2)));
          away = add2(away, two);
        }
      }
    } else {
#pragma unroll
      for (int k = 0; k < 64; ++k) {
        const float x = __uint_as_float(s[k >> 5][k & 31]), y = SCALED || cap_on ? x : x * scale;
        s[k >> 5][k & 31] = __float_as_uint(fmaf(-slope, (float)(abs(pos - k) - nearest), y));
      }
    }
  } else if (!SCALED && !cap_on) {
#pragma unroll
    for (int k = 0; k < 32; ++k) put(k, mul2(get(k), scale2));
  }
}

}  // namespace ac

// grid (blocks_per_seq * n_kv_heads * n_seqs, splits).  Sequences with fewer than rows_from query rows are another kernel's.  Split z takes
// keys [z * chunk, (z + 1) * chunk), the last one all that follow; several leave partial results (accumulator, maximum, sum) of their rows
// to paged_attn_join_kernel.
// map_k, map_v: the pools as [n_pages * n_kv_heads][page_len][HD] with boxes of a page by 64 elements (bf16 only; use_maps 0: not made).
// PAIRS: queries and weights enter as sums of two bf16 (4 bits: of two fp16).
// SC: scores are changed and keys masked as `sc` says; keys are counted from the tile of 128 that the first visible key of the block lies in, and a block
// leaves the number of its splits for every row (part_used).  The change goes over pairs of scores: scale, the polynomial of paged.cuh while no score of
// the warp passes the cap, the distance as a line (keys at or before the row) or an absolute value.
// test_expire: test hook, values are never given back and the loaders give up after about a millisecond, keys of the third tile on their way.
template <typename TC, int HD, bool PAIRS, bool SC>
__global__ void __launch_bounds__(ac::THREADS, 1)
paged_attn_chunk_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, int use_maps,
                        const BatchView b, const Rows q, const Rows out, const TC* __restrict__ Kp, const TC* __restrict__ Vp,
                        const float* __restrict__ Ksc, const float* __restrict__ Vsc, const uint8_t* __restrict__ Kb, const uint8_t* __restrict__ Vb, int group, float scale_log2, bool q_vec, bool out_vec,
                        int blocks_per_seq, int rows_from, int chunk, float* part_acc, float* part_ml, int test_expire, const Scores sc, int* part_used) {
  using namespace ac;
  using L = Layout<HD, PAIRS>;
  constexpr bool SCALED = CacheType<TC>::TOP > 0.f, FOUR = kFour<TC>;
  using Op = std::conditional_t<FOUR, __half, __nv_bfloat16>;    // the products' operands
  // 4 bits: from and to bf16 the values' scales are part of the operands (FOLD), else they join the weights
  constexpr bool FOLD = FOUR && !PAIRS;
  constexpr float LIFT = FOLD ? 16.f : 128.f, BACK = 1.f / LIFT;  // values, or weights, are relative to a power of two (ve) over LIFT
  constexpr int ROWS = L::ROWS;
  // The tensor core's additions truncate, so a long sum comes out smaller (16 384 equal values 3.1e-5, random ones 1e-5): results in fp32
  // have theirs in parts of 256 keys, which are added to nearest (1e-6; 8 chunks of 3-1024 tokens at 1024-4096, 32 heads of 128: 652 us without, 694 with).
  constexpr bool SUMS = FOUR && PAIRS;
  const int sum_mask = SUMS && out.dtype == DT_FP32 ? SUM_HALVES - 1 : 0x7fffffff;
  extern __shared__ unsigned char ac_smem[];
  __shared__ uint64_t bars[4 * STAGES + 13 + SIDE];
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_word;

  pdl_launch_dependents();                                       // the kernel for few rows of the same call may begin beside this one's last blocks

  // the block's rows.  The longest sequences come first, so that no long block is left to the end: sequence number `turn` in
  // order of decreasing length (a block counts for each of up to THREADS sequences how many are longer; more keep their order)
  const int g_head = blockIdx.x % b.n_kv_heads, rest = blockIdx.x / b.n_kv_heads;
  const int blk = rest % blocks_per_seq, turn = rest / blocks_per_seq;
  __shared__ int lens[THREADS];
  __shared__ int4 turn_seq;                                       // number, first row, behind its last row, length
  int4 who;
  if (b.n_seqs > 1 && b.n_seqs <= THREADS) {
    int mine = 0, begin = 0, end = 0;
    if (threadIdx.x < b.n_seqs) { mine = b.len[threadIdx.x]; begin = b.first[threadIdx.x]; end = b.first[threadIdx.x + 1]; }
    lens[threadIdx.x] = mine;
    __syncthreads();
    if (threadIdx.x < b.n_seqs) {
      int ahead = 0;
      for (int i = 0; i < b.n_seqs; ++i) ahead += lens[i] > mine || (lens[i] == mine && i < (int)threadIdx.x);
      if (ahead == turn) turn_seq = make_int4(threadIdx.x, begin, end, mine);
    }
    __syncthreads();
    who = turn_seq;
  } else {
    who = make_int4(turn, b.first[turn], b.first[turn + 1], b.len[turn]);
  }
  const int seq = who.x, f0 = who.y, f1 = who.z, len = b.held_len(who.w);
  int n_new = f1 - f0;
  if (f0 < 0 || n_new < 0 || f1 > b.n_tokens || n_new > b.max_new) {
    if (threadIdx.x == 0) b.bad();
    if (f0 < 0 || n_new < 0) return;
    n_new = min(n_new, min(b.max_new, b.n_tokens - f0));
  }
  const int rows_all = n_new * group;
  if (rows_all < rows_from) return;
  const int blocks = (rows_all + ROWS - 1) / ROWS;
  const int row0 = (blocks - 1 - blk) * ROWS;                   // the rows that see most keys first
  if (row0 < 0) return;
  const long long pos_first = (long long)who.w - (f1 - f0);
  const int splits = gridDim.y, z = blockIdx.y;
  int first_key = 0, first_seen = 0, ends[2] = {0, 0};            // SC: where the block's keys begin; the first that a row sees; where they end for each tile
  if constexpr (SC) {
    __shared__ int span_lo[THREADS / 32], span_hi[THREADS / 32];
    const int t = threadIdx.x >> 8, start = row0 + t * TILE_ROWS;
    const int token = tile_token(start, t < L::TILES ? min(TILE_ROWS, rows_all - start) : 0, group, threadIdx.x & 255);
    Span v{0, -1};
    if (token >= 0) v = visible(sc, f0 + token, pos_first + token, len);
    const int from = __reduce_min_sync(0xffffffffu, v.lo <= v.hi ? v.lo : 0x7fffffff), to = __reduce_max_sync(0xffffffffu, v.hi + 1);
    if ((threadIdx.x & 31) == 0) { span_lo[threadIdx.x >> 5] = from; span_hi[threadIdx.x >> 5] = to; }
    __syncthreads();
    first_key = 0x7fffffff;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) {
      first_key = min(first_key, span_lo[w]);
      ends[w / 8] = max(ends[w / 8], span_hi[w]);
    }
    first_seen = first_key == 0x7fffffff ? 0 : first_key;
    first_key = first_seen & ~(KEYS - 1);
  }
  const int key0 = SC ? (int)min(first_key + (long long)z * chunk, 0x7fffffffll) : z * chunk;  // key numbers below count from key0
  int n_keys[2], n_rows[2], used_splits = 1;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    n_rows[t] = t < L::TILES ? max(0, min(TILE_ROWS, rows_all - row0 - t * TILE_ROWS)) : 0;
    const int last = (row0 + t * TILE_ROWS + n_rows[t] - 1) / group;
    int keys = n_rows[t] ? (int)min(max(pos_first + last + 1, 0ll), (long long)len) : 0;
    if (SC) keys = max(ends[t] - first_key, 0);
    if (splits > 1) {
      used_splits = max(used_splits, ap::splits_of(keys, chunk, splits));
      keys = max(keys - (key0 - first_key), 0);
      if (z < splits - 1) keys = min(keys, chunk);
    }
    n_keys[t] = (keys + HALF - 1) / HALF;                       // halves of key tiles; a later tile of rows sees no fewer
  }
  if (z >= used_splits) return;
  const int n_tiles = (max(n_keys[0], n_keys[1]) + 1) / 2;

  const int warp = uniform((int)threadIdx.x >> 5), lane = threadIdx.x & 31;
  const uint32_t raw = (uint32_t)__cvta_generic_to_shared(ac_smem), base = (raw + 1023u) & ~1023u;
  unsigned char* base_ptr = ac_smem + (base - raw);
  const uint32_t bar0 = (uint32_t)__cvta_generic_to_shared(bars);
  const uint32_t kfull = bar0, kempty = kfull + 8 * STAGES, vfull = kempty + 8 * STAGES, vempty = vfull + 8 * STAGES;
  const uint32_t sfull = vempty + 8 * STAGES, pready = sfull + 32, odone = pready + 32, qfull = odone + 16, drain = qfull + 8, sidefull = drain + 16;
  volatile int* abort_flag = &abort_word;

  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) {
      tc::mbar_init(kfull + 8 * s, 4); tc::mbar_init(kempty + 8 * s, 2);
      tc::mbar_init(vfull + 8 * s, 4); tc::mbar_init(vempty + 8 * s, 2);
    }
    for (int i = 0; i < 4; ++i) { tc::mbar_init(sfull + 8 * i, 1); tc::mbar_init(pready + 8 * i, 4); }      // tile t, half h: 2 t + h
    for (int t = 0; t < 2; ++t) tc::mbar_init(odone + 8 * t, 1);
    tc::mbar_init(qfull, 8);
    tc::mbar_init(drain, 1); tc::mbar_init(drain + 8, 1);
    for (int i = 0; i < SIDE; ++i) tc::mbar_init(sidefull + 8 * i, 4);
    abort_word = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 12) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"((uint32_t)__cvta_generic_to_shared(&tmem_slot)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  // Softmax warps: the thread's query row.  The rows are on their way while the barriers and the tensor memory are prepared.
  const int t = warp >> 2 & 1, r = (warp & 3) * 32 + lane;
  const int row = tile_row(row0, t, n_rows[t], r);
  const int token = row / group, head = g_head * group + row % group;
  int row_last = (int)max(min(pos_first + token, (long long)len - 1), -1ll) - key0;        // last key this row sees
  const float sign = scale_log2 < 0.f ? -1.f : 1.f;             // a negative scale turns the queries round
  float scale = SCALED ? 1.f : fabsf(scale_log2);               // base-2 units of a score, as it comes, that is 1 (8 and 4 bits: the keys' scales have the rest)
  if (warp < 8 && n_rows[t] > 0) {
    // The warp's 32 rows, PIECES lanes to a row, so that a request takes whole lines.  (A row to a thread, 32 lines to a request: 4000 clocks of a block at
    // HD = 64 and 9000 at 128.)
    constexpr int PIECES = HD / 8, AT_ONCE = 32 / PIECES;
    const long long at = (long long)(f0 + token) * q.row_stride + head * q.head_stride;
    const int mine = lane / PIECES, c = lane % PIECES;            // row of a round, piece
    const uint32_t dst = base + L::Q + t * L::TILE;
    auto place = [&](int i) { return dst + piece((warp & 3) * 32 + i * AT_ONCE + mine, c); };
    auto start = [&](int i) { return __shfl_sync(0xffffffffu, at, i * AT_ONCE + mine) + c * 8; };
    auto put = [&](int i, const float (&x)[8]) {
      float turn = sign;
      if constexpr (FOUR) {                                       // fp16 operands: the row is brought near 1 by a power of two
        float top = 0.f;
#pragma unroll
        for (int k = 0; k < 8; ++k) top = fmaxf(top, fabsf(x[k]));
#pragma unroll
        for (int o = 1; o < PIECES; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        const int e = min(max((int)((__float_as_uint(top) >> 23) & 0xff), 2), 252);
        turn *= __uint_as_float((uint32_t)(254 - e) << 23);       // 2^(127 - e)
        const float back = __shfl_sync(0xffffffffu, __uint_as_float((uint32_t)e << 23), lane % AT_ONCE * PIECES);
        if (lane / AT_ONCE == i) scale = back;                    // 2^(e - 127), to the thread whose row it is
      }
      uint32_t hi[4], lo[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if constexpr (PAIRS) ap::split(x[2 * k] * turn, x[2 * k + 1] * turn, hi[k], lo[k], Op{});
        else hi[k] = pack(x[2 * k] * turn, x[2 * k + 1] * turn, Op{});
      }
      sts16(place(i), hi[0], hi[1], hi[2], hi[3]);
      if constexpr (PAIRS) sts16(place(i) + L::Q_LOW, lo[0], lo[1], lo[2], lo[3]);
    };
    if (q_vec && q.dtype != DT_FP32) {
      uint4 x[PIECES];                                            // all on their way together
#pragma unroll
      for (int i = 0; i < PIECES; ++i) x[i] = __ldg(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(q.data) + start(i)));
      if (!PAIRS && !FOUR && q.dtype == DT_BF16) {
        const uint32_t turn = scale_log2 < 0.f ? 0x80008000u : 0u;
#pragma unroll
        for (int i = 0; i < PIECES; ++i) sts16(place(i), x[i].x ^ turn, x[i].y ^ turn, x[i].z ^ turn, x[i].w ^ turn);
      } else {
        const bool is_half = q.dtype == DT_FP16;
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
          const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
          float y[8];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[k]));
            y[2 * k] = is_half ? f.x : __uint_as_float(w[k] << 16);
            y[2 * k + 1] = is_half ? f.y : __uint_as_float(w[k] & 0xffff0000u);
          }
          put(i, y);
        }
      }
    } else {
#pragma unroll
      for (int i0 = 0; i0 < PIECES; i0 += 4) {                    // four rounds' loads on their way together
        float x[4][8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const long long from = start(i0 + i);
          if (q_vec) load8<true>(static_cast<const float*>(q.data) + from, x[i]);
          else ap::load_run<8>(q, from, false, x[i]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) put(i0 + i, x[i]);
      }
    }
    fence_async();
  }
  // loaders: the pages of the first tile of keys
  const int* table = b.pages + (size_t)seq * b.pages_per_seq;
  // Keys from `most` on are filled with zeros, and with masks those ahead of `least`: no row sees them, they may be anything, and their pages need not exist.
  const int most = min((SC ? max(ends[0], ends[1]) : len) - key0, n_tiles * KEYS), least = first_seen - key0;
  // lane i < 16 looks up the page of keys [8 i, 8 i + 8) of a tile
  auto look_up = [&](int j) {
    const int key = j * KEYS + (lane & 15) * 8;
    return j < n_tiles && key < most ? table[(key0 + key) >> b.page_shift] : 0;
  };
  const int page_first = warp >= 8 && warp < 12 ? look_up(0) : 0;
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = tmem_slot;

  if (warp < 8) {
    // ---- softmax: one thread per query row
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(SOFTMAX_REGS));
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t s_addr = tmem + lanes + t * 128, o_addr = tmem + lanes + L::O_COL + t * HD;
    if (lane == 0) arrive(qfull);                                 // the rows are in shared memory since before the block's barriers were

    // the keys that all 32 rows of the warp see: tiles below need no mask
    const int first_token = tile_row(row0, t, n_rows[t], (warp & 3) * 32) / group;
    int all_see = (int)max(min(pos_first + first_token, (long long)len - 1), -1ll) - key0;
    int row_first = 0, all_from = 0, any_from = 0, any_see = 0;  // SC: the first key of this row, the keys that some row of the warp sees
    int row_pos = 0, nearest = 0;                                // the row's position, counted as the keys; the distance of its nearest visible key
    float slope = 0.f, cap = 0.f, inv_cap = 0.f;
    if constexpr (SC) {
      const Span v = visible(sc, f0 + token, pos_first + token, len);
      row_first = v.lo - key0;
      row_last = v.hi - key0;
      all_from = __reduce_max_sync(0xffffffffu, row_first);
      all_see = __reduce_min_sync(0xffffffffu, row_last);
      any_from = __reduce_min_sync(0xffffffffu, v.lo <= v.hi ? row_first : 0x7fffffff);
      any_see = __reduce_max_sync(0xffffffffu, row_last);
      const int p = (int)min(max(pos_first + token, 0ll), 1ll << 30);
      row_pos = p - key0;
      nearest = abs(p - min(max(p, v.lo), v.hi));
      if (sc.slopes && n_rows[t] > 0) slope = sc.slopes[head] * 1.4426950408889634f;
      cap = sc.cap * 1.4426950408889634f;
      inv_cap = sc.cap > 0.f ? 1.f / cap : 0.f;
    }
    float m = -INFINITY, l = 0.f;                                // m in the units of the scores (bf16, 4 bits), or base-2 (8 bits, changed scores)
    const bool changed = SC && (sc.cap > 0.f || sc.slopes);
    const float unit = changed ? 1.f : scale;                    // base-2 units per unit of m
    float ve = 0.f;                                              // 4 bits: what values or their weights are relative to
    bool ok = true;
    // Results in fp32: O of every SUM_HALVES halves is added to a sum beside it, whose unit is behind by `since`.  The product of half i begins anew.
    const uint32_t sum_addr = tmem + lanes + L::SUM_COL + t * HD;
    float since = 1.f;
    auto join = [&](int i) {
      ok = __all_sync(0xffffffffu, tc::mbar_wait(odone + 8 * t, (i - 1) & 1, abort_flag, b.status));
      if (!ok) return false;
      fence_after();
#pragma unroll 1
      for (int c0 = 0; c0 < HD; c0 += 16) {
        uint32_t v[32], old[32], sum[16];
        tc::tmem_ld16(o_addr + c0, v);
        if (i > SUM_HALVES) tc::tmem_ld16(sum_addr + c0, old);
        tmem_wait_ld();
#pragma unroll
        for (int k = 0; k < 16; ++k) sum[k] = i > SUM_HALVES ? __float_as_uint(fmaf(__uint_as_float(old[k]), since, __uint_as_float(v[k]))) : v[k];
        tmem_st16(sum_addr + c0, sum);
      }
      tmem_wait_st();
      since = 1.f;
      return true;
    };
    for (int i = 0; i < n_keys[t]; ++i) {
      const int j = i >> 1, h = i & 1;
      // scales and mask have a barrier of their own; it cannot run a phase ahead of this wait, because the loaders reach tile
      // j + SIDE only after the scores of tile j + 2, which follow this half's weights
      ok = __all_sync(0xffffffffu, tc::mbar_wait(sfull + 8 * (2 * t + h), j & 1, abort_flag, b.status) &&
                                   tc::mbar_wait(sidefull + 8 * (j % SIDE), (j / SIDE) & 1, abort_flag, b.status));
      if (!ok) break;
      fence_after();
      const float* side = reinterpret_cast<const float*>(base_ptr + L::SIDE_OFF + (j & (SIDE - 1)) * L::SIDE_BYTES);
      const uint32_t pages_ok = *reinterpret_cast<const uint32_t*>(side + 2 * KEYS) >> (8 * h) & 0xffu;
      const float ve_now = FOUR ? side[2 * KEYS + 1] : 0.f;      // as large as that of any tile before
      side += h * HALF;
      const uint32_t s_half = s_addr + h * HALF;

      if constexpr (SC) {
        if (i * HALF + HALF - 1 < any_from || i * HALF > any_see) {              // nobody in this warp sees any of them
          const uint32_t none[16] = {};
#pragma unroll
          for (int c = 0; c < (PAIRS ? 4 : 2); ++c) tmem_st16(s_half + 16 * c, none);
          tmem_wait_st();
          if (SUMS && i > 0 && (i & sum_mask) == 0 && !join(i)) break;
          fence_before();
          if (i > 0 && i + 1 == n_keys[t]) {                     // as below
            ok = __all_sync(0xffffffffu, tc::mbar_wait(odone + 8 * t, (i - 1) & 1, abort_flag, b.status));
            if (!ok) break;
          }
          __syncwarp();
          if (lane == 0) arrive(pready + 8 * (2 * t + h));
          continue;
        }
      }
      uint32_t s[2][32];
#pragma unroll
      for (int c = 0; c < 2; ++c) tc::tmem_ld32(s_half + 32 * c, s[c]);
      tmem_wait_ld();
      if (SCALED) {                                              // the key's scale (with the softmax scale and log2 e)
#pragma unroll
        for (int c = 0; c < HALF; c += 4) {
          const float4 k = *reinterpret_cast<const float4*>(side + c);
          uint32_t* x = &s[c >> 5][c & 31];
          float y0, y1, y2, y3;
          un2(mul2(f2(__uint_as_float(x[0]), __uint_as_float(x[1])), f2(k.x, k.y)), y0, y1);
          un2(mul2(f2(__uint_as_float(x[2]), __uint_as_float(x[3])), f2(k.z, k.w)), y2, y3);
          x[0] = __float_as_uint(y0); x[1] = __float_as_uint(y1); x[2] = __float_as_uint(y2); x[3] = __float_as_uint(y3);
        }
      }
      if constexpr (SC) {
        if (changed) change_scores<SCALED && !FOUR>(s, scale, sc.cap > 0.f, cap, inv_cap, sc.slopes != nullptr, slope, row_pos - i * HALF, nearest, sc.hi != nullptr);
      }
      if (i * HALF + HALF - 1 > all_see || pages_ok != 0xffu || (SC && i * HALF < all_from)) {
        const int left = row_last - i * HALF, right = SC ? row_first - i * HALF : 0;          // columns from `right` up to `left` are seen
        uint32_t see[2] = {columns(right, left), columns(right - 32, left - 32)};
        if (pages_ok != 0xffu) { see[0] &= bytes_of(pages_ok); see[1] &= bytes_of(pages_ok >> 4); }
#pragma unroll
        for (int c = 0; c < HALF; ++c)
          if (!(see[c >> 5] & (1u << (c & 31)))) s[c >> 5][c & 31] = 0xff800000u;
      }
      float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
      for (int k = 0; k < 16; k += 2)
#pragma unroll
        for (int c = 0; c < 4; ++c) mx[c] = fmaxf(mx[c], fmaxf(__uint_as_float(s[c >> 1][(c & 1) * 16 + k]), __uint_as_float(s[c >> 1][(c & 1) * 16 + k + 1])));
      const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
      if (__any_sync(0xffffffffu, (top - m) * unit > SLACK || (FOUR && ve_now > ve))) {   // -inf - -inf is NaN: not greater
        const float m_new = fmaxf(m, top);
        float a = m == -INFINITY ? 0.f : ex2((m - m_new) * unit);
        m = m_new;
        l *= a;
        if constexpr (FOUR) {
          a *= ve / ve_now;                                      // powers of two, or 0 over one
          ve = ve_now;
        }
        since *= a;
        if (i > 0) {
          ok = __all_sync(0xffffffffu, tc::mbar_wait(odone + 8 * t, (i - 1) & 1, abort_flag, b.status));
          if (!ok) break;
          fence_after();
#pragma unroll 1
          for (int c0 = 0; c0 < HD; c0 += 16) {
            uint32_t v[32], o16[16];
            tc::tmem_ld16(o_addr + c0, v);
            tmem_wait_ld();
#pragma unroll
            for (int k = 0; k < 16; ++k) o16[k] = __float_as_uint(__uint_as_float(v[k]) * a);
            tmem_st16(o_addr + c0, o16);
          }
          tmem_wait_st();
        }
      }
      const float mb = (m == -INFINITY ? 0.f : -m * unit) + (FOLD ? 7.f : 0.f);      // weights and their sum times 2^7 where fp16 has to hold them
      const F2 unit2 = f2(unit, unit), mb2 = f2(mb, mb);
      F2 sum[2] = {f2(0.f, 0.f), f2(0.f, 0.f)};
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        uint32_t w[16], w_lo[16];
#pragma unroll
        for (int k = 0; k < 16; ++k) {
          F2 x = f2(__uint_as_float(s[c][2 * k]), __uint_as_float(s[c][2 * k + 1]));
          x = SCALED && !FOUR ? add2(x, mb2) : fma2(x, unit2, mb2);
          float p0, p1;
          un2(x, p0, p1);
          p0 = ex2(p0);
          p1 = ex2(p1);
          x = f2(p0, p1);
          sum[k & 1] = add2(sum[k & 1], x);
          if (SCALED && !FOLD) {
            const float2 v = *reinterpret_cast<const float2*>(side + KEYS + c * 32 + 2 * k);
            un2(mul2(x, f2(v.x, v.y)), p0, p1);
          }
          if constexpr (PAIRS) ap::split(p0, p1, w[k], w_lo[k], Op{});
          else w[k] = pack(p0, p1, Op{});
        }
        tmem_st16(s_half + 16 * c, w);                           // over columns that have been read
        if constexpr (PAIRS) tmem_st16(s_half + HALF / 2 + 16 * c, w_lo);
      }
      float a0, a1;
      un2(add2(sum[0], sum[1]), a0, a1);
      l += a0 + a1;
      tmem_wait_st();
      if (SUMS && i > 0 && (i & sum_mask) == 0 && !join(i)) break;
      fence_before();
      // The last half waits here for the product before its own, so that the wait after the loop is for the phase in progress or
      // the one before: a wait looks at a phase's parity only, and one for a phase two back would never end.
      if (i > 0 && i + 1 == n_keys[t]) {
        ok = __all_sync(0xffffffffu, tc::mbar_wait(odone + 8 * t, (i - 1) & 1, abort_flag, b.status));
        if (!ok) break;
      }
      __syncwarp();
      if (lane == 0) arrive(pready + 8 * (2 * t + h));
    }
    if constexpr (SC) {
      if (splits > 1 && z == 0 && r < n_rows[t]) part_used[(size_t)(f0 + token) * (group * b.n_kv_heads) + head] = used_splits;
    }
    if (n_rows[t] > 0 && ok) {
      if (n_keys[t] > 0) {
        ok = __all_sync(0xffffffffu, tc::mbar_wait(odone + 8 * t, (n_keys[t] - 1) & 1, abort_flag, b.status));
        fence_after();
      }
      const bool joined = SUMS && n_keys[t] > SUM_HALVES && sum_mask == SUM_HALVES - 1;
      auto load = [&](int c0, uint32_t (&v)[32]) {               // 32 columns of the row's sums
        tc::tmem_ld32(o_addr + c0, v);
        if (joined) {
          uint32_t old[32];
          tc::tmem_ld32(sum_addr + c0, old);
          tmem_wait_ld();
#pragma unroll
          for (int k = 0; k < 32; ++k) v[k] = __float_as_uint(fmaf(__uint_as_float(old[k]), since, __uint_as_float(v[k])));
        } else {
          tmem_wait_ld();
        }
      };
      if (ok && used_splits == 1) {
        const float inv = l > 0.f ? (FOUR ? ve * BACK : 1.f) / l : 0.f;
        const long long at = (long long)(f0 + token) * out.row_stride + head * out.head_stride;
#pragma unroll 1
        for (int c0 = 0; c0 < HD; c0 += 32) {
          uint32_t v[32];
          if (n_keys[t] > 0) load(c0, v);
          if (r < n_rows[t]) {
#pragma unroll
            for (int i = 0; i < 32; i += 8) {
              float x[8];
#pragma unroll
              for (int k = 0; k < 8; ++k) x[k] = l > 0.f ? __uint_as_float(v[i + k]) * inv : (l == 0.f ? 0.f : l);   // l NaN: NaN
              const long long e = at + c0 + i;
              if (out_vec && out.dtype == DT_BF16) store8<true>(static_cast<__nv_bfloat16*>(out.data) + e, x);
              else if (out_vec && out.dtype == DT_FP16) store8<true>(static_cast<__half*>(out.data) + e, x);
              else if (out_vec) store8<true>(static_cast<float*>(out.data) + e, x);
              else {
#pragma unroll
                for (int k = 0; k < 8; ++k) store_elem(out, e + k, x[k]);
              }
            }
          }
        }
      } else if (ok) {
        // the row's share: sums relative to the maximum, in base-2 units
        const size_t slot = ((size_t)(f0 + token) * (group * b.n_kv_heads) + head) * splits + z;
        const float back = FOUR ? ve * BACK : 1.f;
#pragma unroll 1
        for (int c0 = 0; c0 < HD; c0 += 32) {
          uint32_t v[32] = {};
          if (n_keys[t] > 0) load(c0, v);
          if (r < n_rows[t]) {
#pragma unroll
            for (int i = 0; i < 32; i += 4)
              __stcg(reinterpret_cast<float4*>(part_acc + slot * HD + c0 + i), make_float4(__uint_as_float(v[i]) * back, __uint_as_float(v[i + 1]) * back, __uint_as_float(v[i + 2]) * back, __uint_as_float(v[i + 3]) * back));
          }
        }
        if (r < n_rows[t]) __stcg(reinterpret_cast<float2*>(part_ml + slot * 2), make_float2(m * unit, l));
      }
    }
  } else if (warp < 12) {
    // ---- loaders
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(LOADER_REGS));
    const int w = warp - 8, tid = w * 32 + lane;
    constexpr int E = sizeof(TC), PER_ROW = row_units<TC>(HD) * E / 16;   // 16-byte pieces of a stored key
    constexpr int ROWS_AT_ONCE = 32 / PER_ROW;                    // of a warp
    constexpr int STEPS = KEYS / (4 * ROWS_AT_ONCE);
    auto exists = [&](int j, int page) {
      const int key = j * KEYS + (lane & 15) * 8;
      return __ballot_sync(0xffffffffu, (unsigned)page < (unsigned)b.n_pages || key >= most || (SC && key + 7 < least)) & 0xffffu;
    };
    // this thread's piece in step i: row `key`, piece c
    auto key_of = [&](int i) { return (i * 4 + w) * ROWS_AT_ONCE + lane / PER_ROW; };
    const int c = lane % PER_ROW;
    auto source = [&](const TC* pool, int j, int key, int page, uint32_t pages_ok) -> const TC* {
      page = __shfl_sync(0xffffffffu, page, key >> 3);
      const bool on = j * KEYS + key < most && !(SC && j * KEYS + key < least) && ((pages_ok >> (key >> 3)) & 1u);
      return on ? pool + b.entry(page, g_head, key0 + j * KEYS + key) * row_units<TC>(HD) + c * (16 / E) : nullptr;
    };
    // this thread's key's scales, zeros where there is none
    auto ask_scales = [&](int j, int page, uint32_t pages_ok) {
      page = __shfl_sync(0xffffffffu, page, (tid >> 3) & 15);
      if (!(j * KEYS + tid < most && !(SC && j * KEYS + tid < least) && ((pages_ok >> (tid >> 3)) & 1u))) return make_float2(0.f, 0.f);
      const size_t e = b.entry(page, g_head, key0 + j * KEYS + tid);
      return make_float2(__ldg(Ksc + e), __ldg(Vsc + e));
    };
    // 4 bits: a power of two above all the values' scales so far.  Every warp looks at all 128 of a tile, four a lane, so that none waits for another.
    float ve = 0.f;
    auto ask_values = [&](int j, int page, uint32_t pages_ok) {
      page = __shfl_sync(0xffffffffu, page, lane >> 1);
      const int key = j * KEYS + lane * 4, left = most - key;
      if (left <= 0 || (SC && key + 3 < least) || !((pages_ok >> (lane >> 1)) & 1u)) return 0.f;
      const float4 v = __ldg(reinterpret_cast<const float4*>(Vsc + b.entry(page, g_head, key0 + key)));
      return fmaxf(fmaxf((SC && key < least) ? 0.f : v.x, left > 1 && !(SC && key + 1 < least) ? v.y : 0.f), fmaxf(left > 2 && !(SC && key + 2 < least) ? v.z : 0.f, left > 3 ? v.w : 0.f));
    };
    auto raise = [&](float top) {
      const float all = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(fabsf(top))));
      const int e = min(max((int)((__float_as_uint(all) >> 23) & 0xff) + 1, 14), 254);
      ve = fmaxf(ve, __uint_as_float((uint32_t)e << 23));
    };
    auto begin_side = [&](int j, float2 scales, uint32_t pages_ok) {
      float* side = reinterpret_cast<float*>(base_ptr + L::SIDE_OFF + (j & (SIDE - 1)) * L::SIDE_BYTES);
      if (tid == 0) *reinterpret_cast<uint32_t*>(side + 2 * KEYS) = pages_ok;
      if (pages_ok != 0xffffu && w == 0 && lane == 0) b.bad();
      if (SCALED) {
        side[tid] = scales.x * fabsf(scale_log2);
        if (!FOLD) side[KEYS + tid] = FOUR ? scales.y * (LIFT / ve) : scales.y;
        if (FOUR && tid == 0) side[2 * KEYS + 1] = ve;
      }
      __syncwarp();
      if (lane == 0) arrive(sidefull + 8 * (j % SIDE));
    };
    auto wait_free = [&](uint32_t bar, int j) {
      return j < STAGES || __all_sync(0xffffffffu, tc::mbar_wait(bar + 8 * (j % STAGES), (j / STAGES - 1) & 1, abort_flag, b.status,
                                                                 test_expire ? 2000000ll : tc::kWaitLimit));
    };
    auto announce = [&](uint32_t bar, int j) {                    // plain stores or asynchronous copies that have landed
      fence_async();
      __syncwarp();
      if (lane == 0) arrive(bar + 8 * (j % STAGES));
    };
    bool ok = true;
    int page_next = page_first;
    if constexpr (!SCALED) {
      auto copy = [&](const TC* pool, uint32_t dst, int j, int page, uint32_t pages_ok) {
#pragma unroll 4
        for (int i = 0; i < STEPS; ++i) {
          const int key = key_of(i);
          const TC* src = source(pool, j, key, page, pages_ok);
          pf_cp16(dst + piece(key, c), src ? src : pool, src ? 16 : 0);
        }
        pf_commit();
      };
      // whole pages by tensor copies, a page's half (64 elements) per copy, lane i the page of keys [8 i, ...).  The first warp announces
      // for all four, so that a phase ends when its copies have landed, whatever the other warps do
      auto fetch = [&](const CUtensorMap* map, uint32_t dst, uint32_t bar, int j, int page) {
        const uint32_t full = bar + 8 * (j % STAGES);
        if (w == 0) {
          if (lane == 0) {
            tc::mbar_expect_tx(full, L::TILE);
            arrive(full); arrive(full); arrive(full);
          }
          __syncwarp();
          if (lane < 16 && ((lane * 8) & (b.page_len - 1)) == 0) {
#pragma unroll
            for (int h = 0; h < HD / 64; ++h)
              tma_load_3d(dst + h * (128 * 128) + lane * 1024, map, h * 64, 0, page * b.n_kv_heads + g_head, full);
          }
        }
      };
      int k_asked = 0, v_asked = 0;                               // tiles whose keys, values have been asked for
      uint32_t wholes = 0u;                                       // bit i: tile k_asked - 1 - i came by tensor copies
      for (int j = 0; j < n_tiles; ++j) {
        const int page = page_next;
        page_next = look_up(j + 1);
        const uint32_t pages_ok = exists(j, page);
        const bool whole = use_maps && (j + 1) * KEYS <= most && !(SC && j * KEYS < least) && pages_ok == 0xffffu;
        const uint32_t kt = base + L::K + (j % STAGES) * L::TILE, vt = base + L::V + (j % STAGES) * L::TILE;
        if (!(ok = wait_free(kempty, j))) break;
        begin_side(j, make_float2(0.f, 0.f), pages_ok);
        if (whole) fetch(&map_k, kt, kfull, j, page);
        else copy(Kp, kt, j, page, pages_ok);
        k_asked = j + 1;
        wholes = wholes << 1 | (whole ? 1u : 0u);
        if (!(ok = wait_free(vempty, j))) break;
        v_asked = j + 1;
        if (whole) fetch(&map_v, vt, vfull, j, page);
        else {
          copy(Vp, vt, j, page, pages_ok);
          pf_wait<1>();
          announce(kfull, j);
          pf_wait<0>();
          announce(vfull, j);
        }
      }
      pf_wait<0>();
      if (!ok && w == 0) {
        // giving up: what tensor copies have been asked for must land before the block's memory goes; the last of each stage may be on its way
        auto landed = [&](uint32_t bar, int asked) {
          for (int j = max(asked - STAGES, 0); j < asked; ++j) {
            const long long t0 = clock64();
            if ((wholes >> (k_asked - 1 - j)) & 1u)
              while (!tc::mbar_try(bar + 8 * (j % STAGES), (j / STAGES) & 1) && clock64() - t0 < tc::kWaitLimit) {}
          }
        };
        landed(kfull, k_asked);
        landed(vfull, v_asked);
      }
    } else {
      uint4 k[STEPS], v[STEPS];                                   // the next tile's codes, on their way
      uint32_t kb[FOUR ? STEPS : 1], vb[FOUR ? STEPS : 1];        // and their block scales
      float vs[FOLD ? STEPS : 1];                                 // and, of the values, their scales
      long long entry[FOUR ? STEPS : 1];                          // where the pieces lie, -1: nowhere
      auto locate = [&](int j, int page, uint32_t pages_ok) {
        if constexpr (FOUR) {
#pragma unroll
          for (int i = 0; i < STEPS; ++i) {
            const int key = key_of(i), of = __shfl_sync(0xffffffffu, page, key >> 3);
            entry[i] = j * KEYS + key < most && !(SC && j * KEYS + key < least) && ((pages_ok >> (key >> 3)) & 1u) ? (long long)b.entry(of, g_head, key0 + j * KEYS + key) : -1;
          }
        }
      };
      auto request = [&](const TC* pool, uint4 (&x)[STEPS], const uint8_t* blocks, uint32_t (&xb)[FOUR ? STEPS : 1], int j, int page, uint32_t pages_ok) {
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
          if constexpr (FOUR) {
            x[i] = make_uint4(0u, 0u, 0u, 0u);
            xb[i] = 0u;
            if (entry[i] >= 0) {
              x[i] = __ldg(reinterpret_cast<const uint4*>(pool + entry[i] * row_units<TC>(HD) + c * 16));
              xb[i] = __ldg(reinterpret_cast<const uint16_t*>(blocks + entry[i] * (HD / kBlock) + c * 2));
            }
          } else {
            const TC* src = source(pool, j, key_of(i), page, pages_ok);
            x[i] = src ? __ldg(reinterpret_cast<const uint4*>(src)) : make_uint4(0u, 0u, 0u, 0u);
          }
        }
      };
      auto request_scales = [&] {
        if constexpr (FOLD) {
#pragma unroll
          for (int i = 0; i < STEPS; ++i) vs[i] = entry[i] >= 0 ? __ldg(Vsc + entry[i]) : 0.f;
        }
      };
      // A key's pieces go to the two blocks of 64 elements, whose lines share their banks: lanes of the second block go over theirs in another order
      const bool other = HD == 128 && c >= PER_ROW / 2;
      auto convert = [&](const uint4 (&x)[STEPS], const uint32_t (&xb)[FOUR ? STEPS : 1], uint32_t dst, bool values) {
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
          const int key = key_of(i);
          if constexpr (FOUR) {                                   // 32 codes: two blocks
            uint32_t both = blocks_widen(xb[i]);
            if (FOLD && values) {
              const float2 b2 = e4m3_widen(xb[i]);
              const float f = vs[i] * (LIFT / ve);
              both = pack_f16(b2.x * f, b2.y * f);
            }
            const uint32_t u[2] = {__byte_perm(both, 0u, other ? 0x3232 : 0x1010), __byte_perm(both, 0u, other ? 0x1010 : 0x3232)};
            const uint32_t w[4] = {other ? x[i].z : x[i].x, other ? x[i].w : x[i].y, other ? x[i].x : x[i].z, other ? x[i].y : x[i].w};
#pragma unroll
            for (int n = 0; n < 4; ++n)
              sts16(dst + piece(key, 4 * c + (n ^ (other ? 2 : 0))), hmul2(e2m1_widen<0>(w[n]), u[n >> 1]), hmul2(e2m1_widen<1>(w[n]), u[n >> 1]), hmul2(e2m1_widen<2>(w[n]), u[n >> 1]),
                    hmul2(e2m1_widen<3>(w[n]), u[n >> 1]));
          } else {
            uint32_t o[8];
            to_bf16(other ? x[i].z : x[i].x, o[0], o[1], TC{});
            to_bf16(other ? x[i].w : x[i].y, o[2], o[3], TC{});
            to_bf16(other ? x[i].x : x[i].z, o[4], o[5], TC{});
            to_bf16(other ? x[i].y : x[i].w, o[6], o[7], TC{});
            sts16(dst + piece(key, 2 * c + (other ? 1 : 0)), o[0], o[1], o[2], o[3]);
            sts16(dst + piece(key, 2 * c + (other ? 0 : 1)), o[4], o[5], o[6], o[7]);
          }
        }
      };
      int page = page_next;
      uint32_t pages_ok = exists(0, page);
      float2 scales = ask_scales(0, page, pages_ok);
      float top = FOUR ? ask_values(0, page, pages_ok) : 0.f;
      locate(0, page, pages_ok);
      request(Kp, k, Kb, kb, 0, page, pages_ok);
      request(Vp, v, Vb, vb, 0, page, pages_ok);
      request_scales();
      page_next = look_up(1);
      for (int j = 0; j < n_tiles; ++j) {
        const uint32_t pages_next = exists(j + 1, page_next);
        if (!(ok = wait_free(kempty, j))) break;
        if constexpr (FOUR) raise(top);
        begin_side(j, scales, pages_ok);
        convert(k, kb, base + L::K + (j % STAGES) * L::TILE, false);
        announce(kfull, j);
        if (j + 1 < n_tiles) {
          scales = ask_scales(j + 1, page_next, pages_next);
          if constexpr (FOUR) top = ask_values(j + 1, page_next, pages_next);
          locate(j + 1, page_next, pages_next);
          request(Kp, k, Kb, kb, j + 1, page_next, pages_next);
        }
        if (!(ok = wait_free(vempty, j))) break;
        convert(v, vb, base + L::V + (j % STAGES) * L::TILE, true);
        announce(vfull, j);
        if (j + 1 < n_tiles) {
          request(Vp, v, Vb, vb, j + 1, page_next, pages_next);
          request_scales();
        }
        page = page_next;
        pages_ok = pages_next;
        page_next = look_up(j + 2);
      }
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(PRODUCT_REGS));
    if (warp < 14 && n_tiles > 0) {
      // ---- products: one warp per tile of rows, so that neither waits for the other's softmax
      constexpr uint32_t id_s = idesc(HALF, false, FOUR), id_o = idesc(HD, true, FOUR);
      const int t = warp - 12, tiles = uniform(n_tiles), halves = uniform(t ? n_keys[1] : n_keys[0]);
      const uint32_t tm = uniform(tmem), at = uniform(base), bar = uniform(bar0);
      auto wait = [&](uint32_t which, int phase) { return tc::mbar_wait(bar + (which - bar0), phase & 1, abort_flag, b.status); };
      if (elect()) {
        // each of these announces its completion, and that of everything before it, on the barrier named
        const uint64_t qa = tc::smem_desc(at + L::Q + t * L::TILE);
        auto product_s = [&](int i) {
          const int h = i & 1;
          const uint64_t ka = tc::smem_desc(at + L::K + ((i >> 1) % STAGES) * L::TILE + h * (HALF * 128));
#pragma unroll 1
          for (int part = 0; part < (PAIRS ? 2 : 1); ++part) {
#pragma unroll
            for (int k = 0; k < HD / 16; ++k) {                   // descriptors count 16-byte units
              const uint32_t off = ((k >> 2) * (128 * 128) + (k & 3) * 32) >> 4;
              mma_ss(tm + t * 128 + h * HALF, qa + part * (L::Q_LOW >> 4) + off, ka + off, id_s, k > 0 ? 1u : (uint32_t)part);
            }
          }
          tc::umma_commit(bar + (sfull - bar0) + 8 * (2 * t + h));
        };
        auto product_o = [&](int i) {
          const int h = i & 1;
          const uint64_t va = v_desc(at + L::V + ((i >> 1) % STAGES) * L::TILE + h * (HALF * 128), 128 * 128);
#pragma unroll 1
          for (int part = 0; part < (PAIRS ? 2 : 1); ++part) {
            const uint32_t first = (SUMS ? i & sum_mask : i) + part > 0;
#pragma unroll
            for (int k = 0; k < HALF / 16; ++k)
              mma_ts(tm + L::O_COL + t * HD, tm + t * 128 + h * HALF + part * (HALF / 2) + k * 8, va + k * (2048 >> 4), id_o, k > 0 ? 1u : first);
          }
          tc::umma_commit(bar + (odone - bar0) + 8 * t);
        };
        auto announce = [&](uint32_t which) { tc::umma_commit(bar + (which - bar0)); };
        // the scores of half i, i >= 2, in the columns of half i - 2.  Products with other accumulators are not ordered among each
        // other: its product with the values must have completed.
        auto next_s = [&](int i) {
          if (!wait(odone + 8 * t, i - 2)) return false;
          fence_after();
          product_s(i);
          return true;
        };
        auto next_o = [&](int i) {
          if (!wait(pready + 8 * (2 * t + (i & 1)), i >> 1)) return false;
          fence_after();
          product_o(i);
          return true;
        };
        bool ok = wait(qfull, 0) && wait(kfull, 0);
        if (ok) {
          fence_after();
          if (halves > 0) product_s(0);
          if (halves > 1) product_s(1);
          announce(kempty);
        }
        // every tile of keys is waited for and given back by both warps, also where this one's rows see no more: a warp that
        // gave stages back ahead of the loaders would stand in for the other
        for (int j = 0; j < tiles && ok; ++j) {
          ok = wait(vfull + 8 * (j % STAGES), j / STAGES);
          if (ok && 2 * j < halves) ok = next_o(2 * j);
          if (ok && j + 1 < tiles) {
            ok = wait(kfull + 8 * ((j + 1) % STAGES), (j + 1) / STAGES);
            if (ok && 2 * j + 2 < halves) ok = next_s(2 * j + 2);
          }
          if (ok && 2 * j + 1 < halves) ok = next_o(2 * j + 1);
          if (ok && !test_expire) announce(vempty + 8 * (j % STAGES));
          if (ok && 2 * j + 3 < halves) ok = next_s(2 * j + 3);
          if (ok && j + 1 < tiles) announce(kempty + 8 * ((j + 1) % STAGES));
        }
        if (!ok) {                                                // let what has been issued finish before the memory goes
          announce(drain + 8 * t);
          const long long t0 = clock64();
          while (!tc::mbar_try(drain + 8 * t, 0) && clock64() - t0 < tc::kWaitLimit) {}
        }
      }
      __syncwarp();
    }
  }
  fence_before();
  __syncthreads();
  if (warp == 12) {
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
  }
}

// Adds the shares of a row's splits, in split order.  grid (n_tokens, heads / 8): one warp per row, lane s holds split s's maximum and sum.
// A launch of its own (7..12 us), so that all SMs take part: joined by the last block of each unit, 64 tokens of 32 heads over 60 000
// positions in 16 splits took 158 us instead of 83.
// part_used: how many splits each row has, where its keys alone do not say so; else NULL.
template <int HD>
__global__ void __launch_bounds__(256)
paged_attn_join_kernel(const BatchView b, const Rows out, int group, int rows_from, int block_rows, int chunk, int splits, const float* __restrict__ part_acc,
                       const float* __restrict__ part_ml, const int* __restrict__ part_used) {
  int seq, pos;
  const int tok = blockIdx.x, where = locate_row(b, tok, seq, pos);
  if (where == ROW_PADDING) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, heads = group * b.n_kv_heads, head = blockIdx.y * 8 + warp;
  if (head >= heads) return;
  // the keys that the block of this row went over: those of its last row
  const int f0 = b.first[seq], f1 = b.first[seq + 1], n_new = min(f1 - f0, min(b.max_new, b.n_tokens - f0)), rows_all = n_new * group;
  if (rows_all < rows_from) return;
  const int row = (tok - f0) * group + head % group, last = (min((row / block_rows + 1) * block_rows, rows_all) - 1) / group;
  const int keys = (int)min(max((long long)b.len[seq] - (f1 - f0) + last + 1, 0ll), (long long)b.seq_len(seq));
  const int used = part_used ? min(part_used[(size_t)tok * heads + head], splits) : ap::splits_of(keys, chunk, splits);
  if (used <= 1) return;                                         // written by its block
  const size_t slot = ((size_t)tok * heads + head) * splits;
  const float2 ml = lane < used ? __ldg(reinterpret_cast<const float2*>(part_ml) + slot + lane) : make_float2(-INFINITY, 0.f);
  float top = ml.x;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  const float f = ml.x == -INFINITY ? 0.f : exp2f(ml.x - top);
  constexpr int PER = HD / 32;
  float sum = 0.f, x[PER] = {};
#pragma unroll 8
  for (int k = 0; k < used; ++k) {
    const float w = __shfl_sync(0xffffffffu, f, k);
    sum += w * __shfl_sync(0xffffffffu, ml.y, k);
    const float* src = part_acc + (slot + k) * HD + lane * PER;
    if constexpr (PER == 4) {
      const float4 a = __ldg(reinterpret_cast<const float4*>(src));
      x[0] += w * a.x; x[1] += w * a.y; x[2] += w * a.z; x[3] += w * a.w;
    } else {
      const float2 a = __ldg(reinterpret_cast<const float2*>(src));
      x[0] += w * a.x; x[1] += w * a.y;
    }
  }
#pragma unroll
  for (int k = 0; k < PER; ++k) store_elem(out, (long long)tok * out.row_stride + head * out.head_stride + lane * PER + k, normalised(x[k], sum));
}

}  // namespace sd
