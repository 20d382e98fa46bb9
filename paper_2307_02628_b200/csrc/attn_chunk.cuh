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
// Operands are bf16, the type of a bf16 cache; codes of 8-bit caches are bf16 numbers exactly.  Where queries and results are bf16 too, the only
// rounding is that of the weights, once to 8 bits of significand: relative to 64-bit arithmetic results are 2.3e-3 off, of which their own
// rounding is 1.7e-3.  Queries or results with more bits (fp32, fp16) take the form PAIRS: queries and weights are sums of two
// bf16, 16 bits, in two products each; the weights' lower halves take the other 32 columns of their scores.  Twice the
// products, and at HD = 128 one tile of rows instead of two: 4 chunks of 512 tokens at 2048, 32 heads of 128, bf16: 230 us from and to fp16, 90
// from and to bf16; 2 x 1024 tokens, 32 heads of 64: 66 and 37.  fp32 results go to the kernel for few rows.  A key's scale
// (8-bit caches) multiplies its score in the softmax, a value's scale its weight, before the rounding.
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
  static constexpr int O_COL = 256;                            // tensor memory: S_0 at 0 and 64, S_1 at 128 and 192, O_0, O_1 from 256
};

// bf16 x bf16 -> fp32, 128 rows; b_mn: B is stored with its output axis contiguous
__host__ __device__ constexpr uint32_t idesc(int n, bool b_mn) {
  return (1u << 4) | (1u << 7) | (1u << 10) | (b_mn ? 1u << 16 : 0u) | ((uint32_t)(n >> 3) << 17) | (8u << 24);
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

}  // namespace ac

// grid (blocks_per_seq * n_kv_heads * n_seqs, splits).  Sequences with fewer than rows_from query rows are another kernel's.  Split z takes
// keys [z * chunk, (z + 1) * chunk), the last one all that follow; several leave partial results (accumulator, maximum, sum) of their rows
// to paged_attn_join_kernel.
// map_k, map_v: the pools as [n_pages * n_kv_heads][page_len][HD] with boxes of a page by 64 elements (bf16 only; use_maps 0: not made).
// PAIRS: queries and weights enter as sums of two bf16.
// test_expire: test hook, values are never given back and the loaders give up after about a millisecond, keys of the third tile on their way.
template <typename TC, int HD, bool PAIRS>
__global__ void __launch_bounds__(ac::THREADS, 1)
paged_attn_chunk_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, int use_maps,
                        const BatchView b, const Rows q, const Rows out, const TC* __restrict__ Kp, const TC* __restrict__ Vp,
                        const float* __restrict__ Ksc, const float* __restrict__ Vsc, int group, float scale_log2, bool q_vec, bool out_vec,
                        int blocks_per_seq, int rows_from, int chunk, float* part_acc, float* part_ml, int test_expire) {
  using namespace ac;
  using L = Layout<HD, PAIRS>;
  constexpr bool SCALED = CacheType<TC>::TOP > 0.f;
  constexpr int ROWS = L::ROWS;
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
  __shared__ int turn_seq;
  if (b.n_seqs > 1 && b.n_seqs <= THREADS) {
    const int mine = threadIdx.x < b.n_seqs ? b.len[threadIdx.x] : 0;
    lens[threadIdx.x] = mine;
    __syncthreads();
    if (threadIdx.x < b.n_seqs) {
      int ahead = 0;
      for (int i = 0; i < b.n_seqs; ++i) ahead += lens[i] > mine || (lens[i] == mine && i < (int)threadIdx.x);
      if (ahead == turn) turn_seq = threadIdx.x;
    }
    __syncthreads();
  }
  const int seq = b.n_seqs > 1 && b.n_seqs <= THREADS ? turn_seq : turn;
  const int f0 = b.first[seq], f1 = b.first[seq + 1], len = b.seq_len(seq);
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
  const long long pos_first = (long long)b.len[seq] - (f1 - f0);
  const int splits = gridDim.y, z = blockIdx.y, key0 = z * chunk;  // key numbers below count from key0
  int n_keys[2], n_rows[2], used_splits = 1;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    n_rows[t] = t < L::TILES ? max(0, min(TILE_ROWS, rows_all - row0 - t * TILE_ROWS)) : 0;
    const int last = (row0 + t * TILE_ROWS + n_rows[t] - 1) / group;
    int keys = n_rows[t] ? (int)min(max(pos_first + last + 1, 0ll), (long long)len) : 0;
    if (splits > 1) {
      used_splits = max(used_splits, ap::splits_of(keys, chunk, splits));
      keys = max(keys - key0, 0);
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
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = tmem_slot;

  if (warp < 8) {
    // ---- softmax: one thread per query row
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(SOFTMAX_REGS));
    const int t = warp >> 2, r = (warp & 3) * 32 + lane;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t s_addr = tmem + lanes + t * 128, o_addr = tmem + lanes + L::O_COL + t * HD;
    const int row = row0 + t * TILE_ROWS + min(r, max(n_rows[t] - 1, 0));
    const int token = row / group, head = g_head * group + row % group;
    const int row_last = (int)max(min(pos_first + token, (long long)len - 1), -1ll) - key0; // last key this row sees
    const float scale = fabsf(scale_log2), sign = scale_log2 < 0.f ? -1.f : 1.f;            // a negative scale turns the queries round
    if (n_rows[t] > 0) {
      const long long at = (long long)(f0 + token) * q.row_stride + head * q.head_stride;
      const uint32_t dst = base + L::Q + t * L::TILE;
      if constexpr (PAIRS) {
#pragma unroll 4
        for (int c = 0; c < HD / 8; ++c) {
          float x[8];
          uint32_t hi[4], lo[4];
          ap::load_run<8>(q, at + c * 8, q_vec, x);
#pragma unroll
          for (int i = 0; i < 4; ++i) ap::split(x[2 * i] * sign, x[2 * i + 1] * sign, hi[i], lo[i], __nv_bfloat16{});
          sts16(dst + piece(r, c), hi[0], hi[1], hi[2], hi[3]);
          sts16(dst + L::Q_LOW + piece(r, c), lo[0], lo[1], lo[2], lo[3]);
        }
      } else if (q_vec && q.dtype == DT_BF16) {
        const uint4* src = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(q.data) + at);
        const uint32_t turn = scale_log2 < 0.f ? 0x80008000u : 0u;
        uint4 x[HD / 8];                                          // all on their way together
#pragma unroll
        for (int c = 0; c < HD / 8; ++c) x[c] = __ldg(src + c);
#pragma unroll
        for (int c = 0; c < HD / 8; ++c) sts16(dst + piece(r, c), x[c].x ^ turn, x[c].y ^ turn, x[c].z ^ turn, x[c].w ^ turn);
      } else {
#pragma unroll 8
        for (int c = 0; c < HD / 8; ++c) {
          float x[8];
          ap::load_run<8>(q, at + c * 8, q_vec, x);
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] *= sign;
          sts16(dst + piece(r, c), pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
        }
      }
    }
    fence_async();
    __syncwarp();
    if (lane == 0) arrive(qfull);

    // the keys that all 32 rows of the warp see: tiles below need no mask
    const int first_token = (row0 + t * TILE_ROWS + min((warp & 3) * 32, max(n_rows[t] - 1, 0))) / group;
    const int all_see = (int)max(min(pos_first + first_token, (long long)len - 1), -1ll) - key0;
    float m = -INFINITY, l = 0.f;                                // m in the units of the scores (bf16) or base-2 (8 bits)
    const float unit = SCALED ? 1.f : scale;                     // base-2 units per unit of m
    bool ok = true;
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
      side += h * HALF;
      const uint32_t s_half = s_addr + h * HALF;

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
      if (i * HALF + HALF - 1 > all_see || pages_ok != 0xffu) {
        const int left = row_last - i * HALF;                    // columns up to here are seen
#pragma unroll
        for (int c = 0; c < HALF; ++c)
          if (c > left || !((pages_ok >> (c >> 3)) & 1u)) s[c >> 5][c & 31] = 0xff800000u;
      }
      float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
      for (int k = 0; k < 16; k += 2)
#pragma unroll
        for (int c = 0; c < 4; ++c) mx[c] = fmaxf(mx[c], fmaxf(__uint_as_float(s[c >> 1][(c & 1) * 16 + k]), __uint_as_float(s[c >> 1][(c & 1) * 16 + k + 1])));
      const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
      if (__any_sync(0xffffffffu, (top - m) * unit > SLACK)) {   // -inf - -inf is NaN: not greater
        const float m_new = fmaxf(m, top), a = m == -INFINITY ? 0.f : ex2((m - m_new) * unit);
        m = m_new;
        l *= a;
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
      const float mb = m == -INFINITY ? 0.f : -m * unit;
      const F2 unit2 = f2(unit, unit), mb2 = f2(mb, mb);
      F2 sum[2] = {f2(0.f, 0.f), f2(0.f, 0.f)};
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        uint32_t w[16], w_lo[16];
#pragma unroll
        for (int k = 0; k < 16; ++k) {
          F2 x = f2(__uint_as_float(s[c][2 * k]), __uint_as_float(s[c][2 * k + 1]));
          x = SCALED ? add2(x, mb2) : fma2(x, unit2, mb2);
          float p0, p1;
          un2(x, p0, p1);
          p0 = ex2(p0);
          p1 = ex2(p1);
          x = f2(p0, p1);
          sum[k & 1] = add2(sum[k & 1], x);
          if (SCALED) {
            const float2 v = *reinterpret_cast<const float2*>(side + KEYS + c * 32 + 2 * k);
            un2(mul2(x, f2(v.x, v.y)), p0, p1);
          }
          if constexpr (PAIRS) ap::split(p0, p1, w[k], w_lo[k], __nv_bfloat16{});
          else w[k] = pack_bf16(p0, p1);
        }
        tmem_st16(s_half + 16 * c, w);                           // over columns that have been read
        if constexpr (PAIRS) tmem_st16(s_half + HALF / 2 + 16 * c, w_lo);
      }
      float a0, a1;
      un2(add2(sum[0], sum[1]), a0, a1);
      l += a0 + a1;
      tmem_wait_st();
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
    if (n_rows[t] > 0 && ok) {
      if (n_keys[t] > 0) {
        ok = __all_sync(0xffffffffu, tc::mbar_wait(odone + 8 * t, (n_keys[t] - 1) & 1, abort_flag, b.status));
        fence_after();
      }
      if (ok && used_splits == 1) {
        const float inv = l > 0.f ? 1.f / l : 0.f;
        const long long at = (long long)(f0 + token) * out.row_stride + head * out.head_stride;
#pragma unroll 1
        for (int c0 = 0; c0 < HD; c0 += 32) {
          uint32_t v[32];
          if (n_keys[t] > 0) {
            tc::tmem_ld32(o_addr + c0, v);
            tmem_wait_ld();
          }
          if (r < n_rows[t]) {
#pragma unroll
            for (int i = 0; i < 32; i += 8) {
              float x[8];
#pragma unroll
              for (int k = 0; k < 8; ++k) x[k] = l > 0.f ? __uint_as_float(v[i + k]) * inv : (l == 0.f ? 0.f : l);   // l NaN: NaN
              const long long e = at + c0 + i;
              if (out_vec && out.dtype == DT_BF16) store8<true>(static_cast<__nv_bfloat16*>(out.data) + e, x);
              else if (out_vec && out.dtype == DT_FP16) store8<true>(static_cast<__half*>(out.data) + e, x);
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
#pragma unroll 1
        for (int c0 = 0; c0 < HD; c0 += 32) {
          uint32_t v[32] = {};
          if (n_keys[t] > 0) {
            tc::tmem_ld32(o_addr + c0, v);
            tmem_wait_ld();
          }
          if (r < n_rows[t]) {
#pragma unroll
            for (int i = 0; i < 32; i += 4)
              __stcg(reinterpret_cast<float4*>(part_acc + slot * HD + c0 + i), make_float4(__uint_as_float(v[i]), __uint_as_float(v[i + 1]), __uint_as_float(v[i + 2]), __uint_as_float(v[i + 3])));
          }
        }
        if (r < n_rows[t]) __stcg(reinterpret_cast<float2*>(part_ml + slot * 2), make_float2(m * unit, l));
      }
    }
  } else if (warp < 12) {
    // ---- loaders
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(LOADER_REGS));
    const int w = warp - 8, tid = w * 32 + lane;
    const int* table = b.pages + (size_t)seq * b.pages_per_seq;
    constexpr int E = sizeof(TC), PER_ROW = HD * E / 16;          // 16-byte pieces of a stored key
    constexpr int ROWS_AT_ONCE = 32 / PER_ROW;                    // of a warp
    constexpr int STEPS = KEYS / (4 * ROWS_AT_ONCE);
    const int most = min(len - key0, n_tiles * KEYS);             // keys past it are filled with zeros
    // lane i < 16 looks up the page of keys [8 i, 8 i + 8) of a tile
    auto look_up = [&](int j) {
      const int key = j * KEYS + (lane & 15) * 8;
      return j < n_tiles && key < most ? table[(key0 + key) >> b.page_shift] : 0;
    };
    auto exists = [&](int j, int page) {
      return __ballot_sync(0xffffffffu, (unsigned)page < (unsigned)b.n_pages || j * KEYS + (lane & 15) * 8 >= most) & 0xffffu;
    };
    // this thread's piece in step i: row `key`, piece c
    auto key_of = [&](int i) { return (i * 4 + w) * ROWS_AT_ONCE + lane / PER_ROW; };
    const int c = lane % PER_ROW;
    auto source = [&](const TC* pool, int j, int key, int page, uint32_t pages_ok) -> const TC* {
      page = __shfl_sync(0xffffffffu, page, key >> 3);
      const bool on = j * KEYS + key < most && ((pages_ok >> (key >> 3)) & 1u);
      return on ? pool + b.entry(page, g_head, key0 + j * KEYS + key) * HD + c * (16 / E) : nullptr;
    };
    // this thread's key's scales, zeros where there is none
    auto ask_scales = [&](int j, int page, uint32_t pages_ok) {
      page = __shfl_sync(0xffffffffu, page, (tid >> 3) & 15);
      if (!(j * KEYS + tid < most && ((pages_ok >> (tid >> 3)) & 1u))) return make_float2(0.f, 0.f);
      const size_t e = b.entry(page, g_head, key0 + j * KEYS + tid);
      return make_float2(__ldg(Ksc + e), __ldg(Vsc + e));
    };
    auto begin_side = [&](int j, float2 scales, uint32_t pages_ok) {
      float* side = reinterpret_cast<float*>(base_ptr + L::SIDE_OFF + (j & (SIDE - 1)) * L::SIDE_BYTES);
      if (tid == 0) *reinterpret_cast<uint32_t*>(side + 2 * KEYS) = pages_ok;
      if (pages_ok != 0xffffu && w == 0 && lane == 0) b.bad();
      if (SCALED) {
        side[tid] = scales.x * fabsf(scale_log2);
        side[KEYS + tid] = scales.y;
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
    int page_next = look_up(0);
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
        const bool whole = use_maps && (j + 1) * KEYS <= most && pages_ok == 0xffffu;
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
      auto request = [&](const TC* pool, uint4 (&x)[STEPS], int j, int page, uint32_t pages_ok) {
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
          const TC* src = source(pool, j, key_of(i), page, pages_ok);
          x[i] = src ? __ldg(reinterpret_cast<const uint4*>(src)) : make_uint4(0u, 0u, 0u, 0u);
        }
      };
      auto convert = [&](const uint4 (&x)[STEPS], uint32_t dst) {
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
          const int key = key_of(i);
          uint32_t o[8];
          to_bf16(x[i].x, o[0], o[1], TC{});
          to_bf16(x[i].y, o[2], o[3], TC{});
          to_bf16(x[i].z, o[4], o[5], TC{});
          to_bf16(x[i].w, o[6], o[7], TC{});
          sts16(dst + piece(key, 2 * c), o[0], o[1], o[2], o[3]);
          sts16(dst + piece(key, 2 * c + 1), o[4], o[5], o[6], o[7]);
        }
      };
      int page = page_next;
      uint32_t pages_ok = exists(0, page);
      float2 scales = ask_scales(0, page, pages_ok);
      request(Kp, k, 0, page, pages_ok);
      request(Vp, v, 0, page, pages_ok);
      page_next = look_up(1);
      for (int j = 0; j < n_tiles; ++j) {
        const uint32_t pages_next = exists(j + 1, page_next);
        if (!(ok = wait_free(kempty, j))) break;
        begin_side(j, scales, pages_ok);
        convert(k, base + L::K + (j % STAGES) * L::TILE);
        announce(kfull, j);
        if (j + 1 < n_tiles) {
          scales = ask_scales(j + 1, page_next, pages_next);
          request(Kp, k, j + 1, page_next, pages_next);
        }
        if (!(ok = wait_free(vempty, j))) break;
        convert(v, base + L::V + (j % STAGES) * L::TILE);
        announce(vfull, j);
        if (j + 1 < n_tiles) request(Vp, v, j + 1, page_next, pages_next);
        page = page_next;
        pages_ok = pages_next;
        page_next = look_up(j + 2);
      }
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(PRODUCT_REGS));
    if (warp < 14 && n_tiles > 0) {
      // ---- products: one warp per tile of rows, so that neither waits for the other's softmax
      constexpr uint32_t id_s = idesc(HALF, false), id_o = idesc(HD, true);
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
            const uint32_t first = i + part > 0;
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
template <int HD>
__global__ void __launch_bounds__(256)
paged_attn_join_kernel(const BatchView b, const Rows out, int group, int rows_from, int block_rows, int chunk, int splits, const float* __restrict__ part_acc,
                       const float* __restrict__ part_ml) {
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
  const int used = ap::splits_of(keys, chunk, splits);
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
