// Paged KV cache: storing new tokens' keys and values (fp32, bf16, or 8 bits with a scale per token and head), reading
// them back, and the attention of one row at a time over it.  A pool is [n_pages, n_kv_heads, page_len, head_dim];
// position p of sequence s is slot p % page_len of page pages[s * pages_per_seq + p / page_len].
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "kernels.cuh"

namespace sd {

enum : int { STATUS_BAD_BATCH = 16, STATUS_BAD_SETTING = 32, STATUS_NOT_FINITE = 64 };

struct e4m3 { uint8_t bits; };

// TOP: largest code of the 8-bit types, 0 for the others.  MOST: largest finite value of the others.
template <typename T> struct CacheType;
template <> struct CacheType<float> { static constexpr float TOP = 0.f, MOST = 3.402823466e38f; };
template <> struct CacheType<__nv_bfloat16> { static constexpr float TOP = 0.f, MOST = 3.389531390e38f; };   // (2 - 2^-7) 2^127
template <> struct CacheType<int8_t> { static constexpr float TOP = 127.f, MOST = 0.f; };
template <> struct CacheType<e4m3> { static constexpr float TOP = 448.f, MOST = 0.f; };

// A batch as the kernels see it: the caller's device arrays and the bounds that every index is held to.
struct BatchView {
  const int *pages, *first, *len;
  int n_seqs, pages_per_seq, n_tokens, max_new;
  int n_pages, page_len, page_shift, n_kv_heads;
  int* status;

  __host__ __device__ __forceinline__ void bad() const {
#ifdef __CUDA_ARCH__
    atomicOr(status, STATUS_BAD_BATCH);
#else
    *status |= STATUS_BAD_BATCH;              // the index arithmetic is tested on the host
#endif
  }
  // Positions a sequence can have: len, held to the table.
  __host__ __device__ __forceinline__ int seq_len(int s) const {
    const int l = len[s];
    const long long most = (long long)pages_per_seq << page_shift;
    if (l > most) { bad(); return (int)most; }
    return l > 0 ? l : 0;
  }
  // The page that holds position pos (0 <= pos < the table's reach), or -1 when the table's entry is no page.
  __host__ __device__ __forceinline__ int page_of(int s, int pos) const {
    const int pg = pages[(size_t)s * pages_per_seq + (pos >> page_shift)];
    if ((unsigned)pg < (unsigned)n_pages) return pg;
    bad();
    return -1;
  }
  // Entry (not element) of position pos for key head g inside the pool: 64-bit, a pool may have more than 2^32 elements.
  __host__ __device__ __forceinline__ size_t entry(int page, int g, int pos) const {
    return (((size_t)page * n_kv_heads + g) << page_shift) + (pos & (page_len - 1));
  }
};

enum : int { ROW_PADDING = 0, ROW_NOWHERE = 1, ROW_OK = 2 };

// Which sequence row r belongs to and where it sits; called by all threads of a block.  The rows' owner is found by counting
// how many of first[0..n_seqs] are at most r, one parallel pass instead of a chain of dependent loads.
__device__ __forceinline__ int locate_row(const BatchView& b, int r, int& seq, int& pos) {
  int cnt = 0;
  for (int i0 = 0; i0 <= b.n_seqs; i0 += blockDim.x) {
    const int i = i0 + threadIdx.x;
    cnt += __syncthreads_count(i <= b.n_seqs && b.first[i] <= r);
  }
  seq = cnt - 1;
  pos = -1;
  if (seq < 0 || seq >= b.n_seqs) return ROW_PADDING;
  const int f0 = b.first[seq], f1 = b.first[seq + 1];
  if (f0 < 0 || f0 > r || r >= f1 || r - f0 >= b.max_new) { if (threadIdx.x == 0) b.bad(); return ROW_PADDING; }
  if (threadIdx.x == 0 && b.first[b.n_seqs] > b.n_tokens) b.bad();
  const long long p = (long long)b.len[seq] - f1 + r;
  if (p < 0) return ROW_NOWHERE;
  if (p >= (long long)b.pages_per_seq << b.page_shift) { if (threadIdx.x == 0) b.bad(); return ROW_NOWHERE; }
  pos = (int)p;
  return ROW_OK;
}

// Rows handed in by the caller: [n_tokens, heads, head_dim] with strides in elements.
struct Rows {
  void* data;
  long long row_stride, head_stride;
  int dtype;
};
enum : int { DT_FP32 = 0, DT_BF16 = 1, DT_FP16 = 2 };

// Eight elements in and out.  VEC: 16-byte accesses (the host has checked base and strides).
template <bool VEC> __device__ __forceinline__ void load8(const float* p, float (&o)[8]) {
  if (VEC) {
    const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
    o[0] = a.x; o[1] = a.y; o[2] = a.z; o[3] = a.w; o[4] = b.x; o[5] = b.y; o[6] = b.z; o[7] = b.w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = p[i];
  }
}
template <bool VEC> __device__ __forceinline__ void load8(const __nv_bfloat16* p, float (&o)[8]) {
  if (VEC) Vec16<__nv_bfloat16>::load(p, o);
  else {
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = __bfloat162float(p[i]);
  }
}
template <bool VEC> __device__ __forceinline__ void load8(const __half* p, float (&o)[8]) {
  if (VEC) {
    const uint4 v = __ldg(reinterpret_cast<const uint4*>(p));
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
      o[2 * i] = f.x; o[2 * i + 1] = f.y;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = __half2float(p[i]);
  }
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
  const __half2 v = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}
template <bool VEC> __device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
  if (VEC) {
    reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = v[i];
  }
}
template <bool VEC> __device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&v)[8]) {
  if (VEC) *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
  else {
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = __float2bfloat16_rn(v[i]);
  }
}
// NaN stays NaN: the comparisons of fminf and fmaxf would drop it
__device__ __forceinline__ float sat_f16_nan(float v) { return v != v ? v : sat_f16(v); }
template <bool VEC> __device__ __forceinline__ void store8(__half* p, const float (&v)[8]) {
  float w[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = sat_f16_nan(v[i]);
  if (VEC) *reinterpret_cast<uint4*>(p) = make_uint4(pack_f16(w[0], w[1]), pack_f16(w[2], w[3]), pack_f16(w[4], w[5]), pack_f16(w[6], w[7]));
  else {
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = __float2half_rn(w[i]);
  }
}
__device__ __forceinline__ float load_elem(const Rows& t, long long i) {
  if (t.dtype == DT_FP32) return static_cast<const float*>(t.data)[i];
  if (t.dtype == DT_BF16) return __bfloat162float(static_cast<const __nv_bfloat16*>(t.data)[i]);
  return __half2float(static_cast<const __half*>(t.data)[i]);
}
__device__ __forceinline__ void store_elem(const Rows& t, long long i, float v) {
  if (t.dtype == DT_FP32) static_cast<float*>(t.data)[i] = v;
  else if (t.dtype == DT_BF16) static_cast<__nv_bfloat16*>(t.data)[i] = __float2bfloat16_rn(v);
  else static_cast<__half*>(t.data)[i] = __float2half_rn(sat_f16_nan(v));
}

// ---- codes ------------------------------------------------------------------------------------

__device__ __forceinline__ uint32_t e4m3_pair(float lo, float hi) {
  return (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ float2 e4m3_widen(uint32_t pair) {          // exact: every e4m3 is an fp16
  const __half2_raw r = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)pair, __NV_E4M3);
  return __half22float2(*reinterpret_cast<const __half2*>(&r));
}

// The code nearest to x / s, ties to even, for one element whose fast quotient is too close to a border (or s to the
// smallest floats) to decide.  The quotient of two 24-bit numbers is either a border or at least 2^-25 (relative) away from
// it, so the 53-bit quotient decides exactly; on the way to e4m3 it passes through a float that is rounded to odd, which
// keeps a later rounding to fewer bits correct.
__device__ __noinline__ float quotient_int8(float x, float s) { return (float)fmin(fmax(rint((double)x / (double)s), -127.0), 127.0); }
__device__ __noinline__ float quotient_sticky(float x, float s) {
  const double q = (double)x / (double)s;
  const float f = __double2float_rz(q);
  return (double)f == q ? f : __uint_as_float(__float_as_uint(f) | 1u);
}

// Eight codes of x / s.  inv = 1 / s, or 0 to send every element through the exact route.  The fast quotient x * inv is off
// by less than 2^-22 of itself.
__device__ __forceinline__ uint2 encode8(const float (&x)[8], float s, float inv, int8_t) {
  uint32_t w[2] = {0u, 0u};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float c;
    if (x[i] != x[i] || s == 0.f) c = 0.f;
    else {
      const float y = fminf(fmaxf(x[i] * inv, -127.f), 127.f);
      c = rintf(y);
      if (fabsf(y - c) > 0.4999f || inv == 0.f) c = quotient_int8(x[i], s);      // 127 * 2^-22 = 3e-5 < 1e-4
    }
    w[i >> 2] |= ((uint32_t)(int)c & 0xffu) << (8 * (i & 3));
  }
  return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ uint2 encode8(const float (&x)[8], float s, float inv, e4m3) {
  uint32_t w[2] = {0u, 0u};
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    float y[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) y[j] = (x[i + j] != x[i + j] || s == 0.f) ? 0.f : x[i + j] * inv;
    constexpr float UP = 1.f + 4.f / 16777216.f, DOWN = 1.f - 4.f / 16777216.f;        // 1 +- 2^-22
    uint32_t c = e4m3_pair(y[0] * DOWN, y[1] * DOWN);
    if (c != e4m3_pair(y[0] * UP, y[1] * UP) || inv == 0.f) {
#pragma unroll
      for (int j = 0; j < 2; ++j) y[j] = (x[i + j] != x[i + j] || s == 0.f) ? 0.f : quotient_sticky(x[i + j], s);
      c = e4m3_pair(y[0], y[1]);
    }
    w[i >> 2] |= c << (16 * ((i >> 1) & 1));
  }
  return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ void decode8(uint2 v, float s, float (&o)[8], int8_t) {
  const uint32_t w[2] = {v.x, v.y};
#pragma unroll
  for (int i = 0; i < 8; ++i) o[i] = (float)(int)(int8_t)(w[i >> 2] >> (8 * (i & 3))) * s;
}
__device__ __forceinline__ void decode8(uint2 v, float s, float (&o)[8], e4m3) {
  const uint32_t w[4] = {v.x & 0xffffu, v.x >> 16, v.y & 0xffffu, v.y >> 16};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = e4m3_widen(w[i]);
    o[2 * i] = f.x * s; o[2 * i + 1] = f.y * s;
  }
}

// ---- append -----------------------------------------------------------------------------------
// One block per row.  A group of HD / 8 lanes owns one (head, K or V) of it: each lane holds eight elements, the largest
// magnitude goes round the group by shuffles, and the codes leave as one 8-byte store per lane (16 or 32 bytes in bf16 or
// fp32).  The bytes are read once and written once; there is no other work to speak of.
template <typename TS, typename TC, int HD, bool VEC>
__global__ void __launch_bounds__(256)
cache_append_kernel(const BatchView b, const Rows ks, const Rows vs, TC* __restrict__ Kp, TC* __restrict__ Vp,
                    float* __restrict__ Ksc, float* __restrict__ Vsc) {
  constexpr int LANES = HD / 8;
  int seq, pos;
  if (locate_row(b, blockIdx.x, seq, pos) != ROW_OK) return;
  const int page = b.page_of(seq, pos);
  if (page < 0) return;
  const int total = 2 * b.n_kv_heads * LANES;
  for (int i0 = 0; i0 < total; i0 += blockDim.x) {              // uniform: the shuffles need whole warps
    const int i = i0 + threadIdx.x;
    const bool on = i < total;
    const int unit = on ? i / LANES : 0, sub = i % LANES;
    const bool is_v = unit >= b.n_kv_heads;
    const int g = is_v ? unit - b.n_kv_heads : unit;
    const Rows& src = is_v ? vs : ks;
    float x[8];
    load8<VEC>(static_cast<const TS*>(src.data) + (long long)blockIdx.x * src.row_stride + g * src.head_stride + sub * 8, x);
    const size_t e = b.entry(page, g, pos);
    TC* dst = (is_v ? Vp : Kp) + e * HD + sub * 8;
    float top = 0.f;                                             // of the finite elements
    bool finite = true;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float a = fabsf(x[j]);
      if (a < INFINITY) top = fmaxf(top, a);
      else finite = false;                                       // NaN too
    }
    if (!finite && on) atomicOr(b.status, STATUS_NOT_FINITE);
    if constexpr (CacheType<TC>::TOP > 0.f) {
#pragma unroll
      for (int o = LANES / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      const float s = __fdiv_rn(top, CacheType<TC>::TOP);
      const float inv = s > 1e-30f ? __fdiv_rn(1.f, s) : 0.f;
      if (on) {
        *reinterpret_cast<uint2*>(dst) = encode8(x, s, inv, TC{});
        if (sub == 0) (is_v ? Vsc : Ksc)[e] = s;
      }
    } else if (on) {
      constexpr float MOST = CacheType<TC>::MOST;
      if (!finite || top > MOST) {                               // in bf16 the last half step below 2^128 would round to infinity
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = x[j] != x[j] ? 0.f : fminf(fmaxf(x[j], -MOST), MOST);
      }
      store8<true>(dst, x);                                      // pools are 256-byte aligned, rows multiples of 64 bytes
    }
  }
}

// ---- read -------------------------------------------------------------------------------------
// The same walk the other way.  A row without a place reads as zeros.
template <typename TO, typename TC, int HD, bool VEC>
__global__ void __launch_bounds__(256)
cache_read_kernel(const BatchView b, const Rows ko, const Rows vo, const TC* __restrict__ Kp, const TC* __restrict__ Vp,
                  const float* __restrict__ Ksc, const float* __restrict__ Vsc) {
  constexpr int LANES = HD / 8;
  int seq, pos;
  const int where = locate_row(b, blockIdx.x, seq, pos);
  if (where == ROW_PADDING) return;
  const int page = where == ROW_OK ? b.page_of(seq, pos) : -1;
  const int total = 2 * b.n_kv_heads * LANES;
  for (int i = threadIdx.x; i < total; i += blockDim.x) {
    const int unit = i / LANES, sub = i % LANES;
    const bool is_v = unit >= b.n_kv_heads;
    const int g = is_v ? unit - b.n_kv_heads : unit;
    float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (page >= 0) {
      const size_t e = b.entry(page, g, pos);
      const TC* src = (is_v ? Vp : Kp) + e * HD + sub * 8;
      if constexpr (CacheType<TC>::TOP > 0.f) decode8(*reinterpret_cast<const uint2*>(src), (is_v ? Vsc : Ksc)[e], x, TC{});
      else load8<true>(src, x);
    }
    const Rows& dst = is_v ? vo : ko;
    store8<VEC>(static_cast<TO*>(dst.data) + (long long)blockIdx.x * dst.row_stride + g * dst.head_stride + sub * 8, x);
  }
}

// ---- attention, one row and head per block ------------------------------------------------------
// Any cache type, on the CUDA cores in fp32: the kernel for caches in fp32, whose products the tensor cores would round.
// A group of HD / 8 lanes owns a key at a time (eight elements per lane); every group runs its own base-2 online softmax,
// merged by shuffles inside a warp and through shared memory across warps.
template <typename TC, int HD>
__global__ void __launch_bounds__(128)
paged_attn_row_kernel(const BatchView b, const Rows q, const Rows out, const TC* __restrict__ Kp, const TC* __restrict__ Vp,
                      const float* __restrict__ Ksc, const float* __restrict__ Vsc, int group, float scale_log2) {
  constexpr int LANES = HD / 8, GROUPS = 128 / LANES, NW = 4;
  __shared__ float sm_acc[NW][HD], sm_m[NW], sm_l[NW];
  const int r = blockIdx.x, h = blockIdx.y, g = h / group;
  int seq, pos;
  const int where = locate_row(b, r, seq, pos);
  if (where == ROW_PADDING) return;
  const int n_keys = where == ROW_OK ? pos + 1 : 0;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = threadIdx.x % LANES, grp = threadIdx.x / LANES;
  float qv[8], acc[8], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    qv[j] = load_elem(q, (long long)r * q.row_stride + h * q.head_stride + sub * 8 + j) * scale_log2;
    acc[j] = 0.f;
  }
  for (int j0 = 0; j0 < n_keys; j0 += GROUPS) {                  // uniform bound: the shuffles need whole warps
    const int j = j0 + grp;
    float k[8], v[8];
    const int page = j < n_keys ? b.page_of(seq, j) : -1;
    float s = 0.f;
    if (page >= 0) {
      const size_t e = b.entry(page, g, j);
      if constexpr (CacheType<TC>::TOP > 0.f) {
        decode8(*reinterpret_cast<const uint2*>(Kp + e * HD + sub * 8), Ksc[e], k, TC{});
        decode8(*reinterpret_cast<const uint2*>(Vp + e * HD + sub * 8), Vsc[e], v, TC{});
      } else {
        load8<true>(Kp + e * HD + sub * 8, k);
        load8<true>(Vp + e * HD + sub * 8, v);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) s = fmaf(qv[i], k[i], s);
    }
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (page >= 0) {
      const float mx = fmaxf(m, s);
      const float a = exp2_safe(m, mx), p = exp2f(s - mx);
      l = l * a + p;
#pragma unroll
      for (int i = 0; i < 8; ++i) acc[i] = acc[i] * a + p * v[i];
      m = mx;
    }
  }
#pragma unroll
  for (int o = LANES; o < 32; o <<= 1) {
    const float m2 = __shfl_xor_sync(0xffffffffu, m, o), l2 = __shfl_xor_sync(0xffffffffu, l, o);
    const float mx = fmaxf(m, m2), a = exp2_safe(m, mx), c = exp2_safe(m2, mx);
    l = l * a + l2 * c;
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] = acc[i] * a + __shfl_xor_sync(0xffffffffu, acc[i], o) * c;
    m = mx;
  }
  if (lane < LANES) {
#pragma unroll
    for (int i = 0; i < 8; ++i) sm_acc[warp][sub * 8 + i] = acc[i];
    if (sub == 0) { sm_m[warp] = m; sm_l[warp] = l; }
  }
  __syncthreads();
  float M = -INFINITY, L = 0.f;
#pragma unroll
  for (int w = 0; w < NW; ++w) M = fmaxf(M, sm_m[w]);
#pragma unroll
  for (int w = 0; w < NW; ++w) L += sm_l[w] * exp2_safe(sm_m[w], M);
  for (int c = threadIdx.x; c < HD; c += 128) {
    float a = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) a += sm_acc[w][c] * exp2_safe(sm_m[w], M);
    store_elem(out, (long long)r * out.row_stride + h * out.head_stride + c, L > 0.f ? a / L : 0.f);
  }
}

// ---- rows of a model call -----------------------------------------------------------------------
// minus_pos[r]: minus the position of row r (0 for rows without one): RowMap takes learned positions as "slot minus
// padding", so slot 0 with a padding of minus the position gives the position.  last_row[s]: the row of the sequence's last new token.
__global__ void cache_rows_kernel(const BatchView b, int* __restrict__ minus_pos, int* __restrict__ last_row) {
  int seq, pos;
  const int r = blockIdx.x;
  const int where = locate_row(b, r, seq, pos);
  if (threadIdx.x == 0) minus_pos[r] = where == ROW_OK ? -pos : 0;
  for (int s = r * blockDim.x + threadIdx.x; s < b.n_seqs; s += gridDim.x * blockDim.x)
    last_row[s] = min(max(b.first[s + 1] - 1, 0), b.n_tokens - 1);
}

}  // namespace sd
