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

// The same for up to MOST_ROWS consecutive rows of a block at once, one lane of the first warp per row (its owner by bisection): the
// chain of dependent loads (owner, length, table) is paid once for all of them.  Block 0 also checks the whole description.
constexpr int MOST_ROWS = 2;
struct Places {
  int state[MOST_ROWS], pos[MOST_ROWS], page[MOST_ROWS];         // ROW_*; position; page, -1 where the row has none
};
__device__ __forceinline__ void locate_rows(const BatchView& b, int r0, int n, Places& p) {
  if (threadIdx.x < n) {
    const int r = r0 + threadIdx.x;
    int lo = 0, hi = b.n_seqs + 1;                               // how many of first[0..n_seqs] are at most r
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (b.first[mid] <= r) lo = mid + 1;
      else hi = mid;
    }
    const int seq = lo - 1;
    int state = ROW_PADDING, pos = -1, page = -1;
    if (seq >= 0 && seq < b.n_seqs) {
      const int f0 = b.first[seq], f1 = b.first[seq + 1];
      if (f0 < 0 || f0 > r || r >= f1 || r - f0 >= b.max_new) b.bad();
      else {
        const long long at = (long long)b.len[seq] - f1 + r;
        state = ROW_NOWHERE;
        if (at >= (long long)b.pages_per_seq << b.page_shift) b.bad();
        else if (at >= 0) {
          state = ROW_OK;
          pos = (int)at;
          page = b.page_of(seq, pos);
        }
      }
    }
    p.state[threadIdx.x] = state;
    p.pos[threadIdx.x] = pos;
    p.page[threadIdx.x] = page;
  }
  if (blockIdx.x == 0) {
    for (int i = threadIdx.x; i <= b.n_seqs; i += blockDim.x)
      if (b.first[i] < (i ? b.first[i - 1] : 0) || (i == b.n_seqs && b.first[i] > b.n_tokens)) b.bad();
  }
  __syncthreads();
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

// A result from its weighted sum and the sum of its weights: 0 where no key was seen, NaN where the query was not a number.
__device__ __forceinline__ float normalised(float a, float l) { return l > 0.f ? a / l : (l == 0.f ? 0.f : l); }

// ---- codes ------------------------------------------------------------------------------------

__device__ __forceinline__ uint32_t e4m3_pair(float lo, float hi) {
  return (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ float2 e4m3_widen(uint32_t pair) {          // exact: every e4m3 is an fp16
  const __half2_raw r = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)pair, __NV_E4M3);
  return __half22float2(*reinterpret_cast<const __half2*>(&r));
}

// The code nearest to x / s, ties to even.  The quotient of two 24-bit numbers is either a border or at least 2^-25 (relative) away from
// it, so the 53-bit quotient decides exactly; on the way to e4m3 it passes through a float that is rounded to odd, which
// keeps a later rounding to fewer bits correct.
__device__ __noinline__ float quotient_int8(float x, float s) { return (float)fmin(fmax(rint((double)x / (double)s), -127.0), 127.0); }
__device__ __noinline__ float quotient_sticky(float x, float s) {
  const double q = (double)x / (double)s;
  const float f = __double2float_rz(q);
  return (double)f == q ? f : __uint_as_float(__float_as_uint(f) | 1u);
}

// Eight codes of x / s the exact way, for rows whose fast quotients do not decide, with a tiny scale or with elements that are not finite.
__device__ __forceinline__ uint2 encode8_exact(const float (&x)[8], float s, int8_t) {
  uint32_t w[2] = {0u, 0u};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float c = (x[i] != x[i] || s == 0.f) ? 0.f : quotient_int8(x[i], s);
    w[i >> 2] |= ((uint32_t)(int)c & 0xffu) << (8 * (i & 3));
  }
  return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ uint2 encode8_exact(const float (&x)[8], float s, e4m3) {
  uint32_t w[2] = {0u, 0u};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float y = (x[i] != x[i] || s == 0.f) ? 0.f : quotient_sticky(x[i], s);
    w[i >> 2] |= (e4m3_pair(y, 0.f) & 0xffu) << (8 * (i & 3));
  }
  return make_uint2(w[0], w[1]);
}
// Eight codes of x / s by the fast quotient x * inv, which is off by less than 2^-22 of itself; false where an element is too close
// to a border between two codes for that.  x: finite, inv = 1 / s.
__device__ __forceinline__ bool encode8_fast(const float (&x)[8], float inv, uint2& code, int8_t) {
  uint32_t w[2] = {0u, 0u};
  float far = 0.f;                                 // largest distance from the code
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float y = x[i] * inv;
    const float t = y + 12582912.f;                // 1.5 * 2^23: the code in the low bits
    far = fmaxf(far, fabsf(y - (t - 12582912.f)));
    w[i >> 2] |= (__float_as_uint(t) & 0xffu) << (8 * (i & 3));
  }
  code = make_uint2(w[0], w[1]);
  return far < 0.4999f;                            // 127 * 2^-22 = 3e-5 < 1e-4; at most 127 + 3e-5, so within the codes
}
__device__ __forceinline__ bool encode8_fast(const float (&x)[8], float inv, uint2& code, e4m3) {
  constexpr float UP = 1.f + 4.f / 16777216.f, DOWN = 1.f - 4.f / 16777216.f;          // 1 +- 2^-22
  uint32_t lo[4], hi[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float a = x[2 * i] * inv, b = x[2 * i + 1] * inv;
    lo[i] = e4m3_pair(a * DOWN, b * DOWN);
    hi[i] = e4m3_pair(a * UP, b * UP);
  }
  code = make_uint2(lo[0] | lo[1] << 16, lo[2] | lo[3] << 16);
  return ((code.x ^ (hi[0] | hi[1] << 16)) | (code.y ^ (hi[2] | hi[3] << 16))) == 0u;
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
// One block per few rows.  A group of HD / 8 lanes owns one (row, head, K or V): each lane holds eight elements, the largest
// magnitude goes round the group by shuffles, and the codes leave as one 8-byte store per lane (16 or 32 bytes in bf16 or
// fp32).  The bytes are read once and written once; there is no other work to speak of.  4005 rows of 32 heads of 128 from fp32 to
// e4m3: 46 us, 3.6 TB/s (2000 short blocks, each behind a chain of look-ups before its first load); 8 rows of 12 heads of 64: 4.6 us, of which nearly all is
// a launch and the chain of look-ups (owner, length, page) before the first load.
template <typename TS, typename TC, int HD, bool VEC>
__global__ void __launch_bounds__(256)
cache_append_kernel(const BatchView b, int row_shift, const Rows ks, const Rows vs, TC* __restrict__ Kp, TC* __restrict__ Vp,
                    float* __restrict__ Ksc, float* __restrict__ Vsc) {
  constexpr int LANES = HD / 8;
  __shared__ Places place;
  const int rows = 1 << row_shift, r0 = blockIdx.x << row_shift, n = min(rows, b.n_tokens - r0);
  locate_rows(b, r0, n, place);
  // lanes go over a head's elements, then over the block's rows, then over heads: neighbouring rows are neighbours in a page
  const int total = 2 * b.n_kv_heads * LANES << row_shift;
  constexpr int AT_ONCE = 4;                                     // pieces of a thread whose loads are on their way together
  for (int i0 = 0; i0 < total; i0 += AT_ONCE * blockDim.x) {     // uniform: the shuffles need whole warps
    float x[AT_ONCE][8];
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
      const int i = i0 + u * blockDim.x + threadIdx.x;
      const int row = i / LANES & (rows - 1), unit = i / LANES >> row_shift;
      if (i >= total || row >= n || place.page[row] < 0) {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[u][j] = 0.f;
        continue;
      }
      const bool is_v = unit >= b.n_kv_heads;
      const Rows& src = is_v ? vs : ks;
      load8<VEC>(static_cast<const TS*>(src.data) + (long long)(r0 + row) * src.row_stride + (is_v ? unit - b.n_kv_heads : unit) * src.head_stride + i % LANES * 8, x[u]);
    }
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
      const int i = i0 + u * blockDim.x + threadIdx.x;
      if (i0 + u * (int)blockDim.x >= total) break;              // the same for all threads
      const int row = i / LANES & (rows - 1), unit = i / LANES >> row_shift, sub = i % LANES;
      const bool on = i < total && row < n && place.page[row] >= 0;
      const bool is_v = unit >= b.n_kv_heads;
      const size_t e = on ? b.entry(place.page[row], is_v ? unit - b.n_kv_heads : unit, place.pos[row]) : 0;
      TC* dst = (is_v ? Vp : Kp) + e * HD + sub * 8;
      float top = 0.f;                                           // of the finite elements
      bool finite = true;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float a = fabsf(x[u][j]);
        if (a < INFINITY) top = fmaxf(top, a);
        else finite = false;                                     // NaN too
      }
      if (!finite) atomicOr(b.status, STATUS_NOT_FINITE);
      if constexpr (CacheType<TC>::TOP > 0.f) {
#pragma unroll
        for (int o = LANES / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        const float s = __fdiv_rn(top, CacheType<TC>::TOP);
        const float inv = s > 1e-30f ? __fdiv_rn(1.f, s) : 0.f;
        if (on) {
          uint2 code;
          if (!finite || inv == 0.f || !encode8_fast(x[u], inv, code, TC{})) code = encode8_exact(x[u], s, TC{});
          *reinterpret_cast<uint2*>(dst) = code;
          if (sub == 0) (is_v ? Vsc : Ksc)[e] = s;
        }
      } else if (on) {
        constexpr float MOST = CacheType<TC>::MOST;
        if (!finite || top > MOST) {                             // in bf16 the last half step below 2^128 would round to infinity
#pragma unroll
          for (int j = 0; j < 8; ++j) x[u][j] = x[u][j] != x[u][j] ? 0.f : fminf(fmaxf(x[u][j], -MOST), MOST);
        }
        store8<true>(dst, x[u]);                                 // pools are 256-byte aligned, rows multiples of 64 bytes
      }
    }
  }
}

// ---- read -------------------------------------------------------------------------------------
// The same walk the other way.  A row without a place reads as zeros.  24 sequences of 900..1500 positions, 32 heads of 128, int8 to bf16:
// 131 us, 5.4 TB/s; e4m3 to fp32, 4005 rows: 37 us, 4.5 TB/s.
template <typename TO, typename TC, int HD, bool VEC>
__global__ void __launch_bounds__(256)
cache_read_kernel(const BatchView b, int row_shift, const Rows ko, const Rows vo, const TC* __restrict__ Kp, const TC* __restrict__ Vp,
                  const float* __restrict__ Ksc, const float* __restrict__ Vsc) {
  constexpr int LANES = HD / 8;
  __shared__ Places place;
  const int rows = 1 << row_shift, r0 = blockIdx.x << row_shift, n = min(rows, b.n_tokens - r0);
  locate_rows(b, r0, n, place);
  // lanes go over a head's elements, then over the block's rows, then over heads: neighbouring rows are neighbours in a page
  const int total = 2 * b.n_kv_heads * LANES << row_shift;
  constexpr int AT_ONCE = 4;                                     // pieces of a thread whose loads are on their way together
  for (int i0 = threadIdx.x; i0 < total; i0 += AT_ONCE * blockDim.x) {
    constexpr bool SCALED = CacheType<TC>::TOP > 0.f;
    uint2 code[AT_ONCE];
    float scale[AT_ONCE], x[AT_ONCE][8];
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
      const int i = i0 + u * blockDim.x;
      code[u] = make_uint2(0u, 0u);
      scale[u] = 0.f;
      if constexpr (!SCALED) {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[u][j] = 0.f;
      }
      const int row = i / LANES & (rows - 1), unit = i / LANES >> row_shift;
      if (i >= total || row >= n || place.page[row] < 0) continue;
      const bool is_v = unit >= b.n_kv_heads;
      const size_t e = b.entry(place.page[row], is_v ? unit - b.n_kv_heads : unit, place.pos[row]);
      const TC* src = (is_v ? Vp : Kp) + e * HD + i % LANES * 8;
      if constexpr (SCALED) {
        code[u] = __ldg(reinterpret_cast<const uint2*>(src));
        scale[u] = __ldg((is_v ? Vsc : Ksc) + e);
      } else {
        load8<true>(src, x[u]);
      }
    }
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
      const int i = i0 + u * blockDim.x;
      const int row = i / LANES & (rows - 1), unit = i / LANES >> row_shift;
      if (i >= total || row >= n || place.state[row] == ROW_PADDING) continue;
      const bool is_v = unit >= b.n_kv_heads;
      if constexpr (SCALED) decode8(code[u], scale[u], x[u], TC{});
      const Rows& dst = is_v ? vo : ko;
      store8<VEC>(static_cast<TO*>(dst.data) + (long long)(r0 + row) * dst.row_stride + (is_v ? unit - b.n_kv_heads : unit) * dst.head_stride + i % LANES * 8, x[u]);
    }
  }
}

// ---- attention, one row and head per block ------------------------------------------------------
// Any cache type, on the CUDA cores in fp32: the kernel for caches in fp32, whose products the tensor cores would round.
// A group of HD / 8 lanes owns a key at a time (eight elements per lane); every group runs its own base-2 online softmax,
// merged by shuffles inside a warp and through shared memory across warps.  Every row reads its keys again (from L2): what bounds it is the
// fused multiply-adds and shuffles.  It serves the fp32 configuration, whose sizes are small.
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
    store_elem(out, (long long)r * out.row_stride + h * out.head_stride + c, normalised(a, L));
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
