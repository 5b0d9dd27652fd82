// Paged 8-bit KV cache: what its kernels share.  Layout and conventions: include/tq.h, struct tq_kv8.
#pragma once

#include <cuda_fp8.h>

#include "tq_internal.h"

namespace tq {
namespace kv8 {

constexpr int kPageTokens[] = {16, 32, 64, 128};

// The cache as the kernels see it.
struct Cache {
  uint8_t *k, *v;
  float *k_scale, *v_scale;
  int8_t* bounds;
  int64_t pages;
  int heads, page_shift, d;   // page_tokens = 1 << page_shift
};

// The batch: page table, lengths and the rows of each sequence.
struct Batch {
  const int32_t* table;
  int64_t ldt;
  int width, nseq;
  const int32_t* tokens;
  const int32_t* starts;   // NULL: one row per sequence
  int64_t n;               // rows that the arrays of queries, keys or values hold
};

// Checks shared by the entry points; fills `out`.  0 or a TQ_ERR_* code.
int check_cache(const char* who, const tq_kv8* c, Cache* out);
int check_batch(const char* who, const Cache& c, const int32_t* table, int64_t ldt, int width, int nseq, const int32_t* tokens,
                const int32_t* starts, int64_t n, Batch* out);

#ifdef __CUDACC__
// First and last row of sequence b, whatever the caller's array says: 0 <= begin <= end <= n.
__device__ __forceinline__ void rows_of(const Batch& a, int b, int64_t* begin, int64_t* end) {
  if (a.starts == nullptr) {
    *begin = b;
    *end = b + 1;
    return;
  }
  int64_t s = a.starts[b], e = a.starts[b + 1];
  s = s < 0 ? 0 : (s > a.n ? a.n : s);
  e = e < s ? s : (e > a.n ? a.n : e);
  *begin = s;
  *end = e;
}
// Tokens of sequence b that its row of the table has room for.
__device__ __forceinline__ int64_t tokens_of(const Batch& a, int b, int page_shift) {
  const int64_t t = a.tokens[b], most = (int64_t)a.width << page_shift;
  return t < 0 ? 0 : (t > most ? most : t);
}
// Page of the pool behind logical page j of sequence b, or -1 where there is none.
__device__ __forceinline__ int page_of(const Batch& a, int64_t pages, int b, int64_t j) {
  if (j < 0 || j >= a.width) return -1;
  const int id = a.table[(int64_t)b * a.ldt + j];
  return id >= 0 && id < pages ? id : -1;
}

// Sequence and visible tokens of a row; seq < 0 for rows behind the last sequence.
__device__ __forceinline__ void row_info(const Batch& a, int64_t row, int page_shift, int* seq, int64_t* visible) {
  if (a.starts == nullptr) {
    *seq = (int)row;
    *visible = tokens_of(a, (int)row, page_shift);
    return;
  }
  int lo = 0, hi = a.nseq;   // last b with starts[b] <= row
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (a.starts[mid + 1] <= row) lo = mid + 1; else hi = mid;
  }
  *seq = -1;
  *visible = 0;
  if (lo >= a.nseq) return;
  int64_t r0, r1;
  rows_of(a, lo, &r0, &r1);
  if (row < r0 || row >= r1) return;
  *seq = lo;
  const int64_t t = tokens_of(a, lo, page_shift) - (r1 - 1 - row);
  *visible = t < 0 ? 0 : t;
}

// Powers of two hold every block, so x / s and the change from one scale to another are exact.  a: largest magnitude as the bits of
// a non-negative finite float.  Returns the least 2^e, e >= -126, with a <= most * 2^e, or 0 for a = 0.
template <bool E4M3>
__device__ __forceinline__ float block_scale(uint32_t a) {
  if (a == 0u) return 0.f;
  constexpr int kTop = E4M3 ? 8 : 6;                                  // 448 = 1.75 * 2^8, 127 = 1.984375 * 2^6
  constexpr uint32_t kMantissa = E4M3 ? 0x600000u : 0x7E0000u;
  int e = (int)(a >> 23) - kTop + ((a & 0x7FFFFFu) > kMantissa ? 1 : 0);   // biased exponent of the scale
  if (e < 1) e = 1;
  return __uint_as_float((uint32_t)e << 23);
}
// 1 / s of a power of two (0 for 0, NaN for NaN).
__device__ __forceinline__ float block_inverse(float s) {
  if (s == 0.f) return 0.f;
  return s == s ? __uint_as_float((254u << 23) - __float_as_uint(s)) : s;
}
template <bool E4M3>
__device__ __forceinline__ uint8_t encode(float x) {   // |x| <= 127 or 448; NaN gives 0
  if (!(x == x)) return 0;
  if (E4M3) return (uint8_t)__nv_cvt_float_to_fp8(x, __NV_SATFINITE, __NV_E4M3);
  return (uint8_t)(int8_t)max(-127, min(127, __float2int_rn(x)));
}
// Four at a time, finite and in range.  int8: adding 1.5 * 2^23 rounds to the nearest even integer and leaves it in the low byte.
template <bool E4M3>
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d) {
  if (E4M3) {
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
    return lo | (hi << 16);
  }
  const uint32_t x = __byte_perm(__float_as_uint(a + 12582912.f), __float_as_uint(b + 12582912.f), 0x0040);
  const uint32_t y = __byte_perm(__float_as_uint(c + 12582912.f), __float_as_uint(d + 12582912.f), 0x0040);
  return __byte_perm(x, y, 0x5410);
}
template <bool E4M3>
__device__ __forceinline__ float decode(uint8_t c) {
  if (E4M3) return __half2float(__half(__nv_cvt_fp8_to_halfraw(c, __NV_E4M3)));
  return (float)(int8_t)c;
}
#endif

}  // namespace kv8
}  // namespace tq
