// Attention over a paged 8-bit KV cache: what the few-query and the many-query kernels are given.
#pragma once

#include "tq_kv8.h"

namespace tq {
namespace kv8 {

constexpr int kMaxCols = 16;      // columns of a block of the few-query kernel
constexpr int kPromptRows = 256;  // at most, of a block of the many-query kernel
constexpr float kLift = 6.f;      // (few-query kernel) weights are 2^(score - maximum + kLift): more of the small ones are normal fp16 numbers
constexpr float kSlack = 8.f;     // a maximum only moves when a score exceeds it by this much (in powers of two)
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct Meta {             // an item that begins in a CTA's share of the work and ends in another's
  int row0, col0, cols, head, last_cta, pad[3];
};

struct AttendArgs {
  Cache c;
  Batch b;
  const void* q;
  int64_t ldq, hq;
  int g;                  // query heads per KV head
  int most_cols;          // sequences with more columns (rows x g) are the many-query kernel's
  float scale;
  const int32_t* lists;   // [n, heads, nlist] pages of each row, or NULL: all of the sequence's
  int nlist;
  void* out;
  int64_t ldo, ho;
  float* lse;
  Meta* meta;             // workspace
  float *part_ml, *part_o;   // parts of items: maxima and sums, and outputs divided by these sums
  int pitch;              // columns of a part
  float lift;             // of its weights
  int give_up;            // (many-query kernel) self test of a wait that runs out
};

// The many-query kernel (tq_kv8_prompt.cu): workspace beside the few-query kernel's, and its launch, which is followed by the join.
size_t prompt_space(int sms, int d);
cudaError_t launch_prompt(AttendArgs& a, int dtype, bool e4m3, int sms, void* workspace, cudaStream_t st);
cudaError_t launch_join(const AttendArgs& a, int dtype, int ctas, int cols, cudaStream_t st);   // ctas: shares; cols: of an item, at most

#ifdef __CUDACC__
#define TQ_INF __uint_as_float(0x7F800000u)
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// log2 of a block's scale: exact for a power of two, -inf for 0 and for NaN (whose weights are set apart).
__device__ __forceinline__ float scale_log2(float s) {
  const uint32_t u = __float_as_uint(s);
  if ((u & 0x7FFFFFu) == 0u && u - 1u < 0x7F7FFFFFu) return (float)((int)(u >> 23) - 127);
  return s > 0.f ? __log2f(s) : -TQ_INF;
}
template <typename T>
__device__ __forceinline__ void store_out(T* p, float x);
template <>
__device__ __forceinline__ void store_out<float>(float* p, float x) { *p = x; }
template <>
__device__ __forceinline__ void store_out<__nv_bfloat16>(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }
// A power of two that takes the largest magnitude of a row of queries (its bits) into [2^13, 2^14), and its inverse.
__device__ __forceinline__ float query_scale(uint32_t most, float* inverse) {
  const int e = min(max((int)(most >> 23) - 13, 1), 253);   // both stay normal numbers
  *inverse = __uint_as_float((uint32_t)(254 - e) << 23);
  return __uint_as_float((uint32_t)e << 23);
}
#endif

}  // namespace kv8
}  // namespace tq
