// Paged 8-bit KV cache: argument checks, quantisation of new tokens into their pages, and the choice of pages for sparse attention.
// The interface and the formulas are in include/tq.h; attention itself is in tq_kv8_attend.cu and tq_kv8_prompt.cu.
#include <algorithm>
#include <cstring>

#include "tq_kv8.h"

namespace tq {
namespace kv8 {

int check_cache(const char* who, const tq_kv8* c, Cache* out) {
  TQ_REQUIRE(c != nullptr, TQ_ERR_INVALID_ARG, "%s: cache is NULL", who);
  TQ_REQUIRE(c->code_type == TQ_I8 || c->code_type == TQ_E4M3, TQ_ERR_UNSUPPORTED, "%s: unknown code type %d", who, c->code_type);
  TQ_REQUIRE(c->d >= 32 && c->d <= 128 && c->d % 32 == 0, TQ_ERR_UNSUPPORTED, "%s: head dimension %d (multiples of 32 up to 128)", who, c->d);
  int shift = 0;
  for (int s = 4; s <= 7; ++s)
    if (c->page_tokens == 1 << s) shift = s;
  TQ_REQUIRE(shift != 0, TQ_ERR_UNSUPPORTED, "%s: pages of %d tokens (16, 32, 64 or 128)", who, c->page_tokens);
  TQ_REQUIRE(c->heads >= 1 && c->heads <= 65535, TQ_ERR_UNSUPPORTED, "%s: %d KV heads (1..65535)", who, c->heads);
  TQ_REQUIRE(c->pages >= 0 && c->pages < (1ll << 31), TQ_ERR_INVALID_ARG, "%s: %lld pages", who, (long long)c->pages);
  TQ_REQUIRE(c->pages == 0 || (c->k && c->v && c->k_scale && c->v_scale), TQ_ERR_INVALID_ARG, "%s: a NULL array in the cache", who);
  TQ_REQUIRE(((reinterpret_cast<uintptr_t>(c->k) | reinterpret_cast<uintptr_t>(c->v) | reinterpret_cast<uintptr_t>(c->k_scale) |
               reinterpret_cast<uintptr_t>(c->v_scale) | reinterpret_cast<uintptr_t>(c->k_bounds)) & 15) == 0,
             TQ_ERR_ALIGNMENT, "%s: an array of the cache is not 16-byte aligned", who);
  *out = Cache{c->k, c->v, c->k_scale, c->v_scale, c->k_bounds, c->pages, c->heads, shift, c->d};
  return TQ_OK;
}

int check_batch(const char* who, const Cache& c, const int32_t* table, int64_t ldt, int width, int nseq, const int32_t* tokens,
                const int32_t* starts, int64_t n, Batch* out) {
  TQ_REQUIRE(nseq >= 0 && n >= 0 && width >= 0, TQ_ERR_INVALID_ARG, "%s: negative size", who);
  TQ_REQUIRE(nseq <= (1 << 20) && n < (1ll << 31), TQ_ERR_UNSUPPORTED, "%s: at most 2^20 sequences and 2^31 - 1 rows", who);
  TQ_REQUIRE(width <= (1 << 24), TQ_ERR_UNSUPPORTED, "%s: at most 2^24 pages per sequence", who);
  TQ_REQUIRE(((int64_t)width << c.page_shift) <= (1ll << 31) - 256, TQ_ERR_UNSUPPORTED, "%s: a table of %d pages holds more than 2^31 - 256 tokens", who,
             width);   // positions of tokens, and of the ends of the tiles that they lie in, are 32-bit numbers
  TQ_REQUIRE(nseq == 0 || (tokens && (table || width == 0)), TQ_ERR_INVALID_ARG, "%s: page table or lengths are NULL", who);
  TQ_REQUIRE(ldt >= width, TQ_ERR_INVALID_ARG, "%s: row stride %lld of the table is smaller than its width %d", who, (long long)ldt, width);
  TQ_REQUIRE(starts != nullptr || n == nseq, TQ_ERR_INVALID_ARG, "%s: %lld rows for %d sequences without starts (one row each)", who, (long long)n, nseq);
  *out = Batch{table, ldt, width, nseq, tokens, starts, n};
  return TQ_OK;
}

namespace {

// ---------------------------------------------------------------------------------------------------------------- append
struct Input {
  const void* x;
  int64_t row, head;   // strides, elements
};
struct AppendArgs {
  Cache c;
  Batch b;
  Input in[2];
  int vec;             // rows may be read 16 bytes at a time
};

// 8 consecutive elements; CH of them are in the row.
template <typename T>
__device__ __forceinline__ void load8(const T* p, bool vec, float (&x)[8]) {
  if (vec) {
    if (sizeof(T) == 4) {
      const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
      x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    } else {
      const uint4 a = *reinterpret_cast<const uint4*>(p);
      const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (float)p[i];
  }
}

// Four codes as signed bytes in the order of their values (e4m3: sign and magnitude become two's complement, less one), and back.
template <bool E4M3>
__device__ __forceinline__ uint32_t ordered(uint32_t w) {
  return E4M3 ? w ^ ((w & 0x80808080u) >> 7) * 0x7Fu : w;
}
__device__ __forceinline__ uint32_t max16(uint32_t a, uint32_t b) {
  asm("max.s16x2 %0, %0, %1;" : "+r"(a) : "r"(b));
  return a;
}
__device__ __forceinline__ uint32_t min16(uint32_t a, uint32_t b) {
  asm("min.s16x2 %0, %0, %1;" : "+r"(a) : "r"(b));
  return a;
}
// Largest and smallest code of each channel of a block's first n rows, as ordered bytes: lane l < d / 16 of the warp has channels 16 l to
// 16 l + 15.  Bytes are compared as the upper halves of 16-bit numbers, two at a time in one instruction.
template <bool E4M3>
__device__ __forceinline__ void extremes(const uint8_t* codes, int d, int n, uint32_t (&hi)[4], uint32_t (&lo)[4]) {
  const int lane = threadIdx.x & 31, cpr = d >> 4, rows = 32 / cpr, chunk = lane % cpr;
  constexpr int U = 8;                      // rows that a lane asks for at once
  uint32_t h[8], l[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    h[j] = 0x80008000u;
    l[j] = 0x7F007F00u;
  }
  const uint8_t* from = codes + (lane / cpr) * d + 16 * chunk;
  const int mine = lane < rows * cpr ? n - lane / cpr : 0;    // rows from this lane's first one on
#pragma unroll 1
  for (int r = 0; r < n; r += U * rows) {
    uint4 w[U];
#pragma unroll
    for (int i = 0; i < U; ++i)             // behind the last one: this lane's first row of these again
      if (r < mine) w[i] = *reinterpret_cast<const uint4*>(from + (r + i * rows < mine ? r + i * rows : r) * d);
    if (r < mine) {
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const uint32_t x[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t y = ordered<E4M3>(x[j]), odd = y & 0xFF00FF00u, even = (y << 8) & 0xFF00FF00u;
          h[2 * j] = max16(h[2 * j], even);
          h[2 * j + 1] = max16(h[2 * j + 1], odd);
          l[2 * j] = min16(l[2 * j], even);
          l[2 * j + 1] = min16(l[2 * j + 1], odd);
        }
      }
    }
  }
  for (int s = rows / 2, left = rows; left > 1; left -= s, s = left / 2)   // the last s groups of rows join the first s
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t a = __shfl_down_sync(0xffffffffu, h[j], (left - s) * cpr), b = __shfl_down_sync(0xffffffffu, l[j], (left - s) * cpr);
      if (lane < s * cpr) {
        h[j] = max16(h[j], a);
        l[j] = min16(l[j], b);
      }
    }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    hi[j] = h[2 * j] >> 8 | h[2 * j + 1];
    lo[j] = l[2 * j] >> 8 | l[2 * j + 1];
  }
}

// Which (sequence, page) a slot is: the pages that new tokens fall on, sequence after sequence.  One warp looks it up.
__device__ __forceinline__ void find_slot(const AppendArgs& a, int64_t slot, int lane, int* seq, int64_t* page) {
  int64_t before = 0;
  *seq = -1;
  for (int b0 = 0; b0 < a.b.nseq; b0 += 32) {
    const int b = b0 + lane;
    int64_t first = 0, count = 0;
    if (b < a.b.nseq) {
      int64_t r0, r1;
      rows_of(a.b, b, &r0, &r1);
      const int64_t t = a.b.tokens[b] < 0 ? 0 : a.b.tokens[b];
      first = t >> a.c.page_shift;
      if (r1 > r0) count = ((t + (r1 - r0) - 1) >> a.c.page_shift) - first + 1;
    }
    int64_t upto = count;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t y = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += y;
    }
    const uint32_t hit = __ballot_sync(0xffffffffu, before + upto > slot);
    if (hit) {
      const int w = __ffs(hit) - 1;
      *seq = b0 + w;
      *page = __shfl_sync(0xffffffffu, first + slot - (before + upto - count), w);
      return;
    }
    before += __shfl_sync(0xffffffffu, upto, 31);
  }
}

// One CTA quantises the new tokens of one page and head, keys (blockIdx.z = 0) or values (1): it alone knows the block's largest
// magnitude, and old codes of the page are requantised where the scale grows.  NV vectors of 8 channels per thread hold what is new,
// so the input is read once.  A page per CTA, and not a row: the scale of the page needs all of its new rows at once.  Prompts are bound
// by the input's bytes behind each CTA's chain of dependent loads (lengths, table, rows): 109 MB in 32 us, 3.4 TB/s; one token each of
// 128 sequences by that chain alone, 4.3 us, 0.8 of it for the old codes of the pages, whose bounds are taken anew.
template <typename T, bool E4M3, int NV, int NT>
__global__ void __launch_bounds__(NT) append_kernel(const __grid_constant__ AppendArgs a) {
  __shared__ int found_seq;
  __shared__ int64_t found_page;
  __shared__ uint32_t top;
  __shared__ int hi[128], lo[128];
  const int t = threadIdx.x, lane = t & 31, h = blockIdx.y, d = a.c.d, dv = d >> 3, T_ = 1 << a.c.page_shift;
  const bool isv = blockIdx.z != 0;
  const Input in = a.in[isv];
  int seq;
  int64_t lp;
  wait_for_predecessor();   // lengths, table, cache and inputs may come from the kernel ahead
  if (a.b.starts == nullptr) {
    seq = blockIdx.x;
    const int64_t len = a.b.tokens[seq] < 0 ? 0 : a.b.tokens[seq];
    lp = len >> a.c.page_shift;
  } else {
    if (t < 32) {
      int s;
      int64_t p = 0;
      find_slot(a, blockIdx.x, lane, &s, &p);
      if (lane == 0) {
        found_seq = s;
        found_page = p;
      }
    }
    __syncthreads();
    seq = found_seq;
    lp = found_page;
    if (seq < 0) return;
  }
  int64_t r0, r1;
  rows_of(a.b, seq, &r0, &r1);
  const int64_t len = a.b.tokens[seq] < 0 ? 0 : a.b.tokens[seq];
  const int id = page_of(a.b, a.c.pages, seq, lp);
  if (id < 0) return;
  // slots [p0, p1) of the page are new: row r0 + (lp * T + slot - len) of the input; slots below p0 are old
  const int64_t base = (lp << a.c.page_shift) - len;
  const int p0 = base < 0 ? (int)-base : 0;
  const int p1 = (int)min((int64_t)T_, (r1 - r0) - base);
  const int64_t block = (int64_t)id * a.c.heads + h;
  uint8_t* codes = (isv ? a.c.v : a.c.k) + ((block * d) << a.c.page_shift);
  float* scale = (isv ? a.c.v_scale : a.c.k_scale) + block;
  int8_t* bounds = isv || a.c.bounds == nullptr ? nullptr : a.c.bounds + block * 2 * d;
  const float s0 = p0 > 0 ? *scale : 0.f;
  if (t == 0) top = 0u;
  const T* x = static_cast<const T*>(in.x) + h * in.head;
  float v[NV][8];
  uint32_t most = 0u;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int e = t + i * NT, slot = p0 + e / dv, ch = (e % dv) * 8;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[i][j] = 0.f;
    if (slot < p1) load8(x + (r0 + base + slot) * in.row + ch, a.vec != 0, v[i]);
#pragma unroll
    for (int j = 0; j < 8; ++j) most = max(most, __float_as_uint(v[i][j]) & 0x7FFFFFFFu);
  }
  // Bounds are those of the codes that count, the old ones among them (what is stored may hold tokens that were taken back).  One token
  // each: read here, while the new rows are on their way.
  uint32_t old_hi[4], old_lo[4];
  if (NT == 32) extremes<E4M3>(codes, d, bounds ? p0 : 0, old_hi, old_lo);
  most = __reduce_max_sync(0xffffffffu, most);
  __syncthreads();
  if (lane == 0) atomicMax(&top, most);
  __syncthreads();
  most = top;
  float s1;
  if (most >= 0x7F800000u || !(s0 == s0)) s1 = __uint_as_float(0x7FC00000u);   // not finite: the block reads as NaN from now on
  else s1 = fmaxf(s0, block_scale<E4M3>(most));
  const float inv = block_inverse(s1), ratio = s0 * inv;
  const bool grown = p0 > 0 && s1 == s1 && s1 != s0;
  // One token into blocks whose scale holds it: its lanes have a channel each to themselves.
  const bool one = NT == 32 && !grown;
  if (bounds && !one) {
    for (int c = t; c < d; c += NT) {
      hi[c] = -128;
      lo[c] = 127;
    }
    __syncthreads();
  }
  auto bound = [&](int ch, uint8_t code) {
    const float f = decode<E4M3>(code) * (E4M3 ? 0.25f : 1.f);
    const int u = __float2int_ru(f), w = __float2int_rd(f);
    if (u > hi[ch]) atomicMax(&hi[ch], u);
    if (w < lo[ch]) atomicMin(&lo[ch], w);
  };
  if (grown || (bounds && !one)) {
    for (int e = t; e < p0 * d / 4; e += NT) {
      uint32_t w = reinterpret_cast<uint32_t*>(codes)[e], o = 0u;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint8_t c = (uint8_t)(w >> (8 * j));
        if (grown) c = encode<E4M3>(decode<E4M3>(c) * ratio);
        o |= (uint32_t)c << (8 * j);
        if (bounds) bound((4 * e + j) % d, c);
      }
      if (grown) reinterpret_cast<uint32_t*>(codes)[e] = o;
    }
  }
  uint32_t near_hi[2], near_lo[2];              // old extremes of the 8 channels of this lane's new code
  if (NT == 32) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const uint32_t a = __shfl_sync(0xffffffffu, old_hi[j], t >> 1), b = __shfl_sync(0xffffffffu, old_hi[2 + j], t >> 1);
      const uint32_t c = __shfl_sync(0xffffffffu, old_lo[j], t >> 1), e = __shfl_sync(0xffffffffu, old_lo[2 + j], t >> 1);
      near_hi[j] = t & 1 ? b : a;
      near_lo[j] = t & 1 ? e : c;
    }
  }
  // A block that reads as NaN gets zeros.  Rounding keeps order, so the bounds of a channel's codes are the codes of its largest and
  // smallest value: those are kept per thread where its vectors all hold the same channels.
  const bool number = s1 == s1, aligned = NT % dv == 0;
  float high[8], low[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    high[j] = -__uint_as_float(0x7F800000u);
    low[j] = __uint_as_float(0x7F800000u);
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int e = t + i * NT, slot = p0 + e / dv, ch = (e % dv) * 8;
    if (slot < p1) {
      float y[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        y[j] = number ? v[i][j] * inv : 0.f;
        high[j] = fmaxf(high[j], y[j]);
        low[j] = fminf(low[j], y[j]);
      }
      const uint2 o = make_uint2(encode4<E4M3>(y[0], y[1], y[2], y[3]), encode4<E4M3>(y[4], y[5], y[6], y[7]));
      *reinterpret_cast<uint2*>(codes + slot * d + ch) = o;
      if (bounds && one) {
        uint2* at = reinterpret_cast<uint2*>(bounds + ch);
        uint2* under = reinterpret_cast<uint2*>(bounds + d + ch);
        uint32_t up[2], down[2];                           // int8: a code bounds itself
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          const uint32_t c = ordered<E4M3>(w ? o.y : o.x);
          up[w] = ordered<E4M3>(__vmaxs4(c, near_hi[w]));
          down[w] = ordered<E4M3>(__vmins4(c, near_lo[w]));
          if (E4M3) {
            const uint32_t x = up[w], y = down[w];
            up[w] = down[w] = 0u;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              up[w] |= (uint32_t)(uint8_t)__float2int_ru(decode<E4M3>((uint8_t)(x >> (8 * j))) * 0.25f) << (8 * j);
              down[w] |= (uint32_t)(uint8_t)__float2int_rd(decode<E4M3>((uint8_t)(y >> (8 * j))) * 0.25f) << (8 * j);
            }
          }
        }
        *at = make_uint2(up[0], up[1]);
        *under = make_uint2(down[0], down[1]);
      } else if (bounds && !aligned) {
#pragma unroll
        for (int j = 0; j < 8; ++j) bound(ch + j, (uint8_t)((j < 4 ? o.x : o.y) >> (8 * (j & 3))));
      }
    }
  }
  if (bounds && aligned && !one) {
    for (int x = dv; x < 32; x <<= 1)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        high[j] = fmaxf(high[j], __shfl_xor_sync(0xffffffffu, high[j], x));
        low[j] = fminf(low[j], __shfl_xor_sync(0xffffffffu, low[j], x));
      }
    if (lane < dv && high[0] >= low[0]) {   // some row was here
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        bound((t % dv) * 8 + j, encode<E4M3>(high[j]));
        bound((t % dv) * 8 + j, encode<E4M3>(low[j]));
      }
    }
  }
  if (t == 0) *scale = s1;
  if (bounds && !one) {
    __syncthreads();
    for (int c = t; c < d; c += NT) {
      bounds[c] = (int8_t)hi[c];
      bounds[d + c] = (int8_t)lo[c];
    }
  }
}

template <typename T, bool E4M3>
cudaError_t launch_append(const AppendArgs& a, int64_t slots, cudaStream_t st) {
  const dim3 grid((unsigned)slots, (unsigned)a.c.heads, 2);
  if (a.b.starts == nullptr) return launch_dependent(append_kernel<T, E4M3, 1, 32>, grid, dim3(32), 0, st, a);
  const int vectors = (a.c.d / 8) << a.c.page_shift;   // of a whole page: 64 .. 2048
  if (vectors <= 256) return launch_dependent(append_kernel<T, E4M3, 2, 128>, grid, dim3(128), 0, st, a);
  if (vectors <= 512) return launch_dependent(append_kernel<T, E4M3, 4, 128>, grid, dim3(128), 0, st, a);
  if (vectors <= 1024) return launch_dependent(append_kernel<T, E4M3, 4, 256>, grid, dim3(256), 0, st, a);
  return launch_dependent(append_kernel<T, E4M3, 8, 256>, grid, dim3(256), 0, st, a);
}

// ---------------------------------------------------------------------------------------------------------------- select
struct SelectArgs {
  Cache c;
  Batch b;
  const void* q;
  int64_t ldq, hq;
  int g, k, first, last;
  float unit;           // of a bound, in steps of the block's scale
  uint32_t* keys;       // [rows, heads, width] of this launch
  int64_t row0;         // first row of this launch
  int32_t* lists;       // [n, heads, k]
  int per;              // pages per CTA of the scoring kernel
};

// Order-preserving map of floats to integers; zeros of either sign are one value, NaN (a block that holds one) ranks with +inf.
__device__ __forceinline__ uint32_t rank_key(float x) {
  if (!(x == x)) x = __uint_as_float(0x7F800000u);
  if (x == 0.f) x = 0.f;
  const uint32_t u = __float_as_uint(x);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

constexpr int kScoreWarps = 4;

// score(page) = max over the group's heads j of 2^e_j s unit sum_c (max(qi, 0) B+ + min(qi, 0) B-): an integer product over 2 d bytes,
// so 16 pages x 8 heads x 32 bytes go into one mma with exact int32 sums, and the scores are exact in fp32 (an integer below 2^22
// times powers of two).  A warp takes 16 pages at a time; a lane reads 16 bytes of a page's bounds, in an order of k that the queries
// share.  Bound by the bounds' bytes, 2 d per page and head, and for few rows by latency: 2,048 pages of 8 heads (4 MB) in 4 us.
template <typename T, int D>
__global__ void __launch_bounds__(kScoreWarps * 32) score_kernel(const __grid_constant__ SelectArgs a) {
  constexpr int SEG = D / 32;              // 64-byte pieces of a page's bounds
  extern __shared__ uint4 smem4[];
  int8_t* qs = reinterpret_cast<int8_t*>(smem4);               // [tiles * 8][2 D + 16]
  const int tiles = (a.g + 7) / 8, pitch = 2 * D + 16;
  float* qe = reinterpret_cast<float*>(qs + (size_t)tiles * 8 * pitch);
  const int t = threadIdx.x, warp = t >> 5, lane = t & 31, h = blockIdx.y;
  const int64_t row = a.row0 + blockIdx.z;
  wait_for_predecessor();
  int seq;
  int64_t visible;
  row_info(a.b, row, a.c.page_shift, &seq, &visible);
  const int64_t count = (visible + (1 << a.c.page_shift) - 1) >> a.c.page_shift, p0 = (int64_t)blockIdx.x * a.per;
  if (seq < 0 || p0 >= count || count <= a.k) return;          // all pages are taken: nothing to rank
  const T* q = static_cast<const T*>(a.q) + row * a.ldq + (int64_t)h * a.g * a.hq;
  for (int j = warp; j < tiles * 8; j += kScoreWarps) {
    float x[D / 32];
    uint32_t most = 0u;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      x[i] = j < a.g ? (float)q[j * a.hq + i * 32 + lane] : 0.f;
      most = max(most, __float_as_uint(x[i]) & 0x7FFFFFFFu);
    }
    most = __reduce_max_sync(0xffffffffu, most);
    const float s = most >= 0x7F800000u ? 0.f : block_scale<false>(most), inv = block_inverse(s);
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      const int v = s > 0.f ? max(-127, min(127, __float2int_rn(x[i] * inv))) : 0;
      qs[j * pitch + i * 32 + lane] = (int8_t)max(v, 0);
      qs[j * pitch + D + i * 32 + lane] = (int8_t)min(v, 0);
    }
    if (lane == 0) qe[j] = s;
  }
  __syncthreads();
  const int64_t end = min(count, p0 + a.per);
  uint32_t* keys = a.keys + ((int64_t)blockIdx.z * a.c.heads + h) * a.b.width;
  for (int64_t p = p0 + warp * 16; p < end; p += kScoreWarps * 16) {
    uint4 w[2][SEG];
    float step[2];
    bool live[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int64_t at = p + (lane >> 2) + 8 * r;
      const int id = at < end ? page_of(a.b, a.c.pages, seq, at) : -1;
      live[r] = id >= 0;
      const int64_t block = (int64_t)max(id, 0) * a.c.heads + h;
      step[r] = 0.f;
#pragma unroll
      for (int i = 0; i < SEG; ++i) w[r][i] = make_uint4(0, 0, 0, 0);
      if (live[r]) {
        const uint4* src = reinterpret_cast<const uint4*>(a.c.bounds + block * 2 * D) + (lane & 3);
#pragma unroll
        for (int i = 0; i < SEG; ++i) w[r][i] = __ldg(src + 4 * i);
        step[r] = a.c.k_scale[block] * a.unit;
      }
    }
    float best[2] = {-__uint_as_float(0x7F800000u), -__uint_as_float(0x7F800000u)};
    for (int tile = 0; tile < tiles; ++tile) {
      int acc[4] = {0, 0, 0, 0};
      const uint4* b = reinterpret_cast<const uint4*>(qs + (size_t)(tile * 8 + (lane >> 2)) * pitch) + (lane & 3);
#pragma unroll
      for (int i = 0; i < SEG; ++i) {
        const uint4 y = b[4 * i];
        asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+r"(acc[0]), "+r"(acc[1]), "+r"(acc[2]), "+r"(acc[3])
                     : "r"(w[0][i].x), "r"(w[1][i].x), "r"(w[0][i].y), "r"(w[1][i].y), "r"(y.x), "r"(y.y));
        asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+r"(acc[0]), "+r"(acc[1]), "+r"(acc[2]), "+r"(acc[3])
                     : "r"(w[0][i].z), "r"(w[1][i].z), "r"(w[0][i].w), "r"(w[1][i].w), "r"(y.z), "r"(y.w));
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int j = tile * 8 + 2 * (lane & 3) + e;
        if (j < a.g) {
          best[0] = fmaxf(best[0], (float)acc[e] * qe[j]);
          best[1] = fmaxf(best[1], (float)acc[2 + e] * qe[j]);
        }
      }
    }
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      best[r] = fmaxf(best[r], __shfl_xor_sync(0xffffffffu, best[r], 1));
      best[r] = fmaxf(best[r], __shfl_xor_sync(0xffffffffu, best[r], 2));
      const int64_t at = p + (lane >> 2) + 8 * r;
      if ((lane & 3) == 0 && at < end) {
        uint32_t key = live[r] ? rank_key(best[r] * step[r]) : 0u;
        if (at < a.first || at >= count - a.last) key = 0xFFFFFFFFu;
        keys[at] = key;
      }
    }
  }
}

constexpr int kPickThreads = 512, kPickWarps = kPickThreads / 32, kPickKeys = 8;

// The k best keys of one (row, head) in ascending order of the page number, equal keys by the lower number.  Each round of an 8-bit
// histogram narrows down the value of the last key that is taken, from the first bit in which the keys differ at all, and the rounds
// end as soon as a whole bin is taken; then the pages are numbered through in order.  Up to 4,096 keys are held in registers (REG), more
// are read again from L2.  Latency of a few barriers: one CTA per (row, head).
template <bool REG>
__global__ void __launch_bounds__(kPickThreads) pick_kernel(const __grid_constant__ SelectArgs a) {
  __shared__ uint32_t hist[2][256];
  __shared__ uint32_t low_w[kPickWarps], high_w[kPickWarps], forced_w[kPickWarps];
  __shared__ uint32_t above_w[kPickKeys * kPickWarps], equal_w[kPickKeys * kPickWarps];
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5, h = blockIdx.x;
  const int64_t row = a.row0 + blockIdx.y;
  allow_successor();
  wait_for_predecessor();
  int seq;
  int64_t visible;
  row_info(a.b, row, a.c.page_shift, &seq, &visible);
  if (seq < 0) return;
  int32_t* list = a.lists + (row * a.c.heads + h) * a.k;
  const int count = (int)((visible + (1 << a.c.page_shift) - 1) >> a.c.page_shift);
  if (count <= a.k) {
    for (int i = t; i < a.k; i += kPickThreads) list[i] = i < count ? i : -1;
    return;
  }
  const uint32_t* keys = a.keys + ((int64_t)blockIdx.y * a.c.heads + h) * a.b.width;
  uint32_t own[kPickKeys];
  if (REG) {
#pragma unroll
    for (int j = 0; j < kPickKeys; ++j) own[j] = t + j * kPickThreads < count ? keys[t + j * kPickThreads] : 0u;
  }
  auto each = [&](auto&& f) {   // f(key, page) of this thread's pages
    if (REG) {
#pragma unroll
      for (int j = 0; j < kPickKeys; ++j)
        if (t + j * kPickThreads < count) f(own[j], t + j * kPickThreads);
    } else {
      for (int i = t; i < count; i += kPickThreads) f(keys[i], i);
    }
  };
  // pages that are taken in any case have the largest key; the others' smallest and largest
  uint32_t low = 0xFFFFFFFFu, high = 0u, forced = 0u;
  each([&](uint32_t x, int) {
    if (x == 0xFFFFFFFFu) {
      ++forced;
    } else {
      low = min(low, x);
      high = max(high, x);
    }
  });
  low = __reduce_min_sync(0xffffffffu, low);
  high = __reduce_max_sync(0xffffffffu, high);
  forced = __reduce_add_sync(0xffffffffu, forced);
  if (lane == 0) {
    low_w[warp] = low;
    high_w[warp] = high;
    forced_w[warp] = forced;
  }
  for (int i = t; i < 512; i += kPickThreads) hist[i >> 8][i & 255] = 0u;
  __syncthreads();
  low = __reduce_min_sync(0xffffffffu, low_w[lane % kPickWarps]);
  high = __reduce_max_sync(0xffffffffu, high_w[lane % kPickWarps]);
  forced = __reduce_add_sync(0xffffffffu, lane < kPickWarps ? forced_w[lane] : 0u);
  uint32_t need = (uint32_t)a.k > forced ? (uint32_t)a.k - forced : 0u;   // of the others; there are more of them than that
  // taken: keys above `edge`, and the first `need` of those equal to it
  uint32_t edge = high;
  int rest = low < high ? 32 - __clz(low ^ high) : 0;                     // bits in which keys may differ
  uint32_t prefix = rest == 32 ? 0u : high >> rest;
  bool whole = need == 0u;                                                // all keys at or above `edge` are taken
  if (whole) edge = 0xFFFFFFFFu;
  int round = 0;
  while (rest > 0 && !whole) {
    const int bits = min(rest, 8), shift = rest - bits;
    uint32_t* hb = hist[round & 1];
    each([&](uint32_t x, int) {
      if (x != 0xFFFFFFFFu && (rest == 32 || (x >> rest) == prefix)) atomicAdd(&hb[(x >> shift) & ((1u << bits) - 1u)], 1u);
    });
    __syncthreads();
    // every warp looks for the bin that the need-th largest key falls into: lane l has bins 255 - 8 l .. 248 - 8 l
    uint32_t bins[8], sum = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      bins[i] = hb[255 - 8 * lane - i];
      sum += bins[i];
    }
    uint32_t upto = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t y = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += y;
    }
    uint32_t before = upto - sum, bin = 0u, left = 0u, size = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (before < need && before + bins[i] >= need) {
        bin = 255u - 8u * lane - i;
        left = need - before;
        size = bins[i];
      }
      before += bins[i];
    }
    const int from = __ffs(__ballot_sync(0xffffffffu, size != 0u)) - 1;   // one lane has found it
    bin = __shfl_sync(0xffffffffu, bin, from);
    need = __shfl_sync(0xffffffffu, left, from);
    size = __shfl_sync(0xffffffffu, size, from);
    prefix = rest == 32 ? bin : (prefix << bits) | bin;
    rest = shift;
    edge = prefix << shift;
    whole = need == size;
    // the other histogram was last read before this round's barrier
    for (int i = t; i < 256; i += kPickThreads) hist[(round + 1) & 1][i] = 0u;
    ++round;
    __syncthreads();
  }
  if (whole) need = 0xFFFFFFFFu;
  if (REG) {
    uint32_t bg[kPickKeys], be[kPickKeys];
#pragma unroll
    for (int j = 0; j < kPickKeys; ++j) {
      const bool in = t + j * kPickThreads < count;
      bg[j] = __ballot_sync(0xffffffffu, in && own[j] > edge);
      be[j] = __ballot_sync(0xffffffffu, in && own[j] == edge);
      if (lane == 0) {
        above_w[j * kPickWarps + warp] = __popc(bg[j]);
        equal_w[j * kPickWarps + warp] = __popc(be[j]);
      }
    }
    __syncthreads();
    if (warp == 0) {   // exclusive sums over the 128 (chunk, warp) counts, four per lane
      uint32_t g[4], e[4], sg = 0u, se = 0u;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        g[i] = above_w[4 * lane + i];
        e[i] = equal_w[4 * lane + i];
        sg += g[i];
        se += e[i];
      }
      uint32_t ug = sg, ue = se;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t yg = __shfl_up_sync(0xffffffffu, ug, o), ye = __shfl_up_sync(0xffffffffu, ue, o);
        if (lane >= o) {
          ug += yg;
          ue += ye;
        }
      }
      ug -= sg;
      ue -= se;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        above_w[4 * lane + i] = ug;
        equal_w[4 * lane + i] = ue;
        ug += g[i];
        ue += e[i];
      }
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kPickKeys; ++j) {
      const uint32_t under = (1u << lane) - 1u, g = above_w[j * kPickWarps + warp] + __popc(bg[j] & under),
                     e = equal_w[j * kPickWarps + warp] + __popc(be[j] & under);
      if (((bg[j] >> lane) & 1u) || (((be[j] >> lane) & 1u) && e < need)) list[g + min(e, need)] = t + j * kPickThreads;
    }
  } else {
    uint32_t above = 0u, equal = 0u;   // found before this chunk
    for (int i0 = 0; i0 < count; i0 += kPickThreads) {
      const int i = i0 + t;
      const uint32_t x = i < count ? keys[i] : 0u;
      const bool gt = i < count && x > edge, eq = i < count && x == edge;
      const uint32_t bg = __ballot_sync(0xffffffffu, gt), be = __ballot_sync(0xffffffffu, eq);
      if (lane == 0) {
        above_w[warp] = __popc(bg);
        equal_w[warp] = __popc(be);
      }
      __syncthreads();
      uint32_t ga = above, ge = equal;
      for (int w = 0; w < kPickWarps; ++w) {
        if (w == warp) {
          const uint32_t g = ga + __popc(bg & ((1u << lane) - 1u)), e = ge + __popc(be & ((1u << lane) - 1u));
          if (gt || (eq && e < need)) list[g + min(e, need)] = i;
        }
        ga += above_w[w];
        ge += equal_w[w];
      }
      above = ga;
      equal = ge;
      __syncthreads();
    }
  }
}

template <typename T>
cudaError_t launch_score(const SelectArgs& a, dim3 grid, size_t smem, cudaStream_t st) {
  const dim3 block(kScoreWarps * 32);
  switch (a.c.d) {
    case 32: return launch_dependent(score_kernel<T, 32>, grid, block, smem, st, a);
    case 64: return launch_dependent(score_kernel<T, 64>, grid, block, smem, st, a);
    case 96: return launch_dependent(score_kernel<T, 96>, grid, block, smem, st, a);
    default: return launch_dependent(score_kernel<T, 128>, grid, block, smem, st, a);
  }
}

// Rows that are scored before the next ones: as many as leave the keys within 64 MB, so that many rows need no workspace of their own.
int64_t rows_per_launch(int heads, int width) {
  return std::max<int64_t>(1, std::min<int64_t>(32768, (int64_t)(64 << 20) / ((int64_t)heads * width * (int64_t)sizeof(uint32_t))));
}

}  // namespace
}  // namespace kv8
}  // namespace tq

extern "C" int tq_kv8_append(const tq_kv8* cache, const int32_t* table, int64_t ldt, int width, int nseq, const int32_t* tokens,
                             const int32_t* starts, int64_t n, const void* K, int64_t ldk, int64_t hk, const void* V, int64_t ldv,
                             int64_t hv, int dtype, void* stream) {
  using namespace tq;
  using namespace tq::kv8;
  const char* who = "tq_kv8_append";
  TQ_RANGE(who);
  AppendArgs a;
  std::memset(&a, 0, sizeof(a));
  int rc = check_cache(who, cache, &a.c);
  if (rc == TQ_OK) rc = check_batch(who, a.c, table, ldt, width, nseq, tokens, starts, n, &a.b);
  if (rc != TQ_OK) return rc;
  TQ_REQUIRE(dtype == TQ_F32 || dtype == TQ_BF16, TQ_ERR_UNSUPPORTED, "%s: unknown dtype %d", who, dtype);
  if (nseq == 0 || n == 0 || cache->pages == 0) return TQ_OK;
  TQ_REQUIRE(K != nullptr && V != nullptr, TQ_ERR_INVALID_ARG, "%s: K or V is NULL", who);
  TQ_REQUIRE(ldk >= 0 && hk >= 0 && ldv >= 0 && hv >= 0, TQ_ERR_INVALID_ARG, "%s: negative stride", who);
  const int size = dtype == TQ_F32 ? 4 : 2;
  TQ_REQUIRE(((reinterpret_cast<uintptr_t>(K) | reinterpret_cast<uintptr_t>(V)) & (size - 1)) == 0, TQ_ERR_ALIGNMENT,
             "%s: K or V is not aligned to its elements", who);
  a.in[0] = Input{K, ldk, hk};
  a.in[1] = Input{V, ldv, hv};
  a.vec = ((reinterpret_cast<uintptr_t>(K) | reinterpret_cast<uintptr_t>(V)) & 15) == 0 && ((ldk | hk | ldv | hv) * size) % 16 == 0;
  // a sequence's new tokens fall on at most (count + T - 2) / T + 1 pages, so all of them on at most this many
  const int64_t slots = starts == nullptr ? nseq : (n >> a.c.page_shift) + 2 * (int64_t)std::min<int64_t>(nseq, n);
  TQ_REQUIRE(slots < (1ll << 31), TQ_ERR_UNSUPPORTED, "%s: too many pages in one call", who);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool e4m3 = cache->code_type == TQ_E4M3;
  if (dtype == TQ_F32)
    TQ_CHECK_CUDA((e4m3 ? launch_append<float, true>(a, slots, st) : launch_append<float, false>(a, slots, st)), who);
  else
    TQ_CHECK_CUDA((e4m3 ? launch_append<__nv_bfloat16, true>(a, slots, st) : launch_append<__nv_bfloat16, false>(a, slots, st)), who);
  count_launches(1);
  return TQ_OK;
}

extern "C" size_t tq_kv8_select_workspace_bytes(const tq_kv8* cache, int64_t n, int width) {
  if (cache == nullptr || n <= 0 || width <= 0 || cache->heads <= 0) return 0;
  return (size_t)std::min<int64_t>(n, tq::kv8::rows_per_launch(cache->heads, width)) * cache->heads * width * sizeof(uint32_t);
}

extern "C" int tq_kv8_select(const tq_kv8* cache, const int32_t* table, int64_t ldt, int width, int nseq, const int32_t* tokens,
                             const int32_t* starts, int64_t n, const void* Q, int64_t ldq, int64_t hq, int q_per_kv, int dtype,
                             int first, int last, int k, int32_t* lists, void* workspace, size_t workspace_bytes, void* stream) {
  using namespace tq;
  using namespace tq::kv8;
  const char* who = "tq_kv8_select";
  TQ_RANGE(who);
  SelectArgs a;
  std::memset(&a, 0, sizeof(a));
  int rc = check_cache(who, cache, &a.c);
  if (rc == TQ_OK) rc = check_batch(who, a.c, table, ldt, width, nseq, tokens, starts, n, &a.b);
  if (rc != TQ_OK) return rc;
  TQ_REQUIRE(dtype == TQ_F32 || dtype == TQ_BF16, TQ_ERR_UNSUPPORTED, "%s: unknown dtype %d", who, dtype);
  TQ_REQUIRE(q_per_kv >= 1 && q_per_kv <= 256, TQ_ERR_UNSUPPORTED, "%s: 1..256 queries per KV head", who);
  TQ_REQUIRE(k >= 1 && first >= 0 && last >= 0 && (int64_t)first + last <= k, TQ_ERR_INVALID_ARG,
             "%s: k = %d with %d first and %d last pages", who, k, first, last);
  if (nseq == 0 || n == 0) return TQ_OK;
  TQ_REQUIRE(Q != nullptr && lists != nullptr, TQ_ERR_INVALID_ARG, "%s: Q or lists is NULL", who);
  TQ_REQUIRE(cache->k_bounds != nullptr || cache->pages == 0, TQ_ERR_INVALID_ARG, "%s: the cache keeps no bounds", who);
  TQ_REQUIRE(ldq >= 0 && hq >= 0, TQ_ERR_INVALID_ARG, "%s: negative stride", who);
  TQ_REQUIRE((reinterpret_cast<uintptr_t>(Q) & (dtype == TQ_F32 ? 3 : 1)) == 0 && (reinterpret_cast<uintptr_t>(lists) & 3) == 0,
             TQ_ERR_ALIGNMENT, "%s: Q or lists is not aligned to its elements", who);
  const size_t need = tq_kv8_select_workspace_bytes(cache, n, width);
  TQ_REQUIRE(need == 0 || (workspace != nullptr && workspace_bytes >= need), TQ_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", who,
             workspace_bytes, need);
  TQ_REQUIRE((reinterpret_cast<uintptr_t>(workspace) & 255) == 0, TQ_ERR_ALIGNMENT, "%s: workspace is not 256-byte aligned", who);
  a.q = Q; a.ldq = ldq; a.hq = hq; a.g = q_per_kv; a.k = k; a.first = first; a.last = last;
  a.unit = cache->code_type == TQ_E4M3 ? 4.f : 1.f;
  a.keys = static_cast<uint32_t*>(workspace);
  a.lists = lists;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  int dev = 0, sms = 0;
  TQ_CHECK_CUDA(cudaGetDevice(&dev), who);
  TQ_CHECK_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev), who);
  const int tiles = (q_per_kv + 7) / 8;
  const size_t smem = (size_t)tiles * 8 * (2 * a.c.d + 16) + (size_t)tiles * 8 * sizeof(float);   // at most 71,680 bytes, q_per_kv = 256
  if (smem > 48 * 1024) {
    static std::atomic<unsigned long long> devices[8];
    const void* kern[8] = {(const void*)score_kernel<float, 32>, (const void*)score_kernel<float, 64>, (const void*)score_kernel<float, 96>,
                           (const void*)score_kernel<float, 128>, (const void*)score_kernel<__nv_bfloat16, 32>,
                           (const void*)score_kernel<__nv_bfloat16, 64>, (const void*)score_kernel<__nv_bfloat16, 96>,
                           (const void*)score_kernel<__nv_bfloat16, 128>};
    const int at = (dtype == TQ_F32 ? 0 : 4) + a.c.d / 32 - 1;
    TQ_CHECK_CUDA(allow_largest_smem(kern[at], devices[at]), who);
  }
  const int64_t most = width > 0 ? rows_per_launch(cache->heads, width) : 32768;
  for (int64_t row0 = 0; row0 < n; row0 += most) {
    const int64_t rows = std::min(most, n - row0);
    a.row0 = row0;
    if (width > k) {   // else every page is taken
      // a CTA's queries are quantised once for `per` pages: as many as leave eight CTAs per SM
      const int64_t want = std::max<int64_t>(1, (int64_t)8 * sms / std::max<int64_t>(1, rows * a.c.heads));
      a.per = (int)std::min<int64_t>(round_up64((width + want - 1) / want, kScoreWarps * 16), round_up64(width, kScoreWarps * 16));
      const dim3 grid((unsigned)((width + a.per - 1) / a.per), (unsigned)a.c.heads, (unsigned)rows);
      TQ_CHECK_CUDA(dtype == TQ_F32 ? launch_score<float>(a, grid, smem, st) : launch_score<__nv_bfloat16>(a, grid, smem, st), who);
      count_launches(1);
    }
    TQ_CHECK_CUDA(launch_dependent(width <= kPickKeys * kPickThreads ? pick_kernel<true> : pick_kernel<false>,
                                   dim3((unsigned)a.c.heads, (unsigned)rows), dim3(kPickThreads), 0, st, a), who);
    count_launches(1);
  }
  return TQ_OK;
}
