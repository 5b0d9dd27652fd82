// Attention over a paged 8-bit KV cache for many queries per sequence (prompts, chunks of prompts), on tcgen05.
//
// Mathematics.  Rows are (token, head of the group) pairs of one sequence and KV head; per tile of 128 rows and 128 keys
//   S = Q K^T (TMEM),  p = 2^(s + log2 v - r + lift),  l += 2^(r - log2 v - m) sum p,  O += P V (TMEM, P as the A operand from TMEM),
// out = O 2^(r - m) / l.  As in the few-query kernel queries are scaled per row by a power of two into [2^13, 2^14) and held in fp16 (fp32 ones
// as two limbs), P is one fp16 limb for bf16 outputs and two for fp32 ones, m is the row's running maximum and r that of s + log2 v, whole
// numbers that only rise, when a score exceeds one of them by far: then the row's O in TMEM is rescaled by its own thread.  Sums are fp32.
// v and its like for keys are the tile's units, the largest scales of its blocks.  The codes become fp16 in shared memory times their
// block's scale over the unit, a power of two: from 2^-15 to 1 for keys, exactly; from 2^-2 to 1 for values, as r and with it P's smallest
// step follow the unit for rows too that do not see the block it comes from.  Blocks below that, and values of 0, are left out (masked, as keys
// that nobody sees) and take their turn with units of their own in a second pass over the same tile: what one page holds changes nothing
// for another.  (Pages of 16 tokens of which a third are 2^8 smaller, so that every tile takes two passes: 1,540 us for the 2,048 queries
// below, in place of 579.)
//
// Work.  A CTA per SM; units are (tile of 128 keys) x (block of 256 rows, fp32: 128), numbered through over blocks, heads and sequences,
// and every CTA takes an equal run of them, so that causal triangles and ragged batches are even; runs that end inside a block leave
// parts that the join kernel adds up.
// Warps: two groups of four for the softmax of a row tile each (a thread per row, no shuffles), four and three that expand keys and values
// from global memory through registers into the operand layout, one that issues the MMAs.  While one group works on its S, the tensor cores work for the
// other.  Waits are bounded; a CTA that gives one up writes NaN for the item in hand and for the rest of its run.
//
// Measured, one B200: 2,048 queries x 32 heads (4 per KV head, d = 128, bf16) over 16,384 tokens 581 us = 887 TFLOP/s, 0.54 of cuBLAS (595 in
// calls made one by one); fp32 (twice the MMAs) 1,268 us; a prompt of 4,096 tokens 390 us.  A tile of 128 keys takes about 4,700 cycles,
// its MMAs 2,060 of them and the exponentials 2,050 (both row tiles): what binds is the chain of one row tile, scores - maximum - weights -
// sum - next scores, of which two are in flight.  Scores of 64 keys in two buffers, asked for ahead (694 us), lengthen the MMAs instead: with N = 64 they
// are bound by the reads of the queries from shared memory.  Fewer unrolled copies of the code gained 15 %: 16 warps in four roles fetch
// instructions from one cache.  The copies of codes in registers had to go to warps of their own for keys and values (870 -> 700 us).
#include <algorithm>
#include <cstring>
#include <type_traits>

#include "tq_kv8.h"
#include "tq_kv8_attend.h"
#include "tq_tc.cuh"

namespace tq {
namespace kv8 {
namespace {

std::atomic<int> give_up{0};   // of tq_selftest_kv8_timeout

// Four warps per scheduler, 128 registers each: 8 for the softmax, 4 that expand keys, 3 that expand values, 1 for the MMAs.
constexpr int kThreads = 512, kExpandWarp0 = 8, kKeyWarps = 4, kValueWarps = 3, kMmaWarp = 15;
constexpr int kKeys = 128;                  // of a tile
constexpr uint32_t kPanel = kKeys * 128;    // bytes of 128 rows x 64 fp16

template <typename T, int D>
struct Shape {
  static constexpr int kLimbs = sizeof(T) == 4 ? 2 : 1;
  static constexpr int kTiles = kLimbs == 2 ? 1 : 2;
  static constexpr int kRows = 128 * kTiles;
  static constexpr int kPanels = (D + 63) / 64;
  static constexpr uint32_t kOperand = kPanels * kPanel;          // a tile of 128 rows: queries, keys or values
  static constexpr uint32_t smem = 6 * kOperand + 1024 + 2048;    // two of queries (row tiles, or limbs), two stages of keys and values
};

// Weights are 2^(s - m + kLift), and m moves when a score exceeds it by more than kSlack: rescaling O costs about as much as a tile, and
// 2^15 is the largest power of two in fp16.  With r up to 2^3 above the row's largest product of weight and scale (a whole number, and the
// unit of values up to 2^2 larger), what lies below 2^-16 (bf16) or 2^-19 (fp32) of that may lose bits, 2^-27 or 2^-30 of it each.
template <typename T>
struct Range {
  static constexpr float kLift = sizeof(T) == 4 ? 8.f : 5.f, kSlack = 15.f - kLift;
};

struct Bars {
  uint64_t q_ready, o_done, drain, k_full[2], k_empty[2], v_full[2], v_empty[2], s_ready[2], p_ready[2][2];
};
// ---- work: full blocks of `rows` rows of a sequence see ever more keys; the sum over the first n of them in closed form
__device__ __forceinline__ int64_t quot(int64_t a, int64_t b) {
  return ((a | b) >> 32) == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b;
}
// sum over 0 <= i < n of floor((a i + b) / m), for non-negative a, b
__device__ __noinline__ int64_t floor_sum(int64_t n, int64_t m, int64_t a, int64_t b) {
  int64_t s = 0;
  while (true) {
    if (a >= m) {
      const int64_t q = quot(a, m);
      s += n * (n - 1) / 2 * q;
      a -= q * m;
    }
    if (b >= m) {
      const int64_t q = quot(b, m);
      s += n * q;
      b -= q * m;
    }
    const int64_t top = a * n + b;
    if (top < m) return s;
    n = quot(top, m);
    b = top - n * m;
    const int64_t t = m;
    m = a;
    a = t;
  }
}
struct Seq {              // the host sees to it that columns and units fit 31 bits
  int begin, len_q, tokens, blocks;
};
__device__ __forceinline__ Seq seq_of(const AttendArgs& a, int b, int rows) {
  Seq s;
  int64_t begin, end;
  rows_of(a.b, b, &begin, &end);
  s.begin = (int)begin;
  s.len_q = (int)(end - begin);
  s.tokens = (int)min(tokens_of(a.b, b, a.c.page_shift), (int64_t)INT32_MAX);
  const int cols = s.len_q * a.g;
  s.blocks = cols > a.most_cols ? (cols + rows - 1) / rows : 0;
  return s;
}
// Keys that row c of the sequence's columns sees.
__device__ __forceinline__ int seen_by(const AttendArgs& a, const Seq& s, int c) { return max(s.tokens - (s.len_q - 1 - c / a.g), 0); }
// Key tiles of the first n blocks.
__device__ __forceinline__ int tiles_before(const AttendArgs& a, const Seq& s, int rows, int n) {
  if (n <= 0) return 0;
  int sum = 0;
  if (n == s.blocks) {   // the last block may be short: it sees all keys
    sum = max((int)(((int64_t)s.tokens + kKeys - 1) / kKeys), 1);
    --n;
  }
  // block k sees vis = c + floor((rows k + rows - 1) / g) keys, c = tokens - len_q + 1, and has max(1, ceil(vis / 128)) tiles
  const int64_t c = (int64_t)s.tokens - s.len_q + 1, m = (int64_t)kKeys * a.g;
  int64_t b = rows - 1 + a.g * (c + kKeys - 1);
  int k0 = 0;
  if (b < m) {           // the first blocks have fewer than one: they count as one
    k0 = (int)min((int64_t)n, quot(m - b + rows - 1, rows));
    sum += k0;
    b += (int64_t)k0 * rows;
  }
  if (n > k0) sum += (int)floor_sum(n - k0, m, rows, b);
  return sum;
}

struct Item {
  int b, head, block;
  int row0, col0;        // first row of Q, first column of the block
  int cols, tiles;       // its columns, its key tiles
  int vis_min, vis_max;  // keys that its first and its last column see
  Seq s;
};
struct Shared {
  Bars bar;
  float2 units[4];                          // of passes, by number: scale of the keys, log2 of the values'
  int flags[4];                             // bits 0-7: 16 keys whose values are NaN; 8-15: of no page, or of another pass; 16: the tile has another pass
  uint32_t tmem;
  int abort_flag;
  int sums[16], found[4];
  Item item[kThreads / 32];                 // what each warp is at: registers are for the scores
};

__device__ __forceinline__ void describe(const AttendArgs& a, int rows, Item* it) {
  it->row0 = it->s.begin;
  it->col0 = it->block * rows;
  it->cols = min(it->s.len_q * a.g - it->col0, rows);
  it->vis_min = seen_by(a, it->s, it->col0);
  it->vis_max = seen_by(a, it->s, it->col0 + it->cols - 1);
  it->tiles = max((int)(((int64_t)it->vis_max + kKeys - 1) / kKeys), 1);
}
__device__ __forceinline__ void next_item(const AttendArgs& a, int rows, Item* it) {   // the caller knows that there is one
  if (++it->block == it->s.blocks) {
    it->block = 0;
    if (++it->head == a.c.heads) {
      it->head = 0;
      do it->s = seq_of(a, ++it->b, rows);
      while (it->s.blocks == 0);
    }
  }
  describe(a, rows, it);
}

// ---- tcgen05 forms that the other kernels do not use
// D (+)= A[tmem] B[smem], fp16 operands.
__device__ __forceinline__ void umma_f16_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tmem_st(uint32_t taddr, const uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
        "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
      : "memory");
}
__device__ __forceinline__ void tmem_st(uint32_t taddr, const uint32_t (&v)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}
// Values as the B operand with n (channels) contiguous: rows of 64 channels per key with the 128-byte swizzle, groups of 8 keys 1,024
// bytes apart, the next 64 channels one panel on.
__device__ __forceinline__ uint64_t desc_values(uint32_t addr) {
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | (uint64_t)(kPanel >> 4) << 16 | (uint64_t)(1024u >> 4) << 32 | (uint64_t)1 << 46 |
         (uint64_t)2 << 61;
}
__host__ __device__ constexpr uint32_t idesc_f16(int n, bool b_n_contiguous) {
  return (1u << 4) | (b_n_contiguous ? 1u << 16 : 0u) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
}

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// Two fp32 operations at a time.
__device__ __forceinline__ uint64_t both(float x) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %1};" : "=l"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ void fma2(uint32_t& x, uint32_t& y, uint64_t f, uint64_t c) {
  uint64_t v;
  asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "r"(x), "r"(y));
  asm("fma.rn.f32x2 %0, %0, %1, %2;" : "+l"(v) : "l"(f), "l"(c));
  asm("mov.b64 {%0, %1}, %2;" : "=r"(x), "=r"(y) : "l"(v));
}
__device__ __forceinline__ void add2(uint64_t& s, float x, float y) {
  uint64_t v;
  asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(x), "f"(y));
  asm("add.rn.f32x2 %0, %0, %1;" : "+l"(s) : "l"(v));
}
__device__ __forceinline__ float sum_of(uint64_t s) {
  float x, y;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(s));
  return x + y;
}
// Eight consecutive elements of a row of queries; `vec`: the row is 16-byte aligned.
template <typename T>
__device__ __forceinline__ void row8(const T* p, bool vec, float (&x)[8]) {
  if (!vec) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (float)p[i];
  } else if (sizeof(T) == 4) {
    const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  } else {
    const uint4 a = __ldg(reinterpret_cast<const uint4*>(p));
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
}
// Whole 32-byte sectors: a warp's rows lie apart, and halves of sectors would cost as much each.
__device__ __forceinline__ void store_sector(void* p, const uint32_t (&w)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
               : "memory");
}
// 32 consecutive results of a row; `vec`: the row is 32-byte aligned.
template <typename T>
__device__ __forceinline__ void store32(T* p, bool vec, const uint32_t (&v)[32], float by) {
  if (!vec) {
#pragma unroll
    for (int e = 0; e < 32; ++e) store_out<T>(p + e, __uint_as_float(v[e]) * by);
  } else if (sizeof(T) == 4) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      uint32_t w[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] = __float_as_uint(__uint_as_float(v[8 * e + j]) * by);
      store_sector(p + 8 * e, w);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      uint32_t w[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(__uint_as_float(v[16 * e + 2 * j]) * by, __uint_as_float(v[16 * e + 2 * j + 1]) * by);
        w[j] = *reinterpret_cast<const uint32_t*>(&h);
      }
      store_sector(p + 16 * e, w);
    }
  }
}

// Four codes times r (a power of two up to 1) as fp16, exactly: (1024 + 128 + x) r - 1152 r for int8.
template <bool E4M3>
__device__ __forceinline__ void expand_scaled(uint32_t w, __half2 r, __half2 minus, uint32_t& lo, uint32_t& hi) {
  if (E4M3) {
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}"
        : "=r"(lo), "=r"(hi) : "r"(w));
    const __half2 x = __hmul2(*reinterpret_cast<const __half2*>(&lo), r), y = __hmul2(*reinterpret_cast<const __half2*>(&hi), r);
    lo = *reinterpret_cast<const uint32_t*>(&x);
    hi = *reinterpret_cast<const uint32_t*>(&y);
  } else {
    w ^= 0x80808080u;
    const uint32_t a = __byte_perm(w, 0x64646464u, 0x4140), b = __byte_perm(w, 0x64646464u, 0x4342);
    const __half2 x = __hfma2(*reinterpret_cast<const __half2*>(&a), r, minus), y = __hfma2(*reinterpret_cast<const __half2*>(&b), r, minus);
    lo = *reinterpret_cast<const uint32_t*>(&x);
    hi = *reinterpret_cast<const uint32_t*>(&y);
  }
}

// Chunk i of lane l: row and 16-byte chunk of 16 rows of codes.  The eight lanes of a phase of the 16-byte stores then write to eight
// different bank groups of the swizzled operand, and a warp reads whole sectors.
template <int D>
__device__ __forceinline__ void place(int i, int l, int* row, int* chunk) {
  if (D == 128) {
    *row = (l & 1) | ((l & 2) << 1) | ((i & 1) << 1) | ((i >> 1) << 3);
    *chunk = l >> 2;
  } else if (D == 64) {
    *row = (l & 1) | ((l & 2) << 1) | ((l >> 4) << 1) | (i << 3);
    *chunk = (l >> 2) & 3;
  } else if (D == 32) {
    *row = (l & 1) | ((l & 2) << 1) | (((l >> 3) & 1) << 1) | ((l >> 4) << 3);
    *chunk = (l >> 2) & 1;
  } else {
    const int x = 32 * i + l;
    *row = x / (D / 16);
    *chunk = x % (D / 16);
  }
}

// A wait has run out: NaN for the softmax thread's row of every item from unit u on.  Out of line, as it hardly ever runs.
template <typename T, int D>
__device__ __noinline__ void rest_is_nan(const AttendArgs& a, Item& it, int u, int u_end, int item_at, int per, int row) {
  const float nan = __uint_as_float(0x7FC00000u);
  while (u < u_end) {
    const int n = min(u_end, item_at + it.tiles) - u;
    const bool whole = u == item_at && u + n == item_at + it.tiles;
    if (row < it.cols) {
      const int c = it.col0 + row, q_head = it.head * a.g + c % a.g;
      const int64_t q_row = it.row0 + c / a.g;
      if (whole) {
        T* out = static_cast<T*>(a.out) + q_row * a.ldo + (int64_t)q_head * a.ho;
#pragma unroll 1
        for (int e = 0; e < D; ++e) store_out<T>(out + e, nan);
        if (a.lse) a.lse[q_row * ((int64_t)a.c.heads * a.g) + q_head] = nan;
      } else {                              // a sum of NaN makes the joined row NaN
        a.part_ml[(int64_t)(2 * (int)blockIdx.x + (u == item_at ? 1 : 0)) * 2 * a.pitch + a.pitch + row] = nan;
      }
    }
    if (!whole && u == item_at && row == 0) {
      Meta* meta = a.meta + blockIdx.x;
      meta->row0 = it.row0;
      meta->col0 = it.col0;
      meta->cols = it.cols;
      meta->head = it.head;
      meta->last_cta = (item_at + it.tiles - 1) / per;
    }
    u += n;
    item_at += it.tiles;
    __syncwarp();
    if ((threadIdx.x & 31) == 0 && u < u_end) next_item(a, Shape<T, D>::kRows, &it);
    __syncwarp();
  }
}

template <typename T, int D, bool E4M3>
__global__ void __launch_bounds__(kThreads, 1) prompt_kernel(const __grid_constant__ AttendArgs a, int* status) {
  using S = Shape<T, D>;
  constexpr int TILES = S::kTiles, LIMBS = S::kLimbs, ROWS = S::kRows;
  constexpr uint32_t OP = S::kOperand;
  extern __shared__ uint8_t raw_smem[];
  uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw_smem) + 1023) & ~(uintptr_t)1023);
  uint8_t* q_sm = base;                     // two operands
  uint8_t* k_sm = base + 2 * OP;            // two stages
  uint8_t* v_sm = base + 4 * OP;
  Shared& sh = *reinterpret_cast<Shared*>(base + 6 * OP);
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  volatile int* abort_flag = &sh.abort_flag;

  if (t == 0) {
    sh.abort_flag = 0;
    tc::mbar_init(&sh.bar.q_ready, 128 * TILES);
    tc::mbar_init(&sh.bar.o_done, 1);
    tc::mbar_init(&sh.bar.drain, 1);
    for (int i = 0; i < 2; ++i) {
      tc::mbar_init(&sh.bar.k_full[i], 32 * kKeyWarps);
      tc::mbar_init(&sh.bar.k_empty[i], 1);
      tc::mbar_init(&sh.bar.v_full[i], 32 * kValueWarps);
      tc::mbar_init(&sh.bar.v_empty[i], 1);
      tc::mbar_init(&sh.bar.s_ready[i], 1);
      for (int h = 0; h < 2; ++h) tc::mbar_init(&sh.bar.p_ready[i][h], 128);
    }
    tc::fence_barrier_init();
  }
  allow_successor();
  wait_for_predecessor();
  if (warp == kMmaWarp) tc::tmem_alloc(&sh.tmem, 512);   // (behind the wait: a kernel ahead may have yet to allocate its own)
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  const uint32_t tmem = sh.tmem;
  // S of row tile x at 128 x, P over its first 64 columns (fp32: the low limb 128 further on); O at 256 + 128 x
  constexpr uint32_t O_COL = 256;

  // ---- this CTA's run of units
  int total = 0, before = 0, own = 0, upto = 0;
  auto block_sum = [&](int v) -> int {      // by all threads: the total, and `upto`, the inclusive sum in order
    int x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    __syncthreads();
    if (lane == 31) sh.sums[warp] = x;
    __syncthreads();
    int all = 0;
    for (int w = 0; w < kThreads / 32; ++w) {
      if (w < warp) x += sh.sums[w];
      all += sh.sums[w];
    }
    upto = x;
    return all;
  };
  auto units_of = [&](int b) -> int {
    if (b >= a.b.nseq) return 0;
    const Seq s = seq_of(a, b, ROWS);
    return tiles_before(a, s, ROWS, s.blocks) * a.c.heads;
  };
#pragma unroll 1
  for (int b0 = 0; b0 < a.b.nseq; b0 += kThreads) {
    own = units_of(b0 + t);
    total += block_sum(own);
  }
  const int per = max((total + (int)gridDim.x - 1) / (int)gridDim.x, 1);
  const int u0 = (int)min((int64_t)blockIdx.x * per, (int64_t)total), u_end = min(total, u0 + per);
  Meta* meta = a.meta + blockIdx.x;
  if (t == 0) meta->last_cta = -1;
  int item_at = 0;
  if (u0 < u_end) {
    Item& it = sh.item[warp];
#pragma unroll 1
    for (int b0 = 0;; b0 += kThreads) {
      int all = total;
      if (a.b.nseq > kThreads) {
        own = units_of(b0 + t);
        all = block_sum(own);
      }
      if (before + all > u0) {
        const int from = before + upto - own;
        if (from <= u0 && u0 < from + own) {
          sh.found[0] = b0 + t;
          sh.found[1] = from;
        }
        __syncthreads();
        break;
      }
      before += all;
    }
    {
      Item start;
      start.b = sh.found[0];
      start.s = seq_of(a, start.b, ROWS);
      const int of_head = tiles_before(a, start.s, ROWS, start.s.blocks), rest = u0 - sh.found[1];
      start.head = rest / of_head;
      const int at = rest - start.head * of_head;
      int lo = 0, hi = start.s.blocks - 1;  // the last block whose first unit is not behind u0
#pragma unroll 1
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (tiles_before(a, start.s, ROWS, mid) <= at) lo = mid; else hi = mid - 1;
      }
      start.block = lo;
      item_at = u0 - at + tiles_before(a, start.s, ROWS, lo);
      describe(a, ROWS, &start);
      if (lane == 0) it = start;
      __syncwarp();
    }

    int u = u0;
    int n_item = 0, n_tile = 0;             // of this CTA, for phases and slots
    bool ok = true;
    auto wait_all = [&](uint64_t* bar, uint32_t parity) -> bool {   // one answer for the whole warp, which goes on together
      const bool mine = tc::mbar_wait(bar, parity, abort_flag, status);
      return __all_sync(0xffffffffu, mine);
    };
    if (warp < 4 * TILES) {
      // ================================================================ softmax: thread r of group `tile` has row tile * 128 + r
      const int tile = warp >> 2, r = t & 127;
      const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16);
      const uint32_t s_col = lanes + 128 * tile, p_lo = lanes + 128, o_col = lanes + O_COL + 128 * tile;
      while (u < u_end && ok) {
        const int n = min(u_end, item_at + it.tiles) - u, first = u - item_at;
        const int row = tile * 128 + r;
        const bool mine = row < it.cols;
        const int c = mine ? it.col0 + row : 0, q_head = it.head * a.g + c % a.g;
        const int64_t q_row = it.row0 + c / a.g;
        const int vis = mine ? seen_by(a, it.s, c) : it.vis_max;
        float f;
        {
          const T* q = static_cast<const T*>(a.q) + q_row * a.ldq + (int64_t)q_head * a.hq;
          const bool vec = (reinterpret_cast<uintptr_t>(q) & 15) == 0;
          uint32_t most = 0u;
          if (mine)
#pragma unroll 8
            for (int i = 0; i < D / 8; ++i) {
              float x[8];
              row8(q + 8 * i, vec, x);
#pragma unroll
              for (int j = 0; j < 8; ++j) most = max(most, __float_as_uint(x[j]) & 0x7FFFFFFFu);
            }
          float inv;
          const float s = query_scale(most, &inv);
          // a negative scale goes into the queries: the largest sum is then the largest score
          // a row with an infinity or a NaN has scores of NaN where it sees something: through the queries, so that f leaves -inf what it is
          const bool number = most < 0x7F800000u && fabsf(a.scale) < TQ_INF;
          f = number ? s * fabsf(a.scale * kLog2e) : 1.f;
          inv = !number ? __uint_as_float(0x7FC00000u) : (a.scale < 0.f ? -inv : inv);
#pragma unroll 2
          for (int i = 0; i < D / 8; ++i) {
            float x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = 0.f;
            if (mine) row8(q + 8 * i, vec, x);
            uint32_t hi[4], lo_[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float y = x[2 * j] * inv, z = x[2 * j + 1] * inv;
              hi[j] = pack2(y, z);
              const float2 back = __half22float2(*reinterpret_cast<const __half2*>(&hi[j]));
              lo_[j] = pack2(y - back.x, z - back.y);
            }
            const uint32_t at = (uint32_t)(i >> 3) * kPanel + (uint32_t)r * 128 + (uint32_t)(((i & 7) ^ (r & 7)) << 4);
            *reinterpret_cast<uint4*>(q_sm + tile * OP + at) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
            if (LIMBS == 2) *reinterpret_cast<uint4*>(q_sm + OP + at) = make_uint4(lo_[0], lo_[1], lo_[2], lo_[3]);
          }
        }
        tc::fence_proxy_async();
        tc::mbar_arrive(&sh.bar.q_ready);
        float m = -TQ_INF, mv = -TQ_INF, l = 0.f;
        bool fresh = true;                  // O holds nothing yet
        for (int i = 0; i < n;) {
          const int nt = n_tile++;
          ok = wait_all(&sh.bar.s_ready[tile], nt & 1);
          if (!ok) break;
          tc::tc_fence_after();
          const int t0 = (first + i) * kKeys, flags = sh.flags[nt & 3];
          const float2 unit = sh.units[nt & 3];
          const bool edge = t0 + kKeys > it.vis_min || (flags & 0xFFFF) != 0;
          const float factor = fmaxf(f * unit.x, 1e-30f);   // keys of zeros: all scores are (nearly) 0, and -inf stays what it is
          uint32_t v[2][32];
          auto load_half = [&](int half) {
            tc::tmem_ld32(s_col + 64 * half, v[0]);
            tc::tmem_ld32(s_col + 64 * half + 32, v[1]);
            tc::tmem_ld_wait();
            if (edge) {                     // keys that the row does not see: -inf
#pragma unroll
              for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 32; ++e)
                  if (t0 + 64 * half + 32 * j + e >= vis || ((flags >> (8 + 4 * half + 2 * j + (e >> 4))) & 1)) v[j][e] = 0xFF800000u;
            }
          };
          auto largest = [&]() -> float {
            float x[4];
#pragma unroll
            for (int g = 0; g < 4; ++g) x[g] = __uint_as_float(v[g >> 1][16 * (g & 1)]);
#pragma unroll
            for (int e = 1; e < 15; e += 2)
#pragma unroll
              for (int g = 0; g < 4; ++g)
                x[g] = fmaxf(fmaxf(x[g], __uint_as_float(v[g >> 1][16 * (g & 1) + e])), __uint_as_float(v[g >> 1][16 * (g & 1) + e + 1]));
#pragma unroll
            for (int g = 0; g < 4; ++g) x[g] = fmaxf(x[g], __uint_as_float(v[g >> 1][16 * (g & 1) + 15]));
            return fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
          };
          // Loops that are not unrolled keep the code of all roles small: instructions are fetched while operands wait (618 us against 688)
          float top = -TQ_INF;
#pragma unroll 1
          for (int half = 1; half >= 0; --half) {   // the first half stays
            load_half(half);
            top = fmaxf(top, largest());
          }
          top *= factor;
          const float top_v = top + unit.y;
          const bool higher = top > m + Range<T>::kSlack || top_v > mv + Range<T>::kSlack;
          if (__any_sync(0xffffffffu, higher)) {
            float alpha = 1.f;
            if (higher) {
              const float new_m = fmaxf(m, ceilf(top)), new_v = fmaxf(mv, ceilf(top_v));
              if (new_m > m) l *= ex2(m - new_m);                                 // from -inf: 0
              if (new_v > mv) alpha = ex2(mv - new_v);
              m = new_m;
              mv = new_v;
            }
            if (!fresh) {                   // O is at rest: these scores were asked for after its last sum
#pragma unroll 1
              for (int j = 0; j < D / 16; ++j) {
                uint32_t w[16];
                tc::tmem_ld16(o_col + 16 * j, w);
                tc::tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 16; ++e) w[e] = __float_as_uint(__uint_as_float(w[e]) * alpha);
                tmem_st(o_col + 16 * j, w);
              }
            }
          }
          // p relative to r, but for what lies 2^60 below it: that rounds to 0 in P, and must not in l
          const float below = fmaxf(m - mv + unit.y, -60.f), shift = m == -TQ_INF ? 0.f : Range<T>::kLift - m + below;
          const uint64_t f2 = both(factor), shift2 = both(shift);
          uint64_t sum[2] = {0ull, 0ull};
          constexpr int W = LIMBS == 2 ? 16 : 32;   // keys per store: registers are scarce
          auto weights = [&](auto is_edge, int half) {
#pragma unroll
            for (int g = 0; g < 64 / W; ++g) {
              uint32_t p[W / 2], pl[W / 2];
#pragma unroll
              for (int e = 0; e < W; e += 2) {
                const int key = W * g + e;
                uint32_t &z0 = v[key >> 5][key & 31], &z1 = v[key >> 5][(key & 31) + 1];
                fma2(z0, z1, f2, shift2);
                float x = ex2(__uint_as_float(z0)), y = ex2(__uint_as_float(z1));
                add2(sum[(e >> 1) & 1], x, y);
                // values of a NaN block are zeros in the operand: the weight carries the NaN to the rows that see the block
                if (decltype(is_edge)::value && ((flags >> (4 * half + (key >> 4))) & 1) && t0 + 64 * half + key < vis) x = __uint_as_float(0x7FC00000u);
                p[e >> 1] = pack2(x, y);
                if (LIMBS == 2) {
                  const float2 back = __half22float2(*reinterpret_cast<const __half2*>(&p[e >> 1]));
                  pl[e >> 1] = pack2(x - back.x, y - back.y);
                }
              }
              tmem_st(s_col + 32 * half + W / 2 * g, p);   // over scores that have been read
              if (LIMBS == 2) tmem_st(p_lo + 32 * half + W / 2 * g, pl);
            }
            tc::tmem_st_wait();
            tc::tc_fence_before();
            tc::mbar_arrive(&sh.bar.p_ready[tile][half]);   // the first half is multiplied while the second is computed
          };
#pragma unroll 1
          for (int half = 0; half < 2; ++half) {
            load_half(half);
            if (edge) weights(std::true_type{}, half); else weights(std::false_type{}, half);
          }
          l += (sum_of(sum[0]) + sum_of(sum[1])) * ex2(-below);
          fresh = false;
          i += 1 - (flags >> 16);
        }
        if (ok) ok = wait_all(&sh.bar.o_done, n_item & 1);
        const bool good = ok;
        tc::tc_fence_after();
        const bool whole = u == item_at && u + n == item_at + it.tiles;
        const int slot = 2 * (int)blockIdx.x + (u == item_at ? 1 : 0);
        // an average of the values (parts are averages too); in two steps, as the power may be out of range
        const float x = mv == -TQ_INF ? 0.f : mv - m, x0 = floorf(0.5f * x), by0 = ex2(x0);
        const float by = !good ? __uint_as_float(0x7FC00000u) : (l == 0.f ? 0.f : ex2(x - x0) / l);
        T* out = static_cast<T*>(a.out) + q_row * a.ldo + (int64_t)q_head * a.ho;
        const bool vec_out = (reinterpret_cast<uintptr_t>(out) & 31) == 0;
        float* part = a.part_o + ((int64_t)slot * a.pitch + row) * D;
#pragma unroll 1
        for (int j = 0; j < D / 32; ++j) {
          uint32_t v[32];
          tc::tmem_ld32(o_col + 32 * j, v);
          tc::tmem_ld_wait();
          if (mine) {
#pragma unroll
            for (int e = 0; e < 32; ++e) v[e] = l == 0.f && good ? 0u : __float_as_uint(__uint_as_float(v[e]) * by0);
            if (whole) {
              store32<T>(out + 32 * j, vec_out, v, by);
            } else {
              store32<float>(part + 32 * j, true, v, by);
            }
          }
        }
        if (mine) {
          if (!whole) {
            a.part_ml[(int64_t)slot * 2 * a.pitch + row] = m;
            a.part_ml[(int64_t)slot * 2 * a.pitch + a.pitch + row] = good ? l : by;
          } else if (a.lse) {
            a.lse[q_row * ((int64_t)a.c.heads * a.g) + q_head] =
                !good ? by : (l == 0.f ? -TQ_INF : (m == -TQ_INF ? 0.f : (m - Range<T>::kLift) * kLn2) + logf(l));
          }
        }
        if (!whole && u == item_at && t == 0) {
          meta->row0 = it.row0;
          meta->col0 = it.col0;
          meta->cols = it.cols;
          meta->head = it.head;
          meta->last_cta = (item_at + it.tiles - 1) / per;
        }
        tc::tc_fence_before();
        ++n_item;
        u += n;
        item_at += it.tiles;
        __syncwarp();
        if (lane == 0 && u < u_end) next_item(a, ROWS, &it);
        __syncwarp();
      }
      if (!ok) rest_is_nan<T, D>(a, it, u, u_end, item_at, per, tile * 128 + r);
    } else if (warp >= kExpandWarp0 && warp < kMmaWarp) {
      // ================================================================ codes -> fp16 operands
      const bool isv = warp >= kExpandWarp0 + kKeyWarps;
      // takes keys 16 g .. 16 g + 15 of a tile for g = we, we + stride, ..
      const int we = warp - kExpandWarp0 - (isv ? kKeyWarps : 0), stride = isv ? kValueWarps : kKeyWarps;
      constexpr int G = 3, N = D / 32;      // at most; 16-byte chunks per lane of 16 keys
      uint64_t *full = isv ? sh.bar.v_full : sh.bar.k_full, *empty = isv ? sh.bar.v_empty : sh.bar.k_empty;
      uint8_t* operand = isv ? v_sm : k_sm;
      while (u < u_end && ok) {
        const int n = min(u_end, item_at + it.tiles) - u, first = u - item_at;
        const int32_t* row_pages = a.b.table + (int64_t)it.b * a.b.ldt;
        uint4 raw[G][N];
        // what lane l < 8 knows of keys 16 l .. 16 l + 15 of a tile: page and scales; looked up two tiles ahead
        struct Known { int id; float ks, vs; };
        auto look_up = [&](int tile_no) -> Known {
          Known x{-1, 0.f, 0.f};
          const int64_t t0 = (int64_t)tile_no * kKeys + 16 * (lane & 7);
          if (tile_no < first + n && t0 < it.vis_max) {
            const int id = row_pages[t0 >> a.c.page_shift];
            if (id >= 0 && id < a.c.pages) {
              x.id = id;
              x.ks = a.c.k_scale[(int64_t)id * a.c.heads + it.head];
              x.vs = a.c.v_scale[(int64_t)id * a.c.heads + it.head];
            }
          }
          return x;
        };
        const int64_t head_bytes = (int64_t)D << a.c.page_shift, page_bytes = head_bytes * a.c.heads;
        const uint8_t* codes = (isv ? a.c.v : a.c.k) + it.head * head_bytes;
        auto read = [&](int id8, int tile_no, uint4 (&x)[G][N]) {
#pragma unroll
          for (int g = 0; g < G; ++g) {
            const int grp = we + stride * g, id = __shfl_sync(0xffffffffu, id8, grp & 7);
            const int t0 = tile_no * kKeys + 16 * grp;
            const uint8_t* from = codes + id * page_bytes + (t0 & ((1 << a.c.page_shift) - 1)) * D;
            if (grp < 8 && id >= 0 && t0 + 16 <= it.vis_max) {
#pragma unroll
              for (int i = 0; i < N; ++i) {
                int row, chunk;
                place<D>(i, lane, &row, &chunk);
                x[g][i] = __ldg(reinterpret_cast<const uint4*>(from + row * D + 16 * chunk));
              }
            } else {                        // no page, or keys behind the last one: zeros
#pragma unroll
              for (int i = 0; i < N; ++i) {
                int row, chunk;
                place<D>(i, lane, &row, &chunk);
                x[g][i] = make_uint4(0u, 0u, 0u, 0u);
                if (grp < 8 && id >= 0 && t0 + row < it.vis_max) x[g][i] = __ldg(reinterpret_cast<const uint4*>(from + row * D + 16 * chunk));
              }
            }
          }
        };
        auto write = [&](uint8_t* base, const uint4 (&x)[G][N], float ratio) {
#pragma unroll
          for (int g = 0; g < G; ++g) {
            const int grp = we + stride * g;
            float r = __shfl_sync(0xffffffffu, ratio, grp & 7);
            if (grp >= 8) continue;
            const __half2 r2 = __float2half2_rn(r), minus = __float2half2_rn(-1152.f * r);
#pragma unroll
            for (int i = 0; i < N; ++i) {
              int row, chunk;
              place<D>(i, lane, &row, &chunk);
              const uint32_t w[4] = {x[g][i].x, x[g][i].y, x[g][i].z, x[g][i].w};
              uint32_t y[8];
#pragma unroll
              for (int j = 0; j < 4; ++j) expand_scaled<E4M3>(w[j], r2, minus, y[2 * j], y[2 * j + 1]);
              uint8_t* to = base + (uint32_t)(chunk >> 2) * kPanel + (uint32_t)(16 * grp + row) * 128;
              const int piece = (chunk & 3) * 2;
              *reinterpret_cast<uint4*>(to + ((piece ^ (row & 7)) << 4)) = make_uint4(y[0], y[1], y[2], y[3]);
              *reinterpret_cast<uint4*>(to + (((piece + 1) ^ (row & 7)) << 4)) = make_uint4(y[4], y[5], y[6], y[7]);
            }
          }
        };
        Known now = look_up(first), next = look_up(first + 1);
        read(now.id, first, raw);
        bool left = true;                   // these keys have not been in a pass
        for (int i = 0; i < n;) {
          // units of what is left: scales are positive, so their bits are in their order; keys of 0, and NaN, go with any unit
          const float uk = __uint_as_float(__reduce_max_sync(0xffffffffu, left && now.ks > 0.f ? __float_as_uint(now.ks) : 0u));
          bool in = left && !(now.ks < uk * 0x1p-15f && now.ks > 0.f);
          const float uv = __uint_as_float(__reduce_max_sync(0xffffffffu, in && now.vs > 0.f ? __float_as_uint(now.vs) : 0u));
          in = in && !(now.vs < uv * 0.25f && now.id >= 0);
          const bool again = __any_sync(0xffffffffu, left && !in);
          left = left && !in;
          in = in && now.id >= 0;
          const float x = isv ? now.vs : now.ks, r = !in || (isv && !(x == x)) ? 0.f : x * block_inverse(isv ? uv : uk);
          const int nt = n_tile++, st = nt & 1;
          const int flags = (int)((again ? 1u << 16 : 0u) | (__ballot_sync(0xffffffffu, !in) & 0xFFu) << 8 |
                                  (__ballot_sync(0xffffffffu, in && !(now.vs == now.vs)) & 0xFFu));
          ok = wait_all(&empty[st], ((nt >> 1) & 1) ^ 1);
          if (!ok) break;
          if (!isv && we == 0 && lane == 0) {
            sh.flags[nt & 3] = flags;
            sh.units[nt & 3] = make_float2(uk, uv > 0.f ? scale_log2(uv) : -126.f);
          }
          write(operand + st * OP, raw, r);
          tc::fence_proxy_async();
          tc::mbar_arrive(&full[st]);
          if (!again) {                     // else the same codes once more
            left = true;
            now = next;
            ++i;
            next = look_up(first + i + 1);
          }
          read(now.id, first + i, raw);
        }
        ++n_item;
        u += n;
        item_at += it.tiles;
        __syncwarp();
        if (lane == 0 && u < u_end) next_item(a, ROWS, &it);
        __syncwarp();
      }
    } else if (warp == kMmaWarp && lane == 0) {
      // ================================================================ MMAs
      constexpr uint32_t id_s = idesc_f16(kKeys, false), id_o = idesc_f16(D, true);
      if (a.give_up) {                      // self test: nothing is issued, so that every wait for it runs out
        sh.abort_flag = 1;
        ok = false;
      }
      const uint32_t q_at = tc::smem_u32(q_sm), k_at = tc::smem_u32(k_sm), v_at = tc::smem_u32(v_sm);
      auto scores = [&](int tile, int st) {
#pragma unroll
        for (int x = 0; x < LIMBS; ++x)
#pragma unroll
          for (int k = 0; k < D / 16; ++k) {
            const uint32_t off = (uint32_t)(k >> 2) * kPanel + (uint32_t)(k & 3) * 32;
            tc::umma_bf16(tmem + 128 * tile, tc::smem_desc_sw128(q_at + (tile + x) * OP + off), tc::smem_desc_sw128(k_at + st * OP + off), id_s,
                          (x | k) != 0 ? 1u : 0u);
          }
        tc::umma_commit(&sh.bar.s_ready[tile]);
      };
      auto sums = [&](int tile, int half, int st, bool fresh) {
#pragma unroll
        for (int x = 0; x < LIMBS; ++x)
#pragma unroll
          for (int k = 0; k < 4; ++k)
            umma_f16_ts(tmem + O_COL + 128 * tile, tmem + 128 * (tile + x) + 32 * half + 8 * k, desc_values(v_at + st * OP + 8192 * half + 2048 * k), id_o,
                        !fresh || (x | k) != 0 ? 1u : 0u);
      };
      while (u < u_end && ok) {
        const int n = min(u_end, item_at + it.tiles) - u;
        ok = tc::mbar_wait(&sh.bar.q_ready, n_item & 1, abort_flag, status) &&
             tc::mbar_wait(&sh.bar.k_full[n_tile & 1], (n_tile >> 1) & 1, abort_flag, status);
        if (!ok) break;
        tc::tc_fence_after();
#pragma unroll
        for (int tile = 0; tile < TILES; ++tile) scores(tile, n_tile & 1);
        tc::umma_commit(&sh.bar.k_empty[n_tile & 1]);
        bool fresh = true;
        for (int i = 0; i < n && ok;) {
          const int nt = n_tile++, st = nt & 1;
          i += 1 - (sh.flags[nt & 3] >> 16);     // the pass's keys are there, so its flags are
#pragma unroll
          for (int part = 0; part < 2 * TILES; ++part) {   // the groups are half a tile apart: 0 first half, 0 second, 1 first, 1 second
            const int tile = part >> 1, half = part & 1;
            ok = ok && tc::mbar_wait(&sh.bar.p_ready[tile][half], nt & 1, abort_flag, status);
            if (part == 0) ok = ok && tc::mbar_wait(&sh.bar.v_full[st], (nt >> 1) & 1, abort_flag, status);
            if (!ok) break;
            tc::tc_fence_after();
            sums(tile, half, st, fresh && half == 0);
            if (half == 1 && i < n) {
              if (tile == 0) ok = tc::mbar_wait(&sh.bar.k_full[(nt + 1) & 1], ((nt + 1) >> 1) & 1, abort_flag, status);
              if (!ok) break;
              tc::tc_fence_after();
              scores(tile, (nt + 1) & 1);
            }
          }
          if (!ok) break;
          fresh = false;
          tc::umma_commit(&sh.bar.v_empty[st]);
          if (i < n) tc::umma_commit(&sh.bar.k_empty[(nt + 1) & 1]);
        }
        if (ok) tc::umma_commit(&sh.bar.o_done);
        ++n_item;
        u += n;
        item_at += it.tiles;
        if (u < u_end) next_item(a, ROWS, &it);
      }
      if (!ok) {   // what was issued still reads shared memory and writes TMEM (else the softmax groups have waited for the last commit)
        volatile int never = 0;
        tc::umma_commit(&sh.bar.drain);
        tc::mbar_wait_slow(&sh.bar.drain, 0, &never, status);
      }
    }
  }
  __syncwarp();
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  if (warp == kMmaWarp) tc::tmem_dealloc(tmem, 512);
}

template <typename T, int D, bool E4M3>
cudaError_t launch(const AttendArgs& a, int* status, int sms, cudaStream_t st) {
  static std::atomic<unsigned long long> devices{0};
  const cudaError_t e = allow_largest_smem(reinterpret_cast<const void*>(prompt_kernel<T, D, E4M3>), devices);
  if (e != cudaSuccess) return e;
  return launch_dependent(prompt_kernel<T, D, E4M3>, dim3((unsigned)sms), dim3(kThreads), Shape<T, D>::smem, st, a, status);
}
template <typename T>
cudaError_t launch_t(const AttendArgs& a, bool e4m3, int* status, int sms, cudaStream_t st) {
  switch (a.c.d) {
    case 32: return e4m3 ? launch<T, 32, true>(a, status, sms, st) : launch<T, 32, false>(a, status, sms, st);
    case 64: return e4m3 ? launch<T, 64, true>(a, status, sms, st) : launch<T, 64, false>(a, status, sms, st);
    case 96: return e4m3 ? launch<T, 96, true>(a, status, sms, st) : launch<T, 96, false>(a, status, sms, st);
    default: return e4m3 ? launch<T, 128, true>(a, status, sms, st) : launch<T, 128, false>(a, status, sms, st);
  }
}

struct Space {
  size_t ml, o, status, bytes;
};
Space lay_out(int sms, int d) {
  Space s;
  s.ml = (size_t)round_up64((int64_t)sms * sizeof(Meta), 256);
  s.o = s.ml + (size_t)round_up64((int64_t)sms * 2 * 2 * kPromptRows * sizeof(float), 256);
  s.status = s.o + (size_t)sms * 2 * kPromptRows * d * sizeof(float);
  s.bytes = s.status + 256;
  return s;
}

}  // namespace

size_t prompt_space(int sms, int d) { return lay_out(sms, d).bytes; }

cudaError_t launch_prompt(AttendArgs& a, int dtype, bool e4m3, int sms, void* workspace, cudaStream_t st) {
  const Space s = lay_out(sms, a.c.d);
  char* w = static_cast<char*>(workspace);
  a.meta = reinterpret_cast<Meta*>(w);
  a.part_ml = reinterpret_cast<float*>(w + s.ml);
  a.part_o = reinterpret_cast<float*>(w + s.o);
  a.pitch = kPromptRows;
  a.lift = dtype == TQ_F32 ? Range<float>::kLift : Range<__nv_bfloat16>::kLift;
  a.give_up = give_up.load(std::memory_order_relaxed);
  int* status = reinterpret_cast<int*>(w + s.status);   // only written: a CTA whose wait ran out says so with NaN
  const cudaError_t e = dtype == TQ_F32 ? launch_t<float>(a, e4m3, status, sms, st) : launch_t<__nv_bfloat16>(a, e4m3, status, sms, st);
  if (e != cudaSuccess) return e;
  return launch_join(a, dtype, sms, dtype == TQ_F32 ? 128 : 256, st);
}

}  // namespace kv8
}  // namespace tq

extern "C" int tq_selftest_kv8_timeout(int on) {
  tq::kv8::give_up.store(on != 0, std::memory_order_relaxed);
  return TQ_OK;
}
