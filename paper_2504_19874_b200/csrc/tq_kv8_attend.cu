// Attention over a paged 8-bit KV cache for few queries per sequence (decoding, drafted tokens, listed pages).
//
// Mathematics.  Columns are the queries that share a KV head (q_per_kv heads of up to a few tokens, 8 or 16 at a time); per 16 tokens
//   S^T = K Q^T   (16 tokens x 8 columns, one mma per 16 channels: the codes are the A operand, converted to fp16 exactly),
//   l += 2^(s - m + 6) with the column's running maximum m,   p = 2^(s + log2 v - r + 6),   O^T += V^T P^T
// (P^T is S^T transposed in registers), v the scale of the tile's values and r the column's running maximum of s + log2 v: what goes into
// the matrix product is a weight times a scale, relative to the largest such product so far, so neither a page of far larger or
// smaller values nor its order can push the others' bits out of fp16 or the sums out of fp32.  out = O 2^(r - m) / l.
// m and r are whole numbers and only rise, when a score exceeds one of them by 2^8, so most steps rescale nothing and those that do
// multiply by exact powers of two up to 1; p <= 2^14 stays inside fp16.
// Queries are scaled per row by a power of two into [2^13, 2^14): bf16 values are then exact in fp16 (an element 2^-30 of the row's
// largest loses bits), and fp32 values are two fp16 limbs (2^-23 of each value).  P is one fp16 limb for bf16 outputs (2^-12 of each
// weight, an eighth of the output's own rounding) and two for fp32 ones.  All sums are fp32.
// Scales are powers of two: the key's goes into the score's factor, the value's into p's exponent, both exactly.
//
// Work.  Units of 64 tokens of one (sequence, head) are numbered through; every CTA takes an equal share of them, whatever the lengths,
// and of a unit each of its four warps takes 16 tokens, through a ring of its own in shared memory, some steps ahead.  Warps are
// independent until their share of an item ends; items that several CTAs share are joined by a second, dependent launch in a fixed order.
//
// Measured, one B200, 8 KV heads x 4 queries, d = 128: 37 sequences of 8,192 tokens stream at 5.2 TB/s, a ragged batch of 64 (563 MB) at
// 4.8 TB/s (118 us; 0.73 of the copy bandwidth), one sequence of 32,768 tokens 28 us, of which the loop takes 10 us at the copy bandwidth
// and the chain of first loads, the last sums and the join the rest; 1,000 tokens 9.7 us.  Reading the tiles straight into registers,
// one step ahead, took 228 us for the batch and 43 us for the layer: eight warps per SM had too few bytes on their way.  Long calls
// are bound by HBM (63 % of its cycles in the batch's kernel); half of the issue slots are in use meanwhile.
#include <algorithm>
#include <cstring>

#include "tq_kv8.h"
#include "tq_kv8_attend.h"

namespace tq {
namespace kv8 {
namespace {

constexpr int kWarps = 4, kThreads = kWarps * 32;
constexpr int kUnit = 64;                // tokens
__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint32_t half2_bits(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// Bytes 0, 1 and bytes 2, 3 of a word of codes as pairs of fp16, exactly.  int8: the byte plus 128 is the low byte of 1024 + 128 + x.
template <bool E4M3>
__device__ __forceinline__ void expand(uint32_t w, uint32_t& lo, uint32_t& hi) {
  if (E4M3) {
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}"
        : "=r"(lo), "=r"(hi) : "r"(w));
  } else {
    w ^= 0x80808080u;
    const uint32_t a = __byte_perm(w, 0x64646464u, 0x4140), b = __byte_perm(w, 0x64646464u, 0x4342);
    const __half2 k = __halves2half2(__ushort_as_half(0x6480), __ushort_as_half(0x6480));   // 1152
    const __half2 x = __hsub2(*reinterpret_cast<const __half2*>(&a), k), y = __hsub2(*reinterpret_cast<const __half2*>(&b), k);
    lo = *reinterpret_cast<const uint32_t*>(&x);
    hi = *reinterpret_cast<const uint32_t*>(&y);
  }
}

template <int W>
__device__ __forceinline__ void load_words(const uint8_t* p, uint32_t* w) {   // W words, aligned to the largest power of two in their bytes
  if (W % 4 == 0) {
#pragma unroll
    for (int i = 0; i < W / 4; ++i) {
      const uint4 v = reinterpret_cast<const uint4*>(p)[i];
      w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
    }
  } else if (W % 2 == 0) {
#pragma unroll
    for (int i = 0; i < W / 2; ++i) {
      const uint2 v = reinterpret_cast<const uint2*>(p)[i];
      w[2 * i] = v.x; w[2 * i + 1] = v.y;
    }
  } else {
#pragma unroll
    for (int i = 0; i < W; ++i) w[i] = reinterpret_cast<const uint32_t*>(p)[i];
  }
}
__device__ __forceinline__ void copy16(uint32_t to, const void* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t to, const void* from) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to), "l"(from) : "memory");
}
// Where 16-byte chunk x of row r of a warp's tile is kept: the lanes of a phase of the reads below then touch different banks.
template <int D>
__device__ __forceinline__ int key_chunk(int r, int x) {
  return r * (D / 16) + (D == 128 ? x ^ ((r & 1) << 2) : x);
}
template <int D>
__device__ __forceinline__ int value_chunk(int r, int x) {
  return r * (D / 16) + (D == 128 ? x ^ (r & 6) : (D == 64 ? x ^ (r & 2) : x));
}

// Units of sequence b (all heads and column blocks).  Sequences whose queries go to the many-query kernel have none here.
struct Shape {
  int64_t begin, end, tokens;   // rows, cached tokens
  int blocks;                   // blocks of NC columns
  int units;                    // of one (head, block); the host sees to it that all of a call's units fit 31 bits
};
__device__ __forceinline__ Shape shape_of(const AttendArgs& a, int b, int nc) {
  Shape s;
  rows_of(a.b, b, &s.begin, &s.end);
  s.tokens = tokens_of(a.b, b, a.c.page_shift);
  const int64_t cols = (s.end - s.begin) * a.g;
  s.blocks = cols > a.most_cols ? 0 : (int)((cols + nc - 1) / nc);   // nc is a constant power of two
  s.units = s.blocks == 0 ? 0 : max((int)((s.tokens + kUnit - 1) / kUnit), 1);   // without tokens: one, for the zeros
  return s;
}

__device__ __forceinline__ int block_total(int v, int* sums, int* upto) {   // inclusive sum in order, and the total
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 31) sums[warp] = x;
  __syncthreads();
  int all = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w < warp) x += sums[w];
    all += sums[w];
  }
  *upto = x;
  return all;
}

template <typename T, int D, bool E4M3, int NT>
struct Kernel {
  static constexpr int kLimbs = sizeof(T) == 4 ? 2 : 1;
  static constexpr int NC = 8 * NT;
  static constexpr int KW = D / 16;                       // words of a key row per lane
  static constexpr int KS = D % 64 == 0 ? 4 : 2;          // ... in pieces of that many
  static constexpr int VW = D / 32;                       // words of a value row per lane
  static constexpr int QP = D + 8;                        // pitch of the queries in shared memory, halves
  static constexpr int OP = D + 4;                        // pitch of the warps' results, floats
  static constexpr int kTile = 2 * 16 * D + 16;           // bytes of a warp's stage: keys, values, the two scales
  static constexpr int kStages = D >= 96 ? 4 : 5;
  // 168 registers a thread and a ring of 66 KB let three CTAs share an SM; two fp16 limbs of 16 columns need more
  static constexpr int kCtas = D >= 96 && NT == 2 && kLimbs == 2 ? 2 : 3;
  static constexpr size_t q_bytes = sizeof(__half) * kLimbs * NC * QP;
  static constexpr size_t o_bytes = sizeof(float) * kWarps * NC * OP;
  static constexpr size_t ring = (size_t)kWarps * kStages * kTile;
  static constexpr size_t head = ring > o_bytes ? ring : o_bytes;   // the results take the ring's place
  static constexpr size_t smem = head + q_bytes + sizeof(float) * (2 * kWarps + 3) * NC + 256;
};

template <typename T, int D, bool E4M3, int NT>
__global__ void __launch_bounds__(kThreads, Kernel<T, D, E4M3, NT>::kCtas) attend_kernel(const __grid_constant__ AttendArgs a) {
  using K = Kernel<T, D, E4M3, NT>;
  constexpr int NC = K::NC, KW = K::KW, KS = K::KS, VW = K::VW, LIMBS = K::kLimbs;
  extern __shared__ uint4 smem4[];
  float* osm = reinterpret_cast<float*>(smem4);
  __half* qsm = reinterpret_cast<__half*>(reinterpret_cast<char*>(smem4) + K::head);
  float* msm = reinterpret_cast<float*>(reinterpret_cast<char*>(qsm) + K::q_bytes);   // [warps][NC]
  float* lsm = msm + kWarps * NC;
  float* fsm = lsm + kWarps * NC;       // [NC] factor of a column's scores
  float* top = fsm + NC;                // [NC] maximum, then sum, of all warps
  float* tot = top + NC;
  int* sums = reinterpret_cast<int*>(tot + NC);   // [8]
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5, c4 = lane & 3, n8 = lane >> 2;
  const int cta = blockIdx.x;
  allow_successor();
  wait_for_predecessor();

  // ---- this CTA's share [u, u_end) of all units, and the item that u falls into
  int seq = 0, head = 0, block = 0;
  int item_at = 0;                      // first unit of the item
  int total = 0, per;
  Shape sh;
  int list_units = 0;
  const int T_ = 1 << a.c.page_shift;
  const int grid = gridDim.x;
  // A share that ends one item and begins the next pays for its first loads and last sums twice, about as much as kCross units.  Where
  // there are fewer items than CTAs, shares are therefore laid so that each lies within one item (items count as a multiple of `per`
  // then, the units behind their end being empty), unless that makes them longer by more than that: nine sequences of up to five
  // tokens 19.8 -> 18.0 us, 32,768 tokens 27.7 -> 27.4, the pages of 24 rows 43.1 -> 42.4 (as it was added).
  constexpr int kCross = 4;
  int pad = 1;                          // units of an item are counted up to a multiple of this
  auto padded = [&](int units) -> int { return pad == 1 ? units : (units + pad - 1) / pad * pad; };
  if (a.lists == nullptr) {
    int upto = 0, own = 0;
    auto units_of = [&](int b) -> int {
      if (b >= a.b.nseq) return 0;
      const Shape s = shape_of(a, b, NC);
      return s.units * s.blocks * a.c.heads;
    };
    if (a.b.nseq <= kThreads) {
      Shape s;
      s.units = s.blocks = 0;
      if (t < a.b.nseq) s = shape_of(a, t, NC);
      const int items_of = s.units > 0 ? s.blocks * a.c.heads : 0;
      own = s.units * items_of;
      total = block_total(own, sums, &upto);
      per = max((total + grid - 1) / grid, 1);
      if (per > 1) {
        int before;
        const int items = block_total(items_of, sums, &before);
        if (items < grid) {             // each item ends in at most one share that is not full
          const int even = (total + grid - items - 1) / (grid - items);
          if (even <= per + kCross) {
            per = pad = even;
            own = padded(s.units) * items_of;
            total = block_total(own, sums, &upto);
          }
        }
      }
    } else {
#pragma unroll 1
      for (int b0 = 0; b0 < a.b.nseq; b0 += kThreads) {
        own = units_of(b0 + t);
        total += block_total(own, sums, &upto);
      }
      per = max((total + grid - 1) / grid, 1);
    }
    const int u0 = cta * per;
    if (u0 < total) {
      int before = 0;
#pragma unroll 1
      for (int b0 = 0;; b0 += kThreads) {
        int all = total;
        if (a.b.nseq > kThreads) {
          own = units_of(b0 + t);
          all = block_total(own, sums, &upto);
        }
        if (before + all > u0) {
          const int from = before + upto - own;
          if (from <= u0 && u0 < from + own) {
            sums[4] = b0 + t;
            sums[5] = from;
          }
          __syncthreads();
          break;
        }
        before += all;
      }
      seq = sums[4];
      const int from = sums[5];
      sh = shape_of(a, seq, NC);
      sh.units = padded(sh.units);
      const int i = (u0 - from) / sh.units;
      head = i / sh.blocks;
      block = i - head * sh.blocks;
      item_at = from + i * sh.units;
    }
  } else {                               // rows x heads x blocks of columns, each of as many units as a list holds
    int64_t rows = a.b.nseq;
    if (a.b.starts != nullptr) {
      rows = a.b.starts[a.b.nseq];
      rows = rows < 0 ? 0 : (rows > a.b.n ? a.b.n : rows);
    }
    sh.blocks = (a.g + NC - 1) / NC;
    list_units = max((int)((((int64_t)a.nlist << a.c.page_shift) + kUnit - 1) / kUnit), 1);
    const int of_row = a.c.heads * sh.blocks, items = (int)rows * of_row;
    per = max((items * list_units + grid - 1) / grid, 1);
    if (per > 1 && items <= grid) {
      const int shares = min(grid / items, list_units), even = (list_units + shares - 1) / shares;
      if (even <= per + kCross) {
        per = pad = even;
        list_units = padded(list_units);
      }
    }
    total = items * list_units;
    const int i = cta * per / list_units;
    seq = i / of_row;                                           // a row here
    head = (i - seq * of_row) / sh.blocks;
    block = i - seq * of_row - head * sh.blocks;
    item_at = i * list_units;
  }
  int u = cta * per;
  const int u_end = min(total, u + per);
  Meta* meta = a.meta + cta;
  if (t == 0) meta->last_cta = -1;
  if (u >= u_end) return;

  while (u < u_end) {
    // ---- the item: rows, columns, what each column sees
    int64_t row0, tokens;
    int units;
    int b = seq, cols, width_c = a.g;    // columns of a row
    int64_t len_q;
    const int32_t* list = nullptr;
    if (a.lists == nullptr) {
      row0 = sh.begin;
      len_q = sh.end - sh.begin;
      tokens = sh.tokens;
      cols = (int)min(len_q * a.g - (int64_t)block * NC, (int64_t)NC);
      units = sh.units;
    } else {
      row0 = seq;
      len_q = 1;
      int64_t visible;
      row_info(a.b, row0, a.c.page_shift, &b, &visible);
      tokens = b < 0 ? 0 : visible;
      cols = b < 0 ? 0 : min(a.g - block * NC, NC);   // a row of no sequence is left as it was
      units = list_units;
      list = a.lists + (row0 * a.c.heads + head) * a.nlist;
    }
    const int col0 = block * NC;
    const int u_stop = min(u_end, item_at + units);
    int vis[NT][2];                       // tokens that the column sees
    int vis_min = (int)min(tokens, (int64_t)INT32_MAX), vis_max = vis_min;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int j = nt * 8 + 2 * c4 + e;
        vis[nt][e] = j < cols && a.lists == nullptr ? (int)max(tokens - (len_q - 1 - (col0 + j) / width_c), (int64_t)0) : vis_max;
      }
    if (a.lists == nullptr) {
      vis_min = (int)max(tokens - (len_q - 1 - col0 / width_c), (int64_t)0);
      vis_max = (int)max(tokens - (len_q - 1 - (col0 + cols - 1) / width_c), (int64_t)0);
    }
    float m[NT][2], mv[NT][2], l[NT][2], o[2 * VW][NT][4];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      m[nt][0] = m[nt][1] = mv[nt][0] = mv[nt][1] = -TQ_INF;
      l[nt][0] = l[nt][1] = 0.f;
#pragma unroll
      for (int j = 0; j < 2 * VW; ++j) o[j][nt][0] = o[j][nt][1] = o[j][nt][2] = o[j][nt][3] = 0.f;
    }

    // place s in the sequence, or in the listed pages one after another -> logical page, or -1
    const int32_t* row_pages = a.b.table + (int64_t)b * a.b.ldt;   // not read where b < 0: such a row sees nothing
    const int64_t head_bytes = (int64_t)D << a.c.page_shift, page_bytes = head_bytes * a.c.heads;
    const uint8_t *k_head = a.c.k + head * head_bytes + 16 * lane, *v_head = a.c.v + head * head_bytes + 16 * lane;
    const float* scales = (lane ? a.c.v_scale : a.c.k_scale) + head;
    const int i_first = u - item_at, i_stop = u_stop - item_at;   // of the item's units
    // Pages of 32 steps at a time, one per lane: what step i0 + lane reads.  `pos` is its first token, -1 where there is nothing.
    struct Pages { int id, pos; };
    auto look_up = [&](int i0) -> Pages {
      Pages r{0, -1};
      const int i = i0 + lane;
      if (i >= i_stop) return r;
      const int64_t s = (int64_t)i * kUnit + warp * 16;           // place in the sequence, or in the listed pages one after another
      int64_t lp = s >> a.c.page_shift;
      if (list != nullptr) lp = lp < a.nlist ? list[lp] : -1;
      const int64_t t0 = (lp << a.c.page_shift) + (s & (T_ - 1));
      if (lp < 0 || t0 >= vis_max) return r;
      const int id = row_pages[lp];                               // a token that is seen lies inside the row's width
      if (id < 0 || id >= a.c.pages) return r;
      r.id = id;
      r.pos = (int)t0;
      return r;
    };
    uint8_t* ring = reinterpret_cast<uint8_t*>(smem4) + warp * K::kStages * K::kTile;
    // the queries are read before the first steps' copies queue up, and laid out while those are on their way
    float qx[NC / kWarps][D / 32];
#pragma unroll
    for (int ji = 0; ji < NC / kWarps; ++ji) {
      const int jc = col0 + ji * kWarps + warp;
      const T* q = static_cast<const T*>(a.q) + (row0 + jc / width_c) * a.ldq + (int64_t)(head * a.g + jc % width_c) * a.hq;
#pragma unroll
      for (int i = 0; i < D / 32; ++i) qx[ji][i] = ji * kWarps + warp < cols ? (float)q[i * 32 + lane] : 0.f;
    }
    Pages now = look_up(i_first), then = look_up(i_first + 32);
    int base = i_first, to_issue = i_first;
    auto issue = [&](int stage) {         // starts the copies of step `to_issue`; returns its first token
      if (to_issue == base + 32) {
        now = then;
        base += 32;
        then = look_up(base + 32);
      }
      const int id = __shfl_sync(0xffffffffu, now.id, to_issue - base), pos = __shfl_sync(0xffffffffu, now.pos, to_issue - base);
      ++to_issue;
      if (pos >= 0) {
        const int64_t at = id * page_bytes + (pos & (T_ - 1)) * D;
        const uint32_t to = (uint32_t)__cvta_generic_to_shared(ring + stage * K::kTile);
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
          copy16(to + 16 * key_chunk<D>((lane + 32 * i) / (D / 16), (lane + 32 * i) % (D / 16)), k_head + at + 512 * i);
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
          copy16(to + 16 * D + 16 * value_chunk<D>((lane + 32 * i) / (D / 16), (lane + 32 * i) % (D / 16)), v_head + at + 512 * i);
        if (lane < 2) copy4(to + 32 * D + 4 * lane, scales + (int64_t)id * a.c.heads);
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
      return pos;
    };
    constexpr int S = K::kStages;
    int t0s[S - 1];                      // first tokens of the steps in flight
#pragma unroll
    for (int i = 0; i < S - 1; ++i) t0s[i] = issue(i);
    // ---- queries: scaled to [2^13, 2^14) per column, as fp16 limbs
#pragma unroll
    for (int ji = 0; ji < NC / kWarps; ++ji) {
      const int j = ji * kWarps + warp;
      const float (&x)[D / 32] = qx[ji];
      uint32_t most = 0u;
#pragma unroll
      for (int i = 0; i < D / 32; ++i) most = max(most, __float_as_uint(x[i]) & 0x7FFFFFFFu);
      most = __reduce_max_sync(0xffffffffu, most);
      float inv;
      const float s = query_scale(most, &inv);
#pragma unroll
      for (int i = 0; i < D / 32; ++i) {
        const float y = x[i] * inv;
        const __half hi = __float2half_rn(y);
        qsm[j * K::QP + i * 32 + lane] = hi;
        if (LIMBS == 2) qsm[(NC + j) * K::QP + i * 32 + lane] = __float2half_rn(y - __half2float(hi));
      }
      // a row with an infinity or a NaN has no scores: NaN
      if (lane == 0) fsm[j] = most >= 0x7F800000u ? __uint_as_float(0x7FC00000u) : s * (a.scale * kLog2e);
    }
    __syncthreads();
    float f[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 2; ++e) f[nt][e] = fsm[nt * 8 + 2 * c4 + e];
    uint32_t qf[NT * LIMBS == 1 ? KW : 1][2];
    if (NT * LIMBS == 1) {
#pragma unroll
      for (int w = 0; w < KW; ++w) {
        const uint2 y = *reinterpret_cast<const uint2*>(qsm + n8 * K::QP + 4 * KS * 4 * (w / KS) + 4 * KS * c4 + 4 * (w % KS));
        qf[w][0] = y.x;
        qf[w][1] = y.y;
      }
    }

    auto compute = [&](int t0, int stage) {
      if (t0 < 0) return;
      const uint8_t* tile = ring + stage * K::kTile;
      const float ks = *reinterpret_cast<const float*>(tile + 32 * D), vs = *reinterpret_cast<const float*>(tile + 32 * D + 4);
      float s[NT][4];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) s[nt][0] = s[nt][1] = s[nt][2] = s[nt][3] = 0.f;
      uint32_t kw[2][KW];
#pragma unroll
      for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int i = 0; i < KW / KS; ++i)
          load_words<KS>(tile + (KS == 4 ? 16 * key_chunk<D>(n8 + 8 * r, 4 * i + c4) : (n8 + 8 * r) * D + 32 * i + 8 * c4), &kw[r][KS * i]);
#pragma unroll
      for (int w = 0; w < KW; ++w) {
        uint32_t y[4];
        expand<E4M3>(kw[0][w], y[0], y[2]);
        expand<E4M3>(kw[1][w], y[1], y[3]);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int li = 0; li < LIMBS; ++li) {
            if (NT * LIMBS == 1) {
              mma_f16(s[nt], y, qf[w][0], qf[w][1]);
            } else {
              const uint2 z = *reinterpret_cast<const uint2*>(qsm + (li * NC + nt * 8 + n8) * K::QP + 16 * KS * (w / KS) + 4 * KS * c4 + 4 * (w % KS));
              mma_f16(s[nt], y, z.x, z.y);
            }
          }
      }
      const bool edge = t0 + 16 > vis_min;      // some column does not see all 16 tokens
      const float lv = scale_log2(vs);
      bool higher = false;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int e = 0; e < 4; ++e) s[nt][e] *= f[nt][e & 1] * ks;
        if (edge) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (t0 + n8 + 8 * (e >> 1) >= vis[nt][e & 1]) s[nt][e] = -TQ_INF;
        }
#pragma unroll
        for (int e = 0; e < 2; ++e)     // (values of no scale, mv - lv = NaN or +inf: m alone)
          higher |= fmaxf(s[nt][e], s[nt][2 + e]) > fminf(m[nt][e], mv[nt][e] - lv) + kSlack;
      }
      if (__any_sync(0xffffffffu, higher)) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float g = fmaxf(s[nt][e], s[nt][2 + e]);
            g = fmaxf(g, __shfl_xor_sync(0xffffffffu, g, 4));
            g = fmaxf(g, __shfl_xor_sync(0xffffffffu, g, 8));
            g = fmaxf(g, __shfl_xor_sync(0xffffffffu, g, 16));
            const float top_m = fmaxf(m[nt][e], ceilf(g)), top_v = fmaxf(mv[nt][e], ceilf(g + lv));
            l[nt][e] *= top_m > m[nt][e] ? ex2(m[nt][e] - top_m) : 1.f;                 // from -inf: 0
            const float alpha = top_v > mv[nt][e] ? ex2(mv[nt][e] - top_v) : 1.f;
            m[nt][e] = top_m;
            mv[nt][e] = top_v;
#pragma unroll
            for (int j = 0; j < 2 * VW; ++j) {
              o[j][nt][e] *= alpha;
              o[j][nt][2 + e] *= alpha;
            }
          }
      }
      uint32_t p[NT][LIMBS][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float mm = m[nt][e & 1], mw = mv[nt][e & 1];
          const float x = ex2(s[nt][e] + (mm == -TQ_INF ? 0.f : kLift - mm));
          l[nt][e & 1] += x;
          y[e] = ex2(s[nt][e] + (mw == -TQ_INF ? -TQ_INF : kLift + (lv - mw)));
          if (!(vs == vs)) y[e] = edge && t0 + n8 + 8 * (e >> 1) >= vis[nt][e & 1] ? 0.f : vs;   // NaN for the columns that see it
        }
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const uint32_t hi = half2_bits(y[2 * r], y[2 * r + 1]);
          p[nt][0][r] = transpose8(hi);
          if (LIMBS == 2) {
            const float2 back = __half22float2(*reinterpret_cast<const __half2*>(&hi));
            p[nt][LIMBS - 1][r] = transpose8(half2_bits(y[2 * r] - back.x, y[2 * r + 1] - back.y));
          }
        }
      }
      uint32_t vw[4][VW];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = 2 * c4 + (r & 1) + 8 * (r >> 1);
        load_words<VW>(tile + 16 * D + (VW == 4 ? 16 * value_chunk<D>(row, n8)
                                                : (VW == 2 ? 16 * value_chunk<D>(row, n8 >> 1) + 8 * (n8 & 1) : row * D + 4 * VW * n8)), vw[r]);
      }
      if (edge && E4M3) {                           // slots behind the last token may hold codes of NaN
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (t0 + 2 * c4 + (r & 1) + 8 * (r >> 1) >= vis_max) {
#pragma unroll
            for (int j = 0; j < VW; ++j) vw[r][j] = 0u;
          }
      }
#pragma unroll
      for (int j = 0; j < VW; ++j) {
        uint32_t lo[4], hi[4];                      // of channel 4 j, 4 j + 1 and of 4 j + 2, 4 j + 3
        expand<E4M3>(__byte_perm(vw[0][j], vw[1][j], 0x5140), lo[0], lo[1]);
        expand<E4M3>(__byte_perm(vw[2][j], vw[3][j], 0x5140), lo[2], lo[3]);
        expand<E4M3>(__byte_perm(vw[0][j], vw[1][j], 0x7362), hi[0], hi[1]);
        expand<E4M3>(__byte_perm(vw[2][j], vw[3][j], 0x7362), hi[2], hi[3]);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int li = 0; li < LIMBS; ++li) {
            mma_f16(o[2 * j][nt], lo, p[nt][li][0], p[nt][li][1]);
            mma_f16(o[2 * j + 1][nt], hi, p[nt][li][0], p[nt][li][1]);
          }
      }
    };
    {
      int stage = 0;
#pragma unroll 1
      for (int i = i_first; i < i_stop; ++i) {
        asm volatile("cp.async.wait_group %0;" ::"n"(S - 2) : "memory");
        __syncwarp();                      // the step's bytes are there for all lanes, and the last step's have been read
        const int t0 = t0s[0];
#pragma unroll
        for (int j = 0; j < S - 2; ++j) t0s[j] = t0s[j + 1];
        t0s[S - 2] = issue(stage == 0 ? S - 1 : stage - 1);
        compute(t0, stage);
        stage = stage == S - 1 ? 0 : stage + 1;
      }
      asm volatile("cp.async.wait_group 0;" ::: "memory");
    }

    // ---- the four warps' results as one
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float z = l[nt][e];
        z += __shfl_xor_sync(0xffffffffu, z, 4);
        z += __shfl_xor_sync(0xffffffffu, z, 8);
        z += __shfl_xor_sync(0xffffffffu, z, 16);
        if (n8 == 0) {
          msm[warp * NC + nt * 8 + 2 * c4 + e] = m[nt][e];
          lsm[warp * NC + nt * 8 + 2 * c4 + e] = z;
        }
      }
    __syncthreads();                       // tiles have been read, maxima are there
    if (t < NC) {
      float best = -TQ_INF, sum = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) best = fmaxf(best, msm[w * NC + t]);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) sum += lsm[w * NC + t] * (best == -TQ_INF ? 1.f : ex2(msm[w * NC + t] - best));
      top[t] = best;
      tot[t] = sum;
    }
    __syncthreads();
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int j = nt * 8 + 2 * c4 + e;
        // divided by the whole sum here: an average of the values, in range whatever their scales (in two steps, as 2^x may not be)
        const float x = mv[nt][e] == -TQ_INF ? 0.f : mv[nt][e] - top[j], x0 = floorf(0.5f * x);   // nothing: O is 0, or NaN
        const float w = ex2(x0), w1 = tot[j] == 0.f ? 0.f : ex2(x - x0) / tot[j];
#pragma unroll
        for (int i = 0; i < 2 * VW; ++i) {
          osm[(warp * NC + j) * K::OP + 4 * VW * n8 + 2 * i] = o[i][nt][e] * w * w1;
          osm[(warp * NC + j) * K::OP + 4 * VW * n8 + 2 * i + 1] = o[i][nt][2 + e] * w * w1;
        }
      }
    __syncthreads();
    const bool whole = u == item_at && u_stop == item_at + units;
    const int slot = 2 * cta + (u == item_at ? 1 : 0);
    for (int i = t; i < cols * D; i += kThreads) {
      const int j = i / D, ch = i % D;
      float y = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) y += osm[(w * NC + j) * K::OP + ch];
      if (whole) {
        const int jc = col0 + j;
        T* out = static_cast<T*>(a.out) + (row0 + jc / width_c) * a.ldo + (int64_t)(head * a.g + jc % width_c) * a.ho;
        store_out<T>(out + ch, y);
      } else {
        a.part_o[((int64_t)slot * kMaxCols + j) * D + ch] = y;
      }
    }
    if (t < cols) {
      if (whole) {
        const int jc = col0 + t;
        if (a.lse) a.lse[(row0 + jc / width_c) * ((int64_t)a.c.heads * a.g) + head * a.g + jc % width_c] =
            tot[t] == 0.f ? -TQ_INF : (top[t] == -TQ_INF ? 0.f : (top[t] - kLift) * kLn2) + logf(tot[t]);
      } else {
        a.part_ml[(int64_t)slot * 2 * kMaxCols + t] = top[t];
        a.part_ml[(int64_t)slot * 2 * kMaxCols + kMaxCols + t] = tot[t];
      }
    }
    if (!whole && u == item_at && t == 0) {
      meta->row0 = (int)row0;
      meta->col0 = col0;
      meta->cols = cols;
      meta->head = head;
      meta->last_cta = (item_at + units - 1) / per;
    }
    __syncthreads();                       // shared memory is the next item's
    // ---- the next item
    u = u_stop;
    item_at += units;
    if (u < u_end && ++block == sh.blocks) {
      block = 0;
      if (++head == a.c.heads) {
        head = 0;
        ++seq;
        if (a.lists == nullptr) {
          for (sh = shape_of(a, seq, NC); sh.units == 0; sh = shape_of(a, seq, NC)) ++seq;   // u < total: there is one
          sh.units = padded(sh.units);
        }
      }
    }
  }
}

// Joins the parts of the item that began in CTA blockIdx.x's share, in a fixed order: eight columns per blockIdx.y, whose warps take a
// column's parts in turn.  What the first parts hold is asked for before it is known how many there are (places behind the last part
// are read, never used).  CTAs of 256 threads: most find nothing to do, and 512 threads each cost a ragged batch 3 us of 119; fewer CTAs that
// look after several shares cost short calls 2.
constexpr int kJoinThreads = 256, kJoinWarps = kJoinThreads / 32, kJoinParts = 8;
template <typename T, int D>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const __grid_constant__ AttendArgs a, int c2) {   // c2: 1, 2, 4 or 8 columns at a time
  __shared__ float4 o_s[kJoinWarps][32];
  wait_for_predecessor();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, first = blockIdx.x;
  const int runs = kJoinWarps / c2, run = warp / c2;
  int j = 8 * blockIdx.y + warp % c2;
  auto slot = [&](int i) { return 2 * min(first + i, (int)gridDim.x - 1) + (i == 0 ? 1 : 0); };
  float4 v[kJoinParts];
  auto fetch = [&](int i0) {
    const float* po = a.part_o + (int64_t)j * D + 4 * min(lane, D / 4 - 1);
#pragma unroll
    for (int i = 0; i < kJoinParts; ++i) v[i] = *reinterpret_cast<const float4*>(po + (int64_t)slot(i0 + i * runs) * a.pitch * D);
  };
  const Meta z = a.meta[first];
  float mi[2], li[2];                      // of parts lane and lane + 32
  auto fetch_ml = [&] {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      mi[i] = a.part_ml[(int64_t)slot(lane + 32 * i) * 2 * a.pitch + j];
      li[i] = a.part_ml[(int64_t)slot(lane + 32 * i) * 2 * a.pitch + a.pitch + j];
    }
  };
  fetch_ml();
  fetch(run);
  const int cols = min(z.cols - 8 * (int)blockIdx.y, 8), parts = z.last_cta - first + 1;
  if (z.last_cta < 0) return;
#pragma unroll 1
  for (int base = 0; base < cols; base += c2) {   // once, unless the caller's max_queries was too small
    if (base > 0) {
      j += c2;
      fetch_ml();
      fetch(run);
    }
    const float* ml = a.part_ml + j;
    const bool mine = j - 8 * (int)blockIdx.y < cols;
    auto max_of = [&](int i) { return i < 32 ? mi[0] : (i < 64 ? mi[1] : ml[(int64_t)slot(i) * 2 * a.pitch]); };
    auto sum_of = [&](int i) { return i < 32 ? li[0] : (i < 64 ? li[1] : ml[(int64_t)slot(i) * 2 * a.pitch + a.pitch]); };
    float best = -TQ_INF;
    for (int i = lane; i < parts; i += 32) best = fmaxf(best, max_of(i));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) best = fmaxf(best, __shfl_xor_sync(0xffffffffu, best, o));
    auto weight = [&](int i) { return sum_of(i) * (best == -TQ_INF ? 1.f : ex2(max_of(i) - best)); };
    float sum = 0.f;
    for (int i = lane; i < parts; i += 32) sum += weight(i);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);   // every warp of a column has the whole sum
    float4 y = make_float4(0.f, 0.f, 0.f, 0.f);   // parts are averages of values: with weights that add up to 1 nothing leaves their range
#pragma unroll 1
    for (int p0 = 0; p0 < parts; p0 += 32) {      // weights of 32 parts, one per lane
      const float w = p0 + lane < parts && sum != 0.f ? weight(p0 + lane) / sum : 0.f;
      const int end = min(p0 + 32, parts);
#pragma unroll 1
      for (int i0 = p0 + run; i0 < end; i0 += kJoinParts * runs) {
        if (i0 != run) fetch(i0);
#pragma unroll
        for (int i = 0; i < kJoinParts; ++i) {
          const int at = i0 + i * runs;
          const float wi = __shfl_sync(0xffffffffu, w, (at - p0) & 31);
          if (at < end) {                         // what is behind may not be a number
            y.x = fmaf(v[i].x, wi, y.x); y.y = fmaf(v[i].y, wi, y.y); y.z = fmaf(v[i].z, wi, y.z); y.w = fmaf(v[i].w, wi, y.w);
          }
        }
      }
    }
    if (base > 0) __syncthreads();                // the last columns' results have been read
    o_s[warp][lane] = y;
    __syncthreads();
    if (!mine || run != 0) continue;
    for (int r = 1; r < runs; ++r) {
      const float4 x = o_s[warp + r * c2][lane];
      y.x += x.x; y.y += x.y; y.z += x.z; y.w += x.w;
    }
    const int jc = z.col0 + j, g = a.g;
    const int64_t row = (int64_t)z.row0 + jc / g;
    const int head = z.head * g + jc % g;
    if (lane < D / 4) {
      T* out = static_cast<T*>(a.out) + row * a.ldo + (int64_t)head * a.ho + 4 * lane;
      const float x[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) store_out<T>(out + i, x[i]);
    }
    if (lane == 0 && a.lse) a.lse[row * ((int64_t)a.c.heads * g) + head] =
        sum == 0.f ? -TQ_INF : (best == -TQ_INF ? 0.f : (best - a.lift) * kLn2) + logf(sum);
  }
}

template <typename T, int D, bool E4M3, int NT>
cudaError_t launch(const AttendArgs& a, int sms, int* grid_out, cudaStream_t st) {
  const int grid = *grid_out = sms * Kernel<T, D, E4M3, NT>::kCtas;
  static std::atomic<unsigned long long> devices{0};
  const cudaError_t e = allow_largest_smem(reinterpret_cast<const void*>(attend_kernel<T, D, E4M3, NT>), devices);
  if (e != cudaSuccess) return e;
  return launch_dependent(attend_kernel<T, D, E4M3, NT>, dim3((unsigned)grid), dim3(kThreads), Kernel<T, D, E4M3, NT>::smem, st, a);
}
template <typename T, int D>
cudaError_t launch_d(const AttendArgs& a, bool e4m3, int cols, int sms, cudaStream_t st) {
  const int nt = cols <= 8 ? 1 : 2;
  cudaError_t e;
  int grid = 0;
  if (e4m3) e = nt == 1 ? launch<T, D, true, 1>(a, sms, &grid, st) : launch<T, D, true, 2>(a, sms, &grid, st);
  else e = nt == 1 ? launch<T, D, false, 1>(a, sms, &grid, st) : launch<T, D, false, 2>(a, sms, &grid, st);
  if (e != cudaSuccess) return e;
  return launch_join(a, sizeof(T) == 4 ? TQ_F32 : TQ_BF16, grid, cols, st);
}
template <typename T>
cudaError_t launch_t(const AttendArgs& a, bool e4m3, int cols, int sms, cudaStream_t st) {
  switch (a.c.d) {
    case 32: return launch_d<T, 32>(a, e4m3, cols, sms, st);
    case 64: return launch_d<T, 64>(a, e4m3, cols, sms, st);
    case 96: return launch_d<T, 96>(a, e4m3, cols, sms, st);
    default: return launch_d<T, 128>(a, e4m3, cols, sms, st);
  }
}

constexpr int kMostCtas = 3;   // per SM, of any instance

struct Space {
  size_t meta, ml, o, bytes;
};
Space lay_out(int grid, int d) {
  Space s;
  s.meta = 0;
  s.ml = (size_t)round_up64((int64_t)grid * sizeof(Meta), 256);
  s.o = s.ml + (size_t)round_up64((int64_t)grid * 2 * 2 * kMaxCols * sizeof(float), 256);
  s.bytes = s.o + (size_t)round_up64((int64_t)grid * 2 * kMaxCols * d * sizeof(float), 256);
  return s;
}

}  // namespace

template <typename T>
static cudaError_t join_t(const AttendArgs& a, dim3 grid, int c2, cudaStream_t st) {
  switch (a.c.d) {
    case 32: return launch_dependent(join_kernel<T, 32>, grid, dim3(kJoinThreads), 0, st, a, c2);
    case 64: return launch_dependent(join_kernel<T, 64>, grid, dim3(kJoinThreads), 0, st, a, c2);
    case 96: return launch_dependent(join_kernel<T, 96>, grid, dim3(kJoinThreads), 0, st, a, c2);
    default: return launch_dependent(join_kernel<T, 128>, grid, dim3(kJoinThreads), 0, st, a, c2);
  }
}
cudaError_t launch_join(const AttendArgs& a, int dtype, int ctas, int cols, cudaStream_t st) {
  const dim3 g((unsigned)ctas, (unsigned)((cols + 7) / 8));
  const int c2 = cols > 4 ? 8 : (cols > 2 ? 4 : cols);   // as many as there should be
  return dtype == TQ_F32 ? join_t<float>(a, g, c2, st) : join_t<__nv_bfloat16>(a, g, c2, st);
}

size_t attend_space(int sms, int d) { return lay_out(sms * kMostCtas, d).bytes; }

cudaError_t launch_attend(AttendArgs& a, int dtype, bool e4m3, int cols, int sms, void* workspace, cudaStream_t st) {
  const int grid = sms * kMostCtas;
  const Space s = lay_out(grid, a.c.d);
  char* w = static_cast<char*>(workspace);
  a.meta = reinterpret_cast<Meta*>(w + s.meta);
  a.part_ml = reinterpret_cast<float*>(w + s.ml);
  a.part_o = reinterpret_cast<float*>(w + s.o);
  a.pitch = kMaxCols;
  a.lift = kLift;
  return dtype == TQ_F32 ? launch_t<float>(a, e4m3, cols, sms, st) : launch_t<__nv_bfloat16>(a, e4m3, cols, sms, st);
}

}  // namespace kv8
}  // namespace tq

extern "C" size_t tq_kv8_attend_workspace_bytes(const tq_kv8* cache, int nseq, int64_t n, int q_per_kv, int max_queries, int nlist) {
  using namespace tq;
  using namespace tq::kv8;
  int dev = 0, sms = 0;
  if (cache == nullptr || cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
  (void)nseq; (void)n;
  const bool many = nlist == 0 && (int64_t)std::max(max_queries, 1) * q_per_kv > kMaxCols;
  return attend_space(sms, cache->d) + (many ? prompt_space(sms, cache->d) : 0);
}

extern "C" int tq_kv8_attend(const tq_kv8* cache, const int32_t* table, int64_t ldt, int width, int nseq, const int32_t* tokens,
                             const int32_t* starts, int64_t n, int max_queries, const void* Q, int64_t ldq, int64_t hq, int q_per_kv,
                             int dtype, float scale, const int32_t* lists, int nlist, void* out, int64_t ldo, int64_t ho, float* lse,
                             void* workspace, size_t workspace_bytes, void* stream) {
  using namespace tq;
  using namespace tq::kv8;
  const char* who = "tq_kv8_attend";
  TQ_RANGE(who);
  AttendArgs a;
  std::memset(&a, 0, sizeof(a));
  int rc = check_cache(who, cache, &a.c);
  if (rc == TQ_OK) rc = check_batch(who, a.c, table, ldt, width, nseq, tokens, starts, n, &a.b);
  if (rc != TQ_OK) return rc;
  TQ_REQUIRE(dtype == TQ_F32 || dtype == TQ_BF16, TQ_ERR_UNSUPPORTED, "%s: unknown dtype %d", who, dtype);
  TQ_REQUIRE(q_per_kv >= 1 && q_per_kv <= 256, TQ_ERR_UNSUPPORTED, "%s: 1..256 queries per KV head", who);
  TQ_REQUIRE(max_queries >= 0 && nlist >= 0, TQ_ERR_INVALID_ARG, "%s: negative size", who);
  TQ_REQUIRE(starts != nullptr || max_queries >= 1, TQ_ERR_INVALID_ARG, "%s: max_queries is 0 where every sequence has one row", who);
  TQ_REQUIRE((lists != nullptr) == (nlist > 0), TQ_ERR_INVALID_ARG, "%s: lists of %d pages", who, nlist);
  TQ_REQUIRE(nlist <= (1 << 24), TQ_ERR_UNSUPPORTED, "%s: lists of %d pages", who, nlist);
  if (nseq == 0 || n == 0 || (max_queries == 0 && workspace == nullptr)) return TQ_OK;
  max_queries = std::max(max_queries, 1);   // the figure only chooses kernels: rows that `starts` has all the same are computed
  TQ_REQUIRE(Q != nullptr && out != nullptr, TQ_ERR_INVALID_ARG, "%s: Q or out is NULL", who);
  TQ_REQUIRE(ldq >= 0 && hq >= 0 && ldo >= 0 && ho >= 0, TQ_ERR_INVALID_ARG, "%s: negative stride", who);
  const uintptr_t align = dtype == TQ_F32 ? 3 : 1;
  TQ_REQUIRE(((reinterpret_cast<uintptr_t>(Q) | reinterpret_cast<uintptr_t>(out)) & align) == 0 && (reinterpret_cast<uintptr_t>(lse) & 3) == 0,
             TQ_ERR_ALIGNMENT, "%s: Q, out or lse is not aligned to its elements", who);
  const size_t need = tq_kv8_attend_workspace_bytes(cache, nseq, n, q_per_kv, max_queries, nlist);
  TQ_REQUIRE(workspace != nullptr && workspace_bytes >= need, TQ_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", who, workspace_bytes, need);
  TQ_REQUIRE((reinterpret_cast<uintptr_t>(workspace) & 255) == 0, TQ_ERR_ALIGNMENT, "%s: workspace is not 256-byte aligned", who);
  // units of 64 tokens, over all heads and blocks of eight columns, are numbered in 31 bits
  const double units = (lists != nullptr ? (double)n * (((double)nlist * cache->page_tokens + 63) / 64 + 1) * ((q_per_kv + 7) / 8)
                              : ((double)nseq + (double)n * q_per_kv / 8) * (((double)width * cache->page_tokens + 63) / 64 + 1)) * cache->heads;
  TQ_REQUIRE(units < 2.0e9 && (double)n * q_per_kv < 2.0e9, TQ_ERR_UNSUPPORTED, "%s: %.3g units of 64 tokens in one call", who, units);
  int dev = 0, sms = 0;
  TQ_CHECK_CUDA(cudaGetDevice(&dev), who);
  TQ_CHECK_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev), who);
  a.q = Q; a.ldq = ldq; a.hq = hq; a.g = q_per_kv; a.scale = scale;
  a.lists = lists; a.nlist = nlist; a.out = out; a.ldo = ldo; a.ho = ho; a.lse = lse;
  // Sequences with up to 16 columns (rows x heads of a group) are bound by the cache's bytes and go to the few-query kernel, the others
  // to the many-query one; a batch of both kinds runs both, each over its own.
  const int64_t cols = lists ? q_per_kv : (int64_t)max_queries * q_per_kv;
  const bool e4m3 = cache->code_type == TQ_E4M3, many = lists == nullptr && cols > kMaxCols;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  // A single sequence goes to one kernel, however many rows it turns out to have, and where max_queries says that all are small, sequences
  // that are not are still the few-query kernel's, 16 columns at a time.
  a.most_cols = !many ? INT32_MAX : (nseq == 1 ? 0 : kMaxCols);
  if (many) {
    TQ_CHECK_CUDA(launch_prompt(a, dtype, e4m3, sms, static_cast<char*>(workspace) + attend_space(sms, a.c.d), st), who);
    count_launches(2);
  }
  if (!many || nseq > 1) {
    TQ_CHECK_CUDA(launch_attend(a, dtype, e4m3, (int)std::min<int64_t>(cols, kMaxCols), sms, workspace, st), who);
    count_launches(2);
  }
  return TQ_OK;
}
