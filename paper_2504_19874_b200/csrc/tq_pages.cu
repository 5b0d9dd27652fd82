// Pages of a cache: taking, sharing, copying, freeing and compacting them.  The interface is in include/tq.h.
//
// The only state is the caller's: how many rows of the table hold each page (refs), and the table itself.  A page is free when its
// count is 0, so there is no list of free pages that could fall out of step, and which pages a call takes depends on the counts
// alone: always the lowest free ones, handed out in the order of the requests.  Ranks among the free (or live) pages come from counts
// of 2,048 pages each and a sum over the counts ahead, in two dependent launches; no atomics decide an order.
#include <algorithm>

#include "tq_kv8.h"

namespace tq {
namespace pages {

using kv8::Cache;

constexpr int kThreads = 256, kPer = 8, kChunk = kThreads * kPer;   // pages per CTA of the counting kernels
constexpr int kPiece = 1024;                                        // 16-byte vectors that a CTA copies at a time: four per thread

struct Table {
  int32_t* table;
  int64_t ldt;
  int width, rows;
  int32_t* tokens;
};
struct TakeArgs {
  int32_t* refs;
  int64_t pages;
  Table t;
  const int32_t* next;       // extend: lengths to have room for; fork: NULL
  const int32_t *parents, *children;
  int units, page_shift;     // requests: sequences (extend) or children (fork)
  int32_t *counts, *offsets;           // workspace: free pages of each chunk, first request of each unit
  int32_t* fresh;                      // ... and first entry to fill of each sequence (extend), page of each child (fork)
  int32_t* spare;
};

// Pages that unit u asks for.  *first: extend: the first entry of its row without one, behind those that a sequence that was shortened,
// or that a pool ran short for, still has (read before any entry is filled); fork: the parent's page to copy.
__device__ __forceinline__ int asked(const TakeArgs& a, int u, int* first) {
  const int T1 = (1 << a.page_shift) - 1;
  if (a.next != nullptr) {
    const int64_t have = ((int64_t)max(a.t.tokens[u], 0) + T1) >> a.page_shift;
    const int64_t need = min(((int64_t)max(a.next[u], 0) + T1) >> a.page_shift, (int64_t)a.t.width);
    int64_t j = have;
    for (; j < need; ++j) {
      const int id = a.t.table[(int64_t)u * a.t.ldt + j];
      if (id < 0 || id >= a.pages || a.refs[id] <= 0) break;
    }
    *first = (int)min(j, (int64_t)a.t.width);
    return need > j ? (int)(need - j) : 0;
  }
  *first = 0;
  const int p = a.parents[u], c = a.children[u];
  if (p < 0 || p >= a.t.rows || c < 0 || c >= a.t.rows || p == c) return 0;
  const int len = max(a.t.tokens[p], 0), j = len >> a.page_shift;
  if ((len & T1) == 0 || j >= a.t.width) return 0;
  *first = a.t.table[(int64_t)p * a.t.ldt + j];
  return *first >= 0 && *first < a.pages ? 1 : 0;
}

// Inclusive sum over the CTA's threads in order; *total: that of all of them.
__device__ __forceinline__ int block_sum_upto(int v, int* warp_sums, int* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int s = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, s, o);
    if (lane >= o) s += y;
  }
  __syncthreads();
  if (lane == 31) warp_sums[warp] = s;
  __syncthreads();
  int before = 0, all = 0;
  for (int w = 0; w < kThreads / 32; ++w) {
    if (w < warp) before += warp_sums[w];
    all += warp_sums[w];
  }
  *total = all;
  return s + before;
}

// Bit i: page 8 x + i of the pool is free (live, with LIVE).  refs is 4-byte aligned.
template <bool LIVE>
__device__ __forceinline__ uint32_t page_bits(const int32_t* refs, int64_t pages, int64_t p0) {
  uint32_t bits = 0u;
#pragma unroll
  for (int i = 0; i < kPer; ++i)
    if (p0 + i < pages && (refs[p0 + i] > 0) == LIVE) bits |= 1u << i;
  return bits;
}

// Block c counts the free pages of chunk c; the block behind the last chunk sums up the requests.
__global__ void __launch_bounds__(kThreads) count_kernel(const __grid_constant__ TakeArgs a, int chunks) {
  __shared__ int warp_sums[kThreads / 32];
  const int t = threadIdx.x;
  allow_successor();
  wait_for_predecessor();
  int total;
  if ((int)blockIdx.x < chunks) {
    const int n = __popc(page_bits<false>(a.refs, a.pages, (int64_t)blockIdx.x * kChunk + t * kPer));
    block_sum_upto(n, warp_sums, &total);
    if (t == 0) a.counts[blockIdx.x] = total;
    return;
  }
  int before = 0;
  for (int u0 = 0; u0 < a.units; u0 += kThreads) {
    int first;
    const int n = u0 + t < a.units ? asked(a, u0 + t, &first) : 0;
    const int upto = block_sum_upto(n, warp_sums, &total);
    if (u0 + t < a.units) {
      a.offsets[u0 + t] = before + upto - n;
      if (a.next != nullptr) a.fresh[u0 + t] = first;
    }
    before += total;
  }
  if (t == 0) a.offsets[a.units] = before;
}

// Gives request r (of unit u, its i-th) page id, or none (-1).
__device__ __forceinline__ void give(const TakeArgs& a, int r, int id) {
  int lo = 0, hi = a.units - 1;   // last u with offsets[u] <= r; units without requests share their successor's offset
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.offsets[mid] <= r) lo = mid; else hi = mid - 1;
  }
  if (a.next != nullptr) {
    a.t.table[(int64_t)lo * a.t.ldt + a.fresh[lo] + (r - a.offsets[lo])] = id;
  } else {
    a.fresh[lo] = id;
  }
}

// Chunk c hands its free pages to the requests whose turn it is.
__global__ void __launch_bounds__(kThreads) take_kernel(const __grid_constant__ TakeArgs a, int chunks) {
  __shared__ int warp_sums[kThreads / 32];
  const int t = threadIdx.x;
  allow_successor();
  wait_for_predecessor();
  const int wanted = a.offsets[a.units];
  int ahead = 0, all = 0, total;
  for (int c0 = 0; c0 < chunks; c0 += kThreads) {
    const int n = c0 + t < chunks ? a.counts[c0 + t] : 0;
    block_sum_upto(c0 + t < (int)blockIdx.x ? n : 0, warp_sums, &total);
    ahead += total;
    block_sum_upto(n, warp_sums, &total);
    all += total;
  }
  if (blockIdx.x == 0) {
    if (t == 0) *a.spare = (int32_t)max((int64_t)all - wanted, (int64_t)INT32_MIN);
    for (int r = all + t; r < wanted; r += kThreads) give(a, r, -1);   // the pool is short: spare says by how many
  }
  if (ahead >= wanted) return;
  const int64_t p0 = (int64_t)blockIdx.x * kChunk + t * kPer;
  const uint32_t bits = page_bits<false>(a.refs, a.pages, p0);
  int r = ahead + block_sum_upto(__popc(bits), warp_sums, &total) - __popc(bits);
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    if (((bits >> i) & 1u) && r < wanted) {
      a.refs[p0 + i] = 1;
      give(a, r, (int)(p0 + i));
    }
    r += (bits >> i) & 1u;
  }
}

// Both in one launch, by one CTA, for pools of up to kSmall pages: 2 us less where the launches are all that costs.
constexpr int kSmall = 4 * kChunk;
__global__ void __launch_bounds__(kThreads) take_small_kernel(const __grid_constant__ TakeArgs a) {
  __shared__ int warp_sums[kThreads / 32];
  const int t = threadIdx.x;
  allow_successor();
  wait_for_predecessor();
  constexpr int kMost = kSmall / kChunk;
  uint32_t bits[kMost];                      // chunk c, thread t: pages c kChunk + 8 t and on
#pragma unroll
  for (int c = 0; c < kMost; ++c) bits[c] = page_bits<false>(a.refs, a.pages, (int64_t)c * kChunk + t * kPer);
  int wanted = 0, total;
  for (int u0 = 0; u0 < a.units; u0 += kThreads) {
    int first;
    const int n = u0 + t < a.units ? asked(a, u0 + t, &first) : 0;
    const int upto = block_sum_upto(n, warp_sums, &total);
    if (u0 + t < a.units) {
      a.offsets[u0 + t] = wanted + upto - n;
      if (a.next != nullptr) a.fresh[u0 + t] = first;
    }
    wanted += total;
  }
  if (t == 0) a.offsets[a.units] = wanted;
  __syncthreads();
  int ahead = 0;
#pragma unroll
  for (int c = 0; c < kMost; ++c) {
    int r = ahead + block_sum_upto(__popc(bits[c]), warp_sums, &total) - __popc(bits[c]);
#pragma unroll 1
    for (uint32_t left = bits[c]; left != 0u && r < wanted; left &= left - 1u, ++r) {
      const int page = c * kChunk + t * kPer + __ffs(left) - 1;
      a.refs[page] = 1;
      give(a, r, page);
    }
    ahead += total;
  }
  if (t == 0) *a.spare = ahead - wanted;
  for (int r = ahead + t; r < wanted; r += kThreads) give(a, r, -1);
}

__global__ void __launch_bounds__(kThreads) free_kernel(int32_t* refs, int64_t pages, Table a, const int32_t* seqs) {
  allow_successor();
  wait_for_predecessor();
  const int b = seqs[blockIdx.x];
  if (b < 0 || b >= a.rows) return;
  for (int j = threadIdx.x; j < a.width; j += kThreads) {
    // the exchange makes a sequence that is named twice give its pages back once
    int32_t* at = a.table + (int64_t)b * a.ldt + j;
    if (*at < 0) continue;
    const int id = atomicExch(at, -1);
    if (id >= 0 && id < pages && atomicSub(&refs[id], 1) <= 0) atomicAdd(&refs[id], 1);
  }
  if (threadIdx.x == 0 && a.tokens != nullptr) a.tokens[b] = 0;
}

// ---- data of a page: keys, values and bounds as 16-byte vectors, and the two rows of scales
struct Pool {
  Cache c;
  int64_t codes;   // 16-byte vectors of one page's keys (or values)
  int64_t bounds;  // ... of its bounds, 0 without them
  __host__ __device__ int64_t vectors() const { return 2 * codes + bounds; }
};
Pool pool_of(const Cache& c) {
  const int64_t codes = (((int64_t)c.heads * c.d) << c.page_shift) / 16;
  return Pool{c, codes, c.bounds ? (int64_t)c.heads * 2 * c.d / 16 : 0};
}
__device__ __forceinline__ uint4* vector_at(const Pool& p, int64_t page, int64_t i) {
  if (i < p.codes) return reinterpret_cast<uint4*>(p.c.k) + page * p.codes + i;
  if (i < 2 * p.codes) return reinterpret_cast<uint4*>(p.c.v) + page * p.codes + (i - p.codes);
  return reinterpret_cast<uint4*>(p.c.bounds) + page * p.bounds + (i - 2 * p.codes);
}
// Piece x of page `from` to page `to`: four loads of each thread are in flight before the first store.
__device__ __forceinline__ void copy_piece(const Pool& p, int64_t from, int64_t to, int64_t x) {
  const int64_t n = p.vectors(), i0 = x * kPiece + threadIdx.x;
  uint4 v[kPiece / kThreads];
#pragma unroll
  for (int i = 0; i < kPiece / kThreads; ++i)
    if (i0 + i * kThreads < n) v[i] = __ldcs(vector_at(p, from, i0 + i * kThreads));
#pragma unroll
  for (int i = 0; i < kPiece / kThreads; ++i)
    if (i0 + i * kThreads < n) __stcs(vector_at(p, to, i0 + i * kThreads), v[i]);
  if (x == 0)
    for (int h = threadIdx.x; h < p.c.heads; h += kThreads) {
      p.c.k_scale[to * p.c.heads + h] = p.c.k_scale[from * p.c.heads + h];
      p.c.v_scale[to * p.c.heads + h] = p.c.v_scale[from * p.c.heads + h];
    }
}

__global__ void __launch_bounds__(kThreads) copy_kernel(const __grid_constant__ Pool p, const int32_t* src, const int32_t* dst) {
  wait_for_predecessor();
  const int64_t from = src[blockIdx.x], to = dst[blockIdx.x];
  if (from < 0 || from >= p.c.pages || to < 0 || to >= p.c.pages || from == to) return;
  copy_piece(p, from, to, blockIdx.y);
}

// blockIdx.y = 0: the child's row of the table, which shares the parent's full pages; others: a piece of the page that the parent's
// last tokens fill in part, copied to the child's own.
__global__ void __launch_bounds__(kThreads) fork_kernel(const __grid_constant__ TakeArgs a, const __grid_constant__ Pool p) {
  wait_for_predecessor();
  const int f = blockIdx.x, parent = a.parents[f], child = a.children[f];
  if (parent < 0 || parent >= a.t.rows || child < 0 || child >= a.t.rows || parent == child) return;
  const int len = max(a.t.tokens[parent], 0), full = min(len >> a.page_shift, a.t.width);
  int source;
  const int fresh = asked(a, f, &source) == 1 ? a.fresh[f] : -1;
  const int32_t* from = a.t.table + (int64_t)parent * a.t.ldt;
  if (blockIdx.y == 0) {
    int32_t* to = a.t.table + (int64_t)child * a.t.ldt;
    for (int j = threadIdx.x; j < a.t.width; j += kThreads) {
      int id = -1;
      if (j < full) {
        id = from[j];
        if (id >= 0 && id < a.pages) atomicAdd(&a.refs[id], 1); else id = -1;
      } else if (j == full) {
        id = fresh;
      }
      to[j] = id;
    }
    if (threadIdx.x == 0) a.t.tokens[child] = len;
    return;
  }
  if (fresh >= 0 && fresh < a.pages) copy_piece(p, source, fresh, blockIdx.y - 1);
}

// ---------------------------------------------------------------------------------------------------------------- compact
struct CompactArgs {
  int32_t* refs;
  int64_t pages;
  Table t;
  int32_t *counts, *src, *dst, *rank;   // workspace: live pages of each chunk; moves; number of the move of each page, or -1
  int32_t* moves;                       // how many there are
  int32_t* spare;
};

__global__ void __launch_bounds__(kThreads) live_kernel(const __grid_constant__ CompactArgs a) {
  __shared__ int warp_sums[kThreads / 32];
  allow_successor();
  wait_for_predecessor();
  int total;
  block_sum_upto(__popc(page_bits<true>(a.refs, a.pages, (int64_t)blockIdx.x * kChunk + threadIdx.x * kPer)), warp_sums, &total);
  if (threadIdx.x == 0) a.counts[blockIdx.x] = total;
}

// With L live pages, the i-th live page at or behind L goes to the i-th free one before L: as few moves as there can be, and no
// target is anyone's source, so all of them may run at once.
__global__ void __launch_bounds__(kThreads) moves_kernel(const __grid_constant__ CompactArgs a, int chunks) {
  __shared__ int warp_sums[kThreads / 32];
  const int t = threadIdx.x;
  allow_successor();
  wait_for_predecessor();
  int ahead = 0, live = 0, total;
  for (int c0 = 0; c0 < chunks; c0 += kThreads) {
    const int n = c0 + t < chunks ? a.counts[c0 + t] : 0;
    block_sum_upto(c0 + t < (int)blockIdx.x ? n : 0, warp_sums, &total);
    ahead += total;
    block_sum_upto(n, warp_sums, &total);
    live += total;
  }
  // live pages before page L: whole chunks, and a part of the one that L falls into
  int front = 0;
  const int cl = live / kChunk;
  for (int c0 = 0; c0 < cl; c0 += kThreads) {
    block_sum_upto(c0 + t < cl ? a.counts[c0 + t] : 0, warp_sums, &total);
    front += total;
  }
  const int64_t q0 = (int64_t)cl * kChunk + t * kPer;
  uint32_t bits = page_bits<true>(a.refs, a.pages, q0);
  if (q0 + kPer > live) bits &= q0 >= live ? 0u : (1u << (live - q0)) - 1u;
  block_sum_upto(__popc(bits), warp_sums, &total);
  front += total;
  const int64_t p0 = (int64_t)blockIdx.x * kChunk + t * kPer;
  bits = page_bits<true>(a.refs, a.pages, p0);
  int before = ahead + block_sum_upto(__popc(bits), warp_sums, &total) - __popc(bits);   // live pages ahead of page p0
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int64_t p = p0 + i;
    const bool is = (bits >> i) & 1u;
    if (p < a.pages) {
      a.rank[p] = is && p >= live ? before - front : -1;
      if (is && p >= live) a.src[before - front] = (int32_t)p;
      if (!is && p < live) a.dst[p - before] = (int32_t)p;
    }
    before += is ? 1 : 0;
  }
  if (blockIdx.x == 0 && t == 0) {
    *a.moves = live - front;
    *a.spare = (int32_t)(a.pages - live);
  }
}

// Page data, counts and table entries of the moved pages.
__global__ void __launch_bounds__(kThreads) compact_kernel(const __grid_constant__ CompactArgs a, const __grid_constant__ Pool p, int pieces) {
  wait_for_predecessor();
  const int64_t n = (int64_t)a.t.rows * a.t.width, gt = (int64_t)gridDim.x * kThreads;
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n; i += gt) {
    int32_t* at = a.t.table + (i / a.t.width) * a.t.ldt + i % a.t.width;
    const int id = *at;
    if (id >= 0 && id < a.pages) {
      const int r = a.rank[id];
      if (r >= 0) *at = a.dst[r];
    }
  }
  const int64_t work = (int64_t)*a.moves * pieces;
  for (int64_t w = blockIdx.x; w < work; w += gridDim.x) {
    const int64_t m = w / pieces, x = w % pieces;
    const int64_t from = a.src[m], to = a.dst[m];
    copy_piece(p, from, to, x);
    if (x == 0 && threadIdx.x == 0) {
      a.refs[to] = a.refs[from];
      a.refs[from] = 0;
    }
  }
}

int check_table(const char* who, int64_t pages, const int32_t* refs, int32_t* table, int64_t ldt, int width, int rows, int32_t* tokens,
                bool with_tokens, Table* out) {
  TQ_REQUIRE(pages >= 0 && pages < (1ll << 31) - kChunk, TQ_ERR_INVALID_ARG, "%s: %lld pages", who, (long long)pages);
  TQ_REQUIRE(width >= 0 && rows >= 0 && ldt >= width, TQ_ERR_INVALID_ARG, "%s: table of %d rows and %d entries, row stride %lld", who, rows, width,
             (long long)ldt);
  TQ_REQUIRE(rows <= (1 << 20) && width <= (1 << 24), TQ_ERR_UNSUPPORTED, "%s: at most 2^20 rows of 2^24 entries", who);
  TQ_REQUIRE(pages == 0 || refs != nullptr, TQ_ERR_INVALID_ARG, "%s: refs is NULL", who);
  TQ_REQUIRE(rows == 0 || ((table || width == 0) && (tokens || !with_tokens)), TQ_ERR_INVALID_ARG, "%s: table or tokens is NULL", who);
  *out = Table{table, ldt, width, rows, tokens};
  return TQ_OK;
}

struct Space {
  int32_t *counts, *offsets, *fresh, *src, *dst, *rank, *moves;
  size_t bytes;
};
Space lay_out(void* workspace, int64_t pages, int units) {
  Space s;
  size_t at = 0;
  auto take = [&](int64_t n) {
    int32_t* p = reinterpret_cast<int32_t*>(static_cast<char*>(workspace) + at);
    at += (size_t)round_up64(n * 4, 256);
    return p;
  };
  s.counts = take((pages + kChunk - 1) / kChunk + 1);
  s.offsets = take((int64_t)units + 1);
  s.fresh = take((int64_t)units + 1);
  s.moves = take(1);
  s.src = take(pages);
  s.dst = take(pages);
  s.rank = take(pages);
  s.bytes = at;
  return s;
}

int launch_take(const char* who, TakeArgs& a, cudaStream_t st) {
  if (a.pages <= kSmall) {
    TQ_CHECK_CUDA(launch_dependent(take_small_kernel, dim3(1), dim3(kThreads), 0, st, a), who);
    count_launches(1);
    return TQ_OK;
  }
  const int chunks = std::max<int>(1, (int)((a.pages + kChunk - 1) / kChunk));
  TQ_CHECK_CUDA(launch_dependent(count_kernel, dim3((unsigned)chunks + 1), dim3(kThreads), 0, st, a, chunks), who);
  TQ_CHECK_CUDA(launch_dependent(take_kernel, dim3((unsigned)chunks), dim3(kThreads), 0, st, a, chunks), who);
  count_launches(2);
  return TQ_OK;
}

#define TQ_REQUIRE_SPACE(need)                                                                                                       \
  TQ_REQUIRE(workspace != nullptr && workspace_bytes >= (need), TQ_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", who,     \
             workspace_bytes, (size_t)(need));                                                                                       \
  TQ_REQUIRE((reinterpret_cast<uintptr_t>(workspace) & 255) == 0, TQ_ERR_ALIGNMENT, "%s: workspace is not 256-byte aligned", who)

}  // namespace pages
}  // namespace tq

extern "C" size_t tq_pages_workspace_bytes(int64_t pages, int requests) {
  if (pages < 0 || requests < 0) return 0;
  return tq::pages::lay_out(nullptr, pages, requests).bytes;
}

extern "C" int tq_pages_free(int32_t* refs, int64_t pages, int32_t* table, int64_t ldt, int width, int rows, int32_t* tokens,
                             const int32_t* seqs, int count, void* stream) {
  using namespace tq;
  using namespace tq::pages;
  const char* who = "tq_pages_free";
  TQ_RANGE(who);
  Table t;
  const int rc = check_table(who, pages, refs, table, ldt, width, rows, tokens, false, &t);
  if (rc != TQ_OK) return rc;
  TQ_REQUIRE(count >= 0, TQ_ERR_INVALID_ARG, "%s: negative size", who);
  if (count == 0 || rows == 0) return TQ_OK;
  TQ_REQUIRE(seqs != nullptr, TQ_ERR_INVALID_ARG, "%s: seqs is NULL", who);
  TQ_CHECK_CUDA(launch_dependent(free_kernel, dim3((unsigned)count), dim3(kThreads), 0, static_cast<cudaStream_t>(stream), refs, pages, t, seqs), who);
  count_launches(1);
  return TQ_OK;
}

extern "C" int tq_pages_extend(int32_t* refs, int64_t pages, int32_t* table, int64_t ldt, int width, int rows, const int32_t* tokens,
                               const int32_t* next, int page_tokens, int32_t* spare, void* workspace, size_t workspace_bytes, void* stream) {
  using namespace tq;
  using namespace tq::pages;
  const char* who = "tq_pages_extend";
  TQ_RANGE(who);
  TakeArgs a{};
  const int rc = check_table(who, pages, refs, table, ldt, width, rows, const_cast<int32_t*>(tokens), true, &a.t);
  if (rc != TQ_OK) return rc;
  for (int s = 4; s <= 7; ++s)
    if (page_tokens == 1 << s) a.page_shift = s;
  TQ_REQUIRE(a.page_shift != 0, TQ_ERR_UNSUPPORTED, "%s: pages of %d tokens (16, 32, 64 or 128)", who, page_tokens);
  TQ_REQUIRE((int64_t)rows * width < (1ll << 31), TQ_ERR_UNSUPPORTED, "%s: tables of 2^31 entries and more", who);
  if (rows == 0) return TQ_OK;
  TQ_REQUIRE(next != nullptr && spare != nullptr, TQ_ERR_INVALID_ARG, "%s: next or spare is NULL", who);
  const Space s = lay_out(workspace, pages, rows);
  TQ_REQUIRE_SPACE(s.bytes);
  a.refs = refs; a.pages = pages; a.next = next; a.units = rows; a.counts = s.counts; a.offsets = s.offsets; a.fresh = s.fresh; a.spare = spare;
  return launch_take(who, a, static_cast<cudaStream_t>(stream));
}

extern "C" int tq_pages_fork(const tq_kv8* cache, int32_t* refs, int32_t* table, int64_t ldt, int width, int rows, int32_t* tokens,
                             const int32_t* parents, const int32_t* children, int count, int32_t* spare, void* workspace,
                             size_t workspace_bytes, void* stream) {
  using namespace tq;
  using namespace tq::pages;
  const char* who = "tq_pages_fork";
  TQ_RANGE(who);
  Cache c;
  TakeArgs a{};
  int rc = kv8::check_cache(who, cache, &c);
  if (rc == TQ_OK) rc = check_table(who, c.pages, refs, table, ldt, width, rows, tokens, true, &a.t);
  if (rc != TQ_OK) return rc;
  TQ_REQUIRE(count >= 0, TQ_ERR_INVALID_ARG, "%s: negative size", who);
  if (count == 0 || rows == 0) return TQ_OK;
  TQ_REQUIRE(parents != nullptr && children != nullptr && spare != nullptr, TQ_ERR_INVALID_ARG, "%s: parents, children or spare is NULL", who);
  const Space s = lay_out(workspace, c.pages, count);
  TQ_REQUIRE_SPACE(s.bytes);
  a.refs = refs; a.pages = c.pages; a.parents = parents; a.children = children; a.units = count; a.page_shift = c.page_shift;
  a.counts = s.counts; a.offsets = s.offsets; a.fresh = s.fresh; a.spare = spare;
  const Pool p = pool_of(c);
  const int64_t pieces = (p.vectors() + kPiece - 1) / kPiece;
  TQ_REQUIRE(pieces < 65535, TQ_ERR_UNSUPPORTED, "%s: pages of %lld bytes", who, (long long)p.vectors() * 16);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  rc = launch_take(who, a, st);
  if (rc != TQ_OK) return rc;
  TQ_CHECK_CUDA(launch_dependent(fork_kernel, dim3((unsigned)count, (unsigned)pieces + 1), dim3(kThreads), 0, st, a, p), who);
  count_launches(1);
  return TQ_OK;
}

extern "C" int tq_pages_compact(const tq_kv8* cache, int32_t* refs, int32_t* table, int64_t ldt, int width, int rows, int32_t* spare,
                                void* workspace, size_t workspace_bytes, void* stream) {
  using namespace tq;
  using namespace tq::pages;
  const char* who = "tq_pages_compact";
  TQ_RANGE(who);
  Cache c;
  CompactArgs a{};
  int rc = kv8::check_cache(who, cache, &c);
  if (rc == TQ_OK) rc = check_table(who, c.pages, refs, table, ldt, width, rows, nullptr, false, &a.t);
  if (rc != TQ_OK) return rc;
  if (c.pages == 0) return TQ_OK;
  TQ_REQUIRE(spare != nullptr, TQ_ERR_INVALID_ARG, "%s: spare is NULL", who);
  const Space s = lay_out(workspace, c.pages, 0);
  TQ_REQUIRE_SPACE(s.bytes);
  a.refs = refs; a.pages = c.pages; a.counts = s.counts; a.src = s.src; a.dst = s.dst; a.rank = s.rank; a.moves = s.moves; a.spare = spare;
  int dev = 0, sms = 0;
  TQ_CHECK_CUDA(cudaGetDevice(&dev), who);
  TQ_CHECK_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev), who);
  const Pool p = pool_of(c);
  const int pieces = (int)((p.vectors() + kPiece - 1) / kPiece), chunks = (int)((c.pages + kChunk - 1) / kChunk);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  TQ_CHECK_CUDA(launch_dependent(live_kernel, dim3((unsigned)chunks), dim3(kThreads), 0, st, a), who);
  TQ_CHECK_CUDA(launch_dependent(moves_kernel, dim3((unsigned)chunks), dim3(kThreads), 0, st, a, chunks), who);
  TQ_CHECK_CUDA(launch_dependent(compact_kernel, dim3((unsigned)sms * 8), dim3(kThreads), 0, st, a, p, pieces), who);
  count_launches(3);
  return TQ_OK;
}

extern "C" int tq_pages_copy(const tq_kv8* cache, const int32_t* src, const int32_t* dst, int count, void* stream) {
  using namespace tq;
  using namespace tq::pages;
  const char* who = "tq_pages_copy";
  TQ_RANGE(who);
  Cache c;
  const int rc = kv8::check_cache(who, cache, &c);
  if (rc != TQ_OK) return rc;
  TQ_REQUIRE(count >= 0, TQ_ERR_INVALID_ARG, "%s: negative size", who);
  if (count == 0 || c.pages == 0) return TQ_OK;
  TQ_REQUIRE(src != nullptr && dst != nullptr, TQ_ERR_INVALID_ARG, "%s: src or dst is NULL", who);
  const Pool p = pool_of(c);
  const int64_t pieces = (p.vectors() + kPiece - 1) / kPiece;
  TQ_REQUIRE(pieces <= 65535, TQ_ERR_UNSUPPORTED, "%s: pages of %lld bytes", who, (long long)p.vectors() * 16);
  TQ_CHECK_CUDA(launch_dependent(copy_kernel, dim3((unsigned)count, (unsigned)pieces), dim3(kThreads), 0, static_cast<cudaStream_t>(stream), p, src,
                                 dst), who);
  count_launches(1);
  return TQ_OK;
}
