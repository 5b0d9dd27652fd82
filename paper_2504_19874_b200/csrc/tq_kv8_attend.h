// Attention over a paged 8-bit KV cache: what the few-query and the many-query kernels are given.
#pragma once

#include "tq_kv8.h"

namespace tq {
namespace kv8 {

constexpr int kMaxCols = 16;   // columns of a block of the few-query kernel

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
  float *part_ml, *part_o;
};

}  // namespace kv8
}  // namespace tq
