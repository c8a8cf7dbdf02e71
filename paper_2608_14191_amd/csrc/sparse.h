// Sparse attention over the paged cache: kernel arguments and launchers (sparse.hip).
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "aatc_sparse.h"
#include "paged.h"

namespace aatc {

constexpr int kBoundBytes = 2 * kD;               // of a page and KV head: largest, smallest
constexpr int kMaxSay = 256;                      // query heads of a KV head
constexpr int kMaxMost = 1 << 20;                 // picked pages
constexpr int64_t kMaxSparseGroups = (int64_t)1 << 22;

struct BoundsArgs {
  const char* k;
  int64_t page_stride, head_stride, tok_stride;   // bytes
  const int32_t* table;
  int64_t table_stride;
  const int32_t* held;            // or null: 0
  const int32_t* wanted;
  int8_t* codes;
  float* scales;
  int rows, n_kv_heads, n_pages, max_pages, page_shift, len_max;
};

aatc_status launch_bounds(const BoundsArgs& a, aatc_dtype dtype, void* stream);

struct SparseArgs {
  PagedArgs p;
  const int8_t* codes;
  const float* scales;
  uint32_t* keys;                 // [batch][n_kv_heads][key_stride], in the order of the scores
  int64_t key_stride;
  int32_t* picked;                // [batch][n_kv_heads][most]
  int most, first, last;
  int run;                        // tiles of a workgroup at most
  int parts;                      // workgroups of a row
};

size_t sparse_workspace_bytes(int batch, int n_q_heads, int n_kv_heads, int64_t max_pages);
// Whether the grids of such a call can be launched.
bool sparse_fits(int64_t batch, int n_q_heads, int n_kv_heads, int64_t max_pages);
aatc_status launch_sparse(SparseArgs a, aatc_dtype c_dtype, void* workspace, void* stream);

}  // namespace aatc
