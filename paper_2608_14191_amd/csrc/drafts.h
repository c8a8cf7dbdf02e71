// Drafted tokens over the paged cache: kernel arguments and launchers (drafts.hip).
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "aatc_drafts.h"
#include "paged.h"

namespace aatc {

constexpr int kMaxDrafts = AATC_MAX_DRAFTS;       // a lane, and a bit of 64, for each
constexpr int kMaxColumns = 16384;                // queries of a (sequence, KV head)
constexpr int64_t kMaxTreeGroups = (int64_t)1 << 22;
constexpr int64_t kMaxMoved = (int64_t)1 << 31;   // 16-byte pieces of a token, of all layers: a thread each

struct TreeArgs {
  PagedArgs p;                    // q_stride: from draft to draft
  const int32_t* n_draft;         // or null
  const int32_t* parent;          // or null: a chain
  int drafts;                     // of each sequence at most
  int blocks, block_cols;         // a (sequence, KV head)'s queries: blocks of so many columns
  int units;                      // runs of tokens that fill the chip (each `blocks` workgroups)
  int quantum;                    // tiles
  bool far;                       // pools that do not fit the caches: loads past them
};

size_t tree_workspace_bytes(int batch, int drafts, int n_q_heads, int n_kv_heads);
// Whether the grid of such a call can be launched.
bool tree_fits(int64_t batch, int drafts, int n_q_heads, int n_kv_heads);
aatc_status launch_tree(TreeArgs a, aatc_dtype c_dtype, void* workspace, void* stream);

struct AcceptArgs {
  char* k;
  char* v;
  int64_t page_stride, head_stride, tok_stride, layer_stride;   // bytes
  const int32_t* table;
  int64_t table_stride;
  const int32_t* seq_len;
  const int32_t* n_draft;         // or null
  const int32_t* parent;          // or null
  const int32_t* drafted;
  const int32_t* chosen;
  int32_t* path;
  int32_t* accepted;
  int32_t* next;
  int32_t* len_out;
  int batch, drafts, layers, n_kv_heads, n_pages, max_pages, page_shift, len_max;
  int pieces;                     // 16-byte pieces of a head's token
};

aatc_status launch_tree_accept(const AcceptArgs& a, void* stream);

}  // namespace aatc
