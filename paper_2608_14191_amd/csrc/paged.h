// The paged cache at input precision: kernel arguments and launchers of the rotary, append and
// attention kernels (rope.hip, paged.hip) and of the page-table kernels (pages.hip).
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "aatc_paged.h"
#include "workspace.h"

namespace aatc {

constexpr int kMinPage = 8, kMaxPage = 4096;      // tokens of a page (a power of two)

// Tokens to rotate and store.  Sources: queries, keys, values; rotated queries go to `q_out`,
// keys and values to their slots of the pages.
struct TurnArgs {
  const void* x[3];
  int64_t x_stride[3];            // elements from token to token
  int heads[3];
  void* q_out;
  int64_t q_out_stride;
  int64_t tok0, n_tok;            // tokens tok0 .. n_tok - 1
  const int32_t* seq;             // sequence of each token, or null: the token's own index
  const int32_t* pos;
  bool skip_negative;             // tokens of negative position are left out (append)
  bool copy_rest;                 // q_out is another buffer: its channels behind rot are copied
  const double* freq;             // device [half]
  int half;                       // rotated pairs
  float factor, sign;
  void* k_pages;
  void* v_pages;
  int64_t page_stride, head_stride, tok_stride;   // elements
  int64_t n_pages;
  int page_shift;
  const int32_t* table;
  int64_t table_stride;
  int rows, max_pages;
};

// x_dtype: of x and q_out; c_dtype: of the pages.
aatc_status launch_turn(const TurnArgs& a, aatc_dtype x_dtype, aatc_dtype c_dtype, int layout,
                        void* stream);

struct PagedArgs {
  const char* k;
  const char* v;
  int64_t page_stride, head_stride, tok_stride;   // bytes
  const int32_t* table;
  int64_t table_stride;
  const int32_t* seq_len;
  const void* q;
  int64_t q_stride;               // elements from sequence to sequence
  float* out;                     // [batch][n_q_heads][d], or null: `seg`
  float* lse;                     // [batch][n_q_heads] or null
  Partial* seg;                   // [batch][n_q_heads] softmax partials instead of outputs
  const float* slopes;            // [n_q_heads] or null
  unsigned* counters;
  Partial* parts;
  int parts_bytes, slot_heads;    // of `parts`; partials of a slot
  int batch, n_q_heads, n_kv_heads, G, hg, q_dtype;
  int n_pages, max_pages, page_shift, len_max;    // len_max: tokens that a row can name
  int window, sink;
  float scale, cap;               // cap 0: none
};

// The compressed cache's attention joined with that of pages (decode.hip): `pages` as for
// launch_paged, less its outputs.
aatc_status launch_decode_paged(const void* params_k, const void* params_v, int batch,
                                int n_q_heads, int n_kv_heads, const void* q, aatc_dtype q_dtype,
                                const void* k_codes, const uint16_t* k_alpha, const void* v_codes,
                                const uint16_t* v_alpha, const int32_t* seq_len, int64_t cap,
                                int rk, int rv, float softmax_scale, float* out, void* workspace,
                                void* stream, const PagedArgs& pages, aatc_dtype pages_dtype,
                                void* pages_workspace);

size_t paged_workspace_bytes(int batch, int n_q_heads, int n_kv_heads);
aatc_status launch_paged(PagedArgs a, aatc_dtype c_dtype, void* workspace, void* stream);

aatc_status launch_pages_copy(void* base, int64_t n_pools, int64_t pool_stride, int64_t n_pages,
                              int64_t page_bytes, const int32_t* pairs, int64_t n,
                              const int32_t* n_dev, void* stream);
aatc_status launch_pages_fork(const aatc_page_table& src, const aatc_page_table& dst,
                              int32_t* ref, int64_t n_pages, const int32_t* pairs, int64_t n,
                              void* stream);
aatc_status launch_pages_free(const aatc_page_table& t, int32_t* ref, int64_t n_pages,
                              const int32_t* rows, int64_t n, void* stream);
size_t pages_workspace_bytes(int64_t rows, int64_t n_pages);
aatc_status launch_pages_reserve(const aatc_page_table& t, int32_t* ref, int64_t n_pages,
                                 int page_tokens, const int32_t* held, const int32_t* wanted,
                                 int32_t* pairs, int32_t* lacking, void* workspace, void* stream);
aatc_status launch_pages_compact(const aatc_page_table& t, const int32_t* ref, int64_t n_pages,
                                 const aatc_page_table& t_out, int32_t* ref_out, int32_t* pairs,
                                 int32_t* moves, void* workspace, void* stream);

}  // namespace aatc
