// What the entry points over pages ask of their arguments, and the kernel arguments that they share.
// Host code.
#pragma once

#include <algorithm>
#include <cmath>

#include "aatc_paged.h"
#include "paged.h"
#include "params.h"

namespace aatc {

constexpr int64_t kMaxPages = INT32_MAX;
constexpr int64_t kMaxList = (int64_t)1 << 30;        // tokens or pairs of one call

// Caps from here on change no score (below 1e26 tanh(z / cap) is z / cap in float32, and a softmax
// with larger ones has only zeros and ones), but their products pass float32's range.
constexpr float kNoCap = 1e30f;

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
inline bool known(aatc_dtype t) { return t == AATC_F32 || t == AATC_BF16 || t == AATC_F16; }
inline int size_of(aatc_dtype t) { return t == AATC_F32 ? 4 : 2; }

// A buffer of tokens, `heads` heads of kD elements each.
inline bool tokens_ok(const void* x, aatc_dtype t, int64_t stride, int64_t heads) {
  return x && aligned(x, size_of(t)) && stride >= heads * kD && stride < ((int64_t)1 << 40);
}

inline aatc_status check_rope(const aatc_rope_spec* r) {
  if (!r || !r->freq || !aligned(r->freq, 8)) return AATC_E_INVALID;
  if (r->rot_dim < 2 || r->rot_dim > kD || r->rot_dim % 2) return AATC_E_INVALID;
  if (r->layout != AATC_ROPE_HALF && r->layout != AATC_ROPE_INTERLEAVED) return AATC_E_INVALID;
  return std::isfinite(r->factor) ? AATC_OK : AATC_E_INVALID;
}

inline aatc_status check_cache(const aatc_paged_cache* c) {
  if (!c) return AATC_E_INVALID;
  if (c->d != kD) return AATC_E_UNSUPPORTED;
  if (!c->k_pages || !c->v_pages || !aligned(c->k_pages, 16) || !aligned(c->v_pages, 16))
    return AATC_E_INVALID;
  const aatc_dtype t = (aatc_dtype)c->dtype;
  if (!known(t) || c->n_kv_heads < 1 || c->n_pages < 1 || c->n_pages > kMaxPages)
    return AATC_E_INVALID;
  if (c->page_tokens < kMinPage || c->page_tokens > kMaxPage ||
      (c->page_tokens & (c->page_tokens - 1)))
    return AATC_E_INVALID;
  const int64_t unit = 16 / size_of(t);
  for (int64_t s : {c->page_stride, c->head_stride, c->tok_stride})
    if (s < kD || s % unit || s >= ((int64_t)1 << 40)) return AATC_E_INVALID;
  return AATC_OK;
}

inline aatc_status check_table(const aatc_page_table* t) {
  if (!t || !t->table || !aligned(t->table, 4)) return AATC_E_INVALID;
  if (t->rows < 1 || t->max_pages < 1 || t->stride < t->max_pages) return AATC_E_INVALID;
  return (int64_t)t->rows * t->max_pages <= kMaxList ? AATC_OK : AATC_E_UNSUPPORTED;
}

inline int log2_of(int x) {
  int s = 0;
  while ((1 << s) < x) ++s;
  return s;
}

// Tokens that a row of the table can name.
inline int64_t row_tokens(const aatc_page_table& t, int page_tokens) {
  return std::min<int64_t>((int64_t)t.max_pages * page_tokens, INT32_MAX - 4096);
}

// The plan of the attention counts tiles (16 tokens at least) in 32 bits.
inline bool too_many_tiles(const aatc_paged_cache& c, const aatc_page_table& t, int64_t batch, int hq) {
  const int64_t hg = (hq / c.n_kv_heads + 15) / 16;
  return (row_tokens(t, c.page_tokens) / 16 + 1) > kMaxList / (batch * c.n_kv_heads * hg);
}

inline aatc_status check_counts(const int32_t* ref, int64_t n_pages) {
  return ref && aligned(ref, 4) && n_pages >= 1 && n_pages <= kMaxPages ? AATC_OK
                                                                        : AATC_E_INVALID;
}

// The arguments that the attention over pages alone and with a compressed cache share.
inline PagedArgs paged_args(const aatc_paged_cache& c, const aatc_page_table& t, const int32_t* len,
                     int batch, int n_q_heads, const void* q, aatc_dtype q_dtype,
                     int64_t q_stride, float scale) {
  const int size = size_of((aatc_dtype)c.dtype);
  PagedArgs a{};
  a.k = static_cast<const char*>(c.k_pages);
  a.v = static_cast<const char*>(c.v_pages);
  a.page_stride = c.page_stride * size;
  a.head_stride = c.head_stride * size;
  a.tok_stride = c.tok_stride * size;
  a.table = t.table;
  a.table_stride = t.stride;
  a.seq_len = len;
  a.q = q;
  a.q_stride = q_stride;
  a.batch = batch;
  a.n_q_heads = n_q_heads;
  a.n_kv_heads = c.n_kv_heads;
  a.G = n_q_heads / c.n_kv_heads;
  a.hg = (a.G + 15) / 16;
  a.q_dtype = (int)q_dtype;
  a.n_pages = (int)c.n_pages;
  a.max_pages = t.max_pages;
  a.page_shift = log2_of(c.page_tokens);
  a.len_max = (int)row_tokens(t, c.page_tokens);
  a.scale = scale;
  return a;
}

}  // namespace aatc
