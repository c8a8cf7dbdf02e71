// C ABI of the paged cache (aatc_paged.h): argument validation and dispatch to the HIP
// launchers.  No exception crosses the boundary.
#include <algorithm>
#include <cmath>
#include <cstring>

#include "aatc_paged.h"
#include "launch.h"
#include "paged.h"
#include "paged_checks.h"
#include "params.h"

using namespace aatc;

namespace {

constexpr int64_t kMaxRows = ((int64_t)1 << 24) - 1;  // rows listed: a workgroup of 256 each
constexpr int64_t kMaxForks = (int64_t)1 << 18;       // pairs, each compared with all later ones

}  // namespace

extern "C" aatc_status aatc_rope_frequencies(int32_t rot_dim, double base,
                                             aatc_rope_scaling scaling, double scale,
                                             int64_t trained, double low, double high,
                                             double* freq, float* factor) {
  if (!freq || rot_dim < 2 || rot_dim > kD || rot_dim % 2) return AATC_E_INVALID;
  if (!(base > 1.0) || !std::isfinite(base)) return AATC_E_INVALID;
  if (scaling < AATC_ROPE_PLAIN || scaling > AATC_ROPE_YARN) return AATC_E_INVALID;
  const bool bands = scaling == AATC_ROPE_BANDS || scaling == AATC_ROPE_YARN;
  if (scaling != AATC_ROPE_PLAIN && (!(scale >= 1.0) || !std::isfinite(scale)))
    return AATC_E_INVALID;
  if (scaling == AATC_ROPE_NTK && rot_dim < 4) return AATC_E_INVALID;
  if (bands && (trained < 1 || !(low > 0.0) || !(high > low) || !std::isfinite(high)))
    return AATC_E_INVALID;
  const double two_pi = 6.283185307179586476925;
  if (scaling == AATC_ROPE_NTK) base *= std::pow(scale, (double)rot_dim / (rot_dim - 2));
  // YARN: the pair at which a pair turns u times within the trained positions.
  double from = 0.0, to = 0.0;
  if (scaling == AATC_ROPE_YARN) {
    auto pair_at = [&](double u) {
      return rot_dim * std::log((double)trained / (u * two_pi)) / (2.0 * std::log(base));
    };
    from = std::max(std::floor(pair_at(high)), 0.0);
    to = std::min(std::ceil(pair_at(low)), rot_dim - 1.0);
    to = std::max(to, from + 0.001);
  }
  for (int i = 0; i < rot_dim / 2; ++i) {
    double f = std::pow(base, -2.0 * i / rot_dim);
    double keep = 1.0;                              // share of f in the mix of f and f / scale
    if (scaling == AATC_ROPE_LINEAR) keep = 0.0;
    if (scaling == AATC_ROPE_BANDS)
      keep = std::min(1.0, std::max(0.0, ((double)trained * f / two_pi - low) / (high - low)));
    if (scaling == AATC_ROPE_YARN) keep = 1.0 - std::min(1.0, std::max(0.0, (i - from) / (to - from)));
    if (keep < 1.0) f = keep * f + (1.0 - keep) * (f / scale);
    freq[i] = f;
  }
  if (factor) *factor = scaling == AATC_ROPE_YARN ? (float)(0.1 * std::log(scale) + 1.0) : 1.0f;
  return AATC_OK;
}

extern "C" aatc_status aatc_rope(const void* x, aatc_dtype dtype, int64_t n_tok, int32_t n_heads,
                                 int32_t d, int64_t x_tok_stride, const int32_t* pos,
                                 const aatc_rope_spec* spec, int32_t inverse, void* out,
                                 int64_t out_tok_stride, void* stream) {
  try {
    if (d != kD) return AATC_E_UNSUPPORTED;
    if (!known(dtype) || n_tok < 0 || n_tok > kMaxList || n_heads < 1 || n_heads > 65535)
      return AATC_E_INVALID;
    if (!tokens_ok(x, dtype, x_tok_stride, n_heads) ||
        !tokens_ok(out, dtype, out_tok_stride, n_heads) || !pos || !aligned(pos, 4))
      return AATC_E_INVALID;
    if (x == out && x_tok_stride != out_tok_stride) return AATC_E_INVALID;
    const aatc_status e = check_rope(spec);
    if (e != AATC_OK) return e;
    if (n_tok == 0) return AATC_OK;
    TurnArgs a{};
    a.x[0] = x;
    a.x_stride[0] = x_tok_stride;
    a.heads[0] = n_heads;
    a.q_out = out;
    a.q_out_stride = out_tok_stride;
    a.n_tok = n_tok;
    a.pos = pos;
    a.copy_rest = x != out;
    a.freq = spec->freq;
    a.half = spec->rot_dim / 2;
    a.factor = spec->factor;
    a.sign = inverse ? -1.f : 1.f;
    return launch_turn(a, dtype, dtype, spec->layout, stream);
  } catch (...) {
    return AATC_E_INVALID;
  }
}

extern "C" aatc_status aatc_paged_append(const aatc_paged_cache* cache,
                                         const aatc_page_table* table, int64_t n_tok,
                                         aatc_dtype x_dtype, const void* k, int64_t k_tok_stride,
                                         const void* v, int64_t v_tok_stride, const int32_t* seq,
                                         const int32_t* pos, const aatc_rope_spec* rope,
                                         int32_t n_q_heads, const void* q, int64_t q_tok_stride,
                                         void* q_out, int64_t q_out_tok_stride, void* stream) {
  try {
    aatc_status e = check_cache(cache);
    if (e == AATC_OK) e = check_table(table);
    if (e == AATC_OK && rope) e = check_rope(rope);
    if (e != AATC_OK) return e;
    const int hkv = cache->n_kv_heads;
    if (!known(x_dtype) || n_tok < 0 || n_tok > kMaxList || hkv > 65535) return AATC_E_INVALID;
    if (!tokens_ok(k, x_dtype, k_tok_stride, hkv) || !tokens_ok(v, x_dtype, v_tok_stride, hkv))
      return AATC_E_INVALID;
    if (!pos || !aligned(pos, 4) || !aligned(seq, 4)) return AATC_E_INVALID;
    if (n_q_heads < 0 || n_q_heads > 65535 || (n_q_heads == 0) != (q == nullptr))
      return AATC_E_INVALID;
    if (q && (!tokens_ok(q, x_dtype, q_tok_stride, n_q_heads) ||
              !tokens_ok(q_out, x_dtype, q_out_tok_stride, n_q_heads) ||
              (q == q_out && q_tok_stride != q_out_tok_stride)))
      return AATC_E_INVALID;
    if (n_tok == 0) return AATC_OK;
    TurnArgs a{};
    a.x[0] = q;
    a.x[1] = k;
    a.x[2] = v;
    a.x_stride[0] = q_tok_stride;
    a.x_stride[1] = k_tok_stride;
    a.x_stride[2] = v_tok_stride;
    a.heads[0] = n_q_heads;
    a.heads[1] = a.heads[2] = hkv;
    a.q_out = q_out;
    a.q_out_stride = q_out_tok_stride;
    a.n_tok = n_tok;
    a.seq = seq;
    a.pos = pos;
    a.skip_negative = true;
    a.copy_rest = q != q_out;
    a.freq = rope ? rope->freq : nullptr;
    a.half = rope ? rope->rot_dim / 2 : 0;
    a.factor = rope ? rope->factor : 1.f;
    a.sign = 1.f;
    a.k_pages = cache->k_pages;
    a.v_pages = cache->v_pages;
    a.page_stride = cache->page_stride;
    a.head_stride = cache->head_stride;
    a.tok_stride = cache->tok_stride;
    a.n_pages = cache->n_pages;
    a.page_shift = log2_of(cache->page_tokens);
    a.table = table->table;
    a.table_stride = table->stride;
    a.rows = table->rows;
    a.max_pages = table->max_pages;
    return launch_turn(a, x_dtype, (aatc_dtype)cache->dtype, rope ? rope->layout : AATC_ROPE_HALF,
                       stream);
  } catch (...) {
    return AATC_E_INVALID;
  }
}

extern "C" size_t aatc_paged_decode_workspace_bytes(int32_t batch, int32_t n_q_heads,
                                                    int32_t n_kv_heads) {
  if (batch < 1 || n_q_heads < 1 || n_kv_heads < 1 || n_q_heads % n_kv_heads) return 0;
  return paged_workspace_bytes(batch, n_q_heads, n_kv_heads);
}

extern "C" aatc_status aatc_paged_decode_attention(
    const aatc_paged_cache* cache, const aatc_page_table* table, const int32_t* seq_len,
    int32_t batch, int32_t n_q_heads, const void* q, aatc_dtype q_dtype, int64_t q_stride,
    float softmax_scale, int32_t window, int32_t sink, float softcap, const float* slopes,
    float* out, float* lse, void* workspace, size_t ws_bytes, void* stream) {
  try {
    aatc_status e = check_cache(cache);
    if (e == AATC_OK) e = check_table(table);
    if (e != AATC_OK) return e;
    if (batch < 1 || batch > table->rows || n_q_heads < 1 || n_q_heads % cache->n_kv_heads)
      return AATC_E_INVALID;
    if (!seq_len || !aligned(seq_len, 4) || !known(q_dtype) ||
        !tokens_ok(q, q_dtype, q_stride, n_q_heads))
      return AATC_E_INVALID;
    if (!std::isfinite(softmax_scale) || window < 0 || sink < 0 || !(softcap >= 0.f) ||
        !std::isfinite(softcap) || (softcap > 0.f && !std::isfinite(softmax_scale / softcap)))
      return AATC_E_INVALID;
    if (!out || !aligned(out, 16) || !aligned(lse, 4) || !aligned(slopes, 4) || !workspace ||
        !aligned(workspace, 256))
      return AATC_E_INVALID;
    if (too_many_tiles(*cache, *table, batch, n_q_heads)) return AATC_E_UNSUPPORTED;
    if (ws_bytes < paged_workspace_bytes(batch, n_q_heads, cache->n_kv_heads))
      return AATC_E_WORKSPACE;
    PagedArgs a = paged_args(*cache, *table, seq_len, batch, n_q_heads, q, q_dtype, q_stride,
                             softmax_scale);
    a.window = window;
    a.sink = sink;
    a.cap = softcap < kNoCap ? softcap : 0.f;
    a.slopes = slopes;
    a.out = out;
    a.lse = lse;
    return launch_paged(a, (aatc_dtype)cache->dtype, workspace, stream);
  } catch (...) {
    return AATC_E_INVALID;
  }
}

extern "C" size_t aatc_decode_paged_workspace_bytes(int32_t batch, int32_t n_q_heads,
                                                    int32_t n_kv_heads, int64_t cap) {
  if (batch < 1 || n_q_heads < 1 || n_kv_heads < 1 || n_q_heads % n_kv_heads || cap < 0) return 0;
  return round256(decode_workspace_bytes(batch, n_q_heads, n_kv_heads, cap)) +
         paged_workspace_bytes(batch, n_q_heads, n_kv_heads);
}

extern "C" aatc_status aatc_decode_attention_paged(
    const void* dev_params_k, const void* dev_params_v, int32_t batch, int32_t n_q_heads,
    int32_t n_kv_heads, int32_t d, const void* q, aatc_dtype q_dtype, const void* k_codes,
    const uint16_t* k_alpha, const void* v_codes, const uint16_t* v_alpha,
    const int32_t* seq_len, int64_t cap, int32_t k_record_bytes, int32_t v_record_bytes,
    float softmax_scale, const aatc_paged_cache* cache, const aatc_page_table* table,
    const int32_t* page_len, float* out, void* workspace, size_t ws_bytes, void* stream) {
  try {
    if (d != kD) return AATC_E_UNSUPPORTED;
    aatc_status e = check_cache(cache);
    if (e == AATC_OK) e = check_table(table);
    if (e != AATC_OK) return e;
    if (batch < 1 || batch > table->rows || n_q_heads < 1 || n_kv_heads < 1 ||
        n_q_heads % n_kv_heads || cache->n_kv_heads != n_kv_heads || !page_len ||
        !aligned(page_len, 4))
      return AATC_E_INVALID;
    if (cap < kTile || cap % kTile || cap >= ((int64_t)1 << 31)) return AATC_E_INVALID;
    const size_t own = round256(decode_workspace_bytes(batch, n_q_heads, n_kv_heads, cap));
    e = check_decode(dev_params_k, dev_params_v, batch, n_q_heads, n_kv_heads, d, q, q_dtype,
                     k_codes, k_alpha, v_codes, v_alpha, seq_len, cap, k_record_bytes,
                     v_record_bytes, softmax_scale, out, workspace, ws_bytes);
    if (e != AATC_OK) return e;
    if (too_many_tiles(*cache, *table, batch, n_q_heads)) return AATC_E_UNSUPPORTED;
    if (ws_bytes < own + paged_workspace_bytes(batch, n_q_heads, n_kv_heads))
      return AATC_E_WORKSPACE;
    const PagedArgs a = paged_args(*cache, *table, page_len, batch, n_q_heads, q, q_dtype,
                                   (int64_t)n_q_heads * kD, softmax_scale);
    return launch_decode_paged(dev_params_k, dev_params_v, batch, n_q_heads, n_kv_heads, q,
                               q_dtype, k_codes, k_alpha, v_codes, v_alpha, seq_len, cap,
                               k_record_bytes, v_record_bytes, softmax_scale, out, workspace,
                               stream, a, (aatc_dtype)cache->dtype,
                               static_cast<char*>(workspace) + own);
  } catch (...) {
    return AATC_E_INVALID;
  }
}

extern "C" aatc_status aatc_pages_fork(const aatc_page_table* src, const aatc_page_table* dst,
                                       int32_t* ref, int64_t n_pages, const int32_t* pairs,
                                       int64_t n, void* stream) {
  try {
    aatc_status e = check_table(src);
    if (e == AATC_OK) e = check_table(dst);
    if (e == AATC_OK) e = check_counts(ref, n_pages);
    if (e != AATC_OK) return e;
    if (src->max_pages != dst->max_pages || n < 0 || n > kMaxList || !pairs || !aligned(pairs, 4))
      return AATC_E_INVALID;
    if (n == 0) return AATC_OK;
    if (n > kMaxForks) return AATC_E_UNSUPPORTED;
    return launch_pages_fork(*src, *dst, ref, n_pages, pairs, n, stream);
  } catch (...) {
    return AATC_E_INVALID;
  }
}

extern "C" aatc_status aatc_pages_free(const aatc_page_table* table, int32_t* ref,
                                       int64_t n_pages, const int32_t* rows, int64_t n,
                                       void* stream) {
  try {
    aatc_status e = check_table(table);
    if (e == AATC_OK) e = check_counts(ref, n_pages);
    if (e != AATC_OK) return e;
    if (n < 0 || n > kMaxList || !rows || !aligned(rows, 4)) return AATC_E_INVALID;
    if (n == 0) return AATC_OK;
    if (n > kMaxRows) return AATC_E_UNSUPPORTED;
    return launch_pages_free(*table, ref, n_pages, rows, n, stream);
  } catch (...) {
    return AATC_E_INVALID;
  }
}

extern "C" size_t aatc_pages_workspace_bytes(int64_t rows, int64_t n_pages) {
  if (rows < 1 || rows > kMaxPages || n_pages < 1 || n_pages > kMaxPages) return 0;
  return pages_workspace_bytes(rows, n_pages);
}

extern "C" aatc_status aatc_pages_reserve(const aatc_page_table* table, int32_t* ref,
                                          int64_t n_pages, int32_t page_tokens,
                                          const int32_t* held, const int32_t* wanted,
                                          int32_t* pairs, int32_t* lacking, void* workspace,
                                          size_t ws_bytes, void* stream) {
  try {
    aatc_status e = check_table(table);
    if (e == AATC_OK) e = check_counts(ref, n_pages);
    if (e != AATC_OK) return e;
    if (page_tokens < kMinPage || page_tokens > kMaxPage || (page_tokens & (page_tokens - 1)))
      return AATC_E_INVALID;
    if (!held || !wanted || !pairs || !lacking || !workspace || !aligned(held, 4) ||
        !aligned(wanted, 4) || !aligned(pairs, 4) || !aligned(lacking, 4) ||
        !aligned(workspace, 16))
      return AATC_E_INVALID;
    if (ws_bytes < pages_workspace_bytes(table->rows, n_pages)) return AATC_E_WORKSPACE;
    return launch_pages_reserve(*table, ref, n_pages, page_tokens, held, wanted, pairs, lacking,
                                workspace, stream);
  } catch (...) {
    return AATC_E_INVALID;
  }
}

extern "C" aatc_status aatc_pages_compact(const aatc_page_table* table, const int32_t* ref,
                                          int64_t n_pages, const aatc_page_table* table_out,
                                          int32_t* ref_out, int32_t* pairs, int32_t* moves,
                                          void* workspace, size_t ws_bytes, void* stream) {
  try {
    aatc_status e = check_table(table);
    if (e == AATC_OK) e = check_table(table_out);
    if (e == AATC_OK) e = check_counts(ref, n_pages);
    if (e == AATC_OK) e = check_counts(ref_out, n_pages);
    if (e != AATC_OK) return e;
    if (table->rows != table_out->rows || table->max_pages != table_out->max_pages)
      return AATC_E_INVALID;
    if (table->table == table_out->table && table->stride != table_out->stride)
      return AATC_E_INVALID;
    if (!moves || !aligned(moves, 4) || (n_pages > 1 && (!pairs || !aligned(pairs, 4))) ||
        !workspace || !aligned(workspace, 16))
      return AATC_E_INVALID;
    if (ws_bytes < pages_workspace_bytes(table->rows, n_pages)) return AATC_E_WORKSPACE;
    return launch_pages_compact(*table, ref, n_pages, *table_out, ref_out, pairs, moves,
                                workspace, stream);
  } catch (...) {
    return AATC_E_INVALID;
  }
}

extern "C" aatc_status aatc_pages_copy(void* base, int64_t n_pools, int64_t pool_stride,
                                       int64_t n_pages, int64_t page_bytes, const int32_t* pairs,
                                       int64_t n, const int32_t* n_dev, void* stream) {
  try {
    if (!base || !aligned(base, 16) || n_pools < 1 || n_pools > 65535 || n_pages < 1 ||
        n_pages > kMaxPages || page_bytes < 16 || page_bytes % 16 || pool_stride % 16)
      return AATC_E_INVALID;
    if (n_pools > 1 && pool_stride / page_bytes < n_pages) return AATC_E_INVALID;
    if (n < 0 || n > kMaxList || (n > 0 && !pairs) || !aligned(pairs, 4) || !aligned(n_dev, 4))
      return AATC_E_INVALID;
    if (n == 0) return AATC_OK;
    if (page_bytes / 16 > kMaxList || n * n_pools > INT64_MAX / kMaxList) return AATC_E_UNSUPPORTED;
    return launch_pages_copy(base, n_pools, pool_stride, n_pages, page_bytes, pairs, n, n_dev,
                             stream);
  } catch (...) {
    return AATC_E_INVALID;
  }
}
