// C ABI of sparse attention (aatc_sparse.h): argument validation and dispatch to the HIP launchers.
// No exception crosses the boundary.
#include "aatc_sparse.h"
#include "paged_checks.h"
#include "sparse.h"

using namespace aatc;

namespace {

aatc_status check_bounds(const void* codes, const void* scales) {
  return codes && aligned(codes, 16) && scales && aligned(scales, 4) ? AATC_OK : AATC_E_INVALID;
}

}  // namespace

extern "C" aatc_status aatc_page_bounds(const aatc_paged_cache* cache,
                                        const aatc_page_table* table, const int32_t* held,
                                        const int32_t* wanted, int8_t* codes, float* scales,
                                        void* stream) {
  try {
    aatc_status e = check_cache(cache);
    if (e == AATC_OK) e = check_table(table);
    if (e == AATC_OK) e = check_bounds(codes, scales);
    if (e != AATC_OK) return e;
    if (!wanted || !aligned(wanted, 4) || !aligned(held, 4)) return AATC_E_INVALID;
    if (cache->n_kv_heads > kMaxList / ((int64_t)table->rows * table->max_pages))
      return AATC_E_UNSUPPORTED;
    const int size = size_of((aatc_dtype)cache->dtype);
    BoundsArgs a{};
    a.k = static_cast<const char*>(cache->k_pages);
    a.page_stride = cache->page_stride * size;
    a.head_stride = cache->head_stride * size;
    a.tok_stride = cache->tok_stride * size;
    a.table = table->table;
    a.table_stride = table->stride;
    a.held = held;
    a.wanted = wanted;
    a.codes = codes;
    a.scales = scales;
    a.rows = table->rows;
    a.n_kv_heads = cache->n_kv_heads;
    a.n_pages = (int)cache->n_pages;
    a.max_pages = table->max_pages;
    a.page_shift = log2_of(cache->page_tokens);
    a.len_max = (int)row_tokens(*table, cache->page_tokens);
    return launch_bounds(a, (aatc_dtype)cache->dtype, stream);
  } catch (...) {
    return AATC_E_INVALID;
  }
}

extern "C" size_t aatc_paged_sparse_workspace_bytes(int32_t batch, int32_t n_q_heads,
                                                    int32_t n_kv_heads, int64_t max_pages) {
  if (batch < 1 || n_q_heads < 1 || n_kv_heads < 1 || n_q_heads % n_kv_heads || max_pages < 1 ||
      !sparse_fits(batch, n_q_heads, n_kv_heads, max_pages))
    return 0;
  return sparse_workspace_bytes(batch, n_q_heads, n_kv_heads, max_pages);
}

extern "C" aatc_status aatc_paged_sparse_attention(
    const aatc_paged_cache* cache, const aatc_page_table* table, const int32_t* seq_len,
    const int8_t* codes, const float* scales, int32_t batch, int32_t n_q_heads, const void* q,
    aatc_dtype q_dtype, int64_t q_stride, float softmax_scale, int32_t most, int32_t first,
    int32_t last, float softcap, int32_t* picked, float* out, float* lse, void* workspace,
    size_t ws_bytes, void* stream) {
  try {
    aatc_status e = check_cache(cache);
    if (e == AATC_OK) e = check_table(table);
    if (e == AATC_OK) e = check_bounds(codes, scales);
    if (e != AATC_OK) return e;
    if (batch < 1 || batch > table->rows || n_q_heads < 1 || n_q_heads % cache->n_kv_heads)
      return AATC_E_INVALID;
    if (!seq_len || !aligned(seq_len, 4) || !known(q_dtype) ||
        !tokens_ok(q, q_dtype, q_stride, n_q_heads))
      return AATC_E_INVALID;
    if (!std::isfinite(softmax_scale) || !(softcap >= 0.f) || !std::isfinite(softcap) ||
        (softcap > 0.f && !std::isfinite(softmax_scale / softcap)))
      return AATC_E_INVALID;
    if (most < 1 || first < 0 || last < 0 || (int64_t)first + last > most) return AATC_E_INVALID;
    if (!picked || !aligned(picked, 4) || !out || !aligned(out, 16) || !aligned(lse, 4) ||
        !workspace || !aligned(workspace, 256))
      return AATC_E_INVALID;
    if (most > kMaxMost || too_many_tiles(*cache, *table, batch, n_q_heads) ||
        !sparse_fits(batch, n_q_heads, cache->n_kv_heads, table->max_pages))
      return AATC_E_UNSUPPORTED;
    if (ws_bytes < sparse_workspace_bytes(batch, n_q_heads, cache->n_kv_heads, table->max_pages))
      return AATC_E_WORKSPACE;
    SparseArgs a{};
    a.p = paged_args(*cache, *table, seq_len, batch, n_q_heads, q, q_dtype, q_stride, softmax_scale);
    a.p.cap = softcap < kNoCap ? softcap : 0.f;
    a.p.out = out;
    a.p.lse = lse;
    a.codes = codes;
    a.scales = scales;
    a.picked = picked;
    a.most = most;
    a.first = first;
    a.last = last;
    return launch_sparse(a, (aatc_dtype)cache->dtype, workspace, stream);
  } catch (...) {
    return AATC_E_INVALID;
  }
}
