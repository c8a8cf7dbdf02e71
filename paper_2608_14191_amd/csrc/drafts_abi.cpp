// C ABI of drafted tokens (aatc_drafts.h): argument validation and dispatch to the HIP launchers.
// No exception crosses the boundary.
#include "aatc_drafts.h"
#include "drafts.h"
#include "paged_checks.h"

using namespace aatc;

namespace {

aatc_status check_trees(const int32_t* seq_len, const int32_t* n_draft, const int32_t* parent,
                        int32_t batch, int32_t max_draft, const aatc_page_table& table) {
  if (batch < 1 || batch > table.rows || max_draft < 1) return AATC_E_INVALID;
  if (!seq_len || !aligned(seq_len, 4) || !aligned(n_draft, 4) || !aligned(parent, 4))
    return AATC_E_INVALID;
  return max_draft <= kMaxDrafts ? AATC_OK : AATC_E_UNSUPPORTED;
}

struct List {
  const int32_t* at;
  int64_t n;
};
bool overlap(const List& x, const List& y) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(x.at), b = reinterpret_cast<uintptr_t>(y.at);
  return a && b && a < b + (uintptr_t)y.n * 4 && b < a + (uintptr_t)x.n * 4;
}

}  // namespace

extern "C" size_t aatc_paged_tree_workspace_bytes(int32_t batch, int32_t max_draft,
                                                  int32_t n_q_heads, int32_t n_kv_heads) {
  if (batch < 1 || max_draft < 1 || max_draft > kMaxDrafts || n_q_heads < 1 || n_kv_heads < 1 ||
      n_q_heads % n_kv_heads || !tree_fits(batch, max_draft, n_q_heads, n_kv_heads))
    return 0;
  return tree_workspace_bytes(batch, max_draft, n_q_heads, n_kv_heads);
}

extern "C" aatc_status aatc_paged_tree_attention(
    const aatc_paged_cache* cache, const aatc_page_table* table, const int32_t* seq_len,
    const int32_t* n_draft, const int32_t* parent, int32_t batch, int32_t max_draft,
    int32_t n_q_heads, const void* q, aatc_dtype q_dtype, int64_t q_tok_stride,
    float softmax_scale, int32_t window, int32_t sink, float softcap, const float* slopes,
    float* out, float* lse, void* workspace, size_t ws_bytes, void* stream) {
  try {
    aatc_status e = check_cache(cache);
    if (e == AATC_OK) e = check_table(table);
    if (e == AATC_OK) e = check_trees(seq_len, n_draft, parent, batch, max_draft, *table);
    if (e != AATC_OK) return e;
    if (n_q_heads < 1 || n_q_heads % cache->n_kv_heads) return AATC_E_INVALID;
    if (!known(q_dtype) || !tokens_ok(q, q_dtype, q_tok_stride, n_q_heads)) return AATC_E_INVALID;
    if (!std::isfinite(softmax_scale) || window < 0 || sink < 0 || !(softcap >= 0.f) ||
        !std::isfinite(softcap) || (softcap > 0.f && !std::isfinite(softmax_scale / softcap)))
      return AATC_E_INVALID;
    if (!out || !aligned(out, 16) || !aligned(lse, 4) || !aligned(slopes, 4) || !workspace ||
        !aligned(workspace, 256))
      return AATC_E_INVALID;
    if (too_many_tiles(*cache, *table, batch, n_q_heads) ||
        !tree_fits(batch, max_draft, n_q_heads, cache->n_kv_heads))
      return AATC_E_UNSUPPORTED;
    if (ws_bytes < tree_workspace_bytes(batch, max_draft, n_q_heads, cache->n_kv_heads))
      return AATC_E_WORKSPACE;
    TreeArgs a{};
    a.p = paged_args(*cache, *table, seq_len, batch, n_q_heads, q, q_dtype, q_tok_stride,
                     softmax_scale);
    a.p.window = window;
    a.p.sink = sink;
    a.p.cap = softcap < kNoCap ? softcap : 0.f;
    a.p.slopes = slopes;
    a.p.out = out;
    a.p.lse = lse;
    a.n_draft = n_draft;
    a.parent = parent;
    a.drafts = max_draft;
    return launch_tree(a, (aatc_dtype)cache->dtype, workspace, stream);
  } catch (...) {
    return AATC_E_INVALID;
  }
}

extern "C" aatc_status aatc_paged_tree_accept(
    const aatc_paged_cache* cache, int32_t n_layers, int64_t layer_stride,
    const aatc_page_table* table, const int32_t* seq_len, const int32_t* n_draft,
    const int32_t* parent, int32_t batch, int32_t max_draft, const int32_t* drafted,
    const int32_t* chosen, int32_t* path, int32_t* accepted, int32_t* next, int32_t* len_out,
    void* stream) {
  try {
    aatc_status e = check_cache(cache);
    if (e == AATC_OK) e = check_table(table);
    if (e == AATC_OK) e = check_trees(seq_len, n_draft, parent, batch, max_draft, *table);
    if (e != AATC_OK) return e;
    const int size = size_of((aatc_dtype)cache->dtype);
    if (n_layers < 1 || n_layers > 65535 || cache->n_kv_heads > 65535) return AATC_E_INVALID;
    if (n_layers > 1 && (layer_stride < kD || layer_stride % (16 / size) ||
                         layer_stride >= ((int64_t)1 << 40)))
      return AATC_E_INVALID;
    const int pieces = kD * size / 16;
    if ((int64_t)n_layers * 2 * cache->n_kv_heads * pieces > kMaxMoved) return AATC_E_UNSUPPORTED;
    // (every workgroup of a sequence reads the inputs: no output overlaps one, or another)
    const int64_t each = (int64_t)batch * max_draft;
    const List in[] = {{drafted, each}, {chosen, each}, {seq_len, batch}, {n_draft, batch},
                       {parent, each}, {table->table, (batch - 1) * table->stride + table->max_pages}};
    const List res[] = {{path, each}, {accepted, batch}, {next, batch}, {len_out, batch}};
    for (const List& x : {in[0], in[1], res[0], res[1], res[2], res[3]})
      if (!x.at || !aligned(x.at, 4)) return AATC_E_INVALID;
    for (int i = 0; i < 4; ++i) {
      for (const List& x : in)
        if (overlap(res[i], x)) return AATC_E_INVALID;
      for (int j = 0; j < i; ++j)
        if (overlap(res[i], res[j])) return AATC_E_INVALID;
    }
    AcceptArgs a{};
    a.k = static_cast<char*>(cache->k_pages);
    a.v = static_cast<char*>(cache->v_pages);
    a.page_stride = cache->page_stride * size;
    a.head_stride = cache->head_stride * size;
    a.tok_stride = cache->tok_stride * size;
    a.layer_stride = n_layers > 1 ? layer_stride * size : 0;
    a.table = table->table;
    a.table_stride = table->stride;
    a.seq_len = seq_len;
    a.n_draft = n_draft;
    a.parent = parent;
    a.drafted = drafted;
    a.chosen = chosen;
    a.path = path;
    a.accepted = accepted;
    a.next = next;
    a.len_out = len_out;
    a.batch = batch;
    a.drafts = max_draft;
    a.layers = n_layers;
    a.n_kv_heads = cache->n_kv_heads;
    a.n_pages = (int)cache->n_pages;
    a.max_pages = table->max_pages;
    a.page_shift = log2_of(cache->page_tokens);
    a.len_max = (int)row_tokens(*table, cache->page_tokens);
    a.pieces = pieces;
    return launch_tree_accept(a, stream);
  } catch (...) {
    return AATC_E_INVALID;
  }
}
