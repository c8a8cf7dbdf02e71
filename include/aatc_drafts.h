/*
 * aatc_drafts.h -- C ABI of speculative decoding over the paged cache: attention of a tree of
 * drafted tokens per sequence, and the acceptance of one of its paths.
 *
 * The conventions of aatc.h and aatc_paged.h hold here too.
 *
 * Sequence b has n = seq_len[b] tokens in its pages and m drafted ones behind them: draft i is in
 * the slot of token n + i.  parent[b][i] is the draft that it follows, an earlier one; any other
 * number (-1) makes it follow the sequence itself.  The drafts thus form trees, of depth d(i): 0 for
 * a draft that follows the sequence, else one more than its parent's.  Draft i stands at position
 * n + d(i): that is what its query and key are rotated by (aatc_rope) before aatc_paged_append, given
 * no rotation, stores key and value at n + i.
 */
#ifndef AATC_DRAFTS_H_
#define AATC_DRAFTS_H_

#include "aatc_paged.h"

#ifdef __cplusplus
extern "C" {
#endif

#define AATC_MAX_DRAFTS 64

/*
 * aatc_paged_tree_attention -- attention of the drafts over their sequences' pages.
 *
 * Draft i attends the sequence's tokens, its ancestors and itself.  With pos(t) the position of the
 * token in slot t (t below n, n + d(t - n) from there on), query head j reads KV head
 * j / (n_q_heads / n_kv_heads):
 *   z_t = softcap tanh(softmax_scale q . k_t / softcap) - slopes[j] (pos(n + i) - pos(t)),
 *   out = sum_t softmax(z)_t v_t,   lse = ln sum_t exp(z_t),
 * over those of these tokens whose page exists and, with a window, pos(t) > pos(n + i) - window or
 * t < sink.  For a chain (parent NULL) draft i gets what aatc_paged_decode_attention gives for a
 * sequence of n + i + 1 tokens.  Tokens without weight, infinities and NaN, rounding: as there (an
 * infinity or NaN in a value reaches the drafts that attend it and no others).
 *
 * table     one row per sequence (rows >= batch).
 * seq_len   device [batch] int32, clamped to [0, max_pages * page_tokens].
 * n_draft   device [batch] int32, clamped to [0, max_draft], or NULL: max_draft each.
 * parent    device [batch][max_draft] int32, or NULL: draft i - 1 (a chain).
 * max_draft 1 .. AATC_MAX_DRAFTS (more: AATC_E_UNSUPPORTED).
 * q         device, draft i of sequence b at q + (b * max_draft + i) * q_tok_stride elements,
 *           [n_q_heads][d] contiguous; F32, BF16 or F16.
 * out       device [batch][max_draft][n_q_heads][d] fp32, 16-byte aligned; drafts from n_draft[b] on
 *           are left as they were (here and in lse).
 * lse       device [batch][max_draft][n_q_heads] fp32 or NULL.
 * workspace device scratch of aatc_paged_tree_workspace_bytes bytes, 256-byte aligned, of any content.
 *           Calls that may overlap need one each.
 * Other arguments as in aatc_paged_decode_attention.
 * Errors: AATC_E_INVALID, AATC_E_UNSUPPORTED (d != 128; max_draft; more than 2^30 tiles of 16 tokens;
 * c = max_draft * n_q_heads / n_kv_heads over 16384; (batch * n_kv_heads + 1032) ceil(c / 128) over
 * 2^22), AATC_E_WORKSPACE, AATC_E_DEVICE.
 */
size_t aatc_paged_tree_workspace_bytes(int32_t batch, int32_t max_draft, int32_t n_q_heads,
                                       int32_t n_kv_heads);
aatc_status aatc_paged_tree_attention(const aatc_paged_cache* cache, const aatc_page_table* table,
                                      const int32_t* seq_len, const int32_t* n_draft,
                                      const int32_t* parent, int32_t batch, int32_t max_draft,
                                      int32_t n_q_heads, const void* q, aatc_dtype q_dtype,
                                      int64_t q_tok_stride, float softmax_scale, int32_t window,
                                      int32_t sink, float softcap, const float* slopes, float* out,
                                      float* lse, void* workspace, size_t ws_bytes, void* stream);

/*
 * aatc_paged_tree_accept -- the path of drafts that the model agrees with, and its tokens moved up.
 *
 * Draft 0 is the step's own token, accepted always.  After an accepted draft i follows its child whose
 * token is chosen[b][i], what the model chose there (the earliest of several); where there is none the
 * path ends, and that choice is the next step's token.  The path's keys and values move from the slots
 * n + path[i] to n + i, in every layer; the other slots from n + accepted on are left as they were.
 * A page that is not there is neither read nor written.  Pages written must not be shared with other
 * sequences (aatc_pages_reserve sees to that).
 *
 * cache        of the first layer; layer l's pools are l * layer_stride elements behind its, in both.
 * n_layers     1 .. 65535, for up to 65535 KV heads.
 * layer_stride elements, a multiple of 16 bytes (not read for one layer).
 * drafted      device [batch][max_draft] int32, the drafts' tokens.
 * chosen       device [batch][max_draft] int32.
 * path         device [batch][max_draft] int32: the accepted drafts, ascending, -1 behind them.
 * accepted     device [batch] int32: how many (0 without drafts).
 * next         device [batch] int32: chosen after the last of them (-1 without drafts).
 * len_out      device [batch] int32: seq_len, clamped as below, + accepted.
 * No output overlaps an input or another output: AATC_E_INVALID.
 * seq_len, n_draft, parent, max_draft: as in aatc_paged_tree_attention (seq_len clamped likewise).
 * Errors: AATC_E_INVALID, AATC_E_UNSUPPORTED (d != 128; max_draft; n_layers * n_kv_heads over 2^34 bytes
 * of d elements: 2^26, or 2^25 in float32), AATC_E_DEVICE.
 */
aatc_status aatc_paged_tree_accept(const aatc_paged_cache* cache, int32_t n_layers,
                                   int64_t layer_stride, const aatc_page_table* table,
                                   const int32_t* seq_len, const int32_t* n_draft,
                                   const int32_t* parent, int32_t batch, int32_t max_draft,
                                   const int32_t* drafted, const int32_t* chosen, int32_t* path,
                                   int32_t* accepted, int32_t* next, int32_t* len_out,
                                   void* stream);

#ifdef __cplusplus
}
#endif

#endif /* AATC_DRAFTS_H_ */
