/*
 * aatc_sparse.h -- C ABI of sparse attention over the paged cache: what the keys of each page can
 * score at most, in 8 bits, and attention over the pages that can score most.
 *
 * The conventions of aatc.h and aatc_paged.h hold here too.
 *
 * Bounds.  For page i and KV head h: codes[i][h][0][c] and codes[i][h][1][c] times scales[i][h] are
 * no less than the largest and no more than the smallest value of key channel c in that page.  The
 * scale is a power of two, the smallest (from 2^-50 on) of which 127 reach the page's largest
 * magnitude; the codes are rounded upwards and downwards.  A page with a key that is not finite (or
 * beyond 127 2^100) has the scale +infinity and codes of 0.
 */
#ifndef AATC_SPARSE_H_
#define AATC_SPARSE_H_

#include "aatc_paged.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * aatc_page_bounds -- the bounds of the pages that the tokens held[b] .. wanted[b] - 1 of every row b
 * of the table fall into, each from all of its tokens below wanted[b].
 *
 * Call it for the tokens that an append stored, or for all (held NULL: from 0 on), or after a rollback
 * for those of the last page that stay.  Lengths are clamped to [0, max_pages * page_tokens].  Pages
 * that are not there are skipped, all other pages' bounds left as they were.  Rows that share a page
 * must agree on how many of its tokens they hold.
 *
 * held, wanted  device [rows] int32 (held NULL allowed).
 * codes         device [n_pages][n_kv_heads][2][d] int8, 16-byte aligned.
 * scales        device [n_pages][n_kv_heads] fp32.
 * Errors: AATC_E_INVALID, AATC_E_UNSUPPORTED (d != 128; rows * max_pages * n_kv_heads over 2^30),
 * AATC_E_DEVICE.
 */
aatc_status aatc_page_bounds(const aatc_paged_cache* cache, const aatc_page_table* table,
                             const int32_t* held, const int32_t* wanted, int8_t* codes,
                             float* scales, void* stream);

/*
 * aatc_paged_sparse_attention -- attention of one new token per sequence over the pages that it
 * picks, for every KV head its own.
 *
 * A sequence of n = seq_len[b] tokens has the pages i < ceil(n / page_tokens) that exist.  The first
 * `first` and the last `last` of these indexes are picked always; then the pages with the highest
 * scores, up to `most` in all, the lowest index of equal ones.  With a query head's channels rounded
 * to 8 bits, u_c = q_c / s to the nearest (ties to even; s the power of two that the bounds' rule
 * gives for its largest magnitude; of -q for a negative softmax_scale), a page's score is
 *   max over the KV head's query heads of  (s / s_max) scale sum_c max(u_c hi_c, u_c lo_c),
 * s_max the largest s of them (ratios below 2^-60 count as 2^-60): nearly the most that a key of the
 * page can score, computed without rounding.  Query heads that are not finite have no say; pages
 * whose scale is +infinity score higher than all others.
 *
 * Out and lse are as in aatc_paged_decode_attention over the tokens of the picked pages alone
 * (softcap included; no window, no bias).
 *
 * codes, scales  bounds of the pages, up to date for every page that a sequence has.
 * most       1 or more; first, last >= 0, first + last <= most.
 * picked     device [batch][n_kv_heads][most] int32: table indexes of the picked pages, ascending, -1
 *            behind them.
 * workspace  device scratch of aatc_paged_sparse_workspace_bytes(batch, n_q_heads, n_kv_heads,
 *            max_pages) bytes, 256-byte aligned, zero-filled once after allocation; every call leaves
 *            it reusable, for calls of other shapes that it is large enough for too.  Calls that may
 *            overlap need one each.
 * Other arguments and errors as in aatc_paged_decode_attention; AATC_E_UNSUPPORTED also for
 * batch * n_kv_heads * max_pages over 2^30, batch * n_kv_heads times ceil(max_pages / 64) or times
 * ceil(n_q_heads / n_kv_heads / 16) over 2^22, most over 2^20, and over 256 query heads a KV head.
 */
size_t aatc_paged_sparse_workspace_bytes(int32_t batch, int32_t n_q_heads, int32_t n_kv_heads,
                                         int64_t max_pages);
aatc_status aatc_paged_sparse_attention(const aatc_paged_cache* cache, const aatc_page_table* table,
                                        const int32_t* seq_len, const int8_t* codes,
                                        const float* scales, int32_t batch, int32_t n_q_heads,
                                        const void* q, aatc_dtype q_dtype, int64_t q_stride,
                                        float softmax_scale, int32_t most, int32_t first,
                                        int32_t last, float softcap, int32_t* picked, float* out,
                                        float* lse, void* workspace, size_t ws_bytes,
                                        void* stream);

#ifdef __cplusplus
}
#endif

#endif /* AATC_SPARSE_H_ */
