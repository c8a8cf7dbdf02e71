/*
 * aatc_paged.h -- C ABI of the paged cache at input precision: rotary positions, append,
 * attention over pages (alone and together with a compressed cache) and page tables.
 *
 * The conventions of aatc.h hold here too: caller-owned buffers, arguments validated on the host
 * before anything is launched, asynchronous kernels on `stream` (of the current device, where
 * the buffers are), no allocation and no synchronization, no state between calls.
 */
#ifndef AATC_PAGED_H_
#define AATC_PAGED_H_

#include "aatc.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Rotary positions.  Keys are rotated before they are encoded or stored, queries before they
 * are scored.
 *
 * Pair i of a head, i < rot_dim / 2, is channels (i, i + rot_dim / 2) (HALF) or (2 i, 2 i + 1)
 * (INTERLEAVED); at position p it becomes
 *   (a, b) -> factor (a cos t - b sin t, b cos t + a sin t),  t = p freq[i],
 * and channels from rot_dim on stay as they are.  The angle is reduced in 64 bits, sines,
 * products and sums are in 32 bits, rounded once to the output's type.
 */
typedef enum { AATC_ROPE_HALF = 0, AATC_ROPE_INTERLEAVED = 1 } aatc_rope_layout;

typedef struct {
  const double* freq;   /* device [rot_dim / 2], angle per position (8-byte aligned) */
  int32_t rot_dim;      /* rotated channels: even, 2..128 */
  int32_t layout;       /* aatc_rope_layout */
  float factor;         /* of the rotated channels (1 unless a scaling asks for another) */
} aatc_rope_spec;

/*
 * aatc_rope_frequencies -- the angles per position of rot_dim / 2 pairs (host only).
 *
 * PLAIN: f_i = base^(-2 i / rot_dim).  The others stretch them for contexts `scale` (>= 1) times
 * longer than the `trained` positions:
 *   LINEAR  f_i / scale (position interpolation);
 *   NTK     PLAIN with base scale^(rot_dim / (rot_dim - 2)) (rot_dim > 2);
 *   BANDS   by how often a pair turns within the trained positions, u_i = trained f_i / 2 pi:
 *           f_i from `high` turns on, f_i / scale up to `low` turns, and between them a mix whose
 *           share of f_i grows linearly in u_i (0 < low < high);
 *   YARN    the same two ends, but the share of f_i falls linearly in the pair's index, from
 *           floor(x(high)) to ceil(x(low)), x(u) = rot_dim ln(trained / (2 pi u)) / (2 ln base)
 *           (both kept within 0 .. rot_dim - 1, at least 0.001 apart); *factor = 0.1 ln(scale) + 1.
 * freq    host [rot_dim / 2]; the caller copies it to the device.
 * factor  host, NULL allowed: 1 except for YARN.
 * Errors: AATC_E_INVALID (NULL, rot_dim, base <= 1, scale < 1, trained < 1, bands).
 */
typedef enum {
  AATC_ROPE_PLAIN = 0, AATC_ROPE_LINEAR = 1, AATC_ROPE_NTK = 2, AATC_ROPE_BANDS = 3,
  AATC_ROPE_YARN = 4
} aatc_rope_scaling;
aatc_status aatc_rope_frequencies(int32_t rot_dim, double base, aatc_rope_scaling scaling,
                                  double scale, int64_t trained, double low, double high,
                                  double* freq, float* factor);

/*
 * aatc_rope -- rotates n_tok tokens of n_heads heads, or rotates them back.
 *
 * x        device, token t at x + t * x_tok_stride elements, [n_heads][d] contiguous; F32, BF16
 *          or F16.
 * pos      device [n_tok] int32 positions (negative ones turn the other way).
 * spec     host; its freq is a device pointer.
 * inverse  nonzero: the transposed rotation times factor.  With factor 1 it undoes the forward
 *          one (keys moved to other positions); with any it is its gradient.
 * out      device, like x with out_tok_stride; may be x itself with the same stride (no other
 *          overlap).
 * n_tok == 0 is a no-op.  Errors: AATC_E_INVALID, AATC_E_UNSUPPORTED (d != 128).
 * Speed: 16-byte aligned rows are moved in 16-byte pieces (fastest for INTERLEAVED, and for HALF
 * with a rot_dim / 2 that fills such pieces); others channel by channel, with the same results.
 */
aatc_status aatc_rope(const void* x, aatc_dtype dtype, int64_t n_tok, int32_t n_heads, int32_t d,
                      int64_t x_tok_stride, const int32_t* pos, const aatc_rope_spec* spec,
                      int32_t inverse, void* out, int64_t out_tok_stride, void* stream);

/*
 * The paged cache: tokens at input precision (sequences too short to compress, the recent
 * window, layers left as they are).  A page holds page_tokens consecutive tokens of one sequence,
 * keys in one pool and values in another of the same layout: element c of token slot s of KV
 * head h of page i is at i * page_stride + h * head_stride + s * tok_stride + c.  With
 * token-major pages (tok_stride = n_kv_heads * d) a page is an input of aatc_encode as it is.
 */
typedef struct {
  void* k_pages;        /* device, 16-byte aligned */
  void* v_pages;
  int32_t dtype;        /* aatc_dtype of both pools: F32, BF16 or F16 */
  int32_t n_kv_heads;
  int32_t d;            /* 128 */
  int32_t page_tokens;  /* a power of two, 8..4096 */
  int64_t n_pages;      /* of each pool, 1 .. 2^31 - 1 */
  int64_t page_stride;  /* elements, multiples of 16 bytes, at least d */
  int64_t head_stride;
  int64_t tok_stride;
} aatc_paged_cache;

/*
 * Which pages a sequence has: entry [b][i] is the page of tokens i * page_tokens .. of sequence
 * b, row b at table + b * stride.  Entries outside [0, n_pages) name no page: nothing is stored
 * there and their tokens are not attended.
 */
typedef struct {
  int32_t* table;       /* device */
  int64_t stride;       /* entries from row to row, at least max_pages */
  int32_t rows;
  int32_t max_pages;    /* entries of a row; rows * max_pages at most 2^30 (else
                           AATC_E_UNSUPPORTED) */
} aatc_page_table;

/*
 * aatc_paged_append -- stores new tokens in the pages, rotated on the way.
 *
 * For token t of sequence b = seq[t] at position p = pos[t]: key and value go to slot p %
 * page_tokens of page table[b][p / page_tokens], rounded to the cache's type, the key rotated by
 * `rope`; the token's queries, if given, are rotated into q_out.  Tokens with a negative position
 * are left out altogether (padding); those whose sequence or page does not exist store no key and
 * value.  The (sequence, position) pairs of one call must differ.  A page that several sequences
 * share is written for all of them (aatc_pages_reserve gives the writer a page of its own).
 *
 * k, v     device, token t at k + t * k_tok_stride (v_tok_stride) elements, [n_kv_heads][d]
 *          contiguous, x_dtype F32, BF16 or F16 (as q and q_out).
 * seq      device [n_tok] int32, or NULL: token t belongs to sequence t.
 * pos      device [n_tok] int32.
 * rope     host, or NULL: nothing is rotated.
 * q        device [n_tok] tokens of [n_q_heads][d] at q_tok_stride, or NULL with n_q_heads 0.
 * q_out    device, like q; may be q itself with the same stride.
 * n_tok == 0 is a no-op.  Errors: AATC_E_INVALID, AATC_E_UNSUPPORTED (d != 128).
 */
aatc_status aatc_paged_append(const aatc_paged_cache* cache, const aatc_page_table* table,
                              int64_t n_tok, aatc_dtype x_dtype, const void* k,
                              int64_t k_tok_stride, const void* v, int64_t v_tok_stride,
                              const int32_t* seq, const int32_t* pos, const aatc_rope_spec* rope,
                              int32_t n_q_heads, const void* q, int64_t q_tok_stride, void* q_out,
                              int64_t q_out_tok_stride, void* stream);

/*
 * aatc_paged_decode_attention -- attention of one new token per sequence over its pages.
 *
 * Query head j of sequence b reads KV head j / (n_q_heads / n_kv_heads):
 *   z_t = softcap tanh(softmax_scale q . k_t / softcap) - slopes[j] (seq_len[b] - 1 - t),
 *   out = sum_t softmax(z)_t v_t,   lse = ln sum_t exp(z_t),
 * over tokens t < seq_len[b] whose page exists and, with a window, t >= seq_len[b] - window or
 * t < sink.  A head without any such token gets zeros and lse -infinity.  What the pages hold
 * elsewhere (infinities and NaN among it) does not matter.  NaN in an attended key or in a query
 * gives NaN, an infinity or NaN in an attended value infinities or NaN in its channel.  Infinite
 * scores follow the formula: +infinity gives NaN, -infinity has no weight, with a cap they are
 * +-softcap; a head all of whose attended scores are -infinity gets NaN and lse -infinity.  (Where
 * 16-bit pages meet queries of another type, infinite keys and queries may give NaN instead.)
 * Products are of the stored values, with sums and softmax in 32 bits.  The result does not
 * depend on timing, but in its last bits on how a batch's tokens are split.
 *
 * table     one row per sequence (rows >= batch).
 * seq_len   device [batch] int32, clamped to [0, max_pages * page_tokens].
 * q         device, sequence b at q + b * q_stride elements, [n_q_heads][d] contiguous; F32,
 *           BF16 or F16.
 * window    0: none.  sink: tokens at the start that stay attended with a window, >= 0.
 * softcap   0: none, else > 0 (and softmax_scale / softcap finite); from 1e30 on none either.
 * slopes    device [n_q_heads] fp32 (a bias that falls with distance) or NULL.
 * out       device [batch][n_q_heads][d] fp32, 16-byte aligned.
 * lse       device [batch][n_q_heads] fp32 or NULL.
 * workspace device scratch of aatc_paged_decode_workspace_bytes bytes, 256-byte aligned,
 *           zero-filled once after allocation; every call leaves it reusable, for calls of other
 *           shapes that it is large enough for too.  Calls that may overlap need one each.
 * Errors: AATC_E_INVALID, AATC_E_UNSUPPORTED (d != 128; more than 2^30 tiles of 16 tokens),
 * AATC_E_WORKSPACE, AATC_E_DEVICE.
 */
size_t aatc_paged_decode_workspace_bytes(int32_t batch, int32_t n_q_heads, int32_t n_kv_heads);
aatc_status aatc_paged_decode_attention(const aatc_paged_cache* cache,
                                        const aatc_page_table* table, const int32_t* seq_len,
                                        int32_t batch, int32_t n_q_heads, const void* q,
                                        aatc_dtype q_dtype, int64_t q_stride, float softmax_scale,
                                        int32_t window, int32_t sink, float softcap,
                                        const float* slopes, float* out, float* lse,
                                        void* workspace, size_t ws_bytes, void* stream);

/*
 * aatc_decode_attention_paged -- decode attention over a compressed cache plus pages.
 *
 * aatc_decode_attention_segmented with the tokens at input precision in pages, without its limit
 * of 256: exact softmax attention of each query head over the union of the seq_len[b] compressed
 * tokens and the page_len[b] tokens of the pages (no window, cap or bias; either may be empty).
 * The pages' attention becomes one more partial of the decode launch.
 *
 * q             device [batch][n_q_heads][d] contiguous, F32 or BF16, as aatc_decode_attention.
 * cache         n_kv_heads as the compressed cache's.
 * page_len      device [batch] int32, clamped to [0, max_pages * page_tokens].
 * workspace     of aatc_decode_paged_workspace_bytes bytes, 256-byte aligned, zero-filled once, and
 *               again before calls of another batch, other head counts or another cap.
 * Other arguments and errors as in aatc_decode_attention.
 */
size_t aatc_decode_paged_workspace_bytes(int32_t batch, int32_t n_q_heads, int32_t n_kv_heads,
                                         int64_t cap);
aatc_status aatc_decode_attention_paged(
    const void* dev_params_k, const void* dev_params_v, int32_t batch, int32_t n_q_heads,
    int32_t n_kv_heads, int32_t d, const void* q, aatc_dtype q_dtype, const void* k_codes,
    const uint16_t* k_alpha, const void* v_codes, const uint16_t* v_alpha,
    const int32_t* seq_len, int64_t cap, int32_t k_record_bytes, int32_t v_record_bytes,
    float softmax_scale, const aatc_paged_cache* cache, const aatc_page_table* table,
    const int32_t* page_len, float* out, void* workspace, size_t ws_bytes, void* stream);

/*
 * Page tables on the device.  ref[i] counts the table entries that name page i; pages of count 0
 * are free.  Whole numbers only, and always the same result: nothing depends on timing.  Table
 * entries outside [0, n_pages) are skipped; a new table is filled with -1.
 *
 * aatc_pages_fork -- the rows pairs[i][1] of dst become copies of the rows pairs[i][0] of src
 * (the same or another table, of as many entries per row), and their pages' counts go up: beams
 * and samples share what they have in common.  What the dst rows held is forgotten (not freed).
 * A dst row listed twice takes the last of its sources; rows outside the tables are skipped; no
 * row may be a source and a destination of one call.  n at most 2^18 (more: AATC_E_UNSUPPORTED):
 * every pair is compared with all later ones (32768 pairs 1.5 ms).
 */
aatc_status aatc_pages_fork(const aatc_page_table* src, const aatc_page_table* dst, int32_t* ref,
                            int64_t n_pages, const int32_t* pairs, int64_t n, void* stream);

/* aatc_pages_free -- empties the rows listed (device [n] int32; twice does no harm): the counts
 * of their pages go down and the entries become -1.  n < 2^24 (more: AATC_E_UNSUPPORTED). */
aatc_status aatc_pages_free(const aatc_page_table* table, int32_t* ref, int64_t n_pages,
                            const int32_t* rows, int64_t n, void* stream);

/*
 * aatc_pages_reserve -- makes room for the tokens held[b] .. wanted[b] - 1 of every row b.
 *
 * Entries of the pages that these tokens fall into that name no page (or a free one) take free
 * ones, the lowest first, row after row; a begun page that is not there gets none.  Entries that name a page already
 * (reserved ahead, left by a rollback) keep it where no other entry names it.  Where others do, the
 * row gets a free page of its own and the old one's count goes down (of claims of one call on one
 * page that nobody else holds, the last in the order of rows and entries keeps it).  For the begun
 * page that the first of the tokens falls into, pairs[b] = (old, new) then, for aatc_pages_copy;
 * elsewhere pairs[b] = (-1, -1).  Lengths are clamped to [0, max_pages * page_tokens];
 * wanted[b] <= held[b] asks for nothing.
 * lacking  device [1] int32: 0, or how many free pages there were too few: then nothing but
 *          lacking and pairs (all -1) has been written.
 * held, wanted  device [rows] int32.  pairs  device [rows][2] int32.
 * workspace  of aatc_pages_workspace_bytes bytes, 16-byte aligned, of any content.
 */
size_t aatc_pages_workspace_bytes(int64_t rows, int64_t n_pages);
aatc_status aatc_pages_reserve(const aatc_page_table* table, int32_t* ref, int64_t n_pages,
                               int32_t page_tokens, const int32_t* held, const int32_t* wanted,
                               int32_t* pairs, int32_t* lacking, void* workspace, size_t ws_bytes,
                               void* stream);

/*
 * aatc_pages_compact -- a plan that moves the pages in use to the front of the pool: with L of
 * them, the pages from L on, in order, go to the free ones below L, in order.  The table and the
 * counts as they are after the moves are written to table_out (as many rows and entries) and
 * ref_out, which may be table and ref themselves.  pairs (device [n_pages / 2][2] int32): the
 * moves (from, to), -1 behind the last; moves (device [1] int32): how many.  aatc_pages_copy then
 * moves the contents.  A page that ref counts but no row of this table names is moved too: every
 * table of the pool needs the same call with the counts as they were before.
 */
aatc_status aatc_pages_compact(const aatc_page_table* table, const int32_t* ref, int64_t n_pages,
                               const aatc_page_table* table_out, int32_t* ref_out, int32_t* pairs,
                               int32_t* moves, void* workspace, size_t ws_bytes, void* stream);

/*
 * aatc_pages_copy -- copies page pairs[i][0] to page pairs[i][1] in each of n_pools pools.
 *
 * base         device, 16-byte aligned; page i of pool p at base + p * pool_stride + i *
 *              page_bytes (bytes, multiples of 16; pool_stride >= n_pages * page_bytes).
 * pairs        device [n][2] int32; pairs with a page outside [0, n_pages) are skipped.  The
 *              destinations differ, and none of them is the source of another pair.
 * n_dev        device [1] int32, or NULL: copy no more than that many of the n pairs.
 */
aatc_status aatc_pages_copy(void* base, int64_t n_pools, int64_t pool_stride, int64_t n_pages,
                            int64_t page_bytes, const int32_t* pairs, int64_t n,
                            const int32_t* n_dev, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* AATC_PAGED_H_ */
