/*
 * qcf_turns.h -- C ABI of libqcf, third part: further turns on the paged caches.
 *
 * Requests whose caches live on in pages (qcf_decode.h) get further questions, are answered several
 * times over, and end.  A pass of a further question is one of qcf_decode.h with a chunk of new rows
 * per request in place of drafted ones:
 *   qcf_page_plan            pages, slots and positions of the new rows
 *   per layer:
 *     qcf_norm_rope_store    norm and rotate the new rows, keys and values into their slots
 *     qcf_chunk_attn         attention of the new rows over the pages
 *   qcf_shape_logits         logits to the probabilities that qcf_verify_drafts takes
 * and between passes
 *   qcf_page_fork, qcf_copy_pages   requests that continue others
 *   qcf_page_release                pages that no request holds any more become free
 *
 * The conventions are those of qcf.h and qcf_decode.h.
 */
#ifndef QCF_TURNS_H_
#define QCF_TURNS_H_

#include "qcf_decode.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * qcf_norm_rope_store -- qcf_rope_store for models that norm the queries and keys of every head before
 * they are rotated.  In that call's formulas turn(x, p) becomes turn(norm(x), p) with
 *     norm(x)[j] = x[j] / sqrt( (sum_i x[i]^2) / head_dim + eps ) * w[j]
 * over each head's head_dim elements, w the head's weight for queries or for keys.  Values are
 * stored as they are.  Everything up to the result's one rounding is float32 (the sum of squares too:
 * a head whose squares pass its range gives zeros, squares below 2^-126 lose bits and count as zeros below
 * 2^-149, so that eps decides), the angles float64.
 *   q_weight, k_weight  one weight [head_dim] for all heads (weight stride 0), or a head's own
 *                 (head h's at h * weight stride, >= head_dim, a multiple of 16 bytes), of type dtype;
 *                 NULL: ones (its stride is 0 then).  16-byte aligned
 *   eps           finite and not negative (0: a head of zeros is NaN, one whose squares all count as zeros
 *                 not finite)
 * All other arguments, and rows without a slot or a source, as for qcf_rope_store; without
 * positions rows are normed and not turned.
 * Errors: as for qcf_rope_store; eps, weights or their strides.
 */
qcf_status qcf_norm_rope_store(void* k_cache, void* v_cache, int64_t n_slots, int64_t cache_row_stride,
                               void* q_out, const void* k_new, const void* v_new,
                               int64_t new_row_stride, const void* q_new, int64_t q_row_stride,
                               int64_t n_src_rows, const int32_t* src_idx, qcf_dtype dtype,
                               int64_t n_rows, const int32_t* slots, const int32_t* positions,
                               const double* freq, int rotary_dim, int interleaved, float magnitude,
                               const void* q_weight, int64_t q_weight_stride, const void* k_weight,
                               int64_t k_weight_stride, float eps, int n_q_heads, int n_kv_heads,
                               int head_dim, hipStream_t stream);

/*
 * qcf_chunk_attn -- grouped-query attention of a chunk of new rows of each request over its paged
 * cache.  Request b's row i (packed row r = cu_q[b] + i), whose token is kv_len[b] + i, sees the tokens
 *     t <= kv_len[b] + i,  and with window > 0 only those with t > kv_len[b] + i - window
 * (the window's tokens, its own among them); keys and values of the new rows are in their slots
 * already.  out and lse are those of qcf_tree_attn, and so are its arguments, rows without tokens,
 * logits that are not finite, missing pages and values that a row does not see.  Only tokens that some
 * row sees are read, so that a prompt costs half its square and a windowed layer rows times window.
 *   page_size  at least 16 (UNSUPPORTED below)
 *   window     >= 0; 0: all tokens
 *   max_q      >= every cu_q[b+1] - cu_q[b] (further rows are left alone), at most 2^20 (UNSUPPORTED)
 *   workspace  >= qcf_chunk_attn_workspace_size(...) bytes, 256-byte aligned, wherever there are rows (max_kv = 0
 *              among them: rows that see no token): partial results
 *              of long tiles that are cut over blocks, merged in order by a second kernel
 *              (deterministic).  It needs no initialisation and keeps nothing; calls that
 *              overlap in time need separate ones.  The size for (batch, max_q, max_kv) covers
 *              every call whose three values do not exceed them (other arguments equal).
 * Sums, maxima and partial results are float32; bf16 calls hand the weights exp(x - max) to the matrix
 * units as one bf16 number, after they entered the sum.  A row's bits do not depend on the other
 * rows' values.
 * Errors: as for qcf_tree_attn (all tiles of a batch, of 128 query vectors each, 32 in float32, of one
 * request and KV head, are fewer than 2^31, batch at most 2^30: UNSUPPORTED).
 */
size_t qcf_chunk_attn_workspace_size(int batch, int max_q, int max_kv, int n_q_heads,
                                     int n_kv_heads, int head_dim, qcf_dtype dtype);
qcf_status qcf_chunk_attn(void* out, float* lse, const void* q, int64_t n_rows,
                          const int32_t* cu_q, const void* k_cache, const void* v_cache,
                          int64_t n_slots, int64_t kv_row_stride, const int32_t* block_table,
                          int64_t table_stride, int max_pages, int page_size,
                          const int32_t* kv_len, int window, qcf_dtype dtype, int batch, int max_q,
                          int max_kv, int n_q_heads, int n_kv_heads, int head_dim,
                          float softmax_scale, void* workspace, size_t workspace_bytes,
                          hipStream_t stream);

/*
 * qcf_shape_logits -- a model's logits with the penalties, biases and masks of an answer, as logits or as
 * the probabilities that qcf_verify_drafts takes.  For packed row r of request b and token t:
 *     z  = logits[r, t]
 *     z  = z > 0 ? z / repetition[b] : z * repetition[b]        if t was said
 *     z  = z - frequency[b] * c - presence[b] * (c > 0)         c times in the answer
 *     z  = z + bias of t
 *     z  = -infinity                                            if t is not allowed
 *     out[r, t] = z                                             (probabilities == 0)
 *     out[r, t] = exp(z / T - m) / sum_t' exp(z' / T - m),      m = max z' / T, T = temperature[b]
 * Said in the answer are tokens prompt_len[b] .. hist_len[b] - 1 of row b of `history` and of
 * the pass's new rows those that row r follows: tokens[cu_rows[b] + j] with bit j of row r's tree mask
 * (qcf_page_plan), itself included, or without a mask with j up to its own index; the
 * request's first tokens 0 .. prompt_len[b] - 1 were said as well, outside the answer.
 * With T = 0 the probability is 1 for the largest z (the lowest such token) and 0 elsewhere; however small T is above 0,
 * largest z that are equal share it.  A row without a z
 * above -infinity gives zeros (qcf_verify_drafts: token -1); a NaN z or one of +infinity makes a
 * row of probabilities NaN (T = 0: a NaN z is passed over).  Everything is float32: the quotient by the repetition is the
 * product with its reciprocal, the exponential of z / T 2 to the power of z log2(e) / T, the quotient rounded once.
 * Probabilities, and exponentials on the way to them, below 2^-126 become zero.
 *   out        [n_rows, vocab], rows out_stride elements apart, of type out_dtype; may be the logits
 *              themselves (same type and stride).  Rows at and behind cu_rows[batch] are left as they are
 *   logits     [n_rows, vocab], rows logits_stride elements apart (any stride >= vocab), of type dtype.
 *              Both need only the alignment of their elements
 *   cu_rows    int32 [batch + 1], ascending from 0
 *   history    int32 [batch, history_stride], columns 0 .. max_history - 1 used, or NULL: nothing was said
 *              before the pass; then prompt_len and hist_len are NULL and max_history 0
 *   prompt_len, hist_len  int32 [batch] (a negative one counts as 0, a prompt_len beyond hist_len as that,
 *              a hist_len beyond max_history as that); prompt_len NULL: 0
 *   tokens     int32 [n_rows] or NULL: the pass's rows count as nothing said; tree_mask uint32 [n_rows,
 *              mask_words] or NULL, given with tokens only.  Tokens outside [0, vocab) are passed over
 *   repetition, presence, frequency  float32 [batch] or NULL (1, 0, 0); repetition above 0.  An infinite
 *              presence or frequency bans the answer's tokens (where c = 0 nothing is taken off)
 *   bias_start int32 [batch + 1] or NULL: entries bias_start[b] .. bias_start[b+1] - 1 of bias_token
 *              (int32 [n_bias]) and bias_value (float32 [n_bias]) are request b's; of several
 *              entries of a token the last counts
 *   allowed    uint32 [n_rows, allowed_words] or NULL: bit t % 32 of word t / 32 allows token t; 32 *
 *              allowed_words >= vocab
 *   temperature  float32 [batch] or NULL (1), not negative; not looked at where probabilities == 0.  z / T may
 *              pass float32's range: it is formed of differences to the row's largest z.  An infinite one makes all
 *              finite z equal
 *   workspace  >= qcf_shape_logits_workspace_size(n_rows, vocab) bytes (may be 0), 256-byte
 *              aligned, no initialisation; calls that overlap in time need separate ones.  A size for
 *              more rows serves fewer.
 * Errors: null pointers, strides, vocab <= 0 or beyond 2^28 (UNSUPPORTED), batch or max_history beyond 2^30
 * (UNSUPPORTED), parts that are not given together, workspace.
 */
size_t qcf_shape_logits_workspace_size(int64_t n_rows, int vocab);
qcf_status qcf_shape_logits(void* out, int64_t out_stride, qcf_dtype out_dtype, const void* logits,
                            int64_t logits_stride, qcf_dtype dtype, int64_t n_rows, int vocab,
                            int batch, const int32_t* cu_rows, const int32_t* history,
                            int64_t history_stride, int max_history, const int32_t* prompt_len,
                            const int32_t* hist_len, const int32_t* tokens,
                            const uint32_t* tree_mask, int mask_words, const float* repetition,
                            const float* presence, const float* frequency,
                            const int32_t* bias_start, const int32_t* bias_token,
                            const float* bias_value, int64_t n_bias, const uint32_t* allowed,
                            int64_t allowed_words, const float* temperature, int probabilities,
                            void* workspace, size_t workspace_bytes, hipStream_t stream);

/*
 * qcf_page_fork -- which request continues which.  Request b of the new tables is request s = source[b] of
 * the old ones, at its first n = keep_len[b] tokens (all of kv_len[s] without keep_len, and never more);
 * a source outside [0, batch) ends it (n = 0).  Requests may continue one another in any order, several
 * the same one.  Pages that n fills are shared, the one it starts has to be b's own:
 *     kv_out[b]     = n
 *     held_out[b]   = ceil(n / page_size)         (at most max_pages)
 *     table_out[b]  = the first held_out[b] pages of s, -1 behind
 * but where n ends inside a page, and that page is not the one that b itself has started already (s = b
 * and n / page_size = kv_len[b] / page_size), b gets a page of the free list in its place,
 *     page = free_pages[free_head + (pages that requests before b get)]
 * and its n % page_size rows have to be copied, by qcf_copy_pages:
 *     copy_src[b], copy_dst[b], copy_rows[b] = the source's page, b's, n % page_size; -1, -1, 0 without a copy
 * So a page that is not full belongs to one request, whoever shared its tokens, and qcf_page_plan's rows
 * may follow.  Pages that a request held beyond its tokens (rejected drafts) are not among the new ones.
 * The pages that nobody holds any more are returned by qcf_page_release.
 *   table_out     int32 [batch, table_out_stride], columns 0 .. max_pages-1 are written
 *   block_table   int32 [batch, table_stride]; kv_len, source int32 [batch] (a negative length counts as 0)
 *   keep_len      int32 [batch] or NULL (a negative one counts as 0)
 *   free_pages    int32 [n_free]; free_head int32 [1] (NULL: 0)
 *   free_head_out int32 [1] free_head + pages taken
 * No output may overlap an input.
 * Where the free list ends (free_head_out > n_free then), or the page that it gives lies outside [0,
 * n_pages), the new entry is -1 and there is no copy.  A source's page outside the pool stays what it is,
 * and nothing is taken or copied for it.
 * Errors: null pointers, page_size not a power of two (UNSUPPORTED), n_pages * page_size beyond int32,
 * batch of 2^22 and more (UNSUPPORTED), outputs that are inputs or one another.
 */
qcf_status qcf_page_fork(int32_t* table_out, int64_t table_out_stride, int32_t* kv_out,
                         int32_t* held_out, const int32_t* block_table, int64_t table_stride,
                         int max_pages, int batch, const int32_t* kv_len, const int32_t* source,
                         const int32_t* keep_len, const int32_t* free_pages, int64_t n_free,
                         const int32_t* free_head, int64_t n_pages, int page_size,
                         int32_t* free_head_out, int32_t* copy_src, int32_t* copy_dst,
                         int32_t* copy_rows, hipStream_t stream);

/*
 * qcf_copy_pages -- the first rows[i] rows (all page_size of them without `rows`; a larger number counts as
 * that) of page src_page[i] to page dst_page[i], in every pool, for i < n_pairs: one launch for the keys
 * and values of all layers.  Pairs with a page outside the pool (qcf_page_fork's -1), or of a page
 * with itself, are skipped.  No page may be the destination of two pairs, or the source of one and
 * the destination of another.
 *   pools       [n_pools] in DEVICE memory: base addresses of pools of n_slots rows, all of this geometry,
 *               each 16-byte aligned
 *   row_bytes   bytes copied per row, a multiple of 16, <= row_stride_bytes (a multiple of 16)
 *   src_page, dst_page  int32 [n_pairs]; rows int32 [n_pairs] or NULL
 * Errors: null pointers, sizes, page_size not a power of two (UNSUPPORTED), more than 2^31 copies of 16 KB
 * (UNSUPPORTED).
 */
qcf_status qcf_copy_pages(void* const* pools, int n_pools, int64_t n_slots, int64_t row_bytes,
                          int64_t row_stride_bytes, int page_size, const int32_t* src_page,
                          const int32_t* dst_page, const int32_t* rows, int64_t n_pairs,
                          hipStream_t stream);

/*
 * qcf_page_release -- pages that some request held and none holds any more go back to the free list.  With
 * the tables before and after a change (qcf_page_fork's; requests that end or are shortened hold fewer
 * entries), the released pages are those among the first held_before[b] entries of table_before's rows that
 * are among the first held_after[b] entries of none of table_after's.  They are put in front of the list's
 * first free entry, h = free_head (n_free where it lies beyond the list), in ascending order:
 *     free_pages[h - n .. h - 1] = the n released pages,  free_head_out = h - n
 * Entries in front of free_head are those that were taken, so there is room for every page that was; pages
 * that would go in front of the list are dropped (free_head_out is 0 then).
 *   table_before, table_after  int32 [batch, their stride], columns 0 .. max_pages-1 used; they may be the
 *                same (lengths alone differ)
 *   held_before, held_after  int32 [batch] (negative ones count as 0, those beyond max_pages as that)
 *   free_pages   int32 [n_free], in and out; free_head, free_head_out int32 [1], different ones
 *   workspace    >= qcf_page_release_workspace_size(...) bytes (may be 0), 256-byte aligned: marks of
 *                pages for large tables.  No initialisation; calls that overlap in time need separate
 *                ones.  The size covers every call whose three values do not exceed those given
 * Entries outside [0, n_pages) are no pages.
 * Errors: null pointers, sizes, n_pages beyond int32, outputs that are inputs or one another, 2^22 pieces of 1024
 * entries and more (UNSUPPORTED), workspace.
 */
size_t qcf_page_release_workspace_size(int batch, int max_pages, int64_t n_pages);
qcf_status qcf_page_release(const int32_t* table_before, int64_t before_stride,
                            const int32_t* held_before, const int32_t* table_after,
                            int64_t after_stride, const int32_t* held_after, int max_pages,
                            int batch, int32_t* free_pages, int64_t n_free,
                            const int32_t* free_head, int32_t* free_head_out, int64_t n_pages,
                            void* workspace, size_t workspace_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* QCF_TURNS_H_ */
