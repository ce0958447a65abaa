/*
 * qcf_decode.h -- C ABI of libqcf, second part: answering from the fused cache.
 *
 * The fusion step (qcf.h) ends with a request's fused cache.  Its answer is
 * decoded from it: the cache lives on in pages of a pool, every pass of the
 * model brings a few new rows per request (the last token, or that token and a
 * tree of drafted ones after it), and the drafted tokens are checked against
 * the model's probabilities.  One pass is
 *   qcf_page_plan      pages, slots, positions and tree masks of the new rows
 *   per layer:
 *     qcf_rope_store   rotate the new rows, keys and values into their slots
 *     qcf_tree_attn    attention of the new rows over the pages
 *   qcf_verify_drafts  which drafted tokens stay, and the next token
 *
 * The conventions are those of qcf.h: device pointers owned by the caller,
 * 16-byte aligned; nothing allocated, kept or synchronised; everything on the
 * caller's stream, so that a pass can be captured into a graph; host-visible
 * arguments checked before anything is launched; the contents of device arrays
 * are preconditions, and indices outside the bounds given in the call are
 * skipped, never followed.
 *
 * The new rows of a batch are packed: request b holds rows cu[b] .. cu[b+1]-1.
 * Packed arrays may be longer than cu[batch] (a replayed step of fixed size);
 * what happens to the rows behind it is said at each call.
 *
 * Pages.  A pool of n_slots rows is cut into pages of page_size rows (a power
 * of two); slot p * page_size + i is row i of page p.  block_table [batch,
 * table_stride] holds in row b the pages of request b in the order of its
 * tokens, so token t sits in slot
 *     block_table[b][t / page_size] * page_size + t % page_size.
 */
#ifndef QCF_DECODE_H_
#define QCF_DECODE_H_

#include "qcf.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * qcf_page_plan -- block tables and slot maps from request lengths, on the
 * GPU.  Request b holds kv_len[b] tokens and gets new_len[b] more (a negative
 * length counts as 0).  Its pages are extended to ceil((kv_len + new_len) /
 * page_size), the missing ones taken from the free list in request order:
 *     block_table[b][held + i] = free_pages[free_head + (pages taken by
 *                                requests before b) + i]
 * and for its i-th new row, r = cu_new[b] + i:
 *     slots[r]     = the slot of token kv_len[b] + i
 *     positions[r] = kv_len[b] + i                    without parents
 *                  = kv_len[b] + depth of the row     with parents
 *     tree_mask[r] bit j of word j / 32: row j of the request is row i itself or
 *                  one of its ancestors               with parents
 *   block_table   int32 [batch, table_stride], in and out; columns 0 ..
 *                 max_pages-1 are used.  Only the entries of new pages are written.
 *   kv_len, new_len  int32 [batch]
 *   pages_held    int32 [batch] pages each request has, or NULL: ceil(kv_len /
 *                 page_size).  (After rejected drafts a request holds more
 *                 pages than its tokens fill.)  A smaller number counts as that.
 *   free_pages    int32 [n_free]; free_head int32 [1] (NULL: 0) is the first
 *                 entry that is still free.
 *   parents       int32 [n_rows] or NULL: row parents[r] of the same request is
 *                 the parent of row r; it must be smaller than r's own index.
 *                 Anything else (-1) makes the row a root, of depth 0.
 *   tree_mask     uint32 [n_rows, mask_words], given with parents and only then;
 *                 32 * mask_words >= max_new
 *   max_new       >= every new_len; with parents at most QCF_MAX_TREE.
 *   slots, positions  int32 [n_rows]
 *   cu_new        int32 [batch + 1]
 *   kv_end        int32 [batch] kv_len + new_len, or NULL
 *   pages_held_out  int32 [batch] pages each request has afterwards, or NULL
 *   free_head_out int32 [1] free_head + pages taken, or NULL
 * No output may overlap an input other than block_table (free_head_out must
 * not be free_head: keep two and swap them).
 * Rows at and behind cu_new[batch] get slot and position -1 and an empty mask;
 * rows at and behind n_rows are counted in cu_new, but not written (nor are the
 * table entries of pages that begin with one of them).
 * Where the free list ends (free_head_out > n_free then), where a page number
 * lies outside [0, n_pages) or a request needs more than max_pages pages, the
 * table entry of a new page is -1 (beyond max_pages there is none) and the slots
 * in it are -1; the calls below skip them.
 * Errors: null pointers, page_size not a power of two (UNSUPPORTED),
 * n_pages * page_size beyond int32, max_new > QCF_MAX_TREE with parents (UNSUPPORTED).
 */
#define QCF_MAX_TREE 1024
qcf_status qcf_page_plan(int32_t* block_table, int64_t table_stride, int max_pages, int batch,
                         const int32_t* kv_len, const int32_t* new_len,
                         const int32_t* pages_held, const int32_t* free_pages, int64_t n_free,
                         const int32_t* free_head, int64_t n_pages, int page_size, int max_new,
                         const int32_t* parents, uint32_t* tree_mask, int mask_words,
                         int32_t* slots, int32_t* positions, int64_t n_rows, int32_t* cu_new,
                         int32_t* kv_end, int32_t* pages_held_out, int32_t* free_head_out,
                         hipStream_t stream);

/*
 * qcf_rope_frequencies -- the angular frequencies of rotary pairs j <
 * rotary_dim / 2, in float64 (host function; a model's constant, uploaded once):
 *     w_j = rope_theta^(-2j / rotary_dim)                    QCF_ROPE_UNSCALED
 *     w_j / factor                                           QCF_ROPE_LINEAR
 *     (1 - g_j) w_j / factor + g_j w_j                       QCF_ROPE_BY_PARTS
 * with g_j = clamp((t_j - low_turns) / (high_turns - low_turns), 0, 1) and t_j =
 * trained_len * w_j / (2 pi), the turns that pair j makes over the trained
 * length: pairs of few turns are stretched, pairs of many kept.  A base that is
 * raised instead is another rope_theta.
 *   freq  float64 [rotary_dim / 2] in HOST memory
 * Errors: rotary_dim not even and positive, rope_theta or factor not positive and
 * finite, low_turns >= high_turns or trained_len <= 0 (QCF_ROPE_BY_PARTS only).
 */
typedef enum { QCF_ROPE_UNSCALED = 0, QCF_ROPE_LINEAR = 1, QCF_ROPE_BY_PARTS = 2 } qcf_rope_scaling;
qcf_status qcf_rope_frequencies(double* freq, int rotary_dim, double rope_theta, int scaling,
                                double factor, double low_turns, double high_turns,
                                double trained_len);

/*
 * qcf_rope_store -- rotary positions of new rows in the model's form, keys and
 * values into their slots.  For each r < n_rows with s = src_idx ? src_idx[r] : r
 * and p = positions[r]:
 *     k_cache[slots[r]] = turn(k_new[s], p),  v_cache[slots[r]] = v_new[s]
 *                                             (when k_cache != NULL)
 *     q_out[r]          = turn(q_new[s], p)   (when q_out != NULL)
 * turn() rotates the first rotary_dim elements of every head and copies the
 * rest; pair j turns by the angle p * freq[j], and the turned pair is multiplied
 * by magnitude (the attention factor that goes with some scalings; 1 otherwise).
 * Pairs are (j, j + rotary_dim/2) or, interleaved, (2j, 2j + 1).  Angles are
 * formed in float64, cosine and sine times magnitude rounded to float32, the
 * products are float32.
 *   k_cache, v_cache  [n_slots, cache_row_stride], both or neither
 *   k_new, v_new      [n_src_rows] rows of n_kv_heads * head_dim elements, new_row_stride
 *                     elements apart; q_new rows of n_q_heads * head_dim elements,
 *                     q_row_stride apart (slices of one projection's output)
 *   q_out   [n_rows, n_q_heads, head_dim] dense
 *   slots   int32 [n_rows] (when k_cache != NULL); distinct where inside [0, n_slots);
 *           rows with another slot store nothing, their query is still turned
 *   positions  int32 [n_rows], or NULL: nothing is turned (rows that are turned
 *           already move into pages, or from slot to slot through a copy);
 *           then freq is NULL, rotary_dim 0 and magnitude 1
 *   freq    float64 [rotary_dim / 2] device array; rotary_dim a multiple of 16 up to head_dim
 * Rows whose s is outside [0, n_src_rows) are skipped (their q_out row is left).
 * Outputs may not overlap inputs.
 * Errors: as for qcf_scatter_kv; rotary_dim not a multiple of 16 (UNSUPPORTED).
 */
qcf_status qcf_rope_store(void* k_cache, void* v_cache, int64_t n_slots, int64_t cache_row_stride,
                          void* q_out, const void* k_new, const void* v_new,
                          int64_t new_row_stride, const void* q_new, int64_t q_row_stride,
                          int64_t n_src_rows, const int32_t* src_idx, qcf_dtype dtype,
                          int64_t n_rows, const int32_t* slots, const int32_t* positions,
                          const double* freq, int rotary_dim, int interleaved, float magnitude,
                          int n_q_heads, int n_kv_heads, int head_dim, hipStream_t stream);

/*
 * qcf_tree_attn -- grouped-query attention of each request's new rows over its
 * paged cache.  Request b's row i (packed row r = cu_q[b] + i) and head h:
 *     out[r, h] = sum_t softmax_t( q[r, h] . K[t, h/group] * softmax_scale ) V[t, h/group]
 * over the tokens t < kv_len[b] (all of them) and, of the new rows' own tokens
 * t = kv_len[b] + j (whose keys and values are in their slots already), those
 * whose bit j of row r's mask is set; without a mask those with j <= i (one
 * decoded token, a chain of drafts, a prompt; a long one costs all its rows times
 * all its tokens, whatever they see).  Token t sits in the slot that the
 * block table gives it.  A row that sees no token gets zeros (and lse = -inf); one
 * that sees only logits of -infinity, or a NaN, is NaN (lse too).
 * Values a row does not see never reach it, whatever they hold.
 *   out, q     [n_rows, n_q_heads, head_dim]; rows at and behind cu_q[batch] are
 *              neither read nor written
 *   lse        float32 [n_rows, n_q_heads] natural-log log-sum-exp, or NULL
 *   cu_q       int32 [batch + 1], ascending from 0
 *   k_cache, v_cache  [n_slots, kv_row_stride]; pages p < n_slots / page_size
 *   block_table  int32 [batch, table_stride], columns 0 .. max_pages-1 used; tokens
 *              in pages outside the pool or beyond max_pages are not seen
 *   kv_len     int32 [batch] tokens before the new rows (a negative one counts as 0)
 *   tree_mask  uint32 [n_rows, mask_words] or NULL; bits at and behind the request's row
 *              count and behind 32 * mask_words are not seen
 *   max_q      >= every cu_q[b+1] - cu_q[b] (further rows are left alone)
 *   max_kv     >= every kv_len[b] + (cu_q[b+1] - cu_q[b]) (further tokens are
 *              not seen)
 *   workspace  >= qcf_tree_attn_workspace_size(...) bytes (may be 0), 256-byte aligned:
 *              the partial results of long caches that are cut over blocks, merged in
 *              order by a second kernel (deterministic).  It needs no initialisation
 *              and keeps nothing; calls that overlap in time need separate ones.  The
 *              size for (batch, max_q, max_kv) covers every call whose three values
 *              do not exceed them (other arguments equal).
 * Sums, maxima and partial results are float32; bf16 calls hand the weights
 * exp(x - max) to the matrix units, after they entered the sum, as two bf16 numbers
 * (15 bits) up to max_q * n_q_heads / n_kv_heads = 64, as one beyond.  A row's
 * bits do not depend on the other rows' values.
 * Errors: null pointers, softmax_scale not positive and finite, page_size not a
 * power of two (UNSUPPORTED), row strides of 128 MB and more, batch * max_q *
 * n_q_heads beyond int32, max_kv within 2^20 of it, or, with max_kv up to 2048, 2^23
 * tiles and more (of 16 to 128 query vectors, each of one request and KV head;
 * UNSUPPORTED), workspace.
 */
size_t qcf_tree_attn_workspace_size(int batch, int max_q, int max_kv, int n_q_heads,
                                    int n_kv_heads, int head_dim, qcf_dtype dtype);
qcf_status qcf_tree_attn(void* out, float* lse, const void* q, int64_t n_rows,
                         const int32_t* cu_q, const void* k_cache, const void* v_cache,
                         int64_t n_slots, int64_t kv_row_stride, const int32_t* block_table,
                         int64_t table_stride, int max_pages, int page_size,
                         const int32_t* kv_len, const uint32_t* tree_mask, int mask_words,
                         qcf_dtype dtype, int batch, int max_q, int max_kv, int n_q_heads,
                         int n_kv_heads, int head_dim, float softmax_scale, void* workspace,
                         size_t workspace_bytes, hipStream_t stream);

/*
 * qcf_verify_drafts -- which drafted tokens stay, and the token after them, by
 * sequential rejection against the target's probabilities with random numbers
 * given by the caller.  Row i of request b is a node of its tree; row 0, the
 * root, holds a token that is decided already, and target[r] is the model's
 * distribution after row r.  From the root on, the children of the current node
 * are tested in ascending order.  With P = target row, D = draft row of the
 * current node, x = tokens[child] and u = u_accept[child], a child is accepted if
 *     u * Z * D(x) < R(x),          at first  Z = 1, R = P
 * (D(x) = 1 without draft probabilities), and becomes the current node; else
 *     with draft:     c += Z (c = 0 at first),  R = max(P - c D, 0),  Z = sum R
 *     without draft:  Z = max(Z - R(x), 0),  R(x) = 0
 * and the next child is tested.  Where no child is accepted (or there is none)
 * the next token is drawn from R: the lowest t whose running sum R(0) + .. +
 * R(t) exceeds u_next[b] * sum R.  If R is zero everywhere, P takes its place; if
 * P is too, the token is -1.  Probabilities that are not above zero (NaN too)
 * count as zero.  Sums, products and comparisons are float64.
 *   target, draft  [n_rows, vocab], rows row_stride elements apart (any stride >=
 *              vocab; the same for both); draft may be NULL; vocab <= 2^28 - 8192
 *   tokens     int32 [n_rows]; a child's token outside [0, vocab) is rejected (R unchanged)
 *   parents    int32 [n_rows] index of the parent within the request, below the
 *              row's own (others are not reached), or NULL: a chain, parent i - 1
 *   cu_rows    int32 [batch + 1], batch < 2^22; max_rows >= every request's rows, at most QCF_MAX_TREE
 *              (further rows are ignored)
 *   u_accept   float32 [n_rows], u_next float32 [batch], in [0, 1)
 *   n_out      int32 [batch] accepted drafts + 1 (0 for a request without rows)
 *   path       int32 [batch, max_rows]: the rows of the request that stay, the root first,
 *              n_out of them; -1 behind
 *   out_tokens int32 [batch, max_rows]: the accepted drafts' tokens, then the drawn one;
 *              -1 behind
 *   slots      int32 [n_rows] the rows' slots (qcf_page_plan), or NULL
 *   move_src, move_dst  int32 [batch, max_rows], given with slots and only then: the keys
 *              and values that stay move to the front of the new rows' slots:
 *              entry k < n_out is (slot of row path[k], slot of row k), or -1, -1
 *              where they are the same; -1 behind.  A source may be another entry's
 *              destination: copy them out (qcf_gather_rows) before they are stored
 *              (qcf_rope_store without positions).
 *   workspace  >= qcf_verify_drafts_workspace_size(batch, vocab) bytes, 256-byte
 *              aligned, no initialisation; calls that overlap in time need separate ones
 */
size_t qcf_verify_drafts_workspace_size(int batch, int vocab);
qcf_status qcf_verify_drafts(int32_t* n_out, int32_t* path, int32_t* out_tokens,
                             const void* target, const void* draft, int64_t row_stride,
                             qcf_dtype dtype, int64_t n_rows, int vocab, const int32_t* tokens,
                             const int32_t* parents, int batch, const int32_t* cu_rows,
                             int max_rows, const float* u_accept, const float* u_next,
                             const int32_t* slots, int32_t* move_src, int32_t* move_dst,
                             void* workspace, size_t workspace_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* QCF_DECODE_H_ */
