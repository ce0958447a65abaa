// C ABI of libqcf, third part (qcf_turns.h): host-side validation, then the kernel launchers.
// Every check runs before any HIP call, so a rejected call touches no device
// state (and works on a machine without a GPU).
#include "../../include/qcf_turns.h"

#include <math.h>
#include <stdint.h>

#include "qcf_checks.h"
#include "qcf_turns_launch.h"

namespace {

inline bool element_ok(const void* p, bool empty, qcf_dtype t) {
  return empty || (p && (reinterpret_cast<uintptr_t>(p) & (esize(t) - 1)) == 0);
}
// a weight of all heads, or one per head
inline bool weight_ok(const void* w, int64_t stride, int d, qcf_dtype t) {
  return w ? aligned16(w) && (stride == 0 || kv_stride_ok(stride, 1, d, t)) : stride == 0;
}

}  // namespace

extern "C" {

qcf_status qcf_norm_rope_store(void* k_cache, void* v_cache, int64_t n_slots, int64_t cache_row_stride,
                               void* q_out, const void* k_new, const void* v_new,
                               int64_t new_row_stride, const void* q_new, int64_t q_row_stride,
                               int64_t n_src_rows, const int32_t* src_idx, qcf_dtype dtype,
                               int64_t n_rows, const int32_t* slots, const int32_t* positions,
                               const double* freq, int rotary_dim, int interleaved, float magnitude,
                               const void* q_weight, int64_t q_weight_stride, const void* k_weight,
                               int64_t k_weight_stride, float eps, int n_q_heads, int n_kv_heads,
                               int head_dim, hipStream_t stream) {
  const qcf_status st = check_rope_store(k_cache, v_cache, n_slots, cache_row_stride, q_out, k_new, v_new, new_row_stride,
                                         q_new, q_row_stride, n_src_rows, src_idx, dtype, n_rows, slots, positions,
                                         freq, rotary_dim, magnitude, n_q_heads, n_kv_heads, head_dim);
  if (st != QCF_OK) return st;
  if (!(eps >= 0.f) || !isfinite(eps) || !weight_ok(q_weight, q_weight_stride, head_dim, dtype) ||
      !weight_ok(k_weight, k_weight_stride, head_dim, dtype))
    return QCF_ERR_INVALID_ARG;
  if (n_rows == 0 || n_src_rows == 0 || (!k_cache && !q_out)) return QCF_OK;
  const qcf::NormRopeStore p{{k_cache, v_cache, n_slots, cache_row_stride, q_out, k_new, v_new, new_row_stride, q_new,
                              q_row_stride, n_src_rows, src_idx, n_rows, slots, positions, freq, rotary_dim, magnitude,
                              n_q_heads, n_kv_heads},
                             q_weight, k_weight, q_weight_stride, k_weight_stride, eps};
  return hip_status(qcf::launch_norm_rope_store(p, dtype == QCF_BF16, head_dim, interleaved != 0, stream));
}

size_t qcf_chunk_attn_workspace_size(int batch, int max_q, int max_kv, int n_q_heads,
                                     int n_kv_heads, int head_dim, qcf_dtype dtype) {
  if (!dtype_ok(dtype) || check_heads(n_q_heads, n_kv_heads, head_dim) != QCF_OK) return 0;
  // (rows that see no token go through the same kernels: max_kv does not matter)
  if (batch <= 0 || max_q <= 0 || max_kv < 0) return 0;
  return qcf::chunk_attn_workspace(max_q, n_q_heads, n_kv_heads, head_dim, dtype == QCF_BF16);
}

qcf_status qcf_chunk_attn(void* out, float* lse, const void* q, int64_t n_rows,
                          const int32_t* cu_q, const void* k_cache, const void* v_cache,
                          int64_t n_slots, int64_t kv_row_stride, const int32_t* block_table,
                          int64_t table_stride, int max_pages, int page_size,
                          const int32_t* kv_len, int window, qcf_dtype dtype, int batch, int max_q,
                          int max_kv, int n_q_heads, int n_kv_heads, int head_dim,
                          float softmax_scale, void* workspace, size_t workspace_bytes,
                          hipStream_t stream) {
  if (!dtype_ok(dtype)) return QCF_ERR_UNSUPPORTED;
  const qcf_status st = check_heads(n_q_heads, n_kv_heads, head_dim);
  if (st != QCF_OK) return st;
  if (n_rows < 0 || n_rows > INT32_MAX || n_slots < 0 || n_slots > INT32_MAX || batch < 0 || window < 0 ||
      max_q < 0 || max_kv < 0 || max_pages < 0 || table_stride < max_pages || page_size <= 0)
    return QCF_ERR_INVALID_ARG;
  const int lp = page_log2(page_size);
  if (lp < 4) return QCF_ERR_UNSUPPORTED;
  if (!(softmax_scale > 0.f) || !isfinite(softmax_scale)) return QCF_ERR_INVALID_ARG;
  if (!kv_stride_ok(kv_row_stride, n_kv_heads, head_dim, dtype)) return QCF_ERR_INVALID_ARG;
  // the kernels' 32-bit numbers: offsets inside 16 rows, (row, head) pairs, tokens a few tiles on
  if (kv_row_stride > INT32_MAX / (16 * esize(dtype)) || max_kv > INT32_MAX - (1 << 21) || max_q > 1 << 20 || batch > 1 << 30 ||
      !qcf::chunk_attn_fits(batch, max_q, n_q_heads, n_kv_heads, dtype == QCF_BF16))
    return QCF_ERR_UNSUPPORTED;
  const bool empty = n_rows == 0 || batch == 0 || max_q == 0;
  const bool no_kv = empty || max_kv == 0 || max_pages == 0 || n_slots >> lp == 0;
  if (!tensor_ok(out, empty) || !tensor_ok(q, empty) || !tensor_ok(k_cache, no_kv) ||
      !tensor_ok(v_cache, no_kv) || !index_ok(cu_q, empty) || !index_ok(kv_len, empty) ||
      !index_ok(block_table, no_kv) || !optional_index_ok(lse))
    return QCF_ERR_INVALID_ARG;
  if (!empty && (out == q || out == k_cache || out == v_cache)) return QCF_ERR_INVALID_ARG;
  if (empty) return QCF_OK;
  const size_t need = qcf_chunk_attn_workspace_size(batch, max_q, max_kv, n_q_heads, n_kv_heads, head_dim, dtype);
  if (workspace_bytes < need || (need > 0 && (!workspace || !aligned256(workspace))))
    return QCF_ERR_WORKSPACE;
  // nothing to read: every row sees no token
  const qcf::ChunkAttn p{{out, lse, q, n_rows, cu_q, k_cache, v_cache, no_kv ? 0 : n_slots >> lp, kv_row_stride,
                          block_table, table_stride, no_kv ? 0 : max_pages, lp, kv_len, nullptr, 0, batch, max_q,
                          max_kv, n_q_heads, n_kv_heads, softmax_scale},
                         window};
  return hip_status(qcf::launch_chunk_attn(p, dtype == QCF_BF16, head_dim, workspace, stream));
}

size_t qcf_shape_logits_workspace_size(int64_t n_rows, int vocab) {
  if (n_rows <= 0 || n_rows > INT32_MAX || vocab <= 0 || vocab > qcf::kShapeMaxVocab) return 0;
  return qcf::shape_logits_workspace(n_rows, vocab);
}

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
                            void* workspace, size_t workspace_bytes, hipStream_t stream) {
  if (!dtype_ok(dtype) || !dtype_ok(out_dtype)) return QCF_ERR_UNSUPPORTED;
  if (n_rows < 0 || n_rows > INT32_MAX || vocab <= 0 || batch < 0 || out_stride < vocab || logits_stride < vocab ||
      max_history < 0 || n_bias < 0 || n_bias > INT32_MAX)
    return QCF_ERR_INVALID_ARG;
  // (the kernels' 32-bit counters run a few blocks' width past their ends)
  if (vocab > qcf::kShapeMaxVocab || batch > 1 << 30 || max_history > 1 << 30) return QCF_ERR_UNSUPPORTED;
  const bool empty = n_rows == 0 || batch == 0;
  if (!element_ok(out, empty, out_dtype) || !element_ok(logits, empty, dtype) || !index_ok(cu_rows, empty))
    return QCF_ERR_INVALID_ARG;
  if (!empty && out == logits && (out_dtype != dtype || out_stride != logits_stride)) return QCF_ERR_INVALID_ARG;
  if (history ? !hist_len || history_stride < max_history : prompt_len || hist_len || max_history != 0)
    return QCF_ERR_INVALID_ARG;
  if ((tree_mask && !tokens) || (tree_mask && mask_words <= 0)) return QCF_ERR_INVALID_ARG;
  if (bias_start ? n_bias > 0 && (!bias_token || !bias_value) : bias_token || bias_value || n_bias != 0)
    return QCF_ERR_INVALID_ARG;
  if (allowed && allowed_words < ((int64_t)vocab + 31) / 32) return QCF_ERR_INVALID_ARG;
  for (const void* x : {(const void*)history, (const void*)prompt_len, (const void*)hist_len, (const void*)tokens,
                        (const void*)tree_mask, (const void*)repetition, (const void*)presence,
                        (const void*)frequency, (const void*)bias_start, (const void*)bias_token,
                        (const void*)bias_value, (const void*)allowed, (const void*)temperature})
    if (!optional_index_ok(x)) return QCF_ERR_INVALID_ARG;
  if (empty) return QCF_OK;
  const size_t need = probabilities ? qcf_shape_logits_workspace_size(n_rows, vocab) : 0;
  if (workspace_bytes < need || (need > 0 && (!workspace || !aligned256(workspace)))) return QCF_ERR_WORKSPACE;
  const qcf::ShapeLogits p{out, out_stride, logits, logits_stride, n_rows, vocab, batch, cu_rows, history,
                           history_stride, max_history, prompt_len, hist_len, tokens, tree_mask, mask_words,
                           repetition, presence, frequency, bias_start, bias_token, bias_value, n_bias, allowed,
                           allowed_words, temperature};
  return hip_status(qcf::launch_shape_logits(p, dtype == QCF_BF16, out_dtype == QCF_BF16, probabilities != 0,
                                             workspace, stream));
}

qcf_status qcf_page_fork(int32_t* table_out, int64_t table_out_stride, int32_t* kv_out,
                         int32_t* held_out, const int32_t* block_table, int64_t table_stride,
                         int max_pages, int batch, const int32_t* kv_len, const int32_t* source,
                         const int32_t* keep_len, const int32_t* free_pages, int64_t n_free,
                         const int32_t* free_head, int64_t n_pages, int page_size,
                         int32_t* free_head_out, int32_t* copy_src, int32_t* copy_dst,
                         int32_t* copy_rows, hipStream_t stream) {
  if (batch < 0 || max_pages < 0 || table_out_stride < max_pages || table_stride < max_pages || n_free < 0 ||
      n_free > INT32_MAX || n_pages < 0 || page_size <= 0)
    return QCF_ERR_INVALID_ARG;
  const int lp = page_log2(page_size);
  if (lp < 0 || batch >= 1 << 22) return QCF_ERR_UNSUPPORTED;
  if (n_pages > (int64_t)INT32_MAX >> lp) return QCF_ERR_INVALID_ARG;
  const bool none = batch == 0, no_table = none || max_pages == 0;
  if (!index_ok(table_out, no_table) || !index_ok(block_table, no_table) || !index_ok(kv_out, none) ||
      !index_ok(held_out, none) || !index_ok(kv_len, none) || !index_ok(source, none) || !optional_index_ok(keep_len) ||
      !index_ok(free_pages, n_free == 0) || !optional_index_ok(free_head) || !index_ok(free_head_out, false) ||
      !index_ok(copy_src, none) || !index_ok(copy_dst, none) || !index_ok(copy_rows, none))
    return QCF_ERR_INVALID_ARG;
  // outputs that other blocks still read as inputs
  const void* in[] = {block_table, kv_len, source, keep_len, free_pages, free_head};
  const void* result[] = {table_out, kv_out, held_out, free_head_out, copy_src, copy_dst, copy_rows};
  for (size_t i = 0; i < sizeof result / sizeof *result; ++i) {
    for (const void* x : in)
      if (x && x == result[i]) return QCF_ERR_INVALID_ARG;
    for (size_t j = 0; j < i; ++j)
      if (result[j] && result[j] == result[i]) return QCF_ERR_INVALID_ARG;
  }
  const qcf::PageFork p{table_out, table_out_stride, kv_out, held_out, block_table, table_stride, max_pages, batch,
                        kv_len, source, keep_len, free_pages, n_free, free_head, n_pages, lp, free_head_out, copy_src,
                        copy_dst, copy_rows};
  return hip_status(qcf::launch_page_fork(p, stream));
}

qcf_status qcf_copy_pages(void* const* pools, int n_pools, int64_t n_slots, int64_t row_bytes,
                          int64_t row_stride_bytes, int page_size, const int32_t* src_page,
                          const int32_t* dst_page, const int32_t* rows, int64_t n_pairs,
                          hipStream_t stream) {
  if (n_pools < 0 || n_slots < 0 || n_slots > INT32_MAX || row_bytes <= 0 || row_bytes % 16 != 0 ||
      row_bytes > INT32_MAX || row_stride_bytes < row_bytes || row_stride_bytes % 16 != 0 || page_size <= 0 ||
      n_pairs < 0 || n_pairs > INT32_MAX)
    return QCF_ERR_INVALID_ARG;
  const int lp = page_log2(page_size);
  if (lp < 0) return QCF_ERR_UNSUPPORTED;
  const bool empty = n_pools == 0 || n_pairs == 0 || n_slots >> lp == 0;
  if ((!empty && (!pools || (reinterpret_cast<uintptr_t>(pools) & 7u) != 0)) || !index_ok(src_page, empty) ||
      !index_ok(dst_page, empty) || !optional_index_ok(rows))
    return QCF_ERR_INVALID_ARG;
  if (empty) return QCF_OK;
  const qcf::CopyPages p{pools, n_pools, n_slots >> lp, row_bytes, row_stride_bytes, lp, src_page, dst_page, rows, n_pairs};
  if (qcf::copy_pages_blocks(p) < 0) return QCF_ERR_UNSUPPORTED;
  return hip_status(qcf::launch_copy_pages(p, stream));
}

size_t qcf_page_release_workspace_size(int batch, int max_pages, int64_t n_pages) {
  if (batch <= 0 || max_pages <= 0 || n_pages <= 0 || n_pages > INT32_MAX) return 0;
  return qcf::page_release_workspace(batch, max_pages, n_pages);
}

qcf_status qcf_page_release(const int32_t* table_before, int64_t before_stride,
                            const int32_t* held_before, const int32_t* table_after,
                            int64_t after_stride, const int32_t* held_after, int max_pages,
                            int batch, int32_t* free_pages, int64_t n_free,
                            const int32_t* free_head, int32_t* free_head_out, int64_t n_pages,
                            void* workspace, size_t workspace_bytes, hipStream_t stream) {
  if (batch < 0 || max_pages < 0 || before_stride < max_pages || after_stride < max_pages || n_free < 0 ||
      n_free > INT32_MAX || n_pages < 0 || n_pages > INT32_MAX)
    return QCF_ERR_INVALID_ARG;
  // (a block per 1024 entries of a row of either table)
  if (batch >= 1 << 22 || (int64_t)batch * (((int64_t)max_pages + 1023) / 1024) >= 1 << 22) return QCF_ERR_UNSUPPORTED;
  const bool none = batch == 0, no_table = none || max_pages == 0;
  if (!index_ok(table_before, no_table) || !index_ok(table_after, no_table) || !index_ok(held_before, none) ||
      !index_ok(held_after, none) || !index_ok(free_pages, n_free == 0) || !index_ok(free_head, false) ||
      !index_ok(free_head_out, false))
    return QCF_ERR_INVALID_ARG;
  const void* in[] = {table_before, table_after, held_before, held_after, free_head};
  for (const void* x : in)
    if (x && (x == free_head_out || x == free_pages)) return QCF_ERR_INVALID_ARG;
  if (free_pages == free_head_out) return QCF_ERR_INVALID_ARG;
  const size_t need = qcf_page_release_workspace_size(batch, max_pages, n_pages);
  if (workspace_bytes < need || (need > 0 && (!workspace || !aligned256(workspace)))) return QCF_ERR_WORKSPACE;
  // without a table no page is held, whatever the pool: the workspace is not there then
  const qcf::PageRelease p{table_before, before_stride, held_before, table_after, after_stride, held_after, max_pages,
                           batch, free_pages, n_free, free_head, free_head_out, no_table ? 0 : n_pages};
  return hip_status(qcf::launch_page_release(p, workspace, stream));
}

}  // extern "C"
