// C ABI of libqcf, second part (qcf_decode.h): host-side validation, then the kernel launchers.
// Every check runs before any HIP call, so a rejected call touches no device
// state (and works on a machine without a GPU).
#include "../../include/qcf_decode.h"

#include <math.h>
#include <stdint.h>

#include "qcf_checks.h"
#include "qcf_decode_launch.h"

namespace {

inline bool optional_index_ok(const void* p) { return !p || index_ok(p, false); }

// log2 of a page size, or -1 where it is not a power of two
int page_log2(int page_size) {
  if (page_size <= 0 || (page_size & (page_size - 1)) != 0) return -1;
  return __builtin_ctz((unsigned)page_size);
}

}  // namespace

extern "C" {

qcf_status qcf_page_plan(int32_t* block_table, int64_t table_stride, int max_pages, int batch,
                         const int32_t* kv_len, const int32_t* new_len,
                         const int32_t* pages_held, const int32_t* free_pages, int64_t n_free,
                         const int32_t* free_head, int64_t n_pages, int page_size, int max_new,
                         const int32_t* parents, uint32_t* tree_mask, int mask_words,
                         int32_t* slots, int32_t* positions, int64_t n_rows, int32_t* cu_new,
                         int32_t* kv_end, int32_t* pages_held_out, int32_t* free_head_out,
                         hipStream_t stream) {
  if (batch < 0 || max_pages < 0 || table_stride < max_pages || n_free < 0 || n_free > INT32_MAX ||
      n_pages < 0 || max_new < 0 || n_rows < 0 || n_rows > INT32_MAX || page_size <= 0)
    return QCF_ERR_INVALID_ARG;
  const int lp = page_log2(page_size);
  if (lp < 0) return QCF_ERR_UNSUPPORTED;
  if (n_pages > (int64_t)INT32_MAX >> lp) return QCF_ERR_INVALID_ARG;
  if ((parents == nullptr) != (tree_mask == nullptr) && n_rows > 0) return QCF_ERR_INVALID_ARG;
  if (parents) {
    if (max_new > QCF_MAX_TREE) return QCF_ERR_UNSUPPORTED;
    if (mask_words < 0 || (int64_t)mask_words * 32 < max_new) return QCF_ERR_INVALID_ARG;
    if (!index_ok(parents, false) || !index_ok(tree_mask, false)) return QCF_ERR_INVALID_ARG;
  }
  const bool none = batch == 0;
  if (!index_ok(block_table, none || max_pages == 0) || !index_ok(kv_len, none) ||
      !index_ok(new_len, none) || !index_ok(free_pages, n_free == 0) || !index_ok(cu_new, false) ||
      !index_ok(slots, n_rows == 0) || !index_ok(positions, n_rows == 0))
    return QCF_ERR_INVALID_ARG;
  if (!optional_index_ok(pages_held) || !optional_index_ok(free_head) || !optional_index_ok(kv_end) ||
      !optional_index_ok(pages_held_out) || !optional_index_ok(free_head_out))
    return QCF_ERR_INVALID_ARG;
  // outputs that other blocks still read as inputs
  if ((free_head_out && free_head_out == free_head) ||
      (pages_held_out && (pages_held_out == pages_held || pages_held_out == kv_len)) ||
      (kv_end && (kv_end == kv_len || kv_end == new_len)))
    return QCF_ERR_INVALID_ARG;
  const qcf::PagePlan p{block_table, table_stride, max_pages, batch,      kv_len,  new_len,
                        pages_held,  free_pages,   n_free,    free_head,  n_pages, lp,
                        parents,     tree_mask,    mask_words, slots,     positions, n_rows,
                        cu_new,      kv_end,       pages_held_out, free_head_out};
  return hip_status(qcf::launch_page_plan(p, stream));
}

qcf_status qcf_rope_frequencies(double* freq, int rotary_dim, double rope_theta, int scaling,
                                double factor, double low_turns, double high_turns,
                                double trained_len) {
  if (!freq || rotary_dim <= 0 || rotary_dim % 2 != 0) return QCF_ERR_INVALID_ARG;
  if (!(rope_theta > 0.0) || !isfinite(rope_theta)) return QCF_ERR_INVALID_ARG;
  if (scaling < QCF_ROPE_UNSCALED || scaling > QCF_ROPE_BY_PARTS) return QCF_ERR_UNSUPPORTED;
  if (scaling != QCF_ROPE_UNSCALED && (!(factor > 0.0) || !isfinite(factor))) return QCF_ERR_INVALID_ARG;
  if (scaling == QCF_ROPE_BY_PARTS && (!(low_turns < high_turns) || !(trained_len > 0.0)))
    return QCF_ERR_INVALID_ARG;
  for (int j = 0; j < rotary_dim / 2; ++j) {
    double w = pow(rope_theta, -2.0 * j / rotary_dim);
    if (scaling == QCF_ROPE_LINEAR) w /= factor;
    if (scaling == QCF_ROPE_BY_PARTS) {
      const double turns = trained_len * w / (2.0 * M_PI);
      const double g = fmin(fmax((turns - low_turns) / (high_turns - low_turns), 0.0), 1.0);
      w = (1.0 - g) * w / factor + g * w;
    }
    freq[j] = w;
  }
  return QCF_OK;
}

qcf_status qcf_rope_store(void* k_cache, void* v_cache, int64_t n_slots, int64_t cache_row_stride,
                          void* q_out, const void* k_new, const void* v_new,
                          int64_t new_row_stride, const void* q_new, int64_t q_row_stride,
                          int64_t n_src_rows, const int32_t* src_idx, qcf_dtype dtype,
                          int64_t n_rows, const int32_t* slots, const int32_t* positions,
                          const double* freq, int rotary_dim, int interleaved, float magnitude,
                          int n_q_heads, int n_kv_heads, int head_dim, hipStream_t stream) {
  if (!dtype_ok(dtype)) return QCF_ERR_UNSUPPORTED;
  qcf_status st = check_heads(n_q_heads, n_kv_heads, head_dim);
  if (st != QCF_OK) return st;
  if (n_rows < 0 || n_rows > INT32_MAX || n_slots < 0 || n_slots > INT32_MAX || n_src_rows < 0 ||
      n_src_rows > INT32_MAX)
    return QCF_ERR_INVALID_ARG;
  if ((k_cache == nullptr) != (v_cache == nullptr)) return QCF_ERR_INVALID_ARG;
  if (q_out && !q_new) return QCF_ERR_INVALID_ARG;
  if (rotary_dim < 0 || rotary_dim > head_dim) return QCF_ERR_INVALID_ARG;
  if (rotary_dim % 16 != 0) return QCF_ERR_UNSUPPORTED;
  // positions, frequencies and a rotated part go together
  if (n_rows > 0 && ((positions == nullptr) != (rotary_dim == 0) || (freq == nullptr) != (rotary_dim == 0)))
    return QCF_ERR_INVALID_ARG;
  if (!isfinite(magnitude) || (rotary_dim == 0 && magnitude != 1.f)) return QCF_ERR_INVALID_ARG;
  if (k_cache) {
    if (!kv_stride_ok(cache_row_stride, n_kv_heads, head_dim, dtype) ||
        !kv_stride_ok(new_row_stride, n_kv_heads, head_dim, dtype))
      return QCF_ERR_INVALID_ARG;
    if (!aligned16(k_cache) || !aligned16(v_cache) || !tensor_ok(k_new, n_rows == 0 || n_src_rows == 0) ||
        !tensor_ok(v_new, n_rows == 0 || n_src_rows == 0) || !index_ok(slots, n_rows == 0))
      return QCF_ERR_INVALID_ARG;
  }
  if (q_out && (!aligned16(q_out) || !aligned16(q_new) || q_out == q_new ||
                !kv_stride_ok(q_row_stride, n_q_heads, head_dim, dtype)))
    return QCF_ERR_INVALID_ARG;
  if (!optional_index_ok(positions) || !optional_index_ok(src_idx) ||
      (reinterpret_cast<uintptr_t>(freq) & 7u) != 0)
    return QCF_ERR_INVALID_ARG;
  if (k_cache && (k_cache == k_new || v_cache == v_new)) return QCF_ERR_INVALID_ARG;
  if (n_rows == 0 || n_src_rows == 0 || (!k_cache && !q_out)) return QCF_OK;
  const qcf::RopeStore p{k_cache,  v_cache,    n_slots,   cache_row_stride, q_out,     k_new,  v_new,
                         new_row_stride, q_new, q_row_stride, n_src_rows,   src_idx,   n_rows, slots,
                         positions, freq,      rotary_dim, magnitude,       n_q_heads, n_kv_heads};
  return hip_status(qcf::launch_rope_store(p, dtype == QCF_BF16, head_dim, interleaved != 0, stream));
}

size_t qcf_tree_attn_workspace_size(int batch, int max_q, int max_kv, int n_q_heads,
                                    int n_kv_heads, int head_dim, qcf_dtype dtype) {
  if (!dtype_ok(dtype) || check_heads(n_q_heads, n_kv_heads, head_dim) != QCF_OK) return 0;
  if (batch <= 0 || max_q <= 0 || max_kv <= 0 || (int64_t)batch * max_q > INT32_MAX / n_q_heads) return 0;
  return qcf::tree_attn_workspace(batch, max_q, max_kv, n_q_heads, n_kv_heads, head_dim,
                                  dtype == QCF_BF16);
}

qcf_status qcf_tree_attn(void* out, float* lse, const void* q, int64_t n_rows,
                         const int32_t* cu_q, const void* k_cache, const void* v_cache,
                         int64_t n_slots, int64_t kv_row_stride, const int32_t* block_table,
                         int64_t table_stride, int max_pages, int page_size,
                         const int32_t* kv_len, const uint32_t* tree_mask, int mask_words,
                         qcf_dtype dtype, int batch, int max_q, int max_kv, int n_q_heads,
                         int n_kv_heads, int head_dim, float softmax_scale, void* workspace,
                         size_t workspace_bytes, hipStream_t stream) {
  if (!dtype_ok(dtype)) return QCF_ERR_UNSUPPORTED;
  qcf_status st = check_heads(n_q_heads, n_kv_heads, head_dim);
  if (st != QCF_OK) return st;
  if (n_rows < 0 || n_rows > INT32_MAX || n_slots < 0 || n_slots > INT32_MAX || batch < 0 ||
      max_q < 0 || max_kv < 0 || max_pages < 0 || table_stride < max_pages || page_size <= 0)
    return QCF_ERR_INVALID_ARG;
  const int lp = page_log2(page_size);
  if (lp < 0) return QCF_ERR_UNSUPPORTED;
  if (!(softmax_scale > 0.f) || !isfinite(softmax_scale)) return QCF_ERR_INVALID_ARG;
  if (!kv_stride_ok(kv_row_stride, n_kv_heads, head_dim, dtype)) return QCF_ERR_INVALID_ARG;
  // the kernels' 32-bit numbers: offsets inside 16 rows, (row, head) pairs, tokens a few tiles on
  if (kv_row_stride > INT32_MAX / (16 * esize(dtype)) || max_kv > INT32_MAX - (1 << 20) ||
      (int64_t)batch * max_q > INT32_MAX / n_q_heads ||
      !qcf::tree_attn_fits(batch, max_q, max_kv, n_q_heads, n_kv_heads, dtype == QCF_BF16))
    return QCF_ERR_UNSUPPORTED;
  const bool empty = n_rows == 0 || batch == 0 || max_q == 0;
  const bool no_kv = empty || max_kv == 0 || max_pages == 0 || n_slots >> lp == 0;
  if (!tensor_ok(out, empty) || !tensor_ok(q, empty) || !tensor_ok(k_cache, no_kv) ||
      !tensor_ok(v_cache, no_kv) || !index_ok(cu_q, empty) || !index_ok(kv_len, empty) ||
      !index_ok(block_table, no_kv) || !optional_index_ok(lse) || !optional_index_ok(tree_mask))
    return QCF_ERR_INVALID_ARG;
  if (tree_mask && mask_words <= 0) return QCF_ERR_INVALID_ARG;
  if (!empty && (out == q || out == k_cache || out == v_cache)) return QCF_ERR_INVALID_ARG;
  if (empty) return QCF_OK;
  const size_t need = qcf_tree_attn_workspace_size(batch, max_q, max_kv, n_q_heads, n_kv_heads,
                                                   head_dim, dtype);
  if (workspace_bytes < need || (need > 0 && (!workspace || !aligned256(workspace))))
    return QCF_ERR_WORKSPACE;
  // nothing to read: every row sees no token
  const qcf::TreeAttn p{out,     lse,       q,         n_rows, cu_q,  k_cache, v_cache,
                        no_kv ? 0 : n_slots >> lp,     kv_row_stride, block_table, table_stride,
                        no_kv ? 0 : max_pages,         lp,     kv_len, tree_mask, mask_words,
                        batch,   max_q,     max_kv,    n_q_heads, n_kv_heads, softmax_scale};
  return hip_status(qcf::launch_tree_attn(p, dtype == QCF_BF16, head_dim, workspace, stream));
}

size_t qcf_verify_drafts_workspace_size(int batch, int vocab) {
  if (batch <= 0 || vocab <= 0) return 0;
  return qcf::verify_drafts_workspace(batch, vocab);
}

qcf_status qcf_verify_drafts(int32_t* n_out, int32_t* path, int32_t* out_tokens,
                             const void* target, const void* draft, int64_t row_stride,
                             qcf_dtype dtype, int64_t n_rows, int vocab, const int32_t* tokens,
                             const int32_t* parents, int batch, const int32_t* cu_rows,
                             int max_rows, const float* u_accept, const float* u_next,
                             const int32_t* slots, int32_t* move_src, int32_t* move_dst,
                             void* workspace, size_t workspace_bytes, hipStream_t stream) {
  if (!dtype_ok(dtype)) return QCF_ERR_UNSUPPORTED;
  if (n_rows < 0 || n_rows > INT32_MAX || vocab <= 0 || batch < 0 || max_rows < 0 || row_stride < vocab)
    return QCF_ERR_INVALID_ARG;
  if (max_rows > QCF_MAX_TREE || vocab > qcf::kVerifyMaxVocab || batch > qcf::kVerifyMaxBatch) return QCF_ERR_UNSUPPORTED;
  const bool empty = batch == 0, no_rows = empty || n_rows == 0 || max_rows == 0;
  if (!index_ok(n_out, empty) || !index_ok(path, empty || max_rows == 0) ||
      !index_ok(out_tokens, empty || max_rows == 0) || !index_ok(cu_rows, empty) ||
      !index_ok(u_next, empty) || !index_ok(tokens, no_rows) || !index_ok(u_accept, no_rows) ||
      !tensor_ok(target, no_rows) || !tensor_ok(draft, true) || !optional_index_ok(parents))
    return QCF_ERR_INVALID_ARG;
  if ((slots == nullptr) != (move_src == nullptr) || (slots == nullptr) != (move_dst == nullptr) ||
      !optional_index_ok(slots) || !optional_index_ok(move_src) || !optional_index_ok(move_dst))
    return QCF_ERR_INVALID_ARG;
  if (empty) return QCF_OK;
  const size_t need = qcf_verify_drafts_workspace_size(batch, vocab);
  if (workspace_bytes < need || !workspace || !aligned256(workspace)) return QCF_ERR_WORKSPACE;
  const qcf::VerifyDrafts p{n_out,    path,   out_tokens, target, draft,    row_stride, n_rows,
                            vocab,    tokens, parents,    batch,  cu_rows,  max_rows,   u_accept,
                            u_next,   slots,  move_src,   move_dst};
  return hip_status(qcf::launch_verify_drafts(p, dtype == QCF_BF16, workspace, stream));
}

}  // extern "C"
