// Argument checks shared by the C entry points.  They touch no device state, so a rejected call
// works on a machine without a GPU.
#pragma once
#include <hip/hip_runtime_api.h>
#include <math.h>
#include <stdint.h>

#include "../../include/qcf.h"

namespace {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool aligned256(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 255u) == 0; }
inline bool dtype_ok(qcf_dtype t) { return t == QCF_F32 || t == QCF_BF16; }
inline int64_t esize(qcf_dtype t) { return t == QCF_BF16 ? 2 : 4; }
// a device tensor pointer: non-null and 16-byte aligned (null allowed when empty)
inline bool tensor_ok(const void* p, bool empty) { return empty ? (p == nullptr || aligned16(p)) : (p && aligned16(p)); }
inline bool index_ok(const void* p, bool empty) {
  return empty || (p && (reinterpret_cast<uintptr_t>(p) & 3u) == 0);
}

inline qcf_status check_heads(int hq, int hkv, int d) {
  if (hkv <= 0 || hq <= 0) return QCF_ERR_INVALID_ARG;
  if (d != 64 && d != 128) return QCF_ERR_UNSUPPORTED;
  if (hq % hkv != 0) return QCF_ERR_INVALID_ARG;
  const int grp = hq / hkv;
  if ((grp & (grp - 1)) != 0 || grp > 32) return QCF_ERR_UNSUPPORTED;
  if (hq > 65535) return QCF_ERR_UNSUPPORTED;
  return QCF_OK;
}

inline qcf_status hip_status(hipError_t e) { return e == hipSuccess ? QCF_OK : QCF_ERR_HIP; }

// a K/V row stride: at least one row of heads, a whole number of 16-byte units
inline bool kv_stride_ok(int64_t stride, int hkv, int d, qcf_dtype t) {
  return stride >= (int64_t)hkv * d && (stride * esize(t)) % 16 == 0;
}

inline bool optional_index_ok(const void* p) { return !p || index_ok(p, false); }

// log2 of a page size, or -1 where it is not a power of two
inline int page_log2(int page_size) {
  if (page_size <= 0 || (page_size & (page_size - 1)) != 0) return -1;
  return __builtin_ctz((unsigned)page_size);
}

// what qcf_rope_store refuses
inline qcf_status check_rope_store(const void* k_cache, const void* v_cache, int64_t n_slots, int64_t cache_row_stride,
                                   const void* q_out, const void* k_new, const void* v_new, int64_t new_row_stride,
                                   const void* q_new, int64_t q_row_stride, int64_t n_src_rows,
                                   const int32_t* src_idx, qcf_dtype dtype, int64_t n_rows, const int32_t* slots,
                                   const int32_t* positions, const double* freq, int rotary_dim, float magnitude,
                                   int n_q_heads, int n_kv_heads, int head_dim) {
  if (!dtype_ok(dtype)) return QCF_ERR_UNSUPPORTED;
  const qcf_status st = check_heads(n_q_heads, n_kv_heads, head_dim);
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
  return QCF_OK;
}

}  // namespace
