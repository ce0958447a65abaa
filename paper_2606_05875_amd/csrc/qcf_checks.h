// Argument checks shared by the C entry points.  They touch no device state, so a rejected call
// works on a machine without a GPU.
#pragma once
#include <hip/hip_runtime_api.h>
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

}  // namespace
