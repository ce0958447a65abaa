// Device code shared by the bf16 attention kernels over pages: copies from pages into LDS, and what logits
// and values of any size need.
#pragma once
#include "qcf_attn.h"
#include "qcf_tree.h"

namespace qcf {
namespace {

typedef short v4s __attribute__((ext_vector_type(4)));
typedef v4s __attribute__((address_space(3))) * lds_v4s;

// 16 bytes per lane from base + off into LDS at byte address lds + 16 * lane, past the registers and
// without a wait of the compiler's (the caller counts).  A load that takes its LDS address from m0 needs a wait
// state behind the write of m0, which the compiler does not add inside an asm block.
__device__ __forceinline__ void copy16(const void* base, uint32_t off, uint32_t lds) {
  const uint32_t la = __builtin_amdgcn_readfirstlane(lds);
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               :
               : "s"(la), "v"(off), "s"(uni((int64_t)base))
               : "memory");
}
__device__ __forceinline__ void copy16(const void* from, uint32_t lds) {
  const uint32_t la = __builtin_amdgcn_readfirstlane(lds);
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" : : "s"(la), "v"(from) : "memory");
}

// Weights are exp2(s * scale2 - ref) with a fused multiply-add, which keeps the product exact; its
// difference to the rounded maximum reaches 2^-24 of that, too much to be an exponent where maxima
// pass 2^28.  Such a vector's logits are scaled (and rounded) first; each lane's by its own vector's
// maximum, so that the other vectors' bits do not hang on it.
__device__ __forceinline__ bool is_big(float m) { return fabsf(finite(m)) > 0x1p28f; }

// any of a 16-byte piece's 8 values infinite or NaN
__device__ __forceinline__ bool not_finite(const uint4& x) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    bad = bad || (w[i] & 0x7f80u) == 0x7f80u || (w[i] & 0x7f800000u) == 0x7f800000u;
  return bad;
}

}  // namespace
}  // namespace qcf
