// Rotary positions of new rows in the model's form, keys and values into their slots
// (qcf_rope_store).
//
// Bound: HBM.  Every element is read and written once; a row's angles are formed once and shared
// by all its query and key heads.  The unit of work is a pair of 16-byte vectors of one head: the two
// halves' partners, or, interleaved or not turned, two vectors side by side.
#include "qcf_decode_launch.h"
#include "qcf_device.h"

namespace qcf {
namespace {

constexpr int kThreads = 256;

template <typename T, int D, bool kInter>
__global__ __launch_bounds__(kThreads) void rope_store_kernel(RopeStore p) {
  constexpr int VEC = Vec16<T>::N;
  constexpr int UPH = D / (2 * VEC);  // units per head
  __shared__ float2 cs[D / 2];
  const int64_t r = blockIdx.x;
  const int64_t s = p.src_idx ? (int64_t)p.src_idx[r] : r;
  if (s < 0 || s >= p.n_src_rows) return;
  const int half = p.rotary_dim / 2;
  if (p.positions && (int)threadIdx.x < half)
    cs[threadIdx.x] = angle_cs<true, true>((double)p.positions[r] * p.freq[threadIdx.x], (double)p.magnitude);
  __syncthreads();
  const int64_t slot = p.k_cache ? p.slots[r] : -1;
  const bool store = slot >= 0 && slot < p.n_slots;
  const int nq = p.q_out ? p.hq : 0, nkv = store ? p.hkv : 0;
  for (int u = threadIdx.x; u < (nq + 2 * nkv) * UPH; u += kThreads) {
    const int h = u / UPH, c = u % UPH;
    const T* src;
    T* dst;
    bool turn = p.positions != nullptr && c * 2 * VEC < p.rotary_dim;
    if (h < nq) {
      src = static_cast<const T*>(p.q_new) + s * p.q_stride + h * D;
      dst = static_cast<T*>(p.q_out) + (r * p.hq + h) * D;
    } else if (h < nq + nkv) {
      src = static_cast<const T*>(p.k_new) + s * p.new_stride + (h - nq) * D;
      dst = static_cast<T*>(p.k_cache) + slot * p.cache_stride + (h - nq) * D;
    } else {
      src = static_cast<const T*>(p.v_new) + s * p.new_stride + (h - nq - nkv) * D;
      dst = static_cast<T*>(p.v_cache) + slot * p.cache_stride + (h - nq - nkv) * D;
      turn = false;
    }
    const int a = turn && !kInter ? c * VEC : c * 2 * VEC;
    const int b = turn && !kInter ? a + half : a + VEC;
    uint4 va = ld16(src + a), vb = ld16(src + b);
    if (turn) {
      float x[VEC], y[VEC], xo[VEC], yo[VEC];
      Vec16<T>::unpack(va, x);
      Vec16<T>::unpack(vb, y);
      if (kInter) {
#pragma unroll
        for (int e = 0; e < VEC; e += 2) {
          rope_pair(x[e], x[e + 1], cs[(a + e) / 2], xo[e], xo[e + 1]);
          rope_pair(y[e], y[e + 1], cs[(b + e) / 2], yo[e], yo[e + 1]);
        }
      } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) rope_pair(x[e], y[e], cs[a + e], xo[e], yo[e]);
      }
      va = Vec16<T>::pack(xo);
      vb = Vec16<T>::pack(yo);
    }
    st16(dst + a, va);
    st16(dst + b, vb);
  }
}

template <typename T, int D>
hipError_t launch_t(const RopeStore& p, bool interleaved, hipStream_t stream) {
  const dim3 grid((unsigned)p.n_rows);
  if (interleaved)
    rope_store_kernel<T, D, true><<<grid, kThreads, 0, stream>>>(p);
  else
    rope_store_kernel<T, D, false><<<grid, kThreads, 0, stream>>>(p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rope_store(const RopeStore& p, bool bf16, int head_dim, bool interleaved,
                             hipStream_t stream) {
  if (bf16)
    return head_dim == 64 ? launch_t<uint16_t, 64>(p, interleaved, stream)
                          : launch_t<uint16_t, 128>(p, interleaved, stream);
  return head_dim == 64 ? launch_t<float, 64>(p, interleaved, stream)
                        : launch_t<float, 128>(p, interleaved, stream);
}

}  // namespace qcf
