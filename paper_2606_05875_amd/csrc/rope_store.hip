// Rotary positions of new rows in the model's form, keys and values into their slots
// (qcf_rope_store).
//
// Bound: HBM.  Every element is read and written once; a row's angles are formed once and shared
// by all its query and key heads.  The unit of work is a pair of 16-byte vectors of one head: the two
// halves' partners, or, interleaved or not turned, two vectors side by side.  32896 rows of 64/8 heads of
// 128, bfloat16: 243 us, 5.5 TB/s; 2500 float32 rows of 16/4 heads of 64: 7.8 us, 3.9 TB/s; 48 rows: 4.6 us.
#include "qcf_decode_launch.h"
#include "qcf_device.h"

namespace qcf {
namespace {

constexpr int kThreads = 256;

// One row per block.  The first kAhead units of every thread are asked for, unmasked from clamped units (a
// load under a lane condition waits by itself), before the row's angles are formed (2500 float32 rows 8.5 -> 8.0 us).
constexpr int kAhead = 3;

template <typename T, int D, bool kInter>
__global__ __launch_bounds__(kThreads) void rope_store_kernel(RopeStore p) {
  constexpr int VEC = Vec16<T>::N;
  constexpr int UPH = D / (2 * VEC);  // units per head
  __shared__ float2 cs[D / 2];
  const int64_t r = (int64_t)blockIdx.y << kGridLog2 | blockIdx.x;
  if (r >= p.n_rows) return;
  const int64_t s = p.src_idx ? (int64_t)p.src_idx[r] : r;
  if (s < 0 || s >= p.n_src_rows) return;
  const int half = p.rotary_dim / 2;
  const int64_t slot = p.k_cache ? p.slots[r] : -1;
  const bool store = slot >= 0 && slot < p.n_slots;
  const int nq = p.q_out ? p.hq : 0, nkv = store ? p.hkv : 0;
  const int units = (nq + 2 * nkv) * UPH;
  if (units == 0) return;
  struct Unit {
    uint4 a, b;
    T* dst;
    int ia, ib;
    bool turn;
  };
  auto load = [&](int u) {
    Unit x;
    const int h = u / UPH, c = u % UPH;
    const T* src;
    x.turn = p.positions != nullptr && c * 2 * VEC < p.rotary_dim;
    if (h < nq) {
      src = static_cast<const T*>(p.q_new) + s * p.q_stride + h * D;
      x.dst = static_cast<T*>(p.q_out) + (r * p.hq + h) * D;
    } else if (h < nq + nkv) {
      src = static_cast<const T*>(p.k_new) + s * p.new_stride + (h - nq) * D;
      x.dst = static_cast<T*>(p.k_cache) + slot * p.cache_stride + (h - nq) * D;
    } else {
      src = static_cast<const T*>(p.v_new) + s * p.new_stride + (h - nq - nkv) * D;
      x.dst = static_cast<T*>(p.v_cache) + slot * p.cache_stride + (h - nq - nkv) * D;
      x.turn = false;
    }
    x.ia = x.turn && !kInter ? c * VEC : c * 2 * VEC;
    x.ib = x.turn && !kInter ? x.ia + half : x.ia + VEC;
    x.a = ld16(src + x.ia);
    x.b = ld16(src + x.ib);
    return x;
  };
  auto finish = [&](const Unit& u) {
    uint4 va = u.a, vb = u.b;
    if (u.turn) {
      float x[VEC], y[VEC], xo[VEC], yo[VEC];
      Vec16<T>::unpack(va, x);
      Vec16<T>::unpack(vb, y);
      if (kInter) {
#pragma unroll
        for (int e = 0; e < VEC; e += 2) {
          rope_pair(x[e], x[e + 1], cs[(u.ia + e) / 2], xo[e], xo[e + 1]);
          rope_pair(y[e], y[e + 1], cs[(u.ib + e) / 2], yo[e], yo[e + 1]);
        }
      } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) rope_pair(x[e], y[e], cs[u.ia + e], xo[e], yo[e]);
      }
      va = Vec16<T>::pack(xo);
      vb = Vec16<T>::pack(yo);
    }
    st16(u.dst + u.ia, va);
    st16(u.dst + u.ib, vb);
  };
  Unit x[kAhead];
#pragma unroll
  for (int k = 0; k < kAhead; ++k)
    if (k * kThreads < units) x[k] = load(min((int)threadIdx.x + k * kThreads, units - 1));
  if (p.positions && (int)threadIdx.x < half)
    cs[threadIdx.x] = angle_cs<true, true>((double)p.positions[r] * p.freq[threadIdx.x], (double)p.magnitude);
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kAhead; ++k)
    if ((int)threadIdx.x + k * kThreads < units) finish(x[k]);
  for (int u = threadIdx.x + kAhead * kThreads; u < units; u += kThreads) finish(load(u));
}

template <typename T, int D>
hipError_t launch_t(const RopeStore& p, bool interleaved, hipStream_t stream) {
  const dim3 grid = grid_of(p.n_rows);
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
