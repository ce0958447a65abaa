// Norms of new rows' queries and keys per head and their rotary positions in one pass, keys and values
// into their slots (qcf_norm_rope_store).
//
// norm(x) = x / sqrt(sum x^2 / d + eps) * w, then pairs of norm(x) turn.  Both halves of every pair and all of a
// head lie in the lanes of one wave: a unit of work is a pair of 16-byte vectors of one head (the two halves'
// partners, or, interleaved or not turned, two vectors side by side), a head's units are consecutive
// lanes, and its sum of squares takes log2(units) exchanges between them, so a row is read and written once.
// Bound: HBM for prompts, launch and dependent loads for single rows.
#include "qcf_device.h"
#include "qcf_turns_launch.h"

namespace qcf {
namespace {

constexpr int kThreads = 256;
constexpr int kAhead = 3;    // units of a thread that are asked for before the angles are formed
constexpr int kMaxRows = 8;  // rows of a block

// 2^rows_log2 rows per block, for rows of few units
template <typename T, int D, bool kInter>
__global__ __launch_bounds__(kThreads) void norm_rope_store_kernel(NormRopeStore p, int rows_log2) {
  constexpr int VEC = Vec16<T>::N;
  constexpr int UPH = D / (2 * VEC);  // units per head
  __shared__ float2 cs[kMaxRows * (D / 2)];
  const int64_t r0 = ((int64_t)blockIdx.y << kGridLog2 | blockIdx.x) << rows_log2;
  if (r0 >= p.n_rows) return;
  const int rows = (int)min((int64_t)1 << rows_log2, p.n_rows - r0);
  const int half = p.rotary_dim / 2;
  const int nq = p.q_out ? p.hq : 0, nkv = p.k_cache ? p.hkv : 0;
  const int per_row = (nq + 2 * nkv) * UPH, units = per_row * rows;
  struct Unit {
    uint4 a, b, wa, wb;
    T* dst;  // NULL: nothing is stored
    int ia, ib, cs0;
    bool norm, turn;
  };
  auto load = [&](int u) {
    Unit x;
    const int i = rows_log2 ? u / per_row : 0;
    const int v = u - i * per_row, h = v / UPH, c = v % UPH;
    const int64_t r = r0 + i;
    const int64_t from = p.src_idx ? (int64_t)p.src_idx[r] : r;
    const bool there = from >= 0 && from < p.n_src_rows;
    const int64_t s = there ? from : 0;
    const T *src, *w = nullptr;
    x.norm = true;
    if (h < nq) {
      src = static_cast<const T*>(p.q_new) + s * p.q_stride + h * D;
      x.dst = static_cast<T*>(p.q_out) + (r * p.hq + h) * D;
      if (p.q_weight) w = static_cast<const T*>(p.q_weight) + h * p.q_weight_stride;
    } else {
      const int64_t slot = p.slots[r];
      const bool is_k = h < nq + nkv;
      const int g = h - nq - (is_k ? 0 : nkv);
      src = static_cast<const T*>(is_k ? p.k_new : p.v_new) + s * p.new_stride + g * D;
      x.dst = slot >= 0 && slot < p.n_slots ? static_cast<T*>(is_k ? p.k_cache : p.v_cache) + slot * p.cache_stride + g * D
                                            : nullptr;
      if (is_k && p.k_weight) w = static_cast<const T*>(p.k_weight) + g * p.k_weight_stride;
      x.norm = is_k;
    }
    if (!there) x.dst = nullptr;
    x.turn = x.norm && p.positions != nullptr && c * 2 * VEC < p.rotary_dim;
    x.cs0 = i * (D / 2);
    x.ia = x.turn && !kInter ? c * VEC : c * 2 * VEC;
    x.ib = x.turn && !kInter ? x.ia + half : x.ia + VEC;
    x.a = ld16(src + x.ia);
    x.b = ld16(src + x.ib);
    if (w) {
      x.wa = ld16(w + x.ia);
      x.wb = ld16(w + x.ib);
    } else {
      float one[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) one[e] = 1.f;
      x.wa = x.wb = Vec16<T>::pack(one);
    }
    return x;
  };
  // (all of a head's lanes come here together)
  auto finish = [&](const Unit& u) {
    uint4 va = u.a, vb = u.b;
    float x[VEC], y[VEC];
    Vec16<T>::unpack(va, x);
    Vec16<T>::unpack(vb, y);
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < VEC; ++e) sum = fmaf(x[e], x[e], fmaf(y[e], y[e], sum));
#pragma unroll
    for (int o = UPH / 2; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
    if (u.norm) {
      const float scale = 1.f / sqrtf(sum * (1.f / D) + p.eps);
      float wx[VEC], wy[VEC];
      Vec16<T>::unpack(u.wa, wx);
      Vec16<T>::unpack(u.wb, wy);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        x[e] = x[e] * scale * wx[e];
        y[e] = y[e] * scale * wy[e];
      }
      if (u.turn) {
        float xo[VEC], yo[VEC];
        const float2* c = cs + u.cs0;
        if (kInter) {
#pragma unroll
          for (int e = 0; e < VEC; e += 2) {
            rope_pair(x[e], x[e + 1], c[(u.ia + e) / 2], xo[e], xo[e + 1]);
            rope_pair(y[e], y[e + 1], c[(u.ib + e) / 2], yo[e], yo[e + 1]);
          }
        } else {
#pragma unroll
          for (int e = 0; e < VEC; ++e) rope_pair(x[e], y[e], c[u.ia + e], xo[e], yo[e]);
        }
        va = Vec16<T>::pack(xo);
        vb = Vec16<T>::pack(yo);
      } else {
        va = Vec16<T>::pack(x);
        vb = Vec16<T>::pack(y);
      }
    }
    if (u.dst) {
      st16(u.dst + u.ia, va);
      st16(u.dst + u.ib, vb);
    }
  };
  Unit x[kAhead];
#pragma unroll
  for (int k = 0; k < kAhead; ++k)
    if (k * kThreads < units) x[k] = load(min((int)threadIdx.x + k * kThreads, units - 1));
  if (p.positions)
    for (int t = threadIdx.x; t < rows * half; t += kThreads) {
      const int i = rows_log2 ? t / half : 0, j = t - i * half;
      cs[i * (D / 2) + j] = angle_cs<true, true>((double)p.positions[r0 + i] * p.freq[j], (double)p.magnitude);
    }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kAhead; ++k)
    if ((int)threadIdx.x + k * kThreads < units) finish(x[k]);
  for (int u = threadIdx.x + kAhead * kThreads; u < units; u += kThreads) finish(load(u));
}

template <typename T, int D>
hipError_t launch_t(const NormRopeStore& p, bool interleaved, hipStream_t stream) {
  const int units = ((p.q_out ? p.hq : 0) + (p.k_cache ? 2 * p.hkv : 0)) * (D / (2 * Vec16<T>::N));
  int lg = 0;
  while ((2 << lg) <= kMaxRows && ((int64_t)units << (lg + 1)) <= kThreads && (p.n_rows >> lg) > 512) ++lg;
  const dim3 grid = grid_of(((p.n_rows - 1) >> lg) + 1);
  if (interleaved)
    norm_rope_store_kernel<T, D, true><<<grid, kThreads, 0, stream>>>(p, lg);
  else
    norm_rope_store_kernel<T, D, false><<<grid, kThreads, 0, stream>>>(p, lg);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_norm_rope_store(const NormRopeStore& p, bool bf16, int head_dim, bool interleaved,
                                  hipStream_t stream) {
  if (bf16)
    return head_dim == 64 ? launch_t<uint16_t, 64>(p, interleaved, stream)
                          : launch_t<uint16_t, 128>(p, interleaved, stream);
  return head_dim == 64 ? launch_t<float, 64>(p, interleaved, stream)
                        : launch_t<float, 128>(p, interleaved, stream);
}

}  // namespace qcf
