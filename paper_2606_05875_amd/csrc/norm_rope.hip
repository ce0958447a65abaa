// Norms of new rows' queries and keys per head and their rotary positions in one pass, keys and values
// into their slots (qcf_norm_rope_store).
//
// norm(x) = x / sqrt(sum x^2 / d + eps) * w, then pairs of norm(x) turn.  Both halves of every pair and all of a
// head lie in the lanes of one wave: a unit of work is a pair of 16-byte vectors of one head (the two halves'
// partners, or, interleaved or not turned, two vectors side by side), a head's units are consecutive
// lanes, and its sum of squares takes log2(units) exchanges between them, so a row is read and written once.
// Bound: HBM for prompts (32896 rows of 64/8 heads of 128 in bf16 241 us, 5.6 TB/s), launch and dependent loads for
// single rows (48 rows of 32/8 heads 4.7 us).
#include "qcf_device.h"
#include "qcf_turns_launch.h"

namespace qcf {
namespace {

constexpr int kThreads = 256;
constexpr int kAhead = 3;    // units of a thread that are asked for before the angles are formed
constexpr int kMaxRows = 8;  // rows of a block

// 2^rows_log2 rows per block (kMulti: more than one, for rows of few units that would be more than 512 blocks: 2500 rows of
// 8/2 heads of 64 5.1 us against 7.2 with a block each, 32896 rows 29 against 65, 1000 rows 4.4 against 4.6)
template <typename T, int D, bool kInter, bool kMulti>
__global__ __launch_bounds__(kThreads, 4) void norm_rope_store_kernel(NormRopeStore p, int rows_log2) {
  constexpr int VEC = Vec16<T>::N;
  constexpr int UPH = D / (2 * VEC);  // units per head
  static_assert(kThreads % UPH == 0, "a thread's units are the same part of their heads");
  __shared__ float2 cs[(kMulti ? kMaxRows : 1) * (D / 2)];
  const int64_t block = (int64_t)blockIdx.y << kGridLog2 | blockIdx.x;
  const int64_t r0 = kMulti ? block << rows_log2 : block;
  if (r0 >= p.n_rows) return;
  const int rows = kMulti ? (int)min((int64_t)1 << rows_log2, p.n_rows - r0) : 1;
  const int half = p.rotary_dim / 2;
  const int nq = p.q_out ? p.hq : 0, nkv = p.k_cache ? p.hkv : 0;
  const int per_row = (nq + 2 * nkv) * UPH, units = per_row * rows;
  // this thread's part of every head: 16-byte vectors at ia and ib (values: va and vb)
  const int c = threadIdx.x % UPH;
  const bool turned = p.positions != nullptr && c * 2 * VEC < p.rotary_dim;
  const int va = c * 2 * VEC, vb = va + VEC;
  const int ia = turned && !kInter ? c * VEC : va, ib = turned && !kInter ? ia + half : vb;
  auto row_of = [&](int u) { return kMulti ? u / per_row : 0; };
  auto head_of = [&](int u, int i) { return (u - i * per_row) / UPH; };
  struct Unit {
    uint4 a, b;
  };
  auto load = [&](int u) {
    const int i = row_of(u), h = head_of(u, i);
    const int64_t from = p.src_idx ? (int64_t)p.src_idx[r0 + i] : r0 + i;
    const int64_t s = from >= 0 && from < p.n_src_rows ? from : 0;
    const T* src = h < nq         ? static_cast<const T*>(p.q_new) + s * p.q_stride + h * D
                   : h < nq + nkv ? static_cast<const T*>(p.k_new) + s * p.new_stride + (h - nq) * D
                                  : static_cast<const T*>(p.v_new) + s * p.new_stride + (h - nq - nkv) * D;
    const bool v = h >= nq + nkv;
    return Unit{ld16(src + (v ? va : ia)), ld16(src + (v ? vb : ib))};
  };
  // weights that all heads share are read once
  struct Weight {
    uint4 a, b;
  };
  auto weight = [&](const void* w, int64_t stride, int h) {
    if (w) {
      const T* x = static_cast<const T*>(w) + h * stride;
      return Weight{ld16(x + ia), ld16(x + ib)};
    }
    float one[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) one[e] = 1.f;
    return Weight{Vec16<T>::pack(one), Vec16<T>::pack(one)};
  };
  // (all of a head's lanes come here together)
  auto finish = [&](int u, const Unit& unit, const Weight& qw, const Weight& kw) {
    const int i = row_of(u), h = head_of(u, i);
    const int64_t r = r0 + i;
    const bool is_q = h < nq, is_v = h >= nq + nkv;
    float x[VEC], y[VEC];
    Vec16<T>::unpack(unit.a, x);
    Vec16<T>::unpack(unit.b, y);
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < VEC; ++e) sum = fmaf(x[e], x[e], fmaf(y[e], y[e], sum));
#pragma unroll
    for (int o = UPH / 2; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
    Unit out = unit;
    if (!is_v) {
      const float scale = 1.f / sqrtf(sum * (1.f / D) + p.eps);
      Weight w = is_q ? qw : kw;
      if (is_q && p.q_weight_stride) w = weight(p.q_weight, p.q_weight_stride, h);
      if (!is_q && p.k_weight_stride) w = weight(p.k_weight, p.k_weight_stride, h - nq);
      float wx[VEC], wy[VEC];
      Vec16<T>::unpack(w.a, wx);
      Vec16<T>::unpack(w.b, wy);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        x[e] = x[e] * scale * wx[e];
        y[e] = y[e] * scale * wy[e];
      }
      if (turned) {
        float xo[VEC], yo[VEC];
        const float2* t = cs + i * (D / 2);
        if (kInter) {
#pragma unroll
          for (int e = 0; e < VEC; e += 2) {
            rope_pair(x[e], x[e + 1], t[(ia + e) / 2], xo[e], xo[e + 1]);
            rope_pair(y[e], y[e + 1], t[(ib + e) / 2], yo[e], yo[e + 1]);
          }
        } else {
#pragma unroll
          for (int e = 0; e < VEC; ++e) rope_pair(x[e], y[e], t[ia + e], xo[e], yo[e]);
        }
        out = Unit{Vec16<T>::pack(xo), Vec16<T>::pack(yo)};
      } else {
        out = Unit{Vec16<T>::pack(x), Vec16<T>::pack(y)};
      }
    }
    const int64_t from = p.src_idx ? (int64_t)p.src_idx[r] : r;
    T* dst = nullptr;
    if (is_q) {
      dst = static_cast<T*>(p.q_out) + (r * p.hq + h) * D;
    } else {
      const int64_t slot = p.slots[r];
      if (slot >= 0 && slot < p.n_slots)
        dst = static_cast<T*>(is_v ? p.v_cache : p.k_cache) + slot * p.cache_stride + (is_v ? h - nq - nkv : h - nq) * D;
    }
    if (dst && from >= 0 && from < p.n_src_rows) {
      st16(dst + (is_v ? va : ia), out.a);
      st16(dst + (is_v ? vb : ib), out.b);
    }
  };
  Unit x[kAhead];
#pragma unroll
  for (int k = 0; k < kAhead; ++k)
    if (k * kThreads < units) x[k] = load(min((int)threadIdx.x + k * kThreads, units - UPH + c));
  if (p.positions)
    for (int t = threadIdx.x; t < rows * half; t += kThreads) {
      const int i = kMulti ? t / half : 0, j = t - i * half;
      cs[i * (D / 2) + j] = angle_cs<true, true>((double)p.positions[r0 + i] * p.freq[j], (double)p.magnitude);
    }
  const Weight qw = weight(p.q_weight_stride ? nullptr : p.q_weight, 0, 0);
  const Weight kw = weight(p.k_weight_stride ? nullptr : p.k_weight, 0, 0);
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kAhead; ++k)
    if ((int)threadIdx.x + k * kThreads < units) finish(threadIdx.x + k * kThreads, x[k], qw, kw);
  for (int u = threadIdx.x + kAhead * kThreads; u < units; u += kThreads) finish(u, load(u), qw, kw);
}

template <typename T, int D>
hipError_t launch_t(const NormRopeStore& p, bool interleaved, hipStream_t stream) {
  const int units = ((p.q_out ? p.hq : 0) + (p.k_cache ? 2 * p.hkv : 0)) * (D / (2 * Vec16<T>::N));
  int lg = 0;
  while ((2 << lg) <= kMaxRows && ((int64_t)units << (lg + 1)) <= kThreads && (p.n_rows >> lg) > 512) ++lg;
  const dim3 grid = grid_of(((p.n_rows - 1) >> lg) + 1);
  if (lg > 0) {
    if (interleaved) norm_rope_store_kernel<T, D, true, true><<<grid, kThreads, 0, stream>>>(p, lg);
    else norm_rope_store_kernel<T, D, false, true><<<grid, kThreads, 0, stream>>>(p, lg);
  } else {
    if (interleaved) norm_rope_store_kernel<T, D, true, false><<<grid, kThreads, 0, stream>>>(p, lg);
    else norm_rope_store_kernel<T, D, false, false><<<grid, kThreads, 0, stream>>>(p, lg);
  }
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
