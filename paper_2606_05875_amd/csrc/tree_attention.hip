// Attention of each request's new rows over its paged cache (qcf_tree_attn).
//
// One wave per row and query head, 64 tokens at a time: a lane holds one token's logit, then the
// weights go round the wave and a lane sums its output columns.  The softmax is online (running
// maximum and sum).
#include <math.h>

#include "qcf_decode_launch.h"
#include "qcf_device.h"

namespace qcf {
namespace {

constexpr int kWaves = 4;

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(uint16_t x) { return bf2f(x); }
__device__ __forceinline__ void store_as(float* p, float x) { *p = x; }
__device__ __forceinline__ void store_as(uint16_t* p, float x) { *p = f2bf(x); }

template <typename T, int D>
__global__ __launch_bounds__(kWaves * 64) void tree_attn_kernel(TreeAttn p) {
  constexpr int VEC = Vec16<T>::N, NC = D / 64;
  const int l = threadIdx.x & 63;
  const int h = blockIdx.y * kWaves + (threadIdx.x >> 6);
  const int b = blockIdx.x / p.max_q, i = blockIdx.x % p.max_q;
  if (h >= p.hq) return;
  const int64_t r0 = p.cu_q[b], nr = min((int64_t)p.cu_q[b + 1], p.n_rows) - r0;
  if (r0 < 0 || i >= nr) return;
  const int64_t r = r0 + i;
  const int64_t kv = max(p.kv_len[b], 0);
  const int64_t end = min(kv + nr, (int64_t)p.max_kv);
  const int g = h / (p.hq / p.hkv);
  const T* q = static_cast<const T*>(p.q) + (r * p.hq + h) * D;
  float m = -INFINITY, sum = 0.f, o[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) o[c] = 0.f;
  for (int64_t t0 = 0; t0 < end; t0 += 64) {
    const int64_t t = t0 + l, pg = t >> p.page_log2;
    bool see = t < end && pg < p.max_pages;
    if (see && t >= kv) {
      const int j = (int)(t - kv);
      see = p.tree_mask ? j < 32 * p.mask_words && (p.tree_mask[r * p.mask_words + (j >> 5)] >> (j & 31) & 1)
                        : j <= i;
    }
    int64_t slot = 0;
    if (see) {
      const int64_t page = p.block_table[b * p.table_stride + pg];
      see = page >= 0 && page < p.n_pages;
      slot = (page << p.page_log2) + (t & ((1ll << p.page_log2) - 1));
    }
    float x = -INFINITY;
    if (see) {
      const T* k = static_cast<const T*>(p.k_cache) + slot * p.kv_stride + g * D;
      float dot = 0.f;
      for (int c = 0; c < D; c += VEC) {
        float a[VEC], y[VEC];
        Vec16<T>::unpack(ld16(q + c), a);
        Vec16<T>::unpack(ld16(k + c), y);
#pragma unroll
        for (int e = 0; e < VEC; ++e) dot = fmaf(a[e], y[e], dot);
      }
      x = dot * p.scale;
    }
    const float mn = fmaxf(m, wave_max(x));
    const float ref = mn == -INFINITY ? 0.f : mn;
    const float w = see ? expf(x - ref) : 0.f, alpha = expf(m - ref);
    sum = sum * alpha + wave_sum(w);
    m = mn;
#pragma unroll
    for (int c = 0; c < NC; ++c) o[c] *= alpha;
    uint64_t vis = __ballot(see);
    while (vis) {
      const int k = __builtin_ctzll(vis);
      vis &= vis - 1;
      const float wk = __shfl(w, k, 64);
      const int64_t sk = __shfl(slot, k, 64);
      const T* v = static_cast<const T*>(p.v_cache) + sk * p.kv_stride + g * D;
#pragma unroll
      for (int c = 0; c < NC; ++c) o[c] = fmaf(wk, to_f(v[c * 64 + l]), o[c]);
    }
  }
  T* out = static_cast<T*>(p.out) + (r * p.hq + h) * D;
#pragma unroll
  for (int c = 0; c < NC; ++c) store_as(out + c * 64 + l, m == -INFINITY ? 0.f : o[c] / sum);
  if (p.lse && l == 0) p.lse[r * p.hq + h] = m == -INFINITY ? -INFINITY : m + logf(sum);
}

}  // namespace

size_t tree_attn_workspace(int, int, int, int, int, int, bool) { return 0; }

hipError_t launch_tree_attn(const TreeAttn& p, bool bf16, int head_dim, void*, hipStream_t stream) {
  const int64_t blocks = (int64_t)p.batch * p.max_q;
  if (blocks > 0x7fffffff) return hipErrorInvalidConfiguration;
  const dim3 grid((unsigned)blocks, (unsigned)((p.hq + kWaves - 1) / kWaves));
  if (bf16) {
    if (head_dim == 64) tree_attn_kernel<uint16_t, 64><<<grid, kWaves * 64, 0, stream>>>(p);
    else tree_attn_kernel<uint16_t, 128><<<grid, kWaves * 64, 0, stream>>>(p);
  } else {
    if (head_dim == 64) tree_attn_kernel<float, 64><<<grid, kWaves * 64, 0, stream>>>(p);
    else tree_attn_kernel<float, 128><<<grid, kWaves * 64, 0, stream>>>(p);
  }
  return hipGetLastError();
}

}  // namespace qcf
