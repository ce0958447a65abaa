// Attention of each request's new rows over its paged cache (qcf_tree_attn), float32, on the float32
// matrix instruction v_mfma_f32_16x16x4_f32.
//
// A block holds 16 query vectors of one request and KV head; its four waves take the 16-token tiles in
// turn, each with its own online softmax, and are summed through LDS once per unit.  A lane's fragment is
// 16 contiguous bytes of a row, and no two waves read the same token, so K and V go from the pages to
// registers: K of the next tile is asked for before this tile's softmax, V after its products.
//  * S^T = K Q^T: a lane holds 4 tokens' logits of one vector (register r of lane l: token 4 (l / 16) + r,
//    vector l % 16).  Product (sb, e) takes the d-columns 16 sb + 4 (l / 16) + e of both operands, so both
//    are float4 loads; four accumulators, summed pairwise.
//  * O^T += V^T P^T with P^T straight from those registers: product (r, mb) contracts over the tokens
//    4 (l / 16) + r and fills the d-columns NB (l % 16) + mb, so a lane's V operands are NB contiguous floats.
//  * exp2f, not the bare instruction: weights below 2^-126 stay subnormal numbers.
// Bound: latency at test sizes (3 requests of up to 700 tokens, 8/2 heads of 64: 13.9 us, 4 of them the merge),
// HBM or the float32 matrix rate beyond (each K and V row is read once per 16 vectors; 3 trees over 20000
// tokens, 32/8 heads of 128: 105 us, 4.7 TB/s).
#include "qcf_tree.h"

namespace qcf {
namespace {

constexpr int kW = 4;    // waves
constexpr int kT = 16;   // tokens per wave and step
constexpr int kVt = 16;  // query vectors per block
static_assert(kW * kT == kTreeStep, "a block's waves take a step's tokens");

template <int D, bool kTiny>
__global__ __launch_bounds__(kW * 64, 2) void tree_attn_f32_kernel(TreeAttn p, TreeCut cut, TreeWs ws, int lg) {
  constexpr int SB = D / 16, NB = D / 16;
  __shared__ float4 o_l[kW * kVt * (D / 4)];
  __shared__ float2 ml_l[kW][kVt];
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l = threadIdx.x & 63, li = l & 15, lk = l >> 4;
  const float scale2 = p.scale * kLog2e;

  tree_walk<kW * 64>(p, cut, ws, lg, [&](int b, const TreeRequest& rq, int g, int tile, int first, int n,
                                         int steps, int slot) {
    const_i32 table = (const_i32)(p.block_table + b * p.table_stride);
    const float* kc = static_cast<const float*>(p.k_cache) + (int64_t)g * D;
    const float* vc = static_cast<const float*>(p.v_cache) + (int64_t)g * D;
    constexpr int kHop = kW * kT;
    const int t_first = (first * kW + w) * kT;
    const int vec = tile * kVt + li, idx = vec >> lg;
    const int head = (g << lg) + (vec & ((1 << lg) - 1));
    const int64_t row = rq.r0 + min(idx, rq.rows - 1);
    float4 qf[SB];
#pragma unroll
    for (int sb = 0; sb < SB; ++sb)
      qf[sb] = *reinterpret_cast<const float4*>(static_cast<const float*>(p.q) + (row * p.hq + head) * D + 16 * sb + 4 * lk);

    const bool pool = p.n_pages > 0;
    auto page_at = [&](int i) { return kTiny || i >= n ? -1 : page_of(p, table, t_first + i * kHop, rq.end); };
    // the row of token t0 + r of a tile; without one the pool's first row stands in and is not seen
    auto place = [&](int t0, int page, int r) {
      if (kTiny) return max(slot_of(p, b, t0 + r, rq.end), (int64_t)0) * p.kv_stride;
      return (page < 0 ? 0 : ((int64_t)page << p.page_log2) + (t0 & ((1 << p.page_log2) - 1)) + r) * p.kv_stride;
    };
    float4 kf[SB], vf[4][NB / 4];
    auto load_k = [&](int t0, int page) {
      const float* x = kc + place(t0, page, li) + 4 * lk;
#pragma unroll
      for (int sb = 0; sb < SB; ++sb) kf[sb] = *reinterpret_cast<const float4*>(x + 16 * sb);
    };
    auto load_v = [&](int t0, int page) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float* x = vc + place(t0, page, 4 * lk + r) + NB * li;
#pragma unroll
        for (int c = 0; c < NB / 4; ++c) vf[r][c] = *reinterpret_cast<const float4*>(x + 4 * c);
      }
    };
    f32x4 o[NB];
#pragma unroll
    for (int mb = 0; mb < NB; ++mb) o[mb] = f32x4{};
    float m = -INFINITY, ls = 0.f;  // running maximum in log2 units, this lane's part of the sum
    int page = page_at(0), page1 = page_at(1);
    if (pool && n > 0) {
      load_k(t_first, page);
      load_v(t_first, page);
    }
    // Q has to be there before the loop (a wait for it inside would count the next tile's loads)
#pragma unroll
    for (int sb = 0; sb < SB; ++sb)
      asm volatile("" : "+v"(qf[sb].x), "+v"(qf[sb].y), "+v"(qf[sb].z), "+v"(qf[sb].w));
    for (int i = 0; i < n && pool; ++i) {
      const int t0 = t_first + i * kHop;
      f32x4 s[4] = {};
#pragma unroll
      for (int sb = 0; sb < SB; sb += 4) {
#pragma unroll
        for (int c = 0; c < 4; ++c) s[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[sb + c].x, qf[sb + c].x, s[c], 0, 0, 0);
#pragma unroll
        for (int c = 0; c < 4; ++c) s[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[sb + c].y, qf[sb + c].y, s[c], 0, 0, 0);
#pragma unroll
        for (int c = 0; c < 4; ++c) s[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[sb + c].z, qf[sb + c].z, s[c], 0, 0, 0);
#pragma unroll
        for (int c = 0; c < 4; ++c) s[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[sb + c].w, qf[sb + c].w, s[c], 0, 0, 0);
      }
      const f32x4 dot = (s[0] + s[1]) + (s[2] + s[3]);
      if (i + 1 < n) load_k(t0 + kHop, page1);
      const int page2 = page_at(i + 2);
      // which of the tile's tokens there are, and which of them this lane's vector sees
      uint32_t held = 0xffffu, sees = 0xffffu;
      bool edge = t0 + kT > min(rq.kv, rq.end) || (!kTiny && page < 0);
      if (kTiny) {
        held = (uint32_t)__ballot(slot_of(p, b, t0 + li, rq.end) >= 0) & 0xffffu;
        edge = edge || held != 0xffffu;
      }
      uint32_t loose = 0;  // tokens whose values are added one by one
      if (edge) {
        if (t0 >= rq.end || (!kTiny && page < 0)) held = 0;
        else if (rq.end - t0 < kT) held &= (1u << (rq.end - t0)) - 1u;
        sees = held ? tree_sees<16>(p, rq, row, idx, t0) & held : 0u;
        // a value that a row does not see must not meet its weight 0 where it is not finite: rows that
        // hold no token become zeros, and tokens with such values (rare) are taken out and added to the
        // rows that see them
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const bool there = held >> (4 * lk + r) & 1;
          bool odd = false;
#pragma unroll
          for (int c = 0; c < NB / 4; ++c) {
            const float4 v = vf[r][c];
            odd = odd || !(isfinite(v.x) && isfinite(v.y) && isfinite(v.z) && isfinite(v.w));
          }
          const uint64_t at = __ballot(there && odd);
#pragma unroll
          for (int k = 0; k < 4; ++k) loose |= at >> (16 * k) & 0xffffull ? 1u << (4 * k + r) : 0u;
          const bool keep = there && !(loose >> (4 * lk + r) & 1);
#pragma unroll
          for (int c = 0; c < NB / 4; ++c)
            if (!keep) vf[r][c] = make_float4(0.f, 0.f, 0.f, 0.f);
        }
      }
      float x[4], mt = -INFINITY;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        x[r] = sees >> (4 * lk + r) & 1 ? dot[r] * scale2 : -INFINITY;
        mt = fmaxf(mt, x[r]);
      }
      // lazy rescale: a stale maximum stays unless the vector's grew by more than 2^8 (by each vector's
      // own, so that no row's bits hang on another's)
      if (__ballot(!(mt < m + 8.f))) {  // (no maximum yet: row_scale)
        mt = fmaxf(mt, __shfl_xor(mt, 16, 64));
        mt = fmaxf(mt, __shfl_xor(mt, 32, 64));
        const float mn = mt > m + 8.f ? mt : m;
        const float alpha = exp2f(gap(m, mn));
        ls = fmaf(ls, alpha, mn == -INFINITY && sees ? 1.f : 0.f);
#pragma unroll
        for (int mb = 0; mb < NB; ++mb) o[mb] *= alpha;
        m = mn;
      }
      float pr[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) pr[r] = exp2f(x[r] - finite(m));
      ls += (pr[0] + pr[1]) + (pr[2] + pr[3]);
      for (uint32_t left = loose; left; left &= left - 1) {
        const int k = __builtin_ctz(left);
        float a = 0.f;
#pragma unroll
        for (int r = 0; r < 4; ++r) a = (k & 3) == r ? pr[r] : a;
        const float pk = __shfl(a, (k >> 2) * 16 + li, 64);
        const float* vr = vc + place(t0, page, k);
        if (sees >> k & 1) {
#pragma unroll
          for (int mb = 0; mb < NB; ++mb)
#pragma unroll
            for (int r = 0; r < 4; ++r) o[mb][r] = fmaf(vr[NB * (4 * lk + r) + mb], pk, o[mb][r]);
        }
      }
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int mb = 0; mb < NB; ++mb) {
          const float4 c = vf[r][mb / 4];
          const float ve = mb % 4 == 0 ? c.x : mb % 4 == 1 ? c.y : mb % 4 == 2 ? c.z : c.w;
          o[mb] = __builtin_amdgcn_mfma_f32_16x16x4f32(ve, pr[r], o[mb], 0, 0, 0);
        }
      if (i + 1 < n) load_v(t0 + kHop, page1);
      page = page1;
      page1 = page2;
    }

    // the waves' results, summed in their order.  A lane's columns are NB (4 lk + r) + mb; vector v's
    // columns 4 i .. + 3 sit at i ^ (v % 8).
    ls += __shfl_xor(ls, 16, 64);
    ls += __shfl_xor(ls, 32, 64);
    if (lk == 0) ml_l[w][li] = make_float2(m, ls);
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int c = 0; c < NB / 4; ++c)
        o_l[(w * kVt + li) * (D / 4) + (((4 * lk + r) * (NB / 4) + c) ^ (li & 7))] =
            make_float4(o[4 * c][r], o[4 * c + 1][r], o[4 * c + 2][r], o[4 * c + 3][r]);
    __syncthreads();
    for (int u = threadIdx.x; u < kVt * (D / 4); u += kW * 64) {
      const int v = u / (D / 4), i4 = u % (D / 4);
      const int mine = tile * kVt + v, i = mine >> lg;
      if (i >= rq.rows) continue;
      float2 ml[kW];
      float mx = -INFINITY, lt = 0.f;
#pragma unroll
      for (int k = 0; k < kW; ++k) {
        ml[k] = ml_l[k][v];
        mx = fmaxf(mx, ml[k].x);
      }
      float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k = 0; k < kW; ++k) {
        const float f = exp2f(gap(ml[k].x, mx));
        const float4 y = o_l[(k * kVt + v) * (D / 4) + (i4 ^ (v & 7))];
        lt += f * ml[k].y;
        a.x += f * y.x;
        a.y += f * y.y;
        a.z += f * y.z;
        a.w += f * y.w;
      }
      if (slot >= 0) {
        reinterpret_cast<float4*>(ws.o)[((int64_t)slot * kVt + v) * (D / 4) + i4] = a;
        if (i4 == 0) ws.ml[(int64_t)slot * kVt + v] = make_float2(mx, lt);
      } else {
        const int64_t at = (rq.r0 + i) * p.hq + (g << lg) + (mine & ((1 << lg) - 1));
        const float inv = row_scale(mx, lt);
        store4(static_cast<float*>(p.out) + at * D + 4 * i4, make_float4(a.x * inv, a.y * inv, a.z * inv, a.w * inv));
        if (p.lse && i4 == 0) p.lse[at] = row_lse(mx, lt);
      }
    }
    __syncthreads();  // (the next unit's results go over them)
  });
}

template <int D>
hipError_t launch_t(const TreeAttn& p, void* workspace, hipStream_t stream) {
  const int lg = log2_of(p.hq / p.hkv);
  const TreeCut c = tree_cut(p.batch, p.max_q, p.max_kv, p.hq, p.hkv, false);
  const TreeWs ws = tree_ws(c, p.batch, p.hkv, D, workspace);
  const int64_t blocks = c.blocks ? c.blocks : (int64_t)p.batch * p.hkv * c.tiles;
  const dim3 grid((unsigned)blocks);
  if (p.page_log2 < 4) tree_attn_f32_kernel<D, true><<<grid, kW * 64, 0, stream>>>(p, c, ws, lg);
  else tree_attn_f32_kernel<D, false><<<grid, kW * 64, 0, stream>>>(p, c, ws, lg);
  if (c.blocks) launch_tree_merge<float, D>(p, c, ws, lg, stream);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_tree_attn_f32(const TreeAttn& p, int head_dim, void* ws, hipStream_t stream) {
  return head_dim == 64 ? launch_t<64>(p, ws, stream) : launch_t<128>(p, ws, stream);
}

}  // namespace qcf
