// Attention of a chunk of new rows of each request over its paged cache (qcf_chunk_attn), float32, on the float32
// matrix instruction v_mfma_f32_16x16x4_f32.
//
// A block holds 32 query vectors of one request and KV head, in two groups of 16 that share every K and V
// fragment; its four waves take the 16-token tiles in turn, each with its own online softmax, and are
// summed through LDS once per unit.  A lane's fragment is 16 contiguous bytes of a row, and no two waves read
// the same token, so K and V go from the pages to registers: K of the next tile is asked for before this
// tile's softmax, V after its products.
//  * S^T = K Q^T: a lane holds 4 tokens' logits of one vector of each group (register r of lane l: token
//    4 (l / 16) + r, vector l % 16).  Product (sb, e) takes the d-columns 16 sb + 4 (l / 16) + e of both
//    operands, so both are float4 loads.
//  * O^T += V^T P^T with P^T straight from those registers: product (r, mb) contracts over the tokens
//    4 (l / 16) + r and fills the d-columns NB (l % 16) + mb, so a lane's V operands are NB contiguous floats.
//  * exp2f, not the bare instruction: weights below 2^-126 stay subnormal numbers.
// Bound: latency at test sizes (3 requests of 5 to 70 rows over 33 to 700 tokens, 8/2 heads of 64, 20 us in two
// launches), the float32 matrix rate and the L2 caches beyond (K and V are read once per 32 vectors): 1000 rows over 4000
// tokens, 32/8 heads of 64, 396 us, 93 TFLOP/s; of 128, where 64 registers are in scratch memory, 1113 us, 66 TFLOP/s.
#include "qcf_chunk.h"

namespace qcf {
namespace {

constexpr int kW = 4;    // waves
constexpr int kT = 16;   // tokens per wave and step
constexpr int kNV = 2;   // groups of 16 query vectors
constexpr int kVt = 16 * kNV;
static_assert(kW * kT == kChunkStep, "a block's waves take a step's tokens");

template <int D>
__global__ __launch_bounds__(kW * 64, 2) void chunk_attn_f32_kernel(ChunkAttn p, ChunkCut cut, ChunkWs ws, int lg) {
  constexpr int SB = D / 16, NB = D / 16;
  __shared__ float4 o_l[kW * kVt * (D / 4)];
  __shared__ float2 ml_l[kW][kVt];
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l = threadIdx.x & 63, li = l & 15, lk = l >> 4;
  const float scale2 = p.scale * kLog2e;

  chunk_walk<kW * 64>(p, cut, ws, lg, [&](int b, const TreeRequest& rq, int g, int tile, int first, int n, int slot) {
    const_i32 table = (const_i32)(p.block_table + b * p.table_stride);
    const float* kc = static_cast<const float*>(p.k_cache) + (int64_t)g * D;
    const float* vc = static_cast<const float*>(p.v_cache) + (int64_t)g * D;
    constexpr int kHop = kW * kT;
    const int t_first = (first * kW + w) * kT;
    // tokens that row i of the request sees: from low(i) up to high(i)
    auto low = [&](int i) {
      return p.window ? (int)min(max((int64_t)rq.kv + i - p.window + 1, (int64_t)0), (int64_t)INT32_MAX) : 0;
    };
    auto high = [&](int i) { return (int)min((int64_t)rq.kv + i + 1, (int64_t)rq.end); };
    const int ib0 = (tile * kVt) >> lg, ib1 = min((tile * kVt + kVt - 1) >> lg, rq.rows - 1);
    const int plain_lo = low(ib1), plain_hi = high(ib0);  // tokens that all rows of the unit see
    float4 qf[kNV][SB];
    int r_lo[kNV], r_hi[kNV];
#pragma unroll
    for (int c = 0; c < kNV; ++c) {
      const int vec = tile * kVt + 16 * c + li, idx = min(vec >> lg, rq.rows - 1);
      const int head = (g << lg) + (vec & ((1 << lg) - 1));
      r_lo[c] = low(idx);
      r_hi[c] = high(idx);
      const float* q = static_cast<const float*>(p.q) + ((rq.r0 + idx) * p.hq + head) * D + 4 * lk;
#pragma unroll
      for (int sb = 0; sb < SB; ++sb) qf[c][sb] = *reinterpret_cast<const float4*>(q + 16 * sb);
    }

    const bool pool = p.n_pages > 0;
    auto page_at = [&](int i) { return i >= n ? -1 : page_of(p, table, t_first + i * kHop, rq.end); };
    // row r of the tile at t0; without a page the pool's first rows stand in and are not seen
    auto place = [&](int t0, int page, int r) {
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
    f32x4 o[kNV][NB];
    float m[kNV], ls[kNV];  // running maximum in log2 units, this lane's part of the sum
#pragma unroll
    for (int c = 0; c < kNV; ++c) {
#pragma unroll
      for (int mb = 0; mb < NB; ++mb) o[c][mb] = f32x4{};
      m[c] = -INFINITY;
      ls[c] = 0.f;
    }
    int page = page_at(0), page1 = page_at(1);
    if (pool && n > 0) {
      load_k(t_first, page);
      load_v(t_first, page);
    }
    // Q has to be there before the loop (a wait for it inside would count the next tile's loads)
#pragma unroll
    for (int c = 0; c < kNV; ++c)
#pragma unroll
      for (int sb = 0; sb < SB; ++sb)
        asm volatile("" : "+v"(qf[c][sb].x), "+v"(qf[c][sb].y), "+v"(qf[c][sb].z), "+v"(qf[c][sb].w));
    for (int i = 0; i < n && pool; ++i) {
      const int t0 = t_first + i * kHop;
      f32x4 s[kNV][2] = {};
#pragma unroll
      for (int sb = 0; sb < SB; sb += 2)
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int a = 0; a < 2; ++a)
#pragma unroll
            for (int c = 0; c < kNV; ++c) {
              const float4 k4 = kf[sb + a], q4 = qf[c][sb + a];
              const float ke = e == 0 ? k4.x : e == 1 ? k4.y : e == 2 ? k4.z : k4.w;
              const float qe = e == 0 ? q4.x : e == 1 ? q4.y : e == 2 ? q4.z : q4.w;
              s[c][a] = __builtin_amdgcn_mfma_f32_16x16x4f32(ke, qe, s[c][a], 0, 0, 0);
            }
      if (i + 1 < n) load_k(t0 + kHop, page1);
      const int page2 = page_at(i + 2);
      // which of the tile's tokens there are, and which of them this lane's vectors see
      uint32_t held = 0xffffu, sees[kNV], loose = 0;  // loose: tokens whose values are added one by one
#pragma unroll
      for (int c = 0; c < kNV; ++c) sees[c] = 0xffffu;
      if (t0 + kT > plain_hi || t0 < plain_lo || page < 0) {
        if (t0 >= rq.end || page < 0) held = 0;
        else if (rq.end - t0 < kT) held &= (1u << (rq.end - t0)) - 1u;
#pragma unroll
        for (int c = 0; c < kNV; ++c) {
          const int from = min(max(r_lo[c] - t0, 0), kT), to = min(max(r_hi[c] - t0, 0), kT);
          sees[c] = held & ((1u << to) - 1u) & ~((1u << from) - 1u);
        }
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
      float pr[kNV][4];
#pragma unroll
      for (int c = 0; c < kNV; ++c) {
        const f32x4 dot = s[c][0] + s[c][1];
        float x[4], mt = -INFINITY;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          x[r] = sees[c] >> (4 * lk + r) & 1 ? dot[r] * scale2 : -INFINITY;
          mt = fmaxf(mt, x[r]);
        }
        // lazy rescale: a stale maximum stays unless the vector's grew by more than 2^8 (by each vector's
        // own, so that no row's bits hang on another's)
        if (__ballot(!(mt < m[c] + 8.f))) {  // (no maximum yet: row_scale)
          mt = fmaxf(mt, __shfl_xor(mt, 16, 64));
          mt = fmaxf(mt, __shfl_xor(mt, 32, 64));
          const float mn = mt > m[c] + 8.f ? mt : m[c];
          const float alpha = exp2f(gap(m[c], mn));
          ls[c] = fmaf(ls[c], alpha, mn == -INFINITY && sees[c] ? 1.f : 0.f);
#pragma unroll
          for (int mb = 0; mb < NB; ++mb) o[c][mb] *= alpha;
          m[c] = mn;
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) pr[c][r] = exp2f(x[r] - finite(m[c]));
        ls[c] += (pr[c][0] + pr[c][1]) + (pr[c][2] + pr[c][3]);
      }
      for (uint32_t left = loose; left; left &= left - 1) {
        const int k = __builtin_ctz(left);
        const float* vr = vc + place(t0, page, k);
#pragma unroll
        for (int c = 0; c < kNV; ++c) {
          float a = 0.f;
#pragma unroll
          for (int r = 0; r < 4; ++r) a = (k & 3) == r ? pr[c][r] : a;
          const float pk = __shfl(a, (k >> 2) * 16 + li, 64);
          if (sees[c] >> k & 1) {
#pragma unroll
            for (int mb = 0; mb < NB; ++mb)
#pragma unroll
              for (int r = 0; r < 4; ++r) o[c][mb][r] = fmaf(vr[NB * (4 * lk + r) + mb], pk, o[c][mb][r]);
          }
        }
      }
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int mb = 0; mb < NB; ++mb) {
          const float4 v = vf[r][mb / 4];
          const float ve = mb % 4 == 0 ? v.x : mb % 4 == 1 ? v.y : mb % 4 == 2 ? v.z : v.w;
#pragma unroll
          for (int c = 0; c < kNV; ++c) o[c][mb] = __builtin_amdgcn_mfma_f32_16x16x4f32(ve, pr[c][r], o[c][mb], 0, 0, 0);
        }
      if (i + 1 < n) load_v(t0 + kHop, page1);
      page = page1;
      page1 = page2;
    }

    // the waves' results, summed in their order.  A lane's columns are NB (4 lk + r) + mb; vector v's
    // columns 4 i .. + 3 sit at i ^ (v % 8).
#pragma unroll
    for (int g2 = 0; g2 < kNV; ++g2) {
      ls[g2] += __shfl_xor(ls[g2], 16, 64);
      ls[g2] += __shfl_xor(ls[g2], 32, 64);
      const int v = 16 * g2 + li;
      if (lk == 0) ml_l[w][v] = make_float2(m[g2], ls[g2]);
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int c = 0; c < NB / 4; ++c)
          o_l[(w * kVt + v) * (D / 4) + (((4 * lk + r) * (NB / 4) + c) ^ (v & 7))] =
              make_float4(o[g2][4 * c][r], o[g2][4 * c + 1][r], o[g2][4 * c + 2][r], o[g2][4 * c + 3][r]);
    }
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
hipError_t launch_t(const ChunkAttn& p, void* workspace, hipStream_t stream) {
  const int lg = log2_of(p.hq / p.hkv);
  const ChunkCut c = chunk_cut(p.max_q, p.hq, p.hkv, false);
  const ChunkWs ws = chunk_ws(c, D, workspace);
  chunk_attn_f32_kernel<D><<<dim3((unsigned)c.blocks), kW * 64, 0, stream>>>(p, c, ws, lg);
  launch_chunk_merge<float, D>(p, c, ws, lg, stream);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_chunk_attn_f32(const ChunkAttn& p, int head_dim, void* ws, hipStream_t stream) {
  return head_dim == 64 ? launch_t<64>(p, ws, stream) : launch_t<128>(p, ws, stream);
}

}  // namespace qcf
