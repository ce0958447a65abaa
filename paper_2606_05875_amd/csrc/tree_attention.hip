// Attention of each request's new rows over its paged cache (qcf_tree_attn), bf16.
//
// With the softmax's running maximum m and sum l per query vector, one pass over the tokens suffices:
// S = K Q^T, p = exp2(S - m), O = O alpha + V^T p^T.  Products are transposed, as in the other attention
// kernels of this library: a lane holds tokens' logits of ONE query vector, so its p are the second
// product's operand as they stand.
//
// Weights enter the sum l as float32, and the second product as bf16.  Up to 64 query vectors they are two
// bf16 numbers, p cut short and what that left (15 bits), and the output is off by its own rounding
// alone (1.66e-3 of its norm from 64 bits, 64 decoded rows): a second product per V fragment, which waits for pages
// hide (203.5 -> 204.7 us; 16 trees of 16 rows 114.0 -> 115.3).  Beyond, where products and exponentials
// bound it, they are one bf16 number and the output 2.3e-3 off: two cost 16 trees of 8 to 40 rows 133 -> 170 us,
// 64 rows over 32896 tokens 91 -> 116, over 131584 298 -> 406, and vector registers spill.
//
// Keys and values go from the pages into LDS without passing registers (16 bytes per lane); the
// block table's entries come through the scalar cache, one per 16 tokens, a step ahead.
//  narrow  up to 32 query vectors per request and KV head (one token, short chains).  Bound: HBM.  Four
//          waves take 16-token tiles in turn, each on its own (two stages of LDS, no barrier in the loop),
//          v_mfma_f32_16x16x32/16x16x16_bf16; their results are summed through LDS once per unit.
//          64 decoded rows over 512 to 8192 tokens, 32/8 heads of 128: 204 us with the merge, 5.57 TB/s (a
//          copy reaches 5.1); one row over 8192 tokens 16.7 us, over 32768 32 us.
//  wide    more vectors (trees).  A wave holds 32 of them (v_mfma_f32_32x32x16_bf16) and the 2, 4 or 8
//          waves of a block share every 64-token tile (a ring of stages, one barrier per tile); the
//          products of the next tile's S run beside this tile's exponentials.  Bound: HBM and the latency of
//          pages up to about 128 vectors (16 trees of 8 to 40 rows over 2000 to 12700 tokens, 32/8 heads of
//          128: 133 to 140 us, 3.7 TB/s; all of 40 rows 140 to 146 us), products and exponentials beyond (64 rows
//          of 64/8 heads: 88 to 96 us over 32896 tokens, 0.75 PFLOP/s; 292 to 303 us over 131584, 0.93 PFLOP/s, the
//          matrix units busy 49% of the cycles).
// Pages of fewer than 16 rows are looked up by every lane, and every tile of such pages, as those of a unit with
// a page that is not there, goes the way of the last ones, next products behind the exponentials (64 decoded rows 303
// us against 206, 16 trees of 8 to 40 rows 298 against 140; there, one missing page in every request 194); their
// kernels for head size 128 also spill 2 to 10 vector registers.
// Without a mask, too, a unit goes through all of its request's tokens, and tiles of the new rows' own are such
// last ones: a prompt costs its full rectangle (4096 rows, 64/8 heads of 128, over an empty cache 954 us, 0.29
// PFLOP/s of what its rows see; 2000 rows over 30000 tokens 2.2 ms, 0.92).
#include <math.h>

#include <type_traits>

#include "qcf_paged.h"

namespace qcf {
namespace {

// A weight p as two bf16 numbers, cut_of (the upper half of its bits) and rest_of, which is off by 2^-8 of less than
// 2^-7 p.  Both are above zero wherever p is, so that a product with an infinite value that is seen is infinite and
// never the difference of two, nor 0 times infinity: hence cut, not rounded, 2^-23 p more, and 2^-126 at least
// (as no weight is between that and 0).
__device__ __forceinline__ float cut_of(float p) { return __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, p) & 0xffff0000u); }
__device__ __forceinline__ float rest_of(float p) { return fmaxf(fmaf(p, 0x1.000002p0f, -cut_of(p)), fminf(p, 0x1p-126f)); }

// ---------------------------------------------------------------------------
// narrow
// ---------------------------------------------------------------------------
constexpr int kNW = 4;   // waves
constexpr int kNT = 16;  // tokens per wave and step
static_assert(kNW * kNT == kTreeStep, "a block's waves take a step's tokens");

template <int D, int NV, bool kTiny>
__global__ __launch_bounds__(kNW * 64, 2) void tree_attn_narrow_kernel(TreeAttn p, TreeCut cut, TreeWs ws, int lg) {
  constexpr int CH = D / 8;          // 16-byte chunks per row
  constexpr int RPC = 64 / CH;       // rows per copy
  constexpr int RB = D * 2;          // bytes per row
  constexpr int TB = kNT * RB;       // bytes of a tile of K or V
  constexpr int TC = kNT / RPC;      // copies per tile of K or V
  constexpr int MB = D / 16, ST = D / 32;
  constexpr int VT = 16 * NV;
  __shared__ __attribute__((aligned(1024))) uint8_t ring[kNW * 4 * TB];  // per wave: K, V of two stages
  __shared__ float2 ml_l[kNW][VT];
  static_assert(kNW * VT * D * 4 <= (int)sizeof(ring), "the waves' O fit");

  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l = threadIdx.x & 63, ln = l & 15, lk = l >> 4;
  uint8_t* mine = ring + w * 4 * TB;
  const uint32_t lds0 = lds_addr(mine);
  const uint32_t row_b = (uint32_t)(p.kv_stride * 2);
  const float scale2 = p.scale * kLog2e;

  // copy i of a tile fills rows RPC i + l / CH; chunk c of K row r sits at c ^ r (D = 64: r / 2), of V row r
  // at c ^ 2 (r % 8) (D = 64: 2 (r / 2 % 4)): the fragment reads below are free of conflicts
  uint32_t koff[TC], voff[TC];
#pragma unroll
  for (int i = 0; i < TC; ++i) {
    const int r = RPC * i + l / CH, c = l % CH;
    koff[i] = r * row_b + (c ^ (D == 128 ? r : r >> 1)) * 16;
    voff[i] = r * row_b + (c ^ (D == 128 ? 2 * (r & 7) : 2 * ((r >> 1) & 3))) * 16;
  }
  const int krd = ln * RB, ksw = D == 128 ? ln : ln >> 1;
  const int vr = 4 * lk + ((l >> 2) & 3);  // V row this lane reads for the transposing read
  const int vrd = vr * RB + 8 * (l & 3), vsw = D == 128 ? vr & 7 : (vr >> 1) & 3;

  tree_walk<kNW * 64>(p, cut, ws, lg, [&](int b, const TreeRequest& rq, int g, int tile, int first, int n,
                                          int steps, int slot) {
    const_i32 table = (const_i32)(p.block_table + b * p.table_stride);
    const uint16_t* kc = static_cast<const uint16_t*>(p.k_cache) + (int64_t)g * D;
    const uint16_t* vc = static_cast<const uint16_t*>(p.v_cache) + (int64_t)g * D;
    const int t_first = (first * kNW + w) * kNT;  // this wave's first token; the next ones follow kNW * kNT on
    constexpr int kHop = kNW * kNT;

    bf16x8 qf[NV][ST];
    int64_t row[NV];
    int idx[NV], head[NV];
#pragma unroll
    for (int c = 0; c < NV; ++c) {
      const int v = tile * VT + 16 * c + ln;
      idx[c] = v >> lg;
      head[c] = (g << lg) + (v & ((1 << lg) - 1));
      row[c] = rq.r0 + min(idx[c], rq.rows - 1);
      const uint16_t* q = static_cast<const uint16_t*>(p.q) + (row[c] * p.hq + head[c]) * D + 8 * lk;
#pragma unroll
      for (int st = 0; st < ST; ++st) qf[c][st] = as_bf16x8(ld16(q + 32 * st));
    }
    f32x4 o[NV][MB];
    float m[NV], ls[NV];  // running maximum in log2 units, this lane's part of the sum
    bool big[NV];
#pragma unroll
    for (int c = 0; c < NV; ++c) {
      big[c] = false;
      m[c] = -INFINITY;
      ls[c] = 0.f;
#pragma unroll
      for (int mb = 0; mb < MB; ++mb) o[c][mb] = f32x4{};
    }

    // K and V of the tile at t0 into stage s; returns the rows that hold a token, as bits
    auto copy_tile = [&](int t0, int page, int s) {
      const uint32_t lk0 = lds0 + s * 2 * TB, lv0 = lk0 + TB;
      if (!kTiny) {
        const int64_t base = ((int64_t)max(page, 0) << p.page_log2) + (t0 & ((1 << p.page_log2) - 1));
        const uint16_t* kb = kc + (page < 0 ? 0 : base) * p.kv_stride;
        const uint16_t* vb = vc + (page < 0 ? 0 : base) * p.kv_stride;
#pragma unroll
        for (int i = 0; i < TC; ++i) copy16(kb, koff[i], lk0 + i * 1024);
#pragma unroll
        for (int i = 0; i < TC; ++i) copy16(vb, voff[i], lv0 + i * 1024);
      } else {
#pragma unroll
        for (int i = 0; i < TC; ++i) {
          const int r = RPC * i + l / CH;
          const int64_t at = max(slot_of(p, b, t0 + r, rq.end), (int64_t)0) * p.kv_stride;
          copy16(kc + at + (koff[i] - r * row_b) / 2, lk0 + i * 1024);
          copy16(vc + at + (voff[i] - r * row_b) / 2, lv0 + i * 1024);
        }
      }
    };
    auto page_at = [&](int i) { return kTiny || i >= n ? -1 : page_of(p, table, t_first + i * kHop, rq.end); };

    // the rows of a page are there even where a page ends the pool, so a whole tile can be copied; without
    // a page the pool's first rows stand in and are not seen
    const bool pool = p.n_pages > 0 && (kTiny || p.page_log2 >= 4);
    int page = page_at(0), page1 = page_at(1);
    if (pool) copy_tile(t_first, page, 0);
    // Q has to be there before the loop (and comes with the first tile): a wait for it inside would
    // count the copies in flight
#pragma unroll
    for (int c = 0; c < NV; ++c)
#pragma unroll
      for (int st = 0; st < ST; ++st) asm volatile("" : "+v"(qf[c][st]));
    for (int i = 0; i < n && pool; ++i) {
      const int t0 = t_first + i * kHop;
      asm volatile("" ::: "memory");
      __builtin_amdgcn_s_waitcnt(0xc07f);  // the last tile's LDS reads are done (lgkmcnt 0) before it is overwritten
      if (i + 1 < n) copy_tile(t0 + kHop, page1, (i + 1) & 1);
      const int page2 = page_at(i + 2);
      if (i + 1 < n) wait_vm_lgkm0<2 * TC>();
      else wait_vm_lgkm0<0>();
      asm volatile("" ::: "memory");
      uint8_t* kl = mine + (i & 1) * 2 * TB;
      uint8_t* vl = kl + TB;

      f32x4 s[NV];
#pragma unroll
      for (int c = 0; c < NV; ++c) s[c] = f32x4{};
#pragma unroll
      for (int st = 0; st < ST; ++st) {
        const bf16x8 kf = as_bf16x8(ld16(kl + krd + (((4 * st + lk) ^ ksw) * 16)));
#pragma unroll
        for (int c = 0; c < NV; ++c)
          s[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[c][st], s[c], 0, 0, 0);
      }
      // lane value r of s is token t0 + 4 lk + r
      uint32_t sees[NV];
      uint32_t loose = 0;  // tokens whose values are added one by one
      bool edge = t0 + kNT > min(rq.kv, rq.end) || (!kTiny && page < 0);
      uint32_t held = 0xffffu;
      if (kTiny) {
        held = (uint32_t)__ballot(slot_of(p, b, t0 + ln, rq.end) >= 0) & 0xffffu;
        edge = edge || held != 0xffffu;
      }
      if (edge) {
        if (t0 >= rq.end || (!kTiny && page < 0)) held = 0;
        else if (rq.end - t0 < kNT) held &= (1u << (rq.end - t0)) - 1u;
#pragma unroll
        for (int c = 0; c < NV; ++c) {
          sees[c] = held ? tree_sees<16>(p, rq, row[c], idx[c], t0) & held : 0u;
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (!(sees[c] >> (4 * lk + r) & 1)) s[c][r] = -INFINITY;
        }
        // a value that a row does not see must not meet its weight 0 where it is not finite: rows that
        // hold no token become zeros, and tokens with such values (rare) are taken out and added to the
        // rows that see them
#pragma unroll
        for (int i4 = 0; i4 < TC; ++i4) {
          const int r = RPC * i4 + l / CH;
          uint8_t* at = vl + i4 * 1024 + 16 * l;
          const bool drop = !(held >> r & 1);
          const uint64_t bad = __ballot(!drop && not_finite(ld16(at)));
#pragma unroll
          for (int k = 0; k < RPC; ++k)
            if (bad >> (k * CH) & (CH == 16 ? 0xffffull : 0xffull)) loose |= 1u << (RPC * i4 + k);
          if (drop) st16(at, make_uint4(0, 0, 0, 0));
        }
        asm volatile("" ::: "memory");
      }
      v4s pb[NV], pl[NV];  // weights cut to bf16, and what that left of them
      float pw[NV][4];
#pragma unroll
      for (int c = 0; c < NV; ++c) {
        float mt = fmaxf(fmaxf(s[c][0], s[c][1]), fmaxf(s[c][2], s[c][3])) * scale2;
        // lazy rescale: a stale maximum stays unless the vector's grew by more than 2^8 (by each
        // vector's own, so that no row's bits hang on another's)
        if (__ballot(!(mt < m[c] + 8.f))) {  // (no maximum yet: row_scale)
          mt = fmaxf(mt, __shfl_xor(mt, 16, 64));
          mt = fmaxf(mt, __shfl_xor(mt, 32, 64));
          const float mn = mt > m[c] + 8.f ? mt : m[c];
          const float alpha = __builtin_amdgcn_exp2f(gap(m[c], mn));
          ls[c] = fmaf(ls[c], alpha, mn == -INFINITY && (!edge || sees[c]) ? 1.f : 0.f);
#pragma unroll
          for (int mb = 0; mb < MB; ++mb) o[c][mb] *= alpha;
          m[c] = mn;
          big[c] = is_big(mn);
        }
        const float ref = finite(m[c]);
        const float sc = big[c] ? 1.f : scale2;
        if (__ballot(big[c])) s[c] *= big[c] ? scale2 : 1.f;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          pw[c][r] = __builtin_amdgcn_exp2f(fmaf(s[c][r], sc, -ref));
          pb[c][r] = (short)(__builtin_bit_cast(uint32_t, pw[c][r]) >> 16);
          pl[c][r] = (short)f2bf(rest_of(pw[c][r]));
        }
        ls[c] += (pw[c][0] + pw[c][1]) + (pw[c][2] + pw[c][3]);
      }
      if (loose) {
        for (uint32_t left = loose; left; left &= left - 1) {
          const int k = __builtin_ctz(left);
#pragma unroll
          for (int c = 0; c < NV; ++c) {
            float a = 0.f;
#pragma unroll
            for (int r = 0; r < 4; ++r) a = (k & 3) == r ? pw[c][r] : a;
            const float pk = __shfl(a, (k >> 2) * 16 + ln, 64);
            if (sees[c] >> k & 1) {
              const int sw = D == 128 ? k & 7 : (k >> 1) & 3;
#pragma unroll
              for (int mb = 0; mb < MB; ++mb) {
                const uint16_t* v = reinterpret_cast<const uint16_t*>(vl + k * RB + ((mb ^ sw) << 5) + 8 * lk);
#pragma unroll
                for (int r = 0; r < 4; ++r) o[c][mb][r] = fmaf(pk, bf2f(v[r]), o[c][mb][r]);
              }
            }
          }
        }
        asm volatile("" ::: "memory");
#pragma unroll
        for (int i4 = 0; i4 < TC; ++i4)
          if (loose >> (RPC * i4 + l / CH) & 1) st16(vl + i4 * 1024 + 16 * l, make_uint4(0, 0, 0, 0));
        asm volatile("" ::: "memory");
      }
#pragma unroll
      for (int mb = 0; mb < MB; ++mb) {
        const v4s va = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s)(vl + vrd + ((mb ^ vsw) << 5)));
#pragma unroll
        for (int c = 0; c < NV; ++c) {
          o[c][mb] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(va, pb[c], o[c][mb], 0, 0, 0);
          o[c][mb] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(va, pl[c], o[c][mb], 0, 0, 0);
        }
      }
      page = page1;
      page1 = page2;
    }

    // the waves' results, summed in their order: vector v's columns 4 i .. + 3 at i ^ (v % 8)
    __syncthreads();  // every wave has read its tiles
    float4* o_l = reinterpret_cast<float4*>(ring);
#pragma unroll
    for (int c = 0; c < NV; ++c) {
      ls[c] += __shfl_xor(ls[c], 16, 64);
      ls[c] += __shfl_xor(ls[c], 32, 64);
      const int v = 16 * c + ln;
      if (lk == 0) ml_l[w][v] = make_float2(m[c], ls[c]);
#pragma unroll
      for (int mb = 0; mb < MB; ++mb)
        o_l[(w * VT + v) * (D / 4) + ((4 * mb + lk) ^ (v & 7))] = make_float4(o[c][mb][0], o[c][mb][1], o[c][mb][2], o[c][mb][3]);
    }
    __syncthreads();
    for (int u = threadIdx.x; u < VT * (D / 4); u += kNW * 64) {
      const int v = u / (D / 4), i4 = u % (D / 4);
      const int vec = tile * VT + v, i = vec >> lg;
      if (i >= rq.rows) continue;
      float2 ml[kNW];
      float mx = -INFINITY, lt = 0.f;
#pragma unroll
      for (int k = 0; k < kNW; ++k) {
        ml[k] = ml_l[k][v];
        mx = fmaxf(mx, ml[k].x);
      }
      float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k = 0; k < kNW; ++k) {
        const float f = __builtin_amdgcn_exp2f(gap(ml[k].x, mx));
        const float4 x = o_l[(k * VT + v) * (D / 4) + (i4 ^ (v & 7))];
        lt += f * ml[k].y;
        a.x += f * x.x;
        a.y += f * x.y;
        a.z += f * x.z;
        a.w += f * x.w;
      }
      if (slot >= 0) {
        reinterpret_cast<float4*>(ws.o)[((int64_t)slot * VT + v) * (D / 4) + i4] = a;
        if (i4 == 0) ws.ml[(int64_t)slot * VT + v] = make_float2(mx, lt);
      } else {
        const int64_t at = (rq.r0 + i) * p.hq + (g << lg) + (vec & ((1 << lg) - 1));
        const float inv = row_scale(mx, lt);
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.out) + at * D + 4 * i4) =
            make_uint2(pack_bf16x2(a.x * inv, a.y * inv), pack_bf16x2(a.z * inv, a.w * inv));
        if (p.lse && i4 == 0) p.lse[at] = row_lse(mx, lt);
      }
    }
    // everyone has read the results, which the next unit's tiles go over (stores need not be waited for)
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
  });
}

// ---------------------------------------------------------------------------
// wide
// ---------------------------------------------------------------------------
constexpr int kWT = kTreeStep;
// Stages of the K and V rings: 64 KB, so that a CU holds two blocks, which run beside each other's starts, ends
// and exponentials; 128 KB for 8 waves, which have a CU to themselves
constexpr int wide_stages(int d, int vg) { return d == 64 || vg == 8 ? 4 : 2; }

template <int D, int VG, bool kTiny>
__global__ __launch_bounds__(VG * 64, VG == 2 ? 1 : 2) void tree_attn_wide_kernel(TreeAttn p, TreeCut cut, TreeWs ws, int lg) {
  constexpr int CH = D / 8;        // 16-byte chunks per row
  constexpr int RPC = 64 / CH;     // rows per copy
  constexpr int RB = D * 2;        // bytes per row
  constexpr int TB = kWT * RB;     // bytes of a tile of K or V
  constexpr int VT = 32 * VG;
  constexpr int NB = wide_stages(D, VG);
  constexpr bool kTwo = VG == 2;   // weights of two bf16 numbers
  // Copies go by groups of 16 rows, which lie in one page: wave w takes groups w, w + VG, .. of the
  // tile's four, of 8 waves half of group w / 2
  constexpr int GC = 16 / RPC;               // copies per group, K or V
  constexpr int WC = VG == 8 ? GC / 2 : GC;  // of them a wave's
  constexpr int WG = VG == 8 ? 1 : 4 / VG;   // groups per wave
  constexpr int WI = WG * WC;
  static_assert((VG == 2 || VG == 4 || VG == 8) && GC % 2 == 0, "groups are shared evenly");
  __shared__ __attribute__((aligned(1024))) uint8_t k_ring[NB * TB];
  __shared__ __attribute__((aligned(1024))) uint8_t v_ring[NB * TB];
  __shared__ uint32_t loose_l[2];

  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l = threadIdx.x & 63, lq = l & 31, hi = l >> 5;
  const uint32_t k_lds = lds_addr(k_ring), v_lds = lds_addr(v_ring);
  const uint32_t row_b = (uint32_t)(p.kv_stride * 2);
  const float scale2 = p.scale * kLog2e;
  // Chunk c of K row r sits at c ^ (r % 16) (D = 64: c ^ (r / 2 % 8)), of V row r at c ^ 4 (r % 4)
  // (D = 64: c ^ 4 (r / 2 % 2)): lane fragments st at krd ^ (st << 5), V column blocks mb at vrd ^ (mb << 6)
  const int ky = D == 128 ? lq & 15 : (lq >> 1) & 7;
  int krd = lq * RB + (hi ^ (ky & 1)) * 16 + (ky >> 1) * 32;
  const int tg = l >> 4, te = (l >> 2) & 3, tq = l & 3;
  const int vrd = (4 * (tg >> 1) + te) * RB + (D == 128 ? te : te >> 1) * 64 + 32 * (tg & 1) + 8 * tq;
  // copy i of a group fills rows RPC i + l / CH: the row within the copy and the chunk of K, V before i's
  // part of the exchange (which i's bits give by themselves)
  const int cr = l / CH, cc = l % CH;
  uint32_t coff = cr * row_b, kx = (cc ^ (D == 128 ? cr : cr >> 1)) * 16;
  const uint32_t vx = (cc ^ (4 * (D == 128 ? cr : (cr >> 1) & 1))) * 16;

  tree_walk<VG * 64>(p, cut, ws, lg, [&](int b, const TreeRequest& rq, int g, int tile, int first, int n,
                                         int steps, int slot) {
    const_i32 table = (const_i32)(p.block_table + b * p.table_stride);
    const uint16_t* kc = static_cast<const uint16_t*>(p.k_cache) + (int64_t)g * D;
    const uint16_t* vc = static_cast<const uint16_t*>(p.v_cache) + (int64_t)g * D;
    const bool pool = p.n_pages > 0 && (kTiny || p.page_log2 >= 4);
    const int t_first = first * kWT;
    auto group = [&](int k) { return VG == 8 ? w >> 1 : w + VG * k; };
    const int c0 = VG == 8 ? WC * (w & 1) : 0;  // this wave's first copy of a group
    auto page_at = [&](int t, int k) {
      return kTiny || t >= n ? -1 : page_of(p, table, t_first + t * kWT + 16 * group(k), rq.end);
    };
    // K (V) of this wave's groups of tile t into its stage; without a page the pool's first rows stand in
    // and are not seen
    auto copy = [&](auto is_k, uint32_t lds, int t, const int (&page)[WG]) {
      constexpr bool kK = decltype(is_k)::value;
      const uint16_t* from = kK ? kc : vc;
      const uint32_t to = lds + (t & (NB - 1)) * TB;
      asm volatile("" : "+v"(coff), "+v"(kx));  // (formed anew: every copy's offset kept is a register each)
#pragma unroll
      for (int k = 0; k < WG; ++k) {
        const int t0 = t_first + t * kWT + 16 * group(k);
        const int64_t at = page[k] < 0 ? 0 : ((int64_t)page[k] << p.page_log2) + (t0 & ((1 << p.page_log2) - 1));
#pragma unroll
        for (int i = 0; i < WC; ++i) {
          const uint32_t dst = to + (group(k) * GC + c0 + i) * 1024;
          const uint32_t chunk = kK ? kx ^ ((c0 + i) * 64) : vx;
          if (!kTiny)
            copy16(from + (at + RPC * (c0 + i)) * p.kv_stride, coff + chunk, dst);
          else
            copy16(from + max(slot_of(p, b, t0 + RPC * (c0 + i) + cr, rq.end), (int64_t)0) * p.kv_stride + chunk / 2, dst);
        }
      }
    };
    const std::true_type K{};
    const std::false_type V{};
    const int v0 = tile * VT + 32 * w;
    const int idx = (v0 + lq) >> lg;
    const int head = (g << lg) + ((v0 + lq) & ((1 << lg) - 1));
    const bool valid = idx < rq.rows;
    const bool busy = (v0 >> lg) < rq.rows;  // (the wave has a vector)
    const int64_t row = rq.r0 + min(idx, rq.rows - 1);
    bf16x8 qreg[D / 16];
    {
      const uint16_t* q = static_cast<const uint16_t*>(p.q) + (row * p.hq + head) * D + 8 * hi;
#pragma unroll
      for (int st = 0; st < D / 16; ++st) qreg[st] = as_bf16x8(ld16(q + 16 * st));
    }
    int pages[NB][WG];
#pragma unroll
    for (int t = 0; t < NB; ++t)
#pragma unroll
      for (int k = 0; k < WG; ++k) pages[t][k] = page_at(t, k);
    // pages that are not there are rare: looked for once (by every wave), then tile by tile
    bool bad = kTiny;
    if (!kTiny && pool) {
      const int lp = p.page_log2;
      const int p1 = (int)(((int64_t)min(t_first + n * kWT, rq.end) + (1 << lp) - 1) >> lp);
      for (int i = (t_first >> lp) + l; i < p1; i += 64) {
        const int x = i < p.max_pages ? p.block_table[b * p.table_stride + i] : -1;
        bad = bad || x < 0 || x >= p.n_pages;
      }
    }
    const bool holes = __ballot(bad) != 0;
    // Q has to be there before the copies: a wait for it later would count those in flight
#pragma unroll
    for (int st = 0; st < D / 16; ++st) asm volatile("" : "+v"(qreg[st]));
    // K(0); then K(t + 1), V(t), in this order to the end
    int page[WG], pagev[WG];  // of the next K to be copied, of the next V
    if (pool) {
      copy(K, k_lds, 0, pages[0]);
#pragma unroll
      for (int t = 1; t < NB; ++t) {
        if (t < n) copy(K, k_lds, t, pages[t]);
        if (t <= n) copy(V, v_lds, t - 1, pages[t - 1]);
      }
#pragma unroll
      for (int k = 0; k < WG; ++k) {
        pagev[k] = pages[NB - 1][k];
        page[k] = page_at(NB, k);
      }
    }
    f32x16 o[D / 32];
#pragma unroll
    for (int mb = 0; mb < D / 32; ++mb) o[mb] = f32x16{};
    float m = -INFINITY, ls = 0.f;  // running maximum in log2 units, this lane's part of the sum
    bool big = false;

    // this wave's copies but the last `pairs` (K, V) are there, then the block's
    auto meet = [&](int pairs) {
      asm volatile("" ::: "memory");
      if (NB > 2 && pairs == NB - 2) wait_vm_lgkm0<(NB - 2) * 2 * WI>();
      else if (pairs == NB - 1) wait_vm_lgkm0<(NB - 1) * 2 * WI>();
      else wait_vm_lgkm0<0>();
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
    };
    constexpr int NS = D / 16;  // products per 32 tokens of S
    auto k_frag = [&](const uint8_t* kl, int i) {
      return as_bf16x8(ld16(kl + (i / NS) * 32 * RB + (krd ^ ((i % NS) << 5))));
    };
    auto products = [&](const uint8_t* kl, f32x16 (&s)[2]) {
#pragma unroll
      for (int hb = 0; hb < 2; ++hb) {
        __builtin_amdgcn_sched_barrier(0);
        s[hb] = f32x16{};
#pragma unroll
        for (int st = 0; st < NS; ++st)
          s[hb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_frag(kl, hb * NS + st), qreg[st], s[hb], 0, 0, 0);
      }
    };
    // the running maximum of the tile's logits (with tokens that the vector sees or without), and what the
    // exponentials are taken of
    auto maximum = [&](f32x16 (&s)[2], bool any) {
      float mt = s[0][0];
#pragma unroll
      for (int e = 1; e < 32; ++e) mt = fmaxf(mt, s[e >> 4][e & 15]);
      mt *= scale2;
      // lazily and by each vector's own growth (see the narrow kernel)
      if (__ballot(!(mt < m + 8.f))) {
        mt = fmaxf(mt, __shfl_xor(mt, 32, 64));
        const float mn = mt > m + 8.f ? mt : m;
        const float alpha = __builtin_amdgcn_exp2f(gap(m, mn));
        ls = fmaf(ls, alpha, mn == -INFINITY && any ? 1.f : 0.f);
#pragma unroll
        for (int mb = 0; mb < D / 32; ++mb) o[mb] *= alpha;
        m = mn;
        big = is_big(mn);
      }
      if (__ballot(big)) {
        const float f = big ? scale2 : 1.f;
        s[0] *= f;
        s[1] *= f;
      }
    };
    typedef float f32x2_t __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
    // P of the tile (kTwo: cut, and what that left of it in pl); with kNext S of the next one beside it: one product per fenced group with its K fragment
    // read four groups ahead, a group's arguments, exponentials and sums in three groups in turn
    auto weights = [&](auto next, const uint8_t* kn, f32x16 (&sn)[2], f32x16 (&s)[2], bf16x8 (&pb)[2][2], bf16x8 (&pl)[2][2]) {
      constexpr bool kNext = decltype(next)::value;
      constexpr int NM = 2 * NS, EG = 32 / NM, PF = 4;
      const float nm = -finite(m), sc = big ? 1.f : scale2;
      float psum = 0.f, x[32], pw[32];
      bf16x8 kf[NM];
      auto arg = [&](int i) {
#pragma unroll
        for (int e = EG * i; e < EG * (i + 1); ++e) x[e] = fmaf(s[e >> 4][e & 15], sc, nm);
      };
      auto sum_pack = [&](int i) {
#pragma unroll
        for (int e = EG * i; e < EG * (i + 1); e += 2) {
          psum += pw[e];
          psum += pw[e + 1];
          const bf16x2_t pk = kTwo ? (bf16x2_t){(__bf16)cut_of(pw[e]), (__bf16)cut_of(pw[e + 1])}
                                   : __builtin_convertvector((f32x2_t){pw[e], pw[e + 1]}, bf16x2_t);
          pb[e >> 4][(e >> 3) & 1][e & 7] = pk[0];
          pb[e >> 4][(e >> 3) & 1][(e & 7) + 1] = pk[1];
          if constexpr (kTwo) {
            const bf16x2_t rest = __builtin_convertvector((f32x2_t){rest_of(pw[e]), rest_of(pw[e + 1])}, bf16x2_t);
            pl[e >> 4][(e >> 3) & 1][e & 7] = rest[0];
            pl[e >> 4][(e >> 3) & 1][(e & 7) + 1] = rest[1];
          }
        }
        asm volatile("" : "+v"(psum));  // (in its group, not a chain of 32 sums behind the products)
      };
      if (kNext) {
#pragma unroll
        for (int i = 0; i < PF; ++i) kf[i] = k_frag(kn, i);
      }
      arg(0);
#pragma unroll
      for (int i = 0; i < NM; ++i) {
        __builtin_amdgcn_sched_barrier(0);
        if (kNext) {
          if (i + PF < NM) kf[i + PF] = k_frag(kn, i + PF);
          sn[i / NS] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[i], qreg[i % NS], i % NS == 0 ? f32x16{} : sn[i / NS], 0, 0, 0);
        }
        if (i + 1 < NM) arg(i + 1);
#pragma unroll
        for (int e = EG * i; e < EG * (i + 1); ++e) pw[e] = __builtin_amdgcn_exp2f(x[e]);
        if (i > 0) sum_pack(i - 1);
      }
      __builtin_amdgcn_sched_barrier(0);
      sum_pack(NM - 1);
      ls += psum;
    };
    // O += V^T P^T, one product per fenced group with its V fragment read four groups ahead
    auto products_o = [&](const uint8_t* vl, bf16x8 (&pb)[2][2], bf16x8 (&pl)[2][2]) {
      constexpr int MB = D / 32, NM = 4 * MB, PF = 4;
      auto v_frag = [&](int j) {
        const uint8_t* at = vl + (j / MB) * 16 * RB + (vrd ^ ((j % MB) << 6));
        const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s)(at));
        const v4s up = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s)(at + 8 * RB));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, up, 0, 1, 2, 3, 4, 5, 6, 7));
      };
      bf16x8 vf[NM];
#pragma unroll
      for (int j = 0; j < PF; ++j) vf[j] = v_frag(j);
#pragma unroll
      for (int j = 0; j < NM; ++j) {
        __builtin_amdgcn_sched_barrier(0);
        if (j + PF < NM) vf[j + PF] = v_frag(j + PF);
        o[j % MB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[j], pb[j / (2 * MB)][(j / MB) & 1], o[j % MB], 0, 0, 0);
        if constexpr (kTwo)
          o[j % MB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[j], pl[j / (2 * MB)][(j / MB) & 1], o[j % MB], 0, 0, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
    };

    // K(t + 1) and V(t) are there, and everyone has read K(t) and V(t - 1), whose stages are filled next
    auto begin = [&](int t) {
      meet(t + NB - 1 < n ? NB - 2 : 0);
      // the next page numbers are asked for before the copies and looked at behind them
      int next[WG], at[WG];
#pragma unroll
      for (int k = 0; k < WG; ++k) {
        at[k] = t_first + (t + NB + 1) * kWT + 16 * group(k);
        next[k] = kTiny ? -1 : table[min(at[k] >> p.page_log2, p.max_pages - 1)];
      }
      if (t + NB < n) copy(K, k_lds, t + NB, page);
      if (t + NB - 1 < n) copy(V, v_lds, t + NB - 1, pagev);
#pragma unroll
      for (int k = 0; k < WG; ++k) {
        pagev[k] = page[k];
        const int x = uni(next[k]);
        page[k] = !kTiny && at[k] < rq.end && at[k] >> p.page_log2 < p.max_pages && x < p.n_pages ? max(x, -1) : -1;
      }
    };
    // element e of s is token t0 + 32 (e / 16) + 8 (e / 4 % 4) + 4 hi + e % 4
    // the tiles before the first that is the last one or has tokens that are not there or not seen by all
    const int plain = holes ? 0 : min(n - 1, (min(rq.kv, rq.end) - t_first) / kWT) & ~1;
    auto plain_step = [&](int t, f32x16 (&s)[2], f32x16 (&sn)[2]) {
      bf16x8 pb[2][2], pl[2][2];
      maximum(s, true);
      weights(std::true_type{}, k_ring + ((t + 1) & (NB - 1)) * TB, sn, s, pb, pl);
      products_o(v_ring + (t & (NB - 1)) * TB, pb, pl);
    };
    // Tiles with tokens that are not there or that some row does not see.  held: those that are there, as
    // bits; true if there is something to do (for the whole block).
    auto is_edge = [&](int t, uint64_t& held) {
      const int t0 = t_first + t * kWT;
      held = ~0ull;
      if (holes) held = __ballot(slot_of(p, b, t0 + l, rq.end) >= 0);
      else if (rq.end - t0 < kWT) held = rq.end > t0 ? (1ull << (rq.end - t0)) - 1ull : 0ull;
      return t0 + kWT > rq.kv || held != ~0ull;
    };
    // rows of V that hold no token become zeros; the result is the tokens with a value that is not
    // finite, which are added to the rows that see them one by one (see the narrow kernel) ..
    auto clean = [&](int t, uint64_t held) {
      uint8_t* vl = v_ring + (t & (NB - 1)) * TB;
      if (threadIdx.x < 2) loose_l[threadIdx.x] = 0;
      __syncthreads();
      for (int u = threadIdx.x; u < kWT * CH; u += VG * 64) {
        const int r = u / CH;
        if (!(held >> r & 1)) st16(vl + 16 * u, make_uint4(0, 0, 0, 0));
        else if (not_finite(ld16(vl + 16 * u))) atomicOr(&loose_l[r >> 5], 1u << (r & 31));
      }
      __syncthreads();
      return (uint64_t)(uint32_t)uni((int)loose_l[1]) << 32 | (uint32_t)uni((int)loose_l[0]);
    };
    // .. and taken out once everyone has done so
    auto take_out = [&](int t, uint64_t loose) {
      uint8_t* vl = v_ring + (t & (NB - 1)) * TB;
      __syncthreads();
      for (int u = threadIdx.x; u < kWT * CH; u += VG * 64)
        if (loose >> (u / CH) & 1) st16(vl + 16 * u, make_uint4(0, 0, 0, 0));
      __syncthreads();
    };
    // any step, its next S (into s) after it
    auto other_step = [&](int t, f32x16 (&s)[2]) {
      const int t0 = t_first + t * kWT;
      const uint8_t* kn = k_ring + ((t + 1) & (NB - 1)) * TB;
      const uint8_t* vl = v_ring + (t & (NB - 1)) * TB;
      bf16x8 pb[2][2], pl[2][2];
      uint64_t held, loose = 0;
      uint32_t sees[2] = {0, 0};
      const bool edge = is_edge(t, held);
      if (edge) {
        loose = clean(t, held);
#pragma unroll
        for (int hb = 0; hb < 2; ++hb) {
          const uint32_t h = (uint32_t)(held >> (32 * hb));
          sees[hb] = h ? tree_sees<32>(p, rq, row, idx, t0 + 32 * hb) & h : 0u;
#pragma unroll
          for (int v = 0; v < 16; ++v)
            if (!(sees[hb] >> (8 * (v >> 2) + 4 * hi + (v & 3)) & 1)) s[hb][v] = -INFINITY;
        }
      }
      maximum(s, !edge || (sees[0] | sees[1]) != 0);
      weights(std::false_type{}, kn, s, s, pb, pl);
      if (loose) {
        for (uint64_t left = loose; left; left &= left - 1) {
          const int k = __builtin_ctzll(left);
          float a = 0.f;
#pragma unroll
          for (int e = 0; e < 32; ++e) a = (k >> 3) * 4 + (k & 3) == e ? s[e >> 4][e & 15] : a;
          a = __builtin_amdgcn_exp2f(fmaf(a, big ? 1.f : scale2, -finite(m)));
          const float pk = __shfl(a, ((k >> 2) & 1) * 32 + lq, 64);
          if ((k < 32 ? sees[0] : sees[1]) >> (k & 31) & 1) {
            const int sw = D == 128 ? k & 3 : (k >> 1) & 1;
#pragma unroll
            for (int mb = 0; mb < D / 32; ++mb)
#pragma unroll
              for (int c = 0; c < 4; ++c) {
                // columns 32 mb + 8 c + 4 hi .. + 3: half of chunk 4 mb + c
                const uint16_t* x = reinterpret_cast<const uint16_t*>(vl + k * RB + (((4 * mb + c) ^ (4 * sw)) * 16) + 8 * hi);
#pragma unroll
                for (int e = 0; e < 4; ++e) o[mb][4 * c + e] = fmaf(pk, bf2f(x[e]), o[mb][4 * c + e]);
              }
          }
        }
        take_out(t, loose);
      }
      products_o(vl, pb, pl);
      if (t + 1 < n) products(kn, s);
    };

    if (pool) meet(n >= NB ? NB - 1 : 0);
    if (pool && busy) {
      f32x16 sa[2];
      products(k_ring, sa);
      int t = 0;
      for (; t < plain; t += 2) {
        f32x16 sb[2];
        begin(t);
        plain_step(t, sa, sb);
        begin(t + 1);
        plain_step(t + 1, sb, sa);
      }
      for (; t < n; ++t) {
        begin(t);
        other_step(t, sa);
      }
    } else if (pool) {
      // a wave without vectors takes part in the copies and the block's meetings
      for (int t = 0; t < n; ++t) {
        uint64_t held;
        begin(t);
        if (!is_edge(t, held)) continue;
        const uint64_t loose = clean(t, held);
        if (loose) take_out(t, loose);
      }
    }
    ls += __shfl_xor(ls, 32, 64);
    if (valid) {
      if (slot >= 0) {
        const int64_t at = (int64_t)slot * VT + 32 * w + lq;
        if (hi == 0) ws.ml[at] = make_float2(m, ls);
#pragma unroll
        for (int mb = 0; mb < D / 32; ++mb)
#pragma unroll
          for (int c = 0; c < 4; ++c)
            reinterpret_cast<float4*>(ws.o)[at * (D / 4) + 8 * mb + 2 * c + hi] =
                make_float4(o[mb][4 * c], o[mb][4 * c + 1], o[mb][4 * c + 2], o[mb][4 * c + 3]);
      } else {
        const float inv = row_scale(m, ls);
        const int64_t at = row * p.hq + head;
        uint16_t* out = static_cast<uint16_t*>(p.out) + at * D + 4 * hi;
#pragma unroll
        for (int mb = 0; mb < D / 32; ++mb)
#pragma unroll
          for (int c = 0; c < 4; ++c)
            *reinterpret_cast<uint2*>(out + 32 * mb + 8 * c) =
                make_uint2(pack_bf16x2(o[mb][4 * c] * inv, o[mb][4 * c + 1] * inv),
                           pack_bf16x2(o[mb][4 * c + 2] * inv, o[mb][4 * c + 3] * inv));
        if (p.lse && hi == 0) p.lse[at] = row_lse(m, ls);
      }
    }
    // everyone has read its tiles, which the next unit's go over (stores need not be waited for)
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
  });
}

template <int D>
hipError_t launch_bf16(const TreeAttn& p, void* workspace, hipStream_t stream) {
  const int lg = log2_of(p.hq / p.hkv);
  const TreeCut c = tree_cut(p.batch, p.max_q, p.max_kv, p.hq, p.hkv, true);
  const TreeWs ws = tree_ws(c, p.batch, p.hkv, D, workspace);
  const int64_t blocks = c.blocks ? c.blocks : (int64_t)p.batch * p.hkv * c.tiles;
  const dim3 grid((unsigned)blocks);
  const bool tiny = p.page_log2 < 4;
#define QCF_NARROW(NV)                                                                          \
  do {                                                                                          \
    if (tiny) tree_attn_narrow_kernel<D, NV, true><<<grid, kNW * 64, 0, stream>>>(p, c, ws, lg); \
    else tree_attn_narrow_kernel<D, NV, false><<<grid, kNW * 64, 0, stream>>>(p, c, ws, lg);     \
  } while (0)
#define QCF_WIDE(VG)                                                                            \
  do {                                                                                          \
    if (tiny) tree_attn_wide_kernel<D, VG, true><<<grid, VG * 64, 0, stream>>>(p, c, ws, lg);   \
    else tree_attn_wide_kernel<D, VG, false><<<grid, VG * 64, 0, stream>>>(p, c, ws, lg);       \
  } while (0)
  if (c.vt_log2 == 4) QCF_NARROW(1);
  else if (c.vt_log2 == 5) QCF_NARROW(2);
  else if (c.vt_log2 == 6) QCF_WIDE(2);
  else if (c.vt_log2 == 7) QCF_WIDE(4);
  else QCF_WIDE(8);
#undef QCF_WIDE
#undef QCF_NARROW
  if (c.blocks) launch_tree_merge<uint16_t, D>(p, c, ws, lg, stream);
  return hipGetLastError();
}

}  // namespace

bool tree_attn_fits(int batch, int max_q, int max_kv, int hq, int hkv, bool bf16) {
  const TreeCut c = tree_cut(batch, max_q, max_kv, hq, hkv, bf16);
  return c.blocks || (int64_t)batch * hkv * c.tiles < (int64_t)1 << kGridLog2;  // (up to 512 threads a block)
}

size_t tree_attn_workspace(int batch, int max_q, int max_kv, int hq, int hkv, int head_dim, bool bf16) {
  return tree_ws_layout(tree_cut(batch, max_q, max_kv, hq, hkv, bf16, true), batch, hkv, head_dim).total;
}

hipError_t launch_tree_attn(const TreeAttn& p, bool bf16, int head_dim, void* ws, hipStream_t stream) {
  if (!bf16) return launch_tree_attn_f32(p, head_dim, ws, stream);
  return head_dim == 64 ? launch_bf16<64>(p, ws, stream) : launch_bf16<128>(p, ws, stream);
}

}  // namespace qcf
