// Attention of a chunk of new rows of each request over its paged cache (qcf_chunk_attn), bf16.
//
// One pass over the tokens with the softmax's running maximum m and sum l per query vector: S = K Q^T, p =
// exp2(S - m), O = O alpha + V^T p^T, on v_mfma_f32_32x32x16_bf16.  Products are transposed, as in the other
// attention kernels of this library: a lane holds tokens' logits of ONE query vector, so its p are the
// second product's operand as they stand: one bf16 number each, 2^-8 of it off at most, after they entered the sum in
// float32 (a second number for the rest, as the tree kernel has for few vectors, would be half as many products again).
// A wave holds 32 query vectors (consecutive rows times the heads
// that share a KV head), the 4 waves of a block share every 64-token tile, and the products of the next
// tile's S run beside this tile's exponentials.
//
// Keys and values go from the pages into LDS without passing registers, two stages of each: step t asks for
// K(t+2) and V(t+1) before anything else and ends by waiting for them (in between the products of S(t+1), as the contiguous
// kernels do, the 16 questions below took 2% longer: pages are rarely in the L2).  Wave w copies the tile's
// rows 16 w .. + 15, which lie in one page; the page numbers of a tile's four groups come by one load, a step
// ahead of the copies.
// Two blocks per CU: one's products run beside the other's exponentials, starts and ends.
// Bound: matrix units and vector units together, where tiles are whole and long: 2048 rows over 30848 tokens, 64/8
// heads of 128, 2022 to 2082 us from card to card, 1.03 to 1.06 PFLOP/s.  16 questions of 16 to 128 rows over 2000 to
// 12700 tokens (32/8 heads) 246 to 250 us, 0.67 PFLOP/s: tiles of 32 rows are rounded up, units of a few tiles start
// and end, some are merged, and a fifth is waiting for pages (191 us with all tokens in the same few).  Head size 64
// does half the products per exponential: prompts of 700 to 4000 rows with windows of 1024, 225 to 233 us, 0.52
// PFLOP/s.  64 single rows in such windows (32/8 heads of 128) 77 us, 3.5 TB/s: a tile of 128 vectors holds 4.
#include "qcf_chunk.h"
#include "qcf_paged.h"

namespace qcf {
namespace {

constexpr int kW = 4;            // waves per block
constexpr int kVt = 32 * kW;     // query vectors per block
constexpr int kT = kChunkStep;   // tokens per tile

template <int D>
__global__ __launch_bounds__(kW * 64, 2) void chunk_attn_kernel(ChunkAttn p, ChunkCut cut, ChunkWs ws, int lg) {
  constexpr int CH = D / 8;     // 16-byte chunks per row
  constexpr int RPC = 64 / CH;  // rows per copy
  constexpr int RB = D * 2;     // bytes per row
  constexpr int TB = kT * RB;   // bytes of a tile of K or V
  constexpr int GC = 16 / RPC;  // copies per wave and tile, K or V
  constexpr int NS = D / 16;    // products per 32 tokens of S
  __shared__ __attribute__((aligned(1024))) uint8_t k_ring[2 * TB];
  __shared__ __attribute__((aligned(1024))) uint8_t v_ring[2 * TB];
  __shared__ uint32_t loose_l[2];

  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l = threadIdx.x & 63, lq = l & 31, hi = l >> 5;
  const uint32_t k_lds = lds_addr(k_ring), v_lds = lds_addr(v_ring);
  const uint32_t row_b = (uint32_t)(p.kv_stride * 2);
  const float scale2 = p.scale * kLog2e;
  // Chunk c of K row r sits at c ^ (r % 16) (D = 64: c ^ (r / 2 % 8)), of V row r at c ^ 4 (r % 4)
  // (D = 64: c ^ 4 (r / 2 % 2)): lane fragments st at krd ^ (st << 5), V column blocks mb at vrd ^ (mb << 6)
  const int ky = D == 128 ? lq & 15 : (lq >> 1) & 7;
  const int krd = lq * RB + (hi ^ (ky & 1)) * 16 + (ky >> 1) * 32;
  const int tg = l >> 4, te = (l >> 2) & 3, tq = l & 3;
  const int vrd = (4 * (tg >> 1) + te) * RB + (D == 128 ? te : te >> 1) * 64 + 32 * (tg & 1) + 8 * tq;
  // copy i of a wave fills rows 16 w + RPC i + l / CH: the row within the copy and the chunk of K, V before
  // i's part of the exchange (which i's bits give by themselves)
  const int cr = l / CH, cc = l % CH;
  uint32_t coff = cr * row_b, kx = (cc ^ (D == 128 ? cr : cr >> 1)) * 16;
  const uint32_t vx = (cc ^ (4 * (D == 128 ? cr : (cr >> 1) & 1))) * 16;

  if (threadIdx.x < 2) loose_l[threadIdx.x] = 0;
  chunk_walk<kW * 64>(p, cut, ws, lg, [&](int b, const TreeRequest& rq, int g, int tile, int first, int n, int slot) {
    const int32_t* table = p.block_table + b * p.table_stride;
    const char* kc = static_cast<const char*>(p.k_cache) + (int64_t)g * RB;
    const char* vc = static_cast<const char*>(p.v_cache) + (int64_t)g * RB;
    const bool pool = p.n_pages > 0;
    const int t_first = first * kT;
    // Page numbers of a tile's groups: lane i (i < 4) looks up group i
    auto look = [&](int t) {
      const int at = t_first + t * kT + 16 * (l & 3);
      return pool ? table[min(at >> p.page_log2, p.max_pages - 1)] : -1;
    };
    // the groups of a tile that are there, as bits, and this wave's page (or -1)
    auto pages_of = [&](int t, int x, int& page) {
      const int at = t_first + t * kT + 16 * (l & 3);
      const bool ok = t < n && at < rq.end && at >> p.page_log2 < p.max_pages && x >= 0 && x < p.n_pages;
      page = __builtin_amdgcn_readlane(ok ? x : -1, w);
      return (int)__ballot(ok) & 15;
    };
    // copy i of this wave's part of K (V) of tile t into its stage; without a page the pool's first rows
    // stand in and are not seen
    auto base_of = [&](int t, int page) {
      const int t0 = t_first + t * kT + 16 * w;
      const uint32_t row = page < 0 ? 0u : ((uint32_t)page << p.page_log2) + (t0 & ((1 << p.page_log2) - 1));
      return (uint64_t)row * row_b;
    };
    auto copy_k = [&](int t, uint64_t at, int i) {
      asm volatile("" : "+v"(coff), "+v"(kx));  // (formed anew: every copy's offset kept is a register each)
      const uint32_t c = kx ^ (i * 64);
      copy16(kc + at, coff + i * RPC * row_b + c, k_lds + (t & 1) * TB + (w * GC + i) * 1024);
    };
    auto copy_v = [&](int t, uint64_t at, int i) {
      asm volatile("" : "+v"(coff));
      copy16(vc + at, coff + i * RPC * row_b + vx, v_lds + (t & 1) * TB + (w * GC + i) * 1024);
    };

    const int v0 = tile * kVt + 32 * w;  // this wave's first vector
    const int idx = (v0 + lq) >> lg;
    const int head = (g << lg) + ((v0 + lq) & ((1 << lg) - 1));
    const bool valid = idx < rq.rows;
    const bool busy = (v0 >> lg) < rq.rows;  // (the wave has a vector)
    const int ridx = min(idx, rq.rows - 1);
    const int64_t row = rq.r0 + ridx;
    bf16x8 qreg[D / 16];
    {
      const uint16_t* q = static_cast<const uint16_t*>(p.q) + (row * p.hq + head) * D + 8 * hi;
#pragma unroll
      for (int st = 0; st < D / 16; ++st) qreg[st] = as_bf16x8(ld16(q + 16 * st));
    }
    // tokens that row i of the request sees: from low(i) up to high(i)
    auto low = [&](int i) {
      return p.window ? (int)min(max((int64_t)rq.kv + i - p.window + 1, (int64_t)0), (int64_t)INT32_MAX) : 0;
    };
    auto high = [&](int i) { return (int)min((int64_t)rq.kv + i + 1, (int64_t)rq.end); };
    const int iw0 = min(v0 >> lg, rq.rows - 1), iw1 = min((v0 + 31) >> lg, rq.rows - 1);
    const int w_lo = low(iw0), w_hi = high(iw1);        // tokens that some row of the wave sees
    const int all_lo = low(iw1), all_hi = high(iw0);    // .. that all do
    const int ib0 = (tile * kVt) >> lg, ib1 = min((tile * kVt + kVt - 1) >> lg, rq.rows - 1);
    const int plain_lo = low(ib1), plain_hi = high(ib0);  // .. that all of the block do
    const int r_lo = low(ridx), r_hi = high(ridx);

    int page1, page2;            // this wave's pages of tiles t + 1 (its V) and t + 2 (its K)
    int there0, there1, there2;  // groups that are there, tiles t, t + 1, t + 2
    int next;                    // page numbers of tile t + 3, as loaded
    {
      const int x0 = look(0), x1 = look(1), x2 = look(2);
      int page0;
      there0 = pages_of(0, x0, page0);
      there1 = pages_of(1, x1, page1);
      there2 = pages_of(2, x2, page2);
      // Q has to be there before the copies: a wait for it later would count those in flight
#pragma unroll
      for (int st = 0; st < D / 16; ++st) asm volatile("" : "+v"(qreg[st]));
      if (pool) {
        const uint64_t a0 = base_of(0, page0), a1 = base_of(1, page1);
#pragma unroll
        for (int i = 0; i < GC; ++i) copy_k(0, a0, i);
#pragma unroll
        for (int i = 0; i < GC; ++i) copy_v(0, a0, i);
#pragma unroll
        for (int i = 0; i < GC; ++i) copy_k(1, a1, i);
      }
    }
    f32x16 o[D / 32];
#pragma unroll
    for (int mb = 0; mb < D / 32; ++mb) o[mb] = f32x16{};
    float m = -INFINITY, ls = 0.f;  // running maximum in log2 units, this lane's part of the sum
    bool big = false;

    auto meet = [&]() {  // every copy and LDS access so far is complete, then the block meets
      asm volatile("" ::: "memory");
      wait_vm_lgkm0<0>();
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
    };
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
      // lazy rescale: a stale maximum stays unless the vector's grew by more than 2^8 (by each
      // vector's own, so that no row's bits hang on another's)
      if (__ballot(!(mt < m + 8.f))) {  // (no maximum yet: row_scale)
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
    // P of the tile; with kNext S of the next one beside it: one product per fenced group with its K fragment
    // read four groups ahead, a group's arguments, exponentials and sums in three groups in turn
    auto weights = [&](auto next_s, const uint8_t* kn, f32x16 (&sn)[2], f32x16 (&s)[2], bf16x8 (&pb)[2][2]) {
      constexpr bool kNext = decltype(next_s)::value;
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
          const bf16x2_t pk = __builtin_convertvector((f32x2_t){pw[e], pw[e + 1]}, bf16x2_t);
          pb[e >> 4][(e >> 3) & 1][e & 7] = pk[0];
          pb[e >> 4][(e >> 3) & 1][(e & 7) + 1] = pk[1];
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
    auto products_o = [&](const uint8_t* vl, bf16x8 (&pb)[2][2]) {
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
      }
      __builtin_amdgcn_sched_barrier(0);
    };

    // Tiles with tokens that are not there or that some row of the block does not see: rows of V that hold no
    // token become zeros (an unseen value must not meet its weight 0 where it is not finite); the result
    // is the tokens with a value that is not finite, which are added to the rows that see them one by one ..
    auto clean = [&](int t, uint64_t held) {
      uint8_t* vl = v_ring + (t & 1) * TB;
      for (int u = threadIdx.x; u < kT * CH; u += kW * 64) {
        const int r = u / CH;
        if (!(held >> r & 1)) st16(vl + 16 * u, make_uint4(0, 0, 0, 0));
        else if (not_finite(ld16(vl + 16 * u))) atomicOr(&loose_l[r >> 5], 1u << (r & 31));
      }
      __syncthreads();
      return (uint64_t)(uint32_t)uni((int)loose_l[1]) << 32 | (uint32_t)uni((int)loose_l[0]);
    };
    // .. and taken out once everyone has done so
    auto take_out = [&](int t, uint64_t loose) {
      uint8_t* vl = v_ring + (t & 1) * TB;
      __syncthreads();
      for (int u = threadIdx.x; u < kT * CH; u += kW * 64)
        if (loose >> (u / CH) & 1) st16(vl + 16 * u, make_uint4(0, 0, 0, 0));
      if (threadIdx.x < 2) loose_l[threadIdx.x] = 0;  // (zero between tiles)
      __syncthreads();
    };
    auto add_loose = [&](int t, uint64_t loose, uint64_t sees, const f32x16 (&s)[2]) {
      const uint8_t* vl = v_ring + (t & 1) * TB;
      for (uint64_t left = loose; left; left &= left - 1) {
        const int k = __builtin_ctzll(left);
        float a = 0.f;
#pragma unroll
        for (int e = 0; e < 32; ++e) a = (k >> 3) * 4 + (k & 3) == e ? s[e >> 4][e & 15] : a;
        a = __builtin_amdgcn_exp2f(fmaf(a, big ? 1.f : scale2, -finite(m)));
        const float pk = __shfl(a, ((k >> 2) & 1) * 32 + lq, 64);
        if (sees >> k & 1) {
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
    };

    // the wave has a row that sees a token of the tile at t0
    auto uses = [&](int t0) { return busy && t0 < w_hi && t0 + kT > w_lo; };
    auto on = [&](int t) {  // the page numbers move up
      there0 = there1;
      there1 = there2;
      page1 = page2;
      there2 = pages_of(t + 3, next, page2);
    };
    // a tile that all rows of the block see, its next S (into sn) beside it
    auto plain_step = [&](int t, f32x16 (&s)[2], f32x16 (&sn)[2]) {
      next = look(t + 3);
      bf16x8 pb[2][2];
      const uint64_t ak = base_of(t + 2, page2), av = base_of(t + 1, page1);
#pragma unroll
      for (int i = 0; i < GC; ++i) copy_k(t + 2, ak, i);
#pragma unroll
      for (int i = 0; i < GC; ++i) copy_v(t + 1, av, i);
      maximum(s, true);
      __builtin_amdgcn_s_setprio(1);
      weights(std::true_type{}, k_ring + ((t + 1) & 1) * TB, sn, s, pb);
      __builtin_amdgcn_s_setprio(0);
      products_o(v_ring + (t & 1) * TB, pb);
      meet();
      on(t);
    };
    // any tile, its next S (into s) after it
    auto other_step = [&](int t, f32x16 (&s)[2]) {
      const int t0 = t_first + t * kT;
      const bool now = uses(t0), then = t + 1 < n && uses(t0 + kT);
      next = look(t + 3);
      const uint64_t ak = base_of(t + 2, page2), av = base_of(t + 1, page1);
      if (t + 2 < n)
#pragma unroll
        for (int i = 0; i < GC; ++i) copy_k(t + 2, ak, i);
      if (t + 1 < n)
#pragma unroll
        for (int i = 0; i < GC; ++i) copy_v(t + 1, av, i);
      uint64_t held = ~0ull, loose = 0;
      if (t0 + kT > plain_hi || t0 < plain_lo || there0 != 15) {
        held = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (there0 >> i & 1) held |= 0xffffull << (16 * i);
        if (rq.end - t0 < kT) held &= rq.end > t0 ? (1ull << (rq.end - t0)) - 1ull : 0ull;
        loose = clean(t, held);
      }
      if (now) {
        uint64_t sees = ~0ull;
        if (t0 + kT > all_hi || t0 < all_lo || held != ~0ull) {
          const int from = min(max(r_lo - t0, 0), kT), to = min(max(r_hi - t0, 0), kT);
          sees = held & (to < kT ? (1ull << to) - 1ull : ~0ull) & (from < kT ? ~0ull << from : 0ull);
#pragma unroll
          for (int hb = 0; hb < 2; ++hb) {
            const uint32_t mine = (uint32_t)(sees >> (32 * hb)) >> (4 * hi);
#pragma unroll
            for (int v = 0; v < 16; ++v)
              if (!(mine >> (8 * (v >> 2) + (v & 3)) & 1)) s[hb][v] = -INFINITY;
          }
        }
        maximum(s, sees != 0);
        bf16x8 pb[2][2];
        weights(std::false_type{}, k_ring, s, s, pb);
        if (loose) {
          add_loose(t, loose, sees, s);
          take_out(t, loose);
        }
        products_o(v_ring + (t & 1) * TB, pb);
      } else if (loose) {
        take_out(t, loose);
      }
      if (then) products(k_ring + ((t + 1) & 1) * TB, s);
      meet();
      on(t);
    };

    if (pool) {
      // tiles from plain_at on before plain_end are seen by all rows of the block
      const int plain_end = min((plain_hi - t_first) >> 6, n), plain_at = (max(plain_lo - t_first, 0) + kT - 1) >> 6;
      f32x16 sa[2], sb[2];
      meet();
      if (uses(t_first)) products(k_ring, sa);
      meet();  // K(0) has been read before K(2) takes its place
      for (int t = 0; t < n;) {
        if (busy && t >= plain_at) {
          const int end = min(plain_end - 1, n - 2);
          for (; t < end; t += 2) {
            if ((there0 & there1) != 15) break;
            plain_step(t, sa, sb);
            plain_step(t + 1, sb, sa);
          }
        }
        other_step(t++, sa);
      }
    }
    ls += __shfl_xor(ls, 32, 64);
    if (valid) {
      if (slot >= 0) {
        const int64_t at = (int64_t)slot * kVt + 32 * w + lq;
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
  });
}

template <int D>
hipError_t launch_bf16(const ChunkAttn& p, void* workspace, hipStream_t stream) {
  const int lg = log2_of(p.hq / p.hkv);
  const ChunkCut c = chunk_cut(p.max_q, p.hq, p.hkv, true);
  const ChunkWs ws = chunk_ws(c, D, workspace);
  chunk_attn_kernel<D><<<dim3((unsigned)c.blocks), kW * 64, 0, stream>>>(p, c, ws, lg);
  launch_chunk_merge<uint16_t, D>(p, c, ws, lg, stream);
  return hipGetLastError();
}

}  // namespace

bool chunk_attn_fits(int batch, int max_q, int hq, int hkv, bool bf16) {
  const ChunkCut c = chunk_cut(max_q, hq, hkv, bf16);
  const int64_t units = (int64_t)hkv * c.tiles;
  return batch == 0 || units <= INT32_MAX / batch;
}

size_t chunk_attn_workspace(int max_q, int hq, int hkv, int head_dim, bool bf16) {
  return chunk_ws_layout(chunk_cut(max_q, hq, hkv, bf16), head_dim).total;
}

hipError_t launch_chunk_attn(const ChunkAttn& p, bool bf16, int head_dim, void* ws, hipStream_t stream) {
  if (!bf16) return launch_chunk_attn_f32(p, head_dim, ws, stream);
  return head_dim == 64 ? launch_bf16<64>(p, ws, stream) : launch_bf16<128>(p, ws, stream);
}

}  // namespace qcf
