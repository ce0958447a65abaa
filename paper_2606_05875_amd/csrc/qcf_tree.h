// Device code shared by the kernels of qcf_tree_attn: how the work is cut over blocks, and which of a
// request's own new rows a row sees.
//
// A unit is a tile of query vectors (rows times the heads that share a KV head) of one request and KV
// head; its work is one step per 64 tokens of the request.  Where every block takes one unit there is
// nothing to plan.  Else the steps of all units, laid end to end (request, KV head, tile), are shared
// evenly over a fixed number of blocks, whatever the requests' lengths: a block takes its share unit by
// unit, and a unit that is cut between blocks is merged from float32 partial results.  Beginning and
// ending a unit costs a block about as much as `start` steps, which stand before each unit's own in the
// shares.  A block has at most two partial results: of a unit that others began (slot 2 x) and of one
// that it begins (slot 2 x + 1).
#pragma once
#include <math.h>

#include <algorithm>

#include "qcf_decode_launch.h"
#include "qcf_device.h"

namespace qcf {

constexpr int kTreeStep = 64;  // tokens per step

struct TreeCut {
  int vt_log2; // query vectors per unit
  int blocks;  // blocks that share the steps, 0: one block per unit
  int start;   // what beginning a unit counts as, in steps
  int tiles;   // units of the longest request per KV head
};

// The workspace of a cut call
struct TreeWs {
  int2* held;        // [batch][hkv][tiles]: the blocks that hold a unit's first and last step
  float2* ml;        // [2 * blocks][vt] running maximum (log2 units) and sum
  float* o;          // [2 * blocks][vt][d]
};

// a value that is the same in every lane, in scalar registers
__device__ __forceinline__ int uni(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uni(int64_t x) {
  return (int64_t)((uint64_t)(uint32_t)uni((int)(x >> 32)) << 32 | (uint32_t)uni((int)x));
}

struct TreeRequest {
  int64_t r0;   // first packed row
  int rows;     // new rows
  int kv, end;  // tokens before them, tokens in all
};

__device__ __forceinline__ TreeRequest tree_request(const TreeAttn& p, int b) {
  TreeRequest q;
  const int r0 = p.cu_q[b], r1 = p.cu_q[b + 1], kv = p.kv_len[b];
  q.r0 = r0;
  q.rows = r0 < 0 ? 0 : (int)max(min(min((int64_t)r1, p.n_rows) - r0, (int64_t)p.max_q), (int64_t)0);
  q.kv = max(kv, 0);
  q.end = (int)min((int64_t)q.kv + q.rows, (int64_t)p.max_kv);
  return q;
}

// the same for a request that is the same in every lane
__device__ __forceinline__ TreeRequest tree_request_uni(const TreeAttn& p, int b) {
  TreeRequest q = tree_request(p, b);
  q.r0 = uni(q.r0);
  q.rows = uni(q.rows);
  q.kv = uni(q.kv);
  q.end = uni(q.end);
  return q;
}

__device__ __forceinline__ int tree_tiles(const TreeRequest& q, int lg, const TreeCut& cut) {
  return (int)((((int64_t)q.rows << lg) + (1 << cut.vt_log2) - 1) >> cut.vt_log2);
}
// steps of one unit: at least one, for the rows that see nothing are written too
__device__ __forceinline__ int tree_steps(const TreeRequest& q) {
  return (int)max(((int64_t)q.end + kTreeStep - 1) / kTreeStep, (int64_t)1);
}

// n / d for n >= 0, d > 0, by the short division where it does
__device__ __forceinline__ int64_t quotient(int64_t n, int d) {
  return (uint64_t)n >> 32 ? n / d : (int64_t)((uint32_t)n / (uint32_t)d);
}

// How `all` steps are shared: block x begins at floor(all x / blocks), so that equal units that fill a
// whole number of blocks each are not cut elsewhere.  A share is four steps or more.
struct TreeShares {
  int64_t all;
  int blocks;
  __device__ __forceinline__ TreeShares(int64_t steps, int most) : all(steps) {
    const int n = (int)min((int64_t)most, steps >> 2);
    blocks = max(n >= 64 ? n & ~7 : n, 1);
  }
  __device__ __forceinline__ int64_t first(int x) const { return quotient(all * x, blocks); }
  // the block whose share holds step s < all
  __device__ __forceinline__ int holder(int64_t s) const {
    int x = all >> 31 ? (int)(s * blocks / all) : (int)quotient(s * blocks, (int)all);
    while (x > 0 && first(x) > s) --x;
    while (first(x + 1) <= s) ++x;
    return x;
  }
  // The block at place i of the grid, in an order that gives each of the 8 XCDs (blocks go to them in
  // turn) consecutive shares: tiles of one request and KV head read the same keys.
  __device__ __forceinline__ int block(int i) const {
    return blocks % 8 == 0 ? (i & 7) * (blocks >> 3) + (i >> 3) : i;
  }
};

// Runs `unit(b, request, g, tile, first, n, steps, slot)` for this block's share: steps first .. first+n-1
// of a unit's `steps`, to be written out whole (slot < 0) or as a partial result.  NT threads.
template <int NT, typename F>
__device__ __forceinline__ void tree_walk(const TreeAttn& p, const TreeCut& cut, const TreeWs& ws, int lg,
                                          F&& unit) {
  int b;
  TreeRequest q;
  int64_t before, s, share1, all = 0;  // steps before request b; the share's next and end; of all requests
  int x = 0;
  if (cut.blocks == 0) {
    const int g = blockIdx.x % p.hkv, rest = blockIdx.x / p.hkv;
    const int tile = rest % cut.tiles;
    b = rest / cut.tiles;
    q = tree_request_uni(p, b);
    const int tiles = tree_tiles(q, lg, cut), steps = tree_steps(q);
    if (tile >= tiles) return;
    before = 0;
    s = (int64_t)(g * tiles + tile) * steps;
    share1 = s + steps;
  } else {
    __shared__ int64_t sum_l[NT + 1];  // steps before each thread's requests
    __shared__ int64_t wave_l[NT / 64];
    __shared__ int4 req_l[NT];         // its first request
    const int tid = threadIdx.x, lane = tid & 63;
    const int per = (p.batch + NT - 1) / NT;
    auto cost = [&](const TreeRequest& r) {
      return (int64_t)p.hkv * tree_tiles(r, lg, cut) * (tree_steps(r) + cut.start);
    };
    int64_t own = 0;
    for (int i = tid * per; i < min((tid + 1) * per, p.batch); ++i) {
      const TreeRequest r = tree_request(p, i);
      own += cost(r);
      if (i == tid * per) req_l[tid] = make_int4((int)r.r0, r.rows, r.kv, r.end);
    }
    int64_t sum = own;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int64_t y = __shfl_up(sum, o, 64);
      if (lane >= o) sum += y;
    }
    if (lane == 63) wave_l[tid >> 6] = sum;
    __syncthreads();
    for (int i = 0; i < tid >> 6; ++i) sum += wave_l[i];
    sum_l[tid] = sum - own;
    if (tid == NT - 1) sum_l[NT] = sum;
    __syncthreads();
    const TreeShares shares(uni(sum_l[NT]), cut.blocks);
    if ((int)blockIdx.x >= shares.blocks || shares.all == 0) return;
    x = shares.block(blockIdx.x);
    s = shares.first(x);
    share1 = shares.first(x + 1);
    // the last thread whose requests start at or before s: each lane looks at one of a wave's
    int lo = 0;
#pragma unroll
    for (int i = 0; i < NT; i += 64) lo += __builtin_popcountll(__ballot(sum_l[i + lane] <= s));
    lo = max(lo - 1, 0);
    b = lo * per;
    before = uni(sum_l[lo]);
    const int4 r = req_l[lo];
    q.r0 = uni(r.x);
    q.rows = uni(r.y);
    q.kv = uni(r.z);
    q.end = uni(r.w);
    all = shares.all;
  }
  const int start = cut.blocks ? cut.start : 0;
  while (s < share1) {
    const int steps = tree_steps(q), tiles = tree_tiles(q, lg, cut);
    const int64_t cq = (int64_t)p.hkv * tiles * (steps + start);
    if (before + cq <= s) {  // (ends: the requests' costs sum to more than s)
      before += cq;
      q = tree_request_uni(p, ++b);
      continue;
    }
    const int64_t u = quotient(s - before, steps + start), u0 = before + u * (steps + start);
    const int64_t to = min(u0 + start + steps, share1);
    const int first = (int)max(s - u0 - start, (int64_t)0), n = (int)(to - u0 - start) - first;
    if (n > 0) {
      const int g = uni((int)quotient(u, tiles)), tile = uni((int)(u - (int64_t)g * tiles));
      if (cut.blocks && first == 0 && threadIdx.x == 0) {
        const TreeShares shares(all, cut.blocks);
        ws.held[((int64_t)b * p.hkv + g) * cut.tiles + tile] =
            make_int2(x, n == steps ? x : shares.holder(u0 + start + steps - 1));
      }
      // (uniform values that passed the vector units' division would be taken for vectors', and with them
      // the block table's entries: loads that a wait for copies in flight would follow)
      unit(uni(b), q, g, tile, uni(first), uni(n), uni(steps), n == steps ? -1 : uni(2 * x + (first > 0 ? 0 : 1)));
    }
    s = to;
  }
}

// Bits of the W (<= 32) tokens from t0 on that row `row` (index i of its request) sees, as far as the new
// rows' own tokens go; the tokens before them are all seen.  Tokens at and behind `end` are not.
template <int W>
__device__ __forceinline__ uint32_t tree_sees(const TreeAttn& p, const TreeRequest& q, int64_t row, int i, int t0) {
  constexpr uint32_t kAll = W == 32 ? 0xffffffffu : (1u << W) - 1u;
  const int left = q.end - t0;  // > 0
  const uint32_t in = left >= W ? kAll : (1u << left) - 1u;
  const int j = t0 - q.kv;  // index of the first token among the new rows' own
  if (j + W <= 0) return in;
  uint32_t own;
  if (p.tree_mask) {
    const uint32_t* m = p.tree_mask + row * p.mask_words;
    const int w = j >> 5, sh = j & 31;  // (rounds down: w = -1 for -32 <= j < 0)
    const uint64_t lo = w >= 0 && w < p.mask_words ? m[w] : 0u;
    const uint64_t hi = w + 1 >= 0 && w + 1 < p.mask_words ? m[w + 1] : 0u;
    own = (uint32_t)((hi << 32 | lo) >> sh);
  } else {
    const int n = i - j + 1;  // tokens j .. i
    own = n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u;
  }
  if (j < 0) own |= (1u << -j) - 1u;  // (-j < W <= 32)
  return own & in;
}

// a running maximum as the reference of exponentials: 0 while nothing has been seen
__device__ __forceinline__ float finite(float m) { return m == -INFINITY ? 0.f : m; }

// A row whose maximum stays -infinity either saw no token, and gives zeros, or only logits of -infinity or NaN,
// and is NaN, as 0 / 0 is.  Its sum tells: while the maximum is -infinity, a tile with tokens that it sees adds 1 (or
// the NaN), which the factor of a later, finite maximum turns to nothing.
__device__ __forceinline__ float gap(float m, float to) { return m == to ? 0.f : m - to; }  // exponent of that factor
__device__ __forceinline__ float row_scale(float m, float l) {
  return m != -INFINITY ? 1.f / l : l == 0.f ? 0.f : __builtin_nanf("");
}
__device__ __forceinline__ float row_lse(float m, float l) {
  return m != -INFINITY ? (m + log2f(l)) * kLn2 : l == 0.f ? -INFINITY : __builtin_nanf("");
}

typedef const int32_t __attribute__((address_space(4))) * const_i32;

// The page of 16 tokens from t0 on (t0 a multiple of 16, pages of 16 rows and more), or -1
__device__ __forceinline__ int page_of(const TreeAttn& p, const_i32 table, int t0, int end) {
  const int pg = t0 >> p.page_log2;
  if (t0 >= end || pg >= p.max_pages) return -1;
  const int page = uni(table[pg]);
  return page < p.n_pages ? max(page, -1) : -1;
}

// Pages of fewer than 16 rows: the slot of a lane's token, or -1
__device__ __forceinline__ int64_t slot_of(const TreeAttn& p, int b, int t, int end) {
  const int pg = t >> p.page_log2;
  if (t >= end || pg >= p.max_pages) return -1;
  const int page = p.block_table[b * p.table_stride + pg];
  return page >= 0 && page < p.n_pages ? ((int64_t)page << p.page_log2) + (t & ((1 << p.page_log2) - 1)) : -1;
}

namespace {

__device__ __forceinline__ void store4(uint16_t* p, const float4& a) {
  *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(a.x, a.y), pack_bf16x2(a.z, a.w));
}
__device__ __forceinline__ void store4(float* p, const float4& a) { *reinterpret_cast<float4*>(p) = a; }

// The partial results of a unit that is cut between blocks, in the blocks' order: one wave per row and
// head (those whose unit one block took whole have nothing to do).  Lane j first takes the maximum and sum of
// partial j, then 64 / (D / 4) partials at a time are read and summed, whose sums meet at the end.
// Bound: latency (three loads that wait for each other; 64 rows of 32 heads 5 us), or the partials' bytes (64
// rows of 64 heads in 512 pieces, 34 MB: 9 us).
constexpr int kMergeWaves = 4;
template <typename T, int D>
__global__ __launch_bounds__(kMergeWaves * 64) void tree_attn_merge_kernel(TreeAttn p, TreeCut cut, TreeWs ws, int lg) {
  constexpr int LPR = D / 4, RPW = 64 / LPR, U = 8;
  const int l = threadIdx.x & 63, lc = l % LPR, lr = l / LPR;
  const int64_t block = (int64_t)blockIdx.y << kGridLog2 | blockIdx.x;
  const int64_t item = block * kMergeWaves + uni((int)threadIdx.x >> 6);
  if (item >= (int64_t)p.batch * p.max_q * p.hq) return;
  const int64_t bi = quotient(item, p.hq);
  const int h = (int)(item - bi * p.hq);
  const int b = (int)quotient(bi, p.max_q), i = (int)(bi - (int64_t)b * p.max_q);
  const int g = h >> lg, vec = (i << lg) + (h & ((1 << lg) - 1));
  const int tile = vec >> cut.vt_log2, v = vec - (tile << cut.vt_log2);
  const int2 held = ws.held[((int64_t)b * p.hkv + g) * cut.tiles + tile];
  const TreeRequest q = tree_request(p, b);
  if (i >= q.rows) return;
  const int x0 = uni(held.x), x1 = uni(held.y);
  if (x0 == x1) return;
  auto slot = [&](int x) { return ((int64_t)(2 * x + (x == x0 ? 1 : 0)) << cut.vt_log2) + v; };
  const float4* part = reinterpret_cast<const float4*>(ws.o);
  float mx = -INFINITY, lt = 0.f;
  float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int xb = x0; xb <= x1; xb += 64) {
    const int n = min(64, x1 - xb + 1);
    const float2 ml = l < n ? ws.ml[slot(xb + l)] : make_float2(-INFINITY, 0.f);
    const float mn = fmaxf(mx, wave_max(ml.x));
    const float f = __builtin_amdgcn_exp2f(gap(ml.x, mn)), fa = __builtin_amdgcn_exp2f(gap(mx, mn));
    lt = lt * fa + wave_sum(ml.y * f);
    mx = mn;
    a.x *= fa;
    a.y *= fa;
    a.z *= fa;
    a.w *= fa;
    for (int j0 = 0; j0 < n; j0 += U * RPW) {
      float4 o[U];
#pragma unroll
      for (int k = 0; k < U; ++k) o[k] = part[slot(xb + min(j0 + k * RPW + lr, n - 1)) * LPR + lc];
#pragma unroll
      for (int k = 0; k < U; ++k) {
        const int j = j0 + k * RPW + lr;
        const float fo = __shfl(f, min(j, 63), 64);
        if (j >= n) continue;
        a.x = fmaf(o[k].x, fo, a.x);
        a.y = fmaf(o[k].y, fo, a.y);
        a.z = fmaf(o[k].z, fo, a.z);
        a.w = fmaf(o[k].w, fo, a.w);
      }
    }
  }
#pragma unroll
  for (int m = LPR; m < 64; m <<= 1) {
    a.x += __shfl_xor(a.x, m, 64);
    a.y += __shfl_xor(a.y, m, 64);
    a.z += __shfl_xor(a.z, m, 64);
    a.w += __shfl_xor(a.w, m, 64);
  }
  const float inv = row_scale(mx, lt);
  const int64_t at = (q.r0 + i) * p.hq + h;
  if (lr == 0)
    store4(static_cast<T*>(p.out) + at * D + 4 * lc, make_float4(a.x * inv, a.y * inv, a.z * inv, a.w * inv));
  if (p.lse && l == 0) p.lse[at] = row_lse(mx, lt);
}

inline int log2_of(int x) { return __builtin_ctz((unsigned)x); }

// How a call is cut, from its bounds (lengths are on the device).
//
// Vectors per unit: the fewest that hold a request's, up to 128, since padded ones cost their products (16
// requests of 2000 to 12700 tokens, 32/8 heads of 128: 16 vectors 98 us as 16, 101 as 32, 109 as 128; 64
// vectors 113 as 64, 122 as 128), and more than a unit holds read the keys again (128 vectors: 140 as 128, 173
// as 64; only where all keys stay in the caches is that less, one request of 32896 tokens: 52 and 47).
// Units of 256, which take a CU each, where every CU has 32 steps of KV heads' keys or more and units are cut (160
// vectors: 16 such requests 152 us against 188 as 128, 6 requests 69 against 79; fewer steps lose: 192 vectors
// of one request of 32896 tokens 58 against 53, 64 requests of up to 1980 tokens 140 against 130).  At head size
// 64, where registers too leave one such block per CU: 160 vectors of 16 requests 100 us against 103, of 64 requests
// 359 against 444, of 6 requests 45 against 47; requests of 8 to 40 rows, whose units such bounds leave half empty,
// lose there (95 against 77; at 128 they gain or lose 3%), and the bounds do not tell them apart.  float32
// blocks hold 16 vectors.
//
// Short units are taken whole, one per block: up to 8 steps always (64 decoded rows over up to 500 tokens:
// 21.5 us against 27.0 cut), up to 32 where there is one for every CU (256 units of up to 2000 tokens: 41.6 against
// 47.2; 128 units: 27.8 against 25.2; float32 units, whose steps take longer, not).  Else as many blocks as run at
// once, two per CU (trees, units of 128: 256 blocks 152 us, 512 142, 768 157), with 4 steps each at least.
// `start` 4: 209, 203, 205 us with 0, 4, 8 for 64 decoded rows over 512 to 8192 tokens.
//
// The workspace is sized as if units for every CU were cut too and no unit held 256 (`cut_all`; 256 blocks of
// 256 vectors need what 512 of 128 do): it then grows with every bound, and one for the largest batch serves
// smaller ones.
constexpr int kTreeBlocks = 512;
inline TreeCut tree_cut(int batch, int max_q, int max_kv, int hq, int hkv, bool bf16, bool cut_all = false) {
  const int64_t vectors = (int64_t)max_q * (hq / hkv);
  const int64_t steps = ((int64_t)max_kv + kTreeStep - 1) / kTreeStep;
  const bool cu_wide = vectors > 128 && steps > 32 && (int64_t)batch * hkv * steps >= 16 * kTreeBlocks && !cut_all;
  const int vt = vectors <= 16 || !bf16 ? 16 : vectors <= 32 ? 32 : vectors <= 64 ? 64 : cu_wide ? 256 : 128;
  TreeCut c;
  c.vt_log2 = log2_of(vt);
  c.tiles = (int)((vectors + vt - 1) / vt);
  const int64_t units = (int64_t)batch * hkv * c.tiles;
  c.blocks = 0;
  c.start = 4;
  if (steps > 32 || (steps > 8 && (units < kTreeBlocks / 2 || !bf16 || cut_all)))
    c.blocks = (int)std::max<int64_t>(std::min<int64_t>(vt == 256 ? kTreeBlocks / 2 : kTreeBlocks, units * steps / 4), 1);
  return c;
}

struct TreeWsLayout {
  size_t ml, o, total;
};
inline TreeWsLayout tree_ws_layout(const TreeCut& c, int batch, int hkv, int d) {
  const auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  TreeWsLayout w{};
  if (c.blocks == 0) return w;
  w.ml = up((size_t)batch * hkv * c.tiles * sizeof(int2));
  w.o = w.ml + up(((size_t)2 * c.blocks << c.vt_log2) * 8);
  w.total = w.o + up(((size_t)2 * c.blocks << c.vt_log2) * d * 4);
  return w;
}

inline TreeWs tree_ws(const TreeCut& c, int batch, int hkv, int d, void* workspace) {
  const TreeWsLayout w = tree_ws_layout(c, batch, hkv, d);
  char* base = static_cast<char*>(workspace);
  return TreeWs{reinterpret_cast<int2*>(base), reinterpret_cast<float2*>(base + w.ml),
                reinterpret_cast<float*>(base + w.o)};
}

template <typename T, int D>
inline void launch_tree_merge(const TreeAttn& p, const TreeCut& c, const TreeWs& ws, int lg, hipStream_t stream) {
  const int64_t rows = (int64_t)p.batch * p.max_q * p.hq;
  tree_attn_merge_kernel<T, D><<<grid_of((rows + kMergeWaves - 1) / kMergeWaves), kMergeWaves * 64, 0, stream>>>(p, c, ws, lg);
}

}  // namespace

}  // namespace qcf
