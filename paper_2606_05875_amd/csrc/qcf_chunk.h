// Device code shared by the kernels of qcf_chunk_attn: which tokens a tile of rows sees, and how the work is
// cut over blocks.
//
// A unit is a tile of query vectors (rows times the heads that share a KV head) of one request and KV
// head; its work is one step per 64 tokens between the first that its first row sees and the last one's own.
// Tiles hold a power of two of rows, so the steps of a request's first tiles have a closed form, and
// every block finds its share of all steps by itself.  The steps of all units, laid end to end (request, KV
// head, tile), are shared evenly over a fixed number of blocks; a unit that is cut between blocks is
// merged from float32 partial results.  Beginning and ending a unit counts as `start` steps in the
// shares.  A block has at most two partial results: of a unit that others began (slot 2 x) and of one
// that it begins (slot 2 x + 1), which it enters in a list for the merge.
#pragma once
#include <type_traits>

#include "qcf_tree.h"
#include "qcf_turns_launch.h"

namespace qcf {

constexpr int kChunkStep = 64;  // tokens per step

struct ChunkCut {
  int vt_log2;  // query vectors per unit
  int blocks;   // blocks that share the steps
  int start;    // what beginning a unit counts as, in steps
  int tiles;    // units of the longest request per KV head
};

struct ChunkWs {
  int4* cut;   // [blocks] of the unit that a block begins and others end: first row, rows, KV head, last block; 0 rows: none
  float2* ml;  // [2 * blocks][vt] running maximum (log2 units) and sum
  float* o;    // [2 * blocks][vt][d]
};

// Work of one request per KV head.  Lengths beyond the caller's bound (whose tokens are not seen) count as that.
struct ChunkCost {
  int64_t kv, rows;
  int tiles, rl;  // rows per tile, as a power of two
  int window, start;

  __device__ __forceinline__ ChunkCost(const ChunkAttn& p, const TreeRequest& q, int lg, const ChunkCut& cut) {
    kv = min(q.kv, p.max_kv);
    rows = q.rows;
    rl = cut.vt_log2 - lg;
    tiles = (int)((rows + (1 << rl) - 1) >> rl);
    window = p.window;
    start = cut.start;
  }
  // sum over i < n of floor((a + i * 2^rl) / 64), a >= 0
  __device__ __forceinline__ int64_t floors(int64_t a, int64_t n) const {
    if (rl >= 6) return n * (a >> 6) + ((n * (n - 1) / 2) << (rl - 6));
    const int ml = 6 - rl;
    const auto below = [&](int64_t x) {  // sum over i < x of floor(i / 2^ml)
      const int64_t q = x >> ml, r = x & ((1 << ml) - 1);
      return ((q * (q - 1) / 2) << ml) + q * r;
    };
    return below((a >> rl) + n) - below(a >> rl);
  }
  // the first step of a tile, and the one behind its last
  __device__ __forceinline__ int64_t first(int tile) const {
    return window ? max(kv + ((int64_t)tile << rl) - window + 1, (int64_t)0) >> 6 : 0;
  }
  __device__ __forceinline__ int64_t last(int tile) const {
    return (kv + min((int64_t)(tile + 1) << rl, rows) + 63) >> 6;
  }
  // steps of the first n <= tiles tiles, with their starts
  __device__ __forceinline__ int64_t before(int n) const {
    if (n == 0) return 0;
    int64_t s = floors(kv + (1 << rl) + 63, min(n, tiles - 1)) + (int64_t)start * n;
    if (n == tiles) s += last(tiles - 1);
    if (window) {
      const int64_t a = kv - window + 1;
      const int64_t i0 = a >= 0 ? 0 : min((int64_t)n, ((1 << rl) - 1 - a) >> rl);
      s -= floors(a + (i0 << rl), n - i0);
    }
    return s;
  }
};

// Runs `unit(b, request, g, tile, first, n, slot)` for this block's share: steps first .. first+n-1 (of 64
// tokens, counted from token 0) of a unit, to be written out whole (slot < 0) or as a partial result.  NT threads.
template <int NT, typename F>
__device__ __forceinline__ void chunk_walk(const ChunkAttn& p, const ChunkCut& cut, const ChunkWs& ws, int lg,
                                           F&& unit) {
  __shared__ int64_t sum_l[NT + 1];  // steps before each thread's requests
  __shared__ int64_t wave_l[NT / 64];
  const int tid = threadIdx.x, lane = tid & 63;
  const int per = (p.batch + NT - 1) / NT;
  int64_t own = 0;
  for (int i = tid * per; i < min((tid + 1) * per, p.batch); ++i) {
    const ChunkCost c(p, tree_request(p, i), lg, cut);
    own += p.hkv * c.before(c.tiles);
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
  const bool works = (int)blockIdx.x < shares.blocks && shares.all > 0;
  const int x = works ? shares.block(blockIdx.x) : (int)blockIdx.x;
  if (tid == 0) ws.cut[x] = make_int4(0, 0, 0, 0);
  if (!works) return;
  int64_t s = shares.first(x);
  const int64_t share1 = shares.first(x + 1);
  // the last thread whose requests start at or before s: each lane looks at one of a wave's
  int lo = 0;
#pragma unroll
  for (int i = 0; i < NT; i += 64) lo += __builtin_popcountll(__ballot(sum_l[i + lane] <= s));
  lo = max(lo - 1, 0);
  int b = lo * per;
  int64_t before = uni(sum_l[lo]);
  while (s < share1) {  // (ends: the requests' costs sum to more than s)
    const TreeRequest q = tree_request_uni(p, b);
    const ChunkCost c(p, q, lg, cut);
    const int64_t head = c.before(c.tiles), all = p.hkv * head;
    if (before + all <= s) {
      before += all;
      ++b;
      continue;
    }
    int g = (int)((s - before) / head);
    int64_t h0 = before + g * head;  // where the KV head begins
    int tile = 0;
    for (int n = c.tiles; n > 1;) {  // the last tile that begins at or before s
      const int half = n >> 1;
      if (h0 + c.before(tile + half) <= s) tile += half, n -= half;
      else n = half;
    }
    while (s < share1 && g < p.hkv) {
      const int64_t u0 = h0 + c.before(tile), u1 = h0 + c.before(tile + 1);
      const int64_t to = min(u1, share1);
      const int steps = (int)(u1 - u0) - c.start;
      const int first = (int)max(s - u0 - c.start, (int64_t)0), n = (int)(to - u0) - c.start - first;
      if (n > 0) {
        if (first == 0 && n < steps && tid == 0) 
          ws.cut[x] = make_int4((int)(q.r0 + (tile << c.rl)), (int)min((int64_t)1 << c.rl, c.rows - ((int64_t)tile << c.rl)), g, shares.holder(u1 - 1));
        unit(uni(b), q, uni(g), uni(tile), uni((int)c.first(tile) + first), uni(n),
             n == steps ? -1 : uni(2 * x + (first > 0 ? 0 : 1)));
      }
      s = to;
      if (s == u1 && ++tile == c.tiles) {
        tile = 0;
        h0 += head;
        ++g;
      }
    }
  }
}

namespace {

// The partial results of the units that are cut, in the blocks' order.  A thread sums four columns of one query vector of
// the unit that block x0 begins; the first two partials (most units have no more) go out at once, then eight at a time.
// Bound: the partials' bytes, or latency.
constexpr int kMergeThreads = 256;
template <typename T, int D>
__global__ __launch_bounds__(kMergeThreads) void chunk_merge_kernel(ChunkAttn p, ChunkCut cut, ChunkWs ws, int lg) {
  constexpr int LPR = D / 4, VP = kMergeThreads / LPR;  // vectors of a block
  const int x0 = blockIdx.y;  // (the vectors along x: units are begun by blocks of one XCD where they are cut alike)
  const int4 c = ws.cut[x0];
  const int64_t row0 = c.x;
  const int rows = c.y, g = c.z, x1 = c.w;
  const int lc = threadIdx.x % LPR, v = blockIdx.x * VP + threadIdx.x / LPR;
  const int i = v >> lg, h = (g << lg) + (v & ((1 << lg) - 1));
  if (i >= rows) return;
  const float4* part = reinterpret_cast<const float4*>(ws.o);
  float mx = -INFINITY, lt = 0.f;
  float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
  // (float32: subnormal factors are kept, as the weights are in a unit that is not cut)
  auto factor = [](float x) { return std::is_same<T, float>::value ? exp2f(x) : __builtin_amdgcn_exp2f(x); };
  auto add = [&](auto count, int x) {
    constexpr int J = decltype(count)::value;
    float2 ml[J];
    float4 o[J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int y = min(x + j, x1);
      const int64_t at = ((int64_t)(2 * y + (y == x0 ? 1 : 0)) << cut.vt_log2) + v;
      ml[j] = ws.ml[at];
      o[j] = part[at * LPR + lc];
    }
#pragma unroll
    for (int j = 0; j < J; ++j) {
      if (x + j > x1) break;
      const float mn = fmaxf(mx, ml[j].x);
      const float fa = factor(gap(mx, mn)), fo = factor(gap(ml[j].x, mn));
      mx = mn;
      lt = fmaf(lt, fa, ml[j].y * fo);
      a.x = fmaf(a.x, fa, o[j].x * fo);
      a.y = fmaf(a.y, fa, o[j].y * fo);
      a.z = fmaf(a.z, fa, o[j].z * fo);
      a.w = fmaf(a.w, fa, o[j].w * fo);
    }
  };
  add(std::integral_constant<int, 2>{}, x0);
  for (int x = x0 + 2; x <= x1; x += 8) add(std::integral_constant<int, 8>{}, x);
  const float inv = row_scale(mx, lt);
  const int64_t at = (row0 + i) * p.hq + h;
  store4(static_cast<T*>(p.out) + at * D + 4 * lc, make_float4(a.x * inv, a.y * inv, a.z * inv, a.w * inv));
  if (p.lse && lc == 0) p.lse[at] = row_lse(mx, lt);
}

// How a call is cut, from its bounds (lengths are on the device): tiles of 128 vectors (float32: 32), as many
// blocks as run at once, two per CU.  (Three of head size 64, whose registers would do: 234 us against 233 for
// prompts of 700 to 4000 rows with windows of 1024: the vector units are busy with two.)
constexpr int kChunkBlocks = 512;
inline ChunkCut chunk_cut(int max_q, int hq, int hkv, bool bf16) {
  const int64_t vectors = (int64_t)max_q * (hq / hkv);
  ChunkCut c;
  c.vt_log2 = bf16 ? 7 : 5;
  c.tiles = (int)((vectors + (1 << c.vt_log2) - 1) >> c.vt_log2);
  c.start = 6;  // (what it costs in steps: windows of 1024 252, 233, 233, 232 us with 2, 4, 6, 9; 16 questions 252, 250, 250, 248)
  c.blocks = kChunkBlocks;
  return c;
}

struct ChunkWsLayout {
  size_t ml, o, total;
};
inline ChunkWsLayout chunk_ws_layout(const ChunkCut& c, int d) {
  const auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  ChunkWsLayout w{};
  w.ml = up((size_t)c.blocks * sizeof(int4));
  w.o = w.ml + up(((size_t)2 * c.blocks << c.vt_log2) * 8);
  w.total = w.o + up(((size_t)2 * c.blocks << c.vt_log2) * d * 4);
  return w;
}

inline ChunkWs chunk_ws(const ChunkCut& c, int d, void* workspace) {
  const ChunkWsLayout w = chunk_ws_layout(c, d);
  char* base = static_cast<char*>(workspace);
  return ChunkWs{reinterpret_cast<int4*>(base), reinterpret_cast<float2*>(base + w.ml),
                 reinterpret_cast<float*>(base + w.o)};
}

template <typename T, int D>
inline void launch_chunk_merge(const ChunkAttn& p, const ChunkCut& c, const ChunkWs& ws, int lg, hipStream_t stream) {
  chunk_merge_kernel<T, D><<<dim3((1u << c.vt_log2) / (kMergeThreads / (D / 4)), (unsigned)c.blocks), kMergeThreads, 0, stream>>>(p, c, ws, lg);
}

}  // namespace

}  // namespace qcf
