// Requests that continue others, and the pages behind them (qcf_page_fork, qcf_copy_pages, qcf_page_release).
//
// Pages have no holders' counts: a page is held by whoever's table names it, and what nobody's names any
// more is found by marking the pages of the tables before and after a change in two bit sets.  There is
// nothing to keep in step, and no result hangs on the order of blocks.
#include <algorithm>

#include "qcf_device.h"
#include "qcf_turns_launch.h"

namespace qcf {
namespace {

constexpr int kThreads = 256;

// ---------------------------------------------------------------------------
// fork: one block per request, which counts the pages that the requests before it take on its own (three
// dependent loads each, 256 requests at a time).  Bound: latency
// ---------------------------------------------------------------------------
struct ForkRow {
  int source;      // -1: the request ends
  int64_t n;       // tokens
  int64_t full;    // pages that they fill
  int part;        // rows of the page that they start
  int from;        // that page's number at the source where it has to be copied, else -1
};

__device__ __forceinline__ ForkRow fork_row(const PageFork& p, int b) {
  ForkRow f;
  const int s = p.source[b];
  f.source = s >= 0 && s < p.batch ? s : -1;
  f.n = f.source < 0 ? 0 : max(p.kv_len[f.source], 0);
  if (p.keep_len) f.n = min(f.n, (int64_t)max(p.keep_len[b], 0));
  f.full = f.n >> p.page_log2;
  f.part = (int)(f.n & ((1ll << p.page_log2) - 1));
  f.from = -1;
  if (f.part > 0 && f.full < p.max_pages && !(f.source == b && f.full == max(p.kv_len[b], 0) >> p.page_log2)) {
    const int page = p.block_table[(int64_t)f.source * p.table_stride + f.full];
    if (page >= 0 && page < p.n_pages) f.from = page;
  }
  return f;
}

__global__ __launch_bounds__(kThreads) void page_fork_kernel(PageFork p) {
  __shared__ int taken_l[kThreads / 64];
  const int tid = threadIdx.x, b = blockIdx.x;
  const int64_t head = p.free_head ? p.free_head[0] : 0;
  if (b >= p.batch) {  // (a batch of none)
    if (tid == 0) p.free_head_out[0] = (int)head;
    return;
  }
  const ForkRow f = fork_row(p, b);
  int taken = 0;
  for (int i = tid; i < b; i += kThreads) taken += fork_row(p, i).from >= 0 ? 1 : 0;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) taken += __shfl_xor(taken, o, 64);
  if ((tid & 63) == 0) taken_l[tid >> 6] = taken;
  __syncthreads();
  taken = 0;
#pragma unroll
  for (int i = 0; i < kThreads / 64; ++i) taken += taken_l[i];
  int page = -1;
  if (f.from >= 0) {
    const int64_t at = head + taken;
    if (at >= 0 && at < p.n_free) page = p.free_pages[at];
    if (page < 0 || page >= p.n_pages) page = -1;
  }
  const int held = (int)min(f.full + (f.part > 0 ? 1 : 0), (int64_t)p.max_pages);
  int32_t* out = p.table_out + (int64_t)b * p.table_out_stride;
  const int32_t* in = p.block_table + (int64_t)max(f.source, 0) * p.table_stride;
  for (int c = tid; c < p.max_pages; c += kThreads) {
    int x = -1;
    if (c < held) x = f.from >= 0 && c == f.full ? page : in[c];
    out[c] = x;
  }
  if (tid == 0) {
    p.kv_out[b] = (int)f.n;
    p.held_out[b] = held;
    p.copy_src[b] = page >= 0 ? f.from : -1;
    p.copy_dst[b] = page;
    p.copy_rows[b] = page >= 0 ? f.part : 0;
    if (b == p.batch - 1) p.free_head_out[0] = (int)(head + taken + (f.from >= 0 ? 1 : 0));
  }
}

// ---------------------------------------------------------------------------
// copy: a block moves up to 16 KB of one pair in one pool.  Bound: HBM (or launch, for few rows): with the fork, 7
// continuations that copy 96 rows of 2 KB in 32 pools, 88 MB, 16.8 us (5.2 TB/s); 28 of up to 15 rows in 24 pools 9.6
// ---------------------------------------------------------------------------
constexpr int kCopyBytes = 16384;
constexpr int kCopyUnroll = kCopyBytes / 16 / kThreads;

// rows of one block's part
inline __host__ __device__ int copy_rows_of(int64_t row_bytes) {
  return row_bytes >= kCopyBytes ? 1 : (int)(kCopyBytes / row_bytes);
}

__global__ __launch_bounds__(kThreads) void copy_pages_kernel(CopyPages p, int rows_per, int parts) {
  const int64_t block = (int64_t)blockIdx.y << kGridLog2 | blockIdx.x;
  // parts of a page, then pools, then pairs
  const int64_t item = block / parts;
  const int part = (int)(block - item * parts);
  const int64_t i = item / p.n_pools;
  const int pool = (int)(item - i * p.n_pools);
  if (i >= p.n_pairs) return;
  const int64_t from = p.src_page[i], to = p.dst_page[i];
  const int rows = p.rows ? min(p.rows[i], 1 << p.page_log2) : 1 << p.page_log2;
  if (from < 0 || from >= p.n_pages || to < 0 || to >= p.n_pages || from == to) return;
  const int r0 = part * rows_per, n = min(rows - r0, rows_per);
  if (n <= 0) return;
  char* base = static_cast<char*>(p.pools[pool]);
  const char* src = base + ((from << p.page_log2) + r0) * p.row_stride;
  char* dst = base + ((to << p.page_log2) + r0) * p.row_stride;
  const int per_row = (int)(p.row_bytes >> 4);
  const int64_t vecs = (int64_t)n * per_row;
  for (int64_t v0 = threadIdx.x; v0 < vecs; v0 += kThreads * kCopyUnroll) {
    uint4 x[kCopyUnroll];
    int64_t at[kCopyUnroll];
#pragma unroll
    for (int k = 0; k < kCopyUnroll; ++k) {
      const int64_t v = min(v0 + k * kThreads, vecs - 1);
      const int64_t row = n == 1 ? 0 : (int64_t)((uint32_t)v / (uint32_t)per_row);
      at[k] = row * p.row_stride + (v - row * per_row) * 16;
      x[k] = ld16(src + at[k]);
    }
#pragma unroll
    for (int k = 0; k < kCopyUnroll; ++k)
      if (v0 + k * kThreads < vecs) st16(dst + at[k], x[k]);
  }
}

// ---------------------------------------------------------------------------
// release.  Row i < batch is a request's row of the table before, row batch + i of the one after.
// ---------------------------------------------------------------------------
struct ReleaseRow {
  const int32_t* pages;
  int held;
};
__device__ __forceinline__ ReleaseRow release_row(const PageRelease& p, int i) {
  const bool after = i >= p.batch;
  const int b = after ? i - p.batch : i;
  const int held = after ? p.held_after[b] : p.held_before[b];
  return ReleaseRow{after ? p.after + b * p.after_stride : p.before + b * p.before_stride, min(max(held, 0), p.max_pages)};
}

// Small tables: one block marks the pages of both tables in LDS (two bits per page) and writes those that are only in
// the first.  Bound: latency (16 requests of up to 200 pages 9 us, of three dependent loads; one of 2 pages 6.4).
constexpr int kRelThreads = 1024;
constexpr int kRelWords = 1 << 14;  // of 32 pages, per bit set

__global__ __launch_bounds__(kRelThreads) void page_release_kernel(PageRelease p) {
  __shared__ uint32_t was_l[kRelWords], is_l[kRelWords];
  __shared__ int32_t first_l[kRelThreads];  // 64-entry pieces before each row
  __shared__ int wave_l[kRelThreads / 64];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  constexpr int kWaves = kRelThreads / 64;
  const int64_t head = min(max((int64_t)p.free_head[0], (int64_t)0), p.n_free);

  // inclusive sum over the block's threads of x; `all` is the total
  auto scan = [&](int x, int& all) {
    int sum = x;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int y = __shfl_up(sum, o, 64);
      if (lane >= o) sum += y;
    }
    __syncthreads();
    if (lane == 63) wave_l[w] = sum;
    __syncthreads();
    const int part = lane < kWaves ? wave_l[lane] : 0;
    all = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
      const int x1 = __builtin_amdgcn_readlane(part, i);
      if (i < w) sum += x1;
      all += x1;
    }
    return sum;
  };
  const int words = (int)((p.n_pages + 31) >> 5);
  for (int i = tid; i < words; i += kRelThreads) was_l[i] = is_l[i] = 0;
  for (int i0 = 0; i0 < 2 * p.batch; i0 += kRelThreads) {
    const int mine = i0 + tid < 2 * p.batch ? release_row(p, i0 + tid).held : 0;
    int all;
    const int pieces = (mine + 63) >> 6;
    const int sum = scan(pieces, all);
    first_l[tid] = sum - pieces;
    __syncthreads();
    // the waves share the pieces evenly; each lane looks up one of up to 64 at a time
    const int to = (int)((int64_t)all * (w + 1) / kWaves);
    for (int k0 = (int)((int64_t)all * w / kWaves); k0 < to; k0 += 64) {
      const int piece = min(k0 + lane, to - 1);
      int lo = 0, hi = kRelThreads;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first_l[mid] <= piece) lo = mid; else hi = mid;
      }
      const ReleaseRow row = release_row(p, i0 + lo);
      const int64_t from = reinterpret_cast<int64_t>(row.pages + (piece - first_l[lo]) * 64);
      const int left = row.held - (piece - first_l[lo]) * 64;
      const int which = i0 + lo >= p.batch ? 1 : 0, n = min(64, to - k0);
      constexpr int U = 8;
      for (int k = 0; k < n; k += U) {
        int x[U], set[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int j = min(k + u, n - 1);
          const int32_t* at = reinterpret_cast<const int32_t*>(__shfl(from, j, 64));
          x[u] = at[min(lane, __shfl(left, j, 64) - 1)];
          set[u] = __shfl(which, j, 64);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (x[u] >= 0 && x[u] < p.n_pages) atomicOr(&(set[u] ? is_l : was_l)[x[u] >> 5], 1u << (x[u] & 31));
      }
    }
    __syncthreads();
  }
  const int per = (words + kRelThreads - 1) / kRelThreads;
  const int w0 = min(tid * per, words), w1 = min(w0 + per, words);
  int own = 0, all;
  for (int i = w0; i < w1; ++i) own += __popc(was_l[i] & ~is_l[i]);
  const int before = scan(own, all) - own;
  const int64_t put = head - all;
  if (tid == 0) p.free_head_out[0] = (int)max(put, (int64_t)0);
  int64_t at = put + before;
  for (int i = w0; i < w1; ++i)
    for (uint32_t left = was_l[i] & ~is_l[i]; left; left &= left - 1, ++at)
      if (at >= 0) p.free_pages[at] = i * 32 + __builtin_ctz(left);
}

// Large tables: a byte per page and table in the workspace, set to zero, marked by a block per 1024 entries of a row
// (the same value from everywhere), and gone through by blocks of 16384 pages, each of which counts those before it.
constexpr int kMarkEntries = 1024;

__global__ __launch_bounds__(kThreads) void release_zero_kernel(uint4* marks, int64_t n) {
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (i < n) marks[i] = make_uint4(0, 0, 0, 0);
}

__global__ __launch_bounds__(kThreads) void release_mark_kernel(PageRelease p, uint8_t* marks, int64_t set_bytes, int pieces) {
  const int i = blockIdx.x / pieces, c0 = (blockIdx.x - i * pieces) * kMarkEntries;
  const ReleaseRow row = release_row(p, i);
  if (c0 >= row.held) return;
  uint8_t* set = marks + (i >= p.batch ? set_bytes : 0);
  constexpr int U = kMarkEntries / kThreads;
  int x[U];
#pragma unroll
  for (int u = 0; u < U; ++u) x[u] = row.pages[min(c0 + (int)threadIdx.x + u * kThreads, row.held - 1)];
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (x[u] >= 0 && x[u] < p.n_pages) set[x[u]] = 1;
}

__global__ __launch_bounds__(kRelThreads) void release_list_kernel(PageRelease p, const uint8_t* marks, int64_t set_bytes) {
  __shared__ int sum_l[2][kRelThreads / 64];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const uint4* was = reinterpret_cast<const uint4*>(marks);
  const uint4* is = reinterpret_cast<const uint4*>(marks + set_bytes);
  const int64_t n = set_bytes / 16, mine = (int64_t)blockIdx.x * kRelThreads + tid;
  auto gone = [&](int64_t i) {  // bytes that are 1: released pages 16 i .. 16 i + 15
    const uint4 a = was[i], b = is[i];
    return make_uint4(a.x & ~b.x, a.y & ~b.y, a.z & ~b.z, a.w & ~b.w);
  };
  auto count = [](const uint4& x) { return __popc(x.x) + __popc(x.y) + __popc(x.z) + __popc(x.w); };
  const int64_t head = min(max((int64_t)p.free_head[0], (int64_t)0), p.n_free);
  const uint4 own = mine < n ? gone(mine) : make_uint4(0, 0, 0, 0);
  // pages released in front of this block's, and all
  int before = 0, all = 0;
  constexpr int U = 4;
  for (int64_t i0 = tid; i0 < n; i0 += kRelThreads * U) {
    uint4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = gone(min(i0 + u * kRelThreads, n - 1));
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t i = i0 + u * kRelThreads;
      const int c = i < n ? count(x[u]) : 0;
      all += c;
      if (i < (int64_t)blockIdx.x * kRelThreads) before += c;
    }
  }
  const int mine_n = count(own);
  int sum = mine_n;  // of the wave's threads up to this one
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(sum, o, 64);
    if (lane >= o) sum += y;
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    before += __shfl_xor(before, o, 64);
    all += __shfl_xor(all, o, 64);
  }
  // a wave's threads up to its last, behind what lies before the block
  __shared__ int own_l[kRelThreads / 64];
  if (lane == 63) own_l[w] = sum;
  if (lane == 0) sum_l[0][w] = before, sum_l[1][w] = all;
  __syncthreads();
  before = all = 0;
  for (int i = 0; i < kRelThreads / 64; ++i) {
    before += sum_l[0][i] + (i < w ? own_l[i] : 0);
    all += sum_l[1][i];
  }
  const int64_t put = head - all;
  if (blockIdx.x == 0 && tid == 0) p.free_head_out[0] = (int)max(put, (int64_t)0);
  int64_t at = put + before + sum - mine_n;
  const uint32_t words[4] = {own.x, own.y, own.z, own.w};
#pragma unroll
  for (int k = 0; k < 4; ++k)
    for (uint32_t left = words[k]; left; left &= left - 1, ++at)
      if (at >= 0) p.free_pages[at] = (int)(16 * mine + 4 * k + (__builtin_ctz(left) >> 3));
}

// One block's time grows with the tables, three launches take about 10 us whatever their size (a request of 2 pages 6.4 us
// against 9.4, 16 of 200 9.2 against 9.8, 64 of 100 14.5 against 9.9, 256 of 100 29 against 9.9, 400 of 900 128 against 15).
inline bool release_small(int batch, int max_pages, int64_t n_pages) {
  return (int64_t)batch * max_pages <= 4096 && n_pages <= 32 * kRelWords;
}

}  // namespace

hipError_t launch_page_fork(const PageFork& p, hipStream_t stream) {
  page_fork_kernel<<<dim3((unsigned)(p.batch > 0 ? p.batch : 1)), kThreads, 0, stream>>>(p);
  return hipGetLastError();
}

static int64_t copy_parts(const CopyPages& p) {
  const int64_t rows = copy_rows_of(p.row_bytes);
  return ((1ll << p.page_log2) + rows - 1) / rows;
}

int64_t copy_pages_blocks(const CopyPages& p) {
  const int64_t most = INT32_MAX, parts = copy_parts(p);
  if (p.n_pairs > most / p.n_pools || p.n_pairs * p.n_pools > most / parts) return -1;
  return p.n_pairs * p.n_pools * parts;
}

hipError_t launch_copy_pages(const CopyPages& p, hipStream_t stream) {
  copy_pages_kernel<<<grid_of(copy_pages_blocks(p)), kThreads, 0, stream>>>(p, copy_rows_of(p.row_bytes), (int)copy_parts(p));
  return hipGetLastError();
}

size_t page_release_workspace(int batch, int max_pages, int64_t n_pages) {
  return release_small(batch, max_pages, n_pages) ? 0 : (size_t)((n_pages + 255) / 256 * 256) * 2;
}

hipError_t launch_page_release(const PageRelease& p, void* ws, hipStream_t stream) {
  if (release_small(p.batch, p.max_pages, p.n_pages)) {
    page_release_kernel<<<dim3(1), kRelThreads, 0, stream>>>(p);
    return hipGetLastError();
  }
  const int64_t set_bytes = (p.n_pages + 255) / 256 * 256, vecs = set_bytes * 2 / 16;
  uint8_t* marks = static_cast<uint8_t*>(ws);
  const int pieces = (p.max_pages + kMarkEntries - 1) / kMarkEntries;
  if (vecs > 0)
    release_zero_kernel<<<dim3((unsigned)((vecs + kThreads - 1) / kThreads)), kThreads, 0, stream>>>(reinterpret_cast<uint4*>(marks), vecs);
  release_mark_kernel<<<dim3((unsigned)((int64_t)2 * p.batch * pieces)), kThreads, 0, stream>>>(p, marks, set_bytes, pieces);
  const int64_t blocks = std::max<int64_t>((set_bytes / 16 + kRelThreads - 1) / kRelThreads, 1);
  release_list_kernel<<<dim3((unsigned)blocks), kRelThreads, 0, stream>>>(p, marks, set_bytes);
  return hipGetLastError();
}

}  // namespace qcf
