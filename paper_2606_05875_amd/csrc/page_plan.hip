// Block tables, slot maps, positions and tree masks of a pass's new rows (qcf_page_plan).
//
// Where a request's pages start in the free list and its rows in the packed arrays are prefix
// sums over the requests before it.  Both are needed everywhere, so every block forms them itself
// (256 requests at a time: their lengths packed into one 64-bit scan) on its way to its own tile
// of rows, and nothing has to meet between blocks: one launch, no atomics, the same result in any
// order.  A new page begins with a new row, so whoever writes that row's slot writes the table entry.
//
// Bound: latency (a few dependent loads; the largest calls move about a megabyte): 64 requests of one row 4.3 us,
// 3.2 of them the kernel; 256 trees of up to 40 rows 6.4 us; 16 requests of 117000 rows in all 4.7 us.
#include "qcf_decode_launch.h"
#include "qcf_device.h"

namespace qcf {
namespace {

constexpr int kThreads = 256;
constexpr int kReq = kThreads;      // requests per scan
constexpr int kTile = kThreads;     // rows per block (one per thread: 256 trees of up to 40 rows 14.6 -> 6.8 us against four)
constexpr int kTree = 1024;         // rows of the largest tree (QCF_MAX_TREE)

__device__ __forceinline__ int64_t pages_of(int64_t tokens, int lp) {
  return (tokens + (1ll << lp) - 1) >> lp;
}

__global__ __launch_bounds__(kThreads) void page_plan_kernel(PagePlan p) {
  __shared__ uint64_t wave_sum_l[kThreads / 64];
  __shared__ uint32_t row_l[kReq + 1];   // first row of each request of the scan, from the scan's first
  __shared__ uint32_t page_l[kReq];      // first place in the free list, from the scan's first
  __shared__ int32_t kv_l[kReq], held_l[kReq], need_l[kReq];
  __shared__ int32_t par_l[kTree + kTile];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int64_t t0 = (int64_t)blockIdx.x * kTile;
  if (p.parents) {
    for (int i = tid; i < kTree + kTile; i += kThreads) {
      const int64_t r = t0 - kTree + i;
      par_l[i] = r >= 0 && r < p.n_rows ? p.parents[r] : -1;
    }
  }
  const int64_t head = p.free_head ? p.free_head[0] : 0;
  int64_t row0 = 0, page0 = 0;  // rows and pages of the requests before the scan
  // block 0 goes through every request and writes what is per request
  for (int b0 = 0; b0 < p.batch && (blockIdx.x == 0 || row0 < t0 + kTile); b0 += kReq) {
    const int b = b0 + tid;
    const bool in = b < p.batch;
    const int64_t n = in ? max(p.new_len[b], 0) : 0, kv = in ? max(p.kv_len[b], 0) : 0;
    int64_t held = pages_of(kv, p.page_log2);
    if (in && p.pages_held) held = max(held, (int64_t)p.pages_held[b]);
    held = min(held, (int64_t)p.max_pages);
    const int64_t need = max(held, min(pages_of(kv + n, p.page_log2), (int64_t)p.max_pages));
    const uint64_t own = (uint64_t)(need - held) << 32 | (uint64_t)n;
    uint64_t sum = own;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint64_t x = __shfl_up(sum, o, 64);
      if (lane >= o) sum += x;
    }
    __syncthreads();  // the previous scan's arrays have been read
    if (lane == 63) wave_sum_l[w] = sum;
    __syncthreads();
    uint64_t all = 0;
#pragma unroll
    for (int i = 0; i < kThreads / 64; ++i) {
      if (i < w) sum += wave_sum_l[i];
      all += wave_sum_l[i];
    }
    const uint64_t before = sum - own;
    row_l[tid] = (uint32_t)before;
    page_l[tid] = (uint32_t)(before >> 32);
    if (tid == 0) row_l[kReq] = (uint32_t)all;
    kv_l[tid] = (int32_t)kv;
    held_l[tid] = (int32_t)held;
    need_l[tid] = (int32_t)need;
    if (blockIdx.x == 0 && in) {
      p.cu_new[b] = (int32_t)(row0 + (uint32_t)before);
      if (p.kv_end) p.kv_end[b] = (int32_t)(kv + n);
      if (p.pages_held_out) p.pages_held_out[b] = (int32_t)need;
    }
    __syncthreads();
    const int64_t rows = (uint32_t)all;
    const int64_t t = t0 + tid, rel = t - row0;
    if (rel >= 0 && rel < rows && t < p.n_rows) {
      int lo = 0, hi = kReq;  // the last request that starts at or before the row
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if ((int64_t)row_l[mid] <= rel) lo = mid; else hi = mid;
      }
      const int i = (int)(rel - row_l[lo]);
      const int64_t pos = (int64_t)kv_l[lo] + i;
      const int64_t pg = pos >> p.page_log2;
      int32_t* entry = p.block_table + (int64_t)(b0 + lo) * p.table_stride + pg;
      int64_t page = -1;
      if (pg < held_l[lo]) {
        page = *entry;
        if (page < 0 || page >= p.n_pages) page = -1;
      } else if (pg < need_l[lo]) {
        const int64_t at = head + page0 + page_l[lo] + (pg - held_l[lo]);
        if (at >= 0 && at < p.n_free) page = p.free_pages[at];
        if (page < 0 || page >= p.n_pages) page = -1;
        if ((pos & ((1ll << p.page_log2) - 1)) == 0) *entry = (int32_t)page;
      }
      p.slots[t] = page < 0 ? -1
                            : (int32_t)((page << p.page_log2) + (pos & ((1ll << p.page_log2) - 1)));
      int depth = i;
      if (p.parents) {
        // ancestors have ever smaller indices, so their words are met in falling order
        uint32_t* m = p.tree_mask + t * p.mask_words;
        int word = p.mask_words - 1;
        for (; word > i >> 5; --word) m[word] = 0;
        const int64_t first = t - i;
        uint32_t bits = 0;
        depth = 0;
        for (int a = i;;) {
          for (; word > a >> 5; --word) {
            m[word] = bits;
            bits = 0;
          }
          if (word == a >> 5) bits |= 1u << (a & 31);
          const int64_t at = first + a - (t0 - kTree);
          const int up = at >= 0 ? par_l[at] : -1;
          if (up < 0 || up >= a) break;
          a = up;
          ++depth;
        }
        for (; word >= 0; --word) {
          m[word] = bits;
          bits = 0;
        }
      }
      p.positions[t] = (int32_t)(kv_l[lo] + depth);
    }
    row0 += rows;
    page0 += (int64_t)(all >> 32);
  }
  if (blockIdx.x == 0 && tid == 0) {
    p.cu_new[p.batch] = (int32_t)row0;
    if (p.free_head_out) p.free_head_out[0] = (int32_t)(head + page0);
  }
  // rows behind the last request (a block that left the loop early has none)
  const int64_t t = t0 + tid;
  if (t >= row0 && t < p.n_rows) {
    p.slots[t] = -1;
    p.positions[t] = -1;
    if (p.parents)
      for (int i = 0; i < p.mask_words; ++i) p.tree_mask[t * p.mask_words + i] = 0;
  }
}

}  // namespace

hipError_t launch_page_plan(const PagePlan& p, hipStream_t stream) {
  const int64_t blocks = p.n_rows > 0 ? (p.n_rows + kTile - 1) / kTile : 1;
  page_plan_kernel<<<dim3((unsigned)blocks), kThreads, 0, stream>>>(p);
  return hipGetLastError();
}

}  // namespace qcf
