// Verification of drafted tokens against the target's probabilities (qcf_verify_drafts).
//
//  walk  one block per request reads the few numbers that the tests need (a probability of the
//        target and of the draft per drafted token) into LDS, and its first wave goes down the
//        tree.  Only siblings that are tested after a rejection, with draft probabilities, need a
//        sum over the vocabulary (Z); the block forms it then.
//  sums  the row that the walk ended at, cut over blocks: sum of R (and of P, for an empty R) per
//        kChunk tokens.
//  pick  one block per request: the chunk in which the running sum passes u * sum R, then the token.
//
// R after rejections has a closed form, max(P - c D, 0), because max(max(a, 0) - b, 0) = max(a - b, 0)
// for b >= 0, so no residual row is ever written.
//
// Everything that decides a token is float64 (probabilities are widened exactly): with float32 sums a
// draw next to a border would hang on the order of the additions.
//
// Bound: one vocabulary row of P (and D) per request from HBM; for few requests latency.
#include "qcf_decode_launch.h"
#include "qcf_device.h"

namespace qcf {
namespace {

constexpr int kThreads = 256;
constexpr int kTree = 1024;    // rows of the largest tree (QCF_MAX_TREE)
constexpr int kChunk = 4096;   // tokens per block of the sums

// Where a request's walk ended: row r of the batch (-1: the request has none), its index cur in
// the request, the entry of out_tokens that the drawn token goes to, and R's coefficient c.
struct WalkEnd {
  int64_t row;
  int32_t cur, at;
  double coef;
};

__device__ __forceinline__ float prob(float x) { return x > 0.f ? x : 0.f; }
__device__ __forceinline__ float prob(uint16_t x) { return prob(bf2f(x)); }

__device__ __forceinline__ double wave_sum_d(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

__device__ __forceinline__ int request_rows(const VerifyDrafts& p, int b, int64_t& r0) {
  r0 = p.cu_rows[b];
  if (r0 < 0) return 0;
  return (int)max((int64_t)0, min(min((int64_t)p.cu_rows[b + 1], p.n_rows) - r0, (int64_t)p.max_rows));
}

template <typename T>
__global__ __launch_bounds__(kThreads) void verify_walk_kernel(VerifyDrafts p, WalkEnd* __restrict__ ends) {
  __shared__ int32_t par_l[kTree], tok_l[kTree], path_l[kTree];
  __shared__ float u_l[kTree], p_l[kTree], d_l[kTree];
  __shared__ double red_l[kThreads / 64];
  __shared__ int32_t cur_l, next_l, len_l;
  __shared__ double coef_l, z_l;
  __shared__ bool need_l;
  const T* target = static_cast<const T*>(p.target);
  const T* draft = static_cast<const T*>(p.draft);
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  int64_t r0;
  const int n = request_rows(p, b, r0);
  for (int i = tid; i < n; i += kThreads) {
    const int64_t r = r0 + i;
    const int up = p.parents ? p.parents[r] : i - 1, x = p.tokens[r];
    const bool ok = up >= 0 && up < i && x >= 0 && x < p.vocab;
    const int64_t at = ok ? (r0 + up) * p.row_stride + x : 0;
    par_l[i] = i > 0 && up >= 0 && up < i ? up : -1;
    tok_l[i] = ok ? x : -1;
    u_l[i] = p.u_accept[r];
    p_l[i] = ok ? prob(target[at]) : 0.f;
    d_l[i] = ok && draft ? prob(draft[at]) : 1.f;
  }
  if (tid == 0) {
    cur_l = 0;
    next_l = 1;
    len_l = 1;
    path_l[0] = 0;
    coef_l = 0.;
    z_l = 1.;
  }
  __syncthreads();
  for (;;) {
    if (tid < 64) {
      // one wave, every lane the same state; a window of 64 rows holds a lane's candidate each
      int cur = cur_l, next = next_l, len = len_l;
      double coef = coef_l, z = z_l;
      bool stale = false;  // z has to be summed before the next test
      for (int w0 = next & ~63; w0 < n; w0 += 64) {
        const int i = w0 + lane;
        uint64_t kids = __ballot(i < n && i >= next && par_l[min(i, n - 1)] == cur);
        while (kids) {
          const int j = w0 + __builtin_ctzll(kids);
          kids &= kids - 1;
          const int x = tok_l[j];
          if (x < 0) continue;
          if (stale) {
            next = j;
            w0 = n;  // leave both loops
            break;
          }
          const double px = p_l[j], dx = d_l[j];
          double rx = draft ? fmax(px - coef * dx, 0.) : px;
          if (!draft) {
            // a sibling before it with the same token has taken R(x) away
            bool gone = false;
            for (int v = 0; v < j; v += 64)
              gone = gone || __ballot(v + lane < j && v + lane > cur && par_l[v + lane] == cur && tok_l[v + lane] == x);
            if (gone) rx = 0.;
          }
          if ((double)u_l[j] * z * dx < rx) {
            cur = j;
            next = j + 1;
            if (lane == 0) path_l[len] = j;
            ++len;
            coef = 0.;
            z = 1.;
            kids = __ballot(i < n && i >= next && par_l[min(i, n - 1)] == cur);
          } else {
            next = j + 1;
            if (draft) {
              coef += z;
              stale = true;
            } else {
              z = fmax(z - rx, 0.);
            }
          }
        }
      }
      if (lane == 0) {
        // stale with a child left at `next`: the block sums
        need_l = stale && next < n && par_l[next] == cur && tok_l[next] >= 0;
        cur_l = cur;
        next_l = next;
        len_l = len;
        coef_l = coef;
        z_l = z;
      }
    }
    __syncthreads();
    if (!need_l) break;
    const T* tp = target + (r0 + cur_l) * p.row_stride;
    const T* td = draft + (r0 + cur_l) * p.row_stride;
    const double coef = coef_l;
    double s = 0.;
    for (int t = tid; t < p.vocab; t += kThreads) s += fmax((double)prob(tp[t]) - coef * (double)prob(td[t]), 0.);
    s = wave_sum_d(s);
    if (lane == 0) red_l[tid >> 6] = s;
    __syncthreads();
    if (tid == 0) {
      double z = 0.;
      for (int i = 0; i < kThreads / 64; ++i) z += red_l[i];
      z_l = z;
    }
    __syncthreads();
  }
  const int len = n > 0 ? len_l : 0;
  for (int k = tid; k < p.max_rows; k += kThreads) {
    const int64_t o = (int64_t)b * p.max_rows + k;
    const int at = k < len ? path_l[k] : -1;
    p.path[o] = at;
    p.out_tokens[o] = k + 1 < len ? tok_l[path_l[k + 1]] : -1;
    if (p.slots) {
      const bool move = k < len && at != k;
      p.move_src[o] = move ? p.slots[r0 + at] : -1;
      p.move_dst[o] = move ? p.slots[r0 + k] : -1;
    }
  }
  if (tid == 0) {
    p.n_out[b] = len;
    ends[b] = WalkEnd{n > 0 ? r0 + cur_l : -1, cur_l, len - 1, coef_l};
  }
}

// The tokens of chunk [t0, t0 + kChunk) that the children of the walk's last row hold (all rejected;
// without draft probabilities R is zero there), as bits in LDS.
__device__ __forceinline__ void rejected_bits(const VerifyDrafts& p, const WalkEnd& e, int t0, uint32_t* bits) {
  for (int i = threadIdx.x; i < kChunk / 32; i += kThreads) bits[i] = 0;
  __syncthreads();
  if (!p.draft) {
    int64_t r0;
    const int n = request_rows(p, blockIdx.x, r0);
    for (int i = e.cur + 1 + threadIdx.x; i < n; i += kThreads) {
      const int up = p.parents ? p.parents[r0 + i] : i - 1;
      const int x = p.tokens[r0 + i] - t0;
      if (up == e.cur && x >= 0 && x < kChunk) atomicOr(&bits[x >> 5], 1u << (x & 31));
    }
  }
  __syncthreads();
}

// R and P of token t
template <typename T>
__device__ __forceinline__ double2 residual(const VerifyDrafts& p, const WalkEnd& e, int t, bool gone) {
  const int64_t at = e.row * p.row_stride + t;
  const double pt = prob(static_cast<const T*>(p.target)[at]);
  if (!p.draft) return make_double2(gone ? 0. : pt, pt);
  const double dt = prob(static_cast<const T*>(p.draft)[at]);
  return make_double2(fmax(pt - e.coef * dt, 0.), pt);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void verify_sums_kernel(VerifyDrafts p, const WalkEnd* __restrict__ ends,
                                                               double2* __restrict__ sums) {
  __shared__ uint32_t bits[kChunk / 32];
  __shared__ double2 red_l[kThreads / 64];
  const int b = blockIdx.x, c = blockIdx.y, t0 = c * kChunk;
  const WalkEnd e = ends[b];
  if (e.row < 0) return;
  rejected_bits(p, e, t0, bits);
  double r = 0., q = 0.;
  for (int i = threadIdx.x; i < min(kChunk, p.vocab - t0); i += kThreads) {
    const double2 x = residual<T>(p, e, t0 + i, bits[i >> 5] >> (i & 31) & 1);
    r += x.x;
    q += x.y;
  }
  r = wave_sum_d(r);
  q = wave_sum_d(q);
  if ((threadIdx.x & 63) == 0) red_l[threadIdx.x >> 6] = make_double2(r, q);
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < kThreads / 64; ++i) {
      r += red_l[i].x;
      q += red_l[i].y;
    }
    sums[(int64_t)b * gridDim.y + c] = make_double2(r, q);
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void verify_pick_kernel(VerifyDrafts p, const WalkEnd* __restrict__ ends,
                                                               const double2* __restrict__ sums, int chunks) {
  constexpr int PT = kChunk / kThreads;
  __shared__ uint32_t bits[kChunk / 32];
  __shared__ double wave_l[kThreads / 64];
  __shared__ int32_t hit_l, last_l;
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const WalkEnd e = ends[b];
  if (e.row < 0) return;
  const double2* s = sums + (int64_t)b * chunks;
  // every wave forms the same totals and running sums of the chunks, 64 at a time
  double total = 0., total_p = 0.;
  for (int c = lane; c < chunks; c += 64) {
    total += s[c].x;
    total_p += s[c].y;
  }
  total = wave_sum_d(total);
  total_p = wave_sum_d(total_p);
  const bool empty = !(total > 0.);
  if (empty && !(total_p > 0.)) return;  // the walk left -1
  const double want = (double)p.u_next[b] * (empty ? total_p : total);
  double run = 0., before = 0.;
  int chunk = -1, last = -1;
  for (int c0 = 0; c0 < chunks && chunk < 0; c0 += 64) {
    const double own = c0 + lane < chunks ? (empty ? s[c0 + lane].y : s[c0 + lane].x) : 0.;
    double sum = own;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const double x = __shfl_up(sum, o, 64);
      if (lane >= o) sum += x;
    }
    const uint64_t over = __ballot(own > 0. && run + sum > want), some = __ballot(own > 0.);
    if (over) {
      const int k = __builtin_ctzll(over);
      chunk = c0 + k;
      before = run + __shfl(sum - own, k, 64);
    } else if (some) {
      last = c0 + 63 - __builtin_clzll(some);
    }
    run += __shfl(sum, 63, 64);
  }
  const bool past = chunk < 0;  // rounding, or a number of 1 and more: the last token of all
  if (past) chunk = last;
  if (chunk < 0) return;
  const int t0 = chunk * kChunk;
  if (tid == 0) {
    hit_l = kChunk;
    last_l = -1;
  }
  rejected_bits(p, e, t0, bits);
  double v[PT], own = 0.;
#pragma unroll
  for (int k = 0; k < PT; ++k) {
    const int i = tid * PT + k;
    v[k] = 0.;
    if (t0 + i < p.vocab) {
      const double2 x = residual<T>(p, e, t0 + i, bits[i >> 5] >> (i & 31) & 1);
      v[k] = empty ? x.y : x.x;
    }
    own += v[k];
  }
  double sum = own;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const double x = __shfl_up(sum, o, 64);
    if (lane >= o) sum += x;
  }
  if (lane == 63) wave_l[tid >> 6] = sum;
  __syncthreads();
  double at = before + (sum - own);
  for (int i = 0; i < tid >> 6; ++i) at += wave_l[i];
  int first = kChunk, mine = -1;
#pragma unroll
  for (int k = 0; k < PT; ++k) {
    at += v[k];
    if (v[k] > 0.) {
      mine = tid * PT + k;
      if (!past && at > want) first = min(first, mine);
    }
  }
  if (first < kChunk) atomicMin(&hit_l, first);
  if (mine >= 0) atomicMax(&last_l, mine);
  __syncthreads();
  if (tid == 0) p.out_tokens[(int64_t)b * p.max_rows + e.at] = t0 + (hit_l < kChunk ? hit_l : last_l);
}

int chunk_count(int vocab) { return (int)(((int64_t)vocab + kChunk - 1) / kChunk); }

size_t ends_bytes(int batch) { return ((size_t)batch * sizeof(WalkEnd) + 255) / 256 * 256; }

template <typename T>
hipError_t launch_t(const VerifyDrafts& p, void* ws, hipStream_t stream) {
  WalkEnd* ends = static_cast<WalkEnd*>(ws);
  double2* sums = reinterpret_cast<double2*>(static_cast<char*>(ws) + ends_bytes(p.batch));
  const int chunks = chunk_count(p.vocab);
  verify_walk_kernel<T><<<dim3((unsigned)p.batch), kThreads, 0, stream>>>(p, ends);
  verify_sums_kernel<T><<<dim3((unsigned)p.batch, (unsigned)chunks), kThreads, 0, stream>>>(p, ends, sums);
  verify_pick_kernel<T><<<dim3((unsigned)p.batch), kThreads, 0, stream>>>(p, ends, sums, chunks);
  return hipGetLastError();
}

}  // namespace

size_t verify_drafts_workspace(int batch, int vocab) {
  return ends_bytes(batch) + ((size_t)batch * chunk_count(vocab) * sizeof(double2) + 255) / 256 * 256;
}

hipError_t launch_verify_drafts(const VerifyDrafts& p, bool bf16, void* ws, hipStream_t stream) {
  return bf16 ? launch_t<uint16_t>(p, ws, stream) : launch_t<float>(p, ws, stream);
}

}  // namespace qcf
