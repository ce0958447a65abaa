// Verification of drafted tokens against the target's probabilities (qcf_verify_drafts).
//
//  walk  reads the few numbers that the tests need (a probability of the target and of the draft per
//        drafted token) into LDS; a wave goes down the tree.  Only siblings that are tested after a
//        rejection, with draft probabilities, need a sum over the vocabulary (Z), which the block forms then.
//  sums  the row that the walk ended at, cut over blocks: sum of R (and of P, for an empty R) per
//        kChunk tokens.  Where no walk needs a sum, every block of this kernel walks by itself (a few
//        dependent loads), which saves a launch; else the walk is a kernel of its own.
//  pick  one block per request: the chunk in which the running sum passes u * sum R, then the token.
//
// R after rejections has a closed form, max(P - c D, 0), because max(max(a, 0) - b, 0) = max(a - b, 0)
// for b >= 0, so no residual row is ever written.
//
// Everything that decides a token is float64 (probabilities are widened exactly): with float32 sums a
// draw next to a border would hang on the order of the additions.
//
// Bound: one vocabulary row of P (and D) per request from HBM; for few requests latency.  64 chains of 5 over
// 128000 float32 probabilities of both: 24.6 us (66 MB; sums 14, pick 8); 16 trees over 150001 of bfloat16
// without D 14.7 us, one tree 12.6.  64 trees of 5 with D 57 us: siblings' sums wait for each other on one CU each (31).
#include "qcf_decode_launch.h"
#include "qcf_device.h"

namespace qcf {
namespace {

constexpr int kThreads = 256;
constexpr int kWalkThreads = 1024;  // of a walk that sums over the vocabulary
constexpr int kTree = 1024;         // rows of the largest tree (QCF_MAX_TREE)
constexpr int kChunk = 4096;        // tokens per block of the sums
constexpr int kPer = kChunk / kThreads;

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
  const int64_t r1 = p.cu_rows[b + 1];
  return r0 < 0 ? 0 : (int)max((int64_t)0, min(min(r1, p.n_rows) - r0, (int64_t)p.max_rows));
}

// One vocabulary row in 16-byte pieces.  Rows may begin anywhere: pieces lie on the tensor's own 16-byte
// grid, `lead` elements of the first one before the row.
template <typename T>
struct Row {
  static constexpr int VEC = Vec16<T>::N;
  int64_t first;  // element where the first piece begins
  int lead, vocab;
  __device__ __forceinline__ Row(const VerifyDrafts& p, int64_t row) {
    const int64_t at = row * p.row_stride;
    lead = (int)(at & (VEC - 1));
    first = at - lead;
    vocab = p.vocab;
  }
  // pieces j0 .. j1 - 1 hold tokens of this row only
  __device__ __forceinline__ bool inside(int64_t j0, int64_t j1) const { return j0 >= lead && j1 <= (int64_t)vocab + lead; }
  // the piece that begins with token j - lead (j a multiple of VEC), which is inside the row ..
  __device__ __forceinline__ uint4 load(const T* x, int64_t j) const { return ld16(x + first + j); }
  // .. or anywhere: elements outside the row are zeros.  No load is under a lane's condition, where each would
  // wait by itself: four elements are read from clamped places (64 chains of float32: 24.6 us a call, 28.0 the
  // other way), of eight the whole piece, and only the row's ends by element (16 trees of bfloat16: 50 us, 57).
  __device__ __forceinline__ uint4 load_any(const T* x, int64_t j) const {
    const int64_t end = (int64_t)lead + vocab;
    if constexpr (VEC == 4) {
      uint32_t w[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) w[e] = __builtin_bit_cast(uint32_t, x[first + min(max(j + e, (int64_t)lead), end - 1)]);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        asm volatile("" : "+v"(w[e]));
        if (j + e < lead || j + e >= end) w[e] = 0;
      }
      return make_uint4(w[0], w[1], w[2], w[3]);
    } else {
      const int64_t lo = lead ? VEC : 0, hi = (end & ~(int64_t)(VEC - 1)) - VEC;  // the first and the last whole piece
      uint4 v = make_uint4(0, 0, 0, 0);
      if (lo <= hi) v = load(x, min(max(j, lo), hi));
      if (j < lo || j > hi) {
        T w[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) w[e] = j + e >= lead && j + e < end ? x[first + j + e] : T(0);
        v = __builtin_bit_cast(uint4, w);
      }
      return v;
    }
  }
  __device__ __forceinline__ static void unpack(const uint4& x, float (&v)[VEC]) {
    Vec16<T>::unpack(x, v);
#pragma unroll
    for (int e = 0; e < VEC; ++e) v[e] = prob(v[e]);
  }
};

// kCap: rows of the largest request
template <int kCap>
struct WalkLds {
  int32_t par[kCap], tok[kCap], path[kCap];
  float u[kCap], p[kCap], d[kCap];
  double red[kWalkThreads / 64];
  int32_t cur, next, len;
  double coef, z;
  bool need;
};

template <typename T, int NT, int kCap>
__device__ __forceinline__ void walk(const VerifyDrafts& p, int64_t r0, int n, WalkLds<kCap>& s) {
  const T* target = static_cast<const T*>(p.target);
  const T* draft = static_cast<const T*>(p.draft);
  const int tid = threadIdx.x, lane = tid & 63;
  for (int i = tid; i < n; i += NT) {
    const int64_t r = r0 + i;
    const int up = p.parents ? p.parents[r] : i - 1, x = p.tokens[r];
    const bool ok = up >= 0 && up < i && x >= 0 && x < p.vocab;
    const int64_t at = ok ? (r0 + up) * p.row_stride + x : 0;
    s.par[i] = i > 0 && up >= 0 && up < i ? up : -1;
    s.tok[i] = ok ? x : -1;
    s.u[i] = p.u_accept[r];
    s.p[i] = ok ? prob(target[at]) : 0.f;
    s.d[i] = ok && draft ? prob(draft[at]) : 1.f;
  }
  if (tid == 0) {
    s.cur = 0;
    s.next = 1;
    s.len = 1;
    s.path[0] = 0;
    s.coef = 0.;
    s.z = 1.;
  }
  __syncthreads();
  for (;;) {
    if (tid < 64) {
      // one wave, every lane the same state; a window of 64 rows holds a lane's candidate each
      int cur = s.cur, next = s.next, len = s.len;
      double coef = s.coef, z = s.z;
      bool stale = false;  // z has to be summed before the next test
      for (int w0 = next & ~63; w0 < n; w0 += 64) {
        const int i = w0 + lane;
        const int par = s.par[min(i, n - 1)];
        uint64_t kids = __ballot(i < n && i >= next && par == cur);
        while (kids) {
          const int j = w0 + __builtin_ctzll(kids);
          kids &= kids - 1;
          const int x = s.tok[j];
          if (x < 0) continue;
          if (stale) {
            next = j;
            w0 = n;  // leave both loops
            break;
          }
          const double px = s.p[j], dx = s.d[j];
          double rx = draft ? fmax(px - coef * dx, 0.) : px;
          if (!draft) {
            // a sibling before it with the same token has taken R(x) away
            bool gone = false;
            for (int v = cur & ~63; v < j; v += 64) {
              const int k = v + lane;
              gone = gone || __ballot(k < j && k > cur && s.par[k] == cur && s.tok[k] == x);
            }
            if (gone) rx = 0.;
          }
          if ((double)s.u[j] * z * dx < rx) {
            cur = j;
            next = j + 1;
            if (lane == 0) s.path[len] = j;
            ++len;
            coef = 0.;
            z = 1.;
            kids = __ballot(i < n && i >= next && par == cur);
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
        s.need = stale && next < n && s.par[next] == cur && s.tok[next] >= 0;
        s.cur = cur;
        s.next = next;
        s.len = len;
        s.coef = coef;
        s.z = z;
      }
    }
    __syncthreads();
    if (!s.need) return;
    const Row<T> row(p, r0 + s.cur);
    const double coef = s.coef;
    double sum = 0.;
    constexpr int VEC = Vec16<T>::N, U = 4;
    const int64_t end = (int64_t)p.vocab + row.lead;
    for (int64_t j0 = 0; j0 < end; j0 += NT * VEC * U) {
      const int64_t j = j0 + (int64_t)tid * VEC;
      uint4 a[U], d[U];
      if (row.inside(j0, j0 + NT * VEC * U)) {  // (for the whole block: a load under a lane's condition waits by itself)
#pragma unroll
        for (int k = 0; k < U; ++k) {
          a[k] = row.load(target, j + k * NT * VEC);
          d[k] = row.load(draft, j + k * NT * VEC);
        }
      } else {
#pragma unroll
        for (int k = 0; k < U; ++k) {
          const int64_t jk = j0 + (int64_t)k * NT * VEC;
          if (row.inside(jk, jk + NT * VEC)) {
            a[k] = row.load(target, j + k * NT * VEC);
            d[k] = row.load(draft, j + k * NT * VEC);
          } else if (jk < end) {
            a[k] = row.load_any(target, j + k * NT * VEC);
            d[k] = row.load_any(draft, j + k * NT * VEC);
          } else {
            a[k] = d[k] = make_uint4(0, 0, 0, 0);
          }
        }
      }
#pragma unroll
      for (int k = 0; k < U; ++k) {
        float x[VEC], y[VEC];
        Row<T>::unpack(a[k], x);
        Row<T>::unpack(d[k], y);
#pragma unroll
        for (int e = 0; e < VEC; ++e) sum += fmax((double)x[e] - coef * (double)y[e], 0.);
      }
    }
    sum = wave_sum_d(sum);
    if (lane == 0) s.red[tid >> 6] = sum;
    __syncthreads();
    if (tid == 0) {
      double z = 0.;
      for (int i = 0; i < NT / 64; ++i) z += s.red[i];
      s.z = z;
    }
    __syncthreads();
  }
}

// the walk's results, by one block of the request
template <int NT, int kCap>
__device__ __forceinline__ void write_walk(const VerifyDrafts& p, int b, int64_t r0, int n, const WalkLds<kCap>& s,
                                           WalkEnd* __restrict__ ends) {
  const int len = n > 0 ? s.len : 0;
  for (int k = threadIdx.x; k < p.max_rows; k += NT) {
    const int64_t o = (int64_t)b * p.max_rows + k;
    const int at = k < len ? s.path[k] : -1;
    p.path[o] = at;
    p.out_tokens[o] = k + 1 < len ? s.tok[s.path[k + 1]] : -1;
    if (p.slots) {
      const bool move = k < len && at != k;
      p.move_src[o] = move ? p.slots[r0 + at] : -1;
      p.move_dst[o] = move ? p.slots[r0 + k] : -1;
    }
  }
  if (threadIdx.x == 0) {
    p.n_out[b] = len;
    ends[b] = WalkEnd{n > 0 ? r0 + s.cur : -1, s.cur, len - 1, s.coef};
  }
}

template <typename T>
__global__ __launch_bounds__(kWalkThreads) void verify_walk_kernel(VerifyDrafts p, WalkEnd* __restrict__ ends) {
  __shared__ WalkLds<kTree> s;
  int64_t r0;
  const int n = request_rows(p, blockIdx.x, r0);
  walk<T, kWalkThreads, kTree>(p, r0, n, s);
  write_walk<kWalkThreads, kTree>(p, blockIdx.x, r0, n, s, ends);
}

// P and D of VEC tokens of a row
template <typename T>
struct Residual {
  static constexpr int VEC = Vec16<T>::N;
  uint4 a, d;
  __device__ __forceinline__ void load(const VerifyDrafts& p, const Row<T>& row, int64_t j) {
    a = row.load(static_cast<const T*>(p.target), j);
    if (p.draft) d = row.load(static_cast<const T*>(p.draft), j);
  }
  __device__ __forceinline__ void load_any(const VerifyDrafts& p, const Row<T>& row, int64_t j) {
    a = row.load_any(static_cast<const T*>(p.target), j);
    if (p.draft) d = row.load_any(static_cast<const T*>(p.draft), j);
  }
  // R and P of each token; bits: rejected ones without draft probabilities
  template <typename F>
  __device__ __forceinline__ void each(const VerifyDrafts& p, double coef, uint32_t bits, F&& f) const {
    float x[VEC], y[VEC];
    Row<T>::unpack(a, x);
    if (p.draft) Row<T>::unpack(d, y);
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const double q = x[e];
      f(e, p.draft ? fmax(q - coef * (double)y[e], 0.) : bits >> e & 1 ? 0. : q, q);
    }
  }
};

// Tokens that children of row cur hold, as bits of the chunk that begins at token t0 (all were rejected)
__device__ __forceinline__ void mark_rejected(uint32_t* bits, int par, int tok, int cur, int64_t t0) {
  const int64_t x = tok - t0;
  if (par == cur && tok >= 0 && x >= 0 && x < kChunk) atomicOr(&bits[x >> 5], 1u << (x & 31));
}

template <typename T, bool kWalk, int kCap>
__global__ __launch_bounds__(kThreads) void verify_sums_kernel(VerifyDrafts p, WalkEnd* __restrict__ ends,
                                                               double2* __restrict__ sums) {
  constexpr int VEC = Vec16<T>::N, NV = kPer / VEC;
  __shared__ WalkLds<kCap> s;
  __shared__ uint32_t bits[kChunk / 32];
  __shared__ double2 red_l[kThreads / 64];
  const int b = blockIdx.x, c = blockIdx.y, tid = threadIdx.x;
  if (tid < kChunk / 32) bits[tid] = 0;
  int64_t r0, at;
  const int n = request_rows(p, b, r0);
  int cur;
  double coef;
  if (kWalk) {
    walk<T, kThreads, kCap>(p, r0, n, s);
    if (c == 0) write_walk<kThreads, kCap>(p, b, r0, n, s, ends);
    cur = s.cur;
    coef = s.coef;
    at = n > 0 ? r0 + cur : -1;
  } else {
    const WalkEnd e = ends[b];
    cur = e.cur;
    coef = e.coef;
    at = e.row;
    __syncthreads();
  }
  if (at < 0) return;
  const Row<T> row(p, at);
  Residual<T> x[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int64_t jk = (int64_t)c * kChunk + k * kThreads * VEC;
    if (row.inside(jk, jk + kThreads * VEC)) x[k].load(p, row, jk + tid * VEC);
    else if (jk < (int64_t)p.vocab + row.lead) x[k].load_any(p, row, jk + tid * VEC);
    else x[k].a = x[k].d = make_uint4(0, 0, 0, 0);
  }
  if (kWalk && !p.draft) {
    for (int i = cur + 1 + tid; i < n; i += kThreads) mark_rejected(bits, s.par[i], s.tok[i], cur, (int64_t)c * kChunk - row.lead);
    __syncthreads();
  }
  double r = 0., q = 0.;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int j = (k * kThreads + tid) * VEC;
    x[k].each(p, coef, bits[j >> 5] >> (j & 31), [&](int, double rt, double pt) {
      r += rt;
      q += pt;
    });
  }
  r = wave_sum_d(r);
  q = wave_sum_d(q);
  if ((tid & 63) == 0) red_l[tid >> 6] = make_double2(r, q);
  __syncthreads();
  if (tid == 0) {
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
  constexpr int VEC = Vec16<T>::N, NV = kPer / VEC;
  __shared__ uint32_t bits[kChunk / 32];
  __shared__ double wave_l[kThreads / 64];
  __shared__ int32_t hit_l, last_l;
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  // what does not wait for the walk's end is asked for with it
  const WalkEnd e = ends[b];
  const double2* s = sums + (int64_t)b * chunks;
  const double u = (double)p.u_next[b];
  double2 mine0 = lane < chunks ? s[lane] : make_double2(0., 0.);
  int64_t r0;
  const int n = request_rows(p, b, r0);
  int par = -1, tok = -1;
  if (!p.draft && tid < n) {
    par = p.parents ? p.parents[r0 + tid] : tid - 1;
    tok = p.tokens[r0 + tid];
  }
  if (tid < kChunk / 32) bits[tid] = 0;
  if (tid == 0) {
    hit_l = kChunk;
    last_l = -1;
  }
  if (e.row < 0) return;
  // every wave forms the same totals and running sums of the chunks, 64 at a time (up to 64, which is
  // 262137 tokens, the running sums give the total too)
  auto scan = [&](double x) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const double y = __shfl_up(x, o, 64);
      if (lane >= o) x += y;
    }
    return x;
  };
  double sum = scan(mine0.x), total = __shfl(sum, 63, 64);
  if (chunks > 64) {
    total = mine0.x;
    for (int c = 64 + lane; c < chunks; c += 64) total += s[c].x;
    total = wave_sum_d(total);
  }
  const bool empty = !(total > 0.);
  if (empty) {
    total = mine0.y;
    for (int c = 64 + lane; c < chunks; c += 64) total += s[c].y;
    total = wave_sum_d(total);
    if (!(total > 0.)) return;  // the walk left -1
    sum = scan(mine0.y);
  }
  const double want = u * total;
  double run = 0., before = 0.;
  int chunk = -1, last = -1;
  for (int c0 = 0; c0 < chunks && chunk < 0; c0 += 64) {
    if (c0) {
      mine0 = c0 + lane < chunks ? s[c0 + lane] : make_double2(0., 0.);
      sum = scan(empty ? mine0.y : mine0.x);
    }
    const double own = empty ? mine0.y : mine0.x;
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
  const Row<T> row(p, e.row);
  const int64_t j0 = (int64_t)chunk * kChunk, t0 = j0 - row.lead;
  Residual<T> x[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    if (row.inside(j0, j0 + kChunk)) x[k].load(p, row, j0 + tid * kPer + k * VEC);
    else x[k].load_any(p, row, j0 + tid * kPer + k * VEC);
  }
  __syncthreads();  // (bits, hit_l, last_l)
  if (!p.draft) {
    if (tid > e.cur) mark_rejected(bits, par, tok, e.cur, t0);
    for (int i = max(kThreads, e.cur + 1 - (e.cur + 1) % kThreads) + tid; i < n; i += kThreads)
      if (i > e.cur) mark_rejected(bits, p.parents ? p.parents[r0 + i] : i - 1, p.tokens[r0 + i], e.cur, t0);
    __syncthreads();
  }
  double v[kPer], own = 0.;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int j = tid * kPer + k * VEC;
    x[k].each(p, e.coef, bits[j >> 5] >> (j & 31), [&](int i, double rt, double pt) {
      v[k * VEC + i] = empty ? pt : rt;
      own += v[k * VEC + i];
    });
  }
  sum = scan(own);
  if (lane == 63) wave_l[tid >> 6] = sum;
  __syncthreads();
  double at = before + (sum - own);
  for (int i = 0; i < tid >> 6; ++i) at += wave_l[i];
  int first = kChunk, mine = -1;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    at += v[k];
    if (v[k] > 0.) {
      mine = tid * kPer + k;
      if (!past && at > want) first = min(first, mine);
    }
  }
  if (first < kChunk) atomicMin(&hit_l, first);
  if (mine >= 0) atomicMax(&last_l, mine);
  __syncthreads();
  if (tid == 0) p.out_tokens[(int64_t)b * p.max_rows + e.at] = (int32_t)(t0 + (hit_l < kChunk ? hit_l : last_l));
}

// pieces of a row that begins up to 7 elements into one
int chunk_count(int vocab) { return (int)(((int64_t)vocab + 7 + kChunk - 1) / kChunk); }

size_t ends_bytes(int batch) { return ((size_t)batch * sizeof(WalkEnd) + 255) / 256 * 256; }

template <typename T>
hipError_t launch_t(const VerifyDrafts& p, void* ws, hipStream_t stream) {
  WalkEnd* ends = static_cast<WalkEnd*>(ws);
  double2* sums = reinterpret_cast<double2*>(static_cast<char*>(ws) + ends_bytes(p.batch));
  const int chunks = chunk_count(p.vocab);
  const dim3 grid((unsigned)p.batch, (unsigned)chunks);
  if (p.draft && p.parents) {
    verify_walk_kernel<T><<<dim3((unsigned)p.batch), kWalkThreads, 0, stream>>>(p, ends);
    verify_sums_kernel<T, false, 1><<<grid, kThreads, 0, stream>>>(p, ends, sums);
  } else if (p.max_rows <= 128) {
    // (the LDS of the largest trees lets 6 blocks share a CU, 128 rows 8)
    verify_sums_kernel<T, true, 128><<<grid, kThreads, 0, stream>>>(p, ends, sums);
  } else {
    verify_sums_kernel<T, true, kTree><<<grid, kThreads, 0, stream>>>(p, ends, sums);
  }
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
