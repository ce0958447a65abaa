// Logits with penalties for what was said, biases and masks, as logits or as probabilities (qcf_shape_logits).
//
// A block takes a piece of one row.  How often each of the piece's tokens was said is counted in LDS from the
// request's history and the drafted tokens that the row follows (32 bits per token: bit 0 said at all, the
// count in the answer above it; whole numbers, so the order of the additions is of no account), and which
// entry of the bias list is a token's last beside it.  Probabilities take two launches: a piece's maximum and its sum
// of exponentials, then the row's from all of them (in the pieces' order) and the values; a row
// of one piece takes one.  z is formed the same way both times, so nothing is stored in between.
// Bound: HBM and the scan of the history by every block.
#include "qcf_device.h"
#include "qcf_turns_launch.h"

namespace qcf {
namespace {

constexpr int kThreads = 256;
constexpr int kVec = 8;                              // tokens of a thread at a time
constexpr int kVecs = 4;                             // times
constexpr int kPiece = kThreads * kVec * kVecs;      // tokens of a block
constexpr int kWaves = kThreads / 64;

enum Mode { kLogits, kStats, kWrite, kWhole };

struct Stat {
  float m, s;  // maximum, sum of exp(x - m)
  int at;      // lowest token with the maximum (T = 0)
  int pad;
};

// exp(y), y <= 0 (or NaN): the product's rounding error goes into the result, which is off by 2^-23 or so for any
// y where 2^(y log2 e) alone is off by |y| 2^-24
__device__ __forceinline__ float exp_of(float y) {
  y = y < -200.f ? -200.f : y;  // (0 already)
  const float t = y * kLog2e;
  const float e = __builtin_amdgcn_exp2f(t);
  return fmaf(e, fmaf(y, kLog2e, -t) * kLn2, e);
}

template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&x)[kVec]) {  // (aligned as its elements are)
  T v[kVec];
  __builtin_memcpy(v, p, sizeof v);
#pragma unroll
  for (int e = 0; e < kVec; ++e) x[e] = sizeof(T) == 2 ? bf2f((uint16_t)v[e]) : (float)v[e];
}
__device__ __forceinline__ void load8(const float* p, float (&x)[kVec]) { __builtin_memcpy(x, p, sizeof x); }
__device__ __forceinline__ float as_float(uint16_t x) { return bf2f(x); }
__device__ __forceinline__ float as_float(float x) { return x; }
__device__ __forceinline__ void put(uint16_t* p, float x) { *p = f2bf(x); }
__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void store8(uint16_t* p, const float (&x)[kVec]) {
  const uint4 v = Vec16<uint16_t>::pack(x);
  __builtin_memcpy(p, &v, sizeof v);
}
__device__ __forceinline__ void store8(float* p, const float (&x)[kVec]) { __builtin_memcpy(p, x, sizeof x); }

template <typename In, typename Out, int kMode, bool kBias>
__global__ __launch_bounds__(kThreads) void shape_kernel(ShapeLogits p, Stat* stats, int pieces) {
  __shared__ __attribute__((aligned(16))) uint32_t said_l[kPiece];
  __shared__ __attribute__((aligned(16))) uint32_t bias_l[kBias ? kPiece : 4];
  __shared__ float red_l[kWaves];
  __shared__ int redi_l[kWaves];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int64_t block = (int64_t)blockIdx.y << kGridLog2 | blockIdx.x;
  const int64_t r = block / pieces;
  if (r >= p.n_rows) return;
  const int piece = (int)(block - r * pieces), p0 = piece * kPiece;
  auto sum_i = [&](int x) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o, 64);
    __syncthreads();
    if (lane == 0) redi_l[w] = x;
    __syncthreads();
    x = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) x += redi_l[i];
    return x;
  };
  auto min_i = [&](int x) {
    x = wave_min_i(x);
    __syncthreads();
    if (lane == 0) redi_l[w] = x;
    __syncthreads();
    x = redi_l[0];
#pragma unroll
    for (int i = 1; i < kWaves; ++i) x = min(x, redi_l[i]);
    return x;
  };
  auto max_f = [&](float x) {
    x = wave_max(x);
    __syncthreads();
    if (lane == 0) red_l[w] = x;
    __syncthreads();
    x = red_l[0];
#pragma unroll
    for (int i = 1; i < kWaves; ++i) x = fmaxf(x, red_l[i]);
    return x;
  };
  auto sum_f = [&](float x) {
    x = wave_sum(x);
    __syncthreads();
    if (lane == 0) red_l[w] = x;
    __syncthreads();
    x = 0.f;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) x += red_l[i];
    return x;
  };
  // the row's request: as many end at or before it
  int before = 0;
  for (int i = tid; i < p.batch; i += kThreads) before += (int64_t)p.cu_rows[i + 1] <= r ? 1 : 0;
  const int b = sum_i(before);
  if (b >= p.batch) return;

  // what was said of the piece's tokens
  for (int i = tid; i < kPiece / 4; i += kThreads) {
    reinterpret_cast<uint4*>(said_l)[i] = make_uint4(0, 0, 0, 0);
    if (kBias) reinterpret_cast<uint4*>(bias_l)[i] = make_uint4(0, 0, 0, 0);
  }
  __syncthreads();
  if (p.history) {
    const int n = min(max(p.hist_len[b], 0), p.max_history);
    const int prompt = p.prompt_len ? p.prompt_len[b] : 0;
    const int32_t* h = p.history + (int64_t)b * p.history_stride;
    constexpr int U = 8;
    for (int i0 = tid; i0 < n; i0 += kThreads * U) {
      int t[U];
#pragma unroll
      for (int k = 0; k < U; ++k) t[k] = h[min(i0 + k * kThreads, n - 1)];
#pragma unroll
      for (int k = 0; k < U; ++k) {
        const int i = i0 + k * kThreads;
        const uint32_t x = (uint32_t)t[k] - (uint32_t)p0;
        if (i < n && t[k] >= 0 && x < (uint32_t)kPiece) {
          if (i < prompt) atomicOr(&said_l[x], 1u);
          else atomicAdd(&said_l[x], 2u);
        }
      }
    }
  }
  if (p.tokens) {
    const int64_t first = p.cu_rows[b];
    const int own = (int)(r - first);
    const int64_t last = min((int64_t)p.cu_rows[b + 1], p.n_rows);
    const int rows = (int)(last - first);
    const uint32_t* m = p.tree_mask ? p.tree_mask + r * p.mask_words : nullptr;
    const int end = m ? (int)min((int64_t)rows, (int64_t)p.mask_words * 32) : own + 1;
    for (int j = tid; j < end; j += kThreads) {
      const int t = p.tokens[first + j];
      const uint32_t x = (uint32_t)t - (uint32_t)p0;
      if (t >= 0 && x < (uint32_t)kPiece && (!m || (m[j >> 5] >> (j & 31) & 1))) atomicAdd(&said_l[x], 2u);
    }
  }
  int64_t bias0 = 0;
  if (kBias) {
    bias0 = max((int64_t)p.bias_start[b], (int64_t)0);
    const int64_t bias1 = min((int64_t)p.bias_start[b + 1], p.n_bias);
    for (int64_t e = bias0 + tid; e < bias1; e += kThreads) {
      const int t = p.bias_token[e];
      const uint32_t x = (uint32_t)t - (uint32_t)p0;
      if (t >= 0 && x < (uint32_t)kPiece) atomicMax(&bias_l[x], (uint32_t)(e - bias0) + 1u);
    }
  }
  __syncthreads();

  const float rep = p.repetition ? p.repetition[b] : 1.f, pres = p.presence ? p.presence[b] : 0.f;
  const float freq = p.frequency ? p.frequency[b] : 0.f;
  const float temp = kMode != kLogits && p.temperature ? p.temperature[b] : 1.f;
  const bool cold = temp == 0.f;
  const float inv_t = cold ? 1.f : 1.f / temp;
  const In* in = static_cast<const In*>(p.logits) + r * p.logits_stride;
  Out* out = static_cast<Out*>(p.out) + r * p.out_stride;
  const uint32_t* allowed = p.allowed ? p.allowed + r * p.allowed_words : nullptr;

  // x = z / T of the thread's tokens, -infinity behind the vocabulary
  float x[kVecs][kVec];
#pragma unroll
  for (int k = 0; k < kVecs; ++k) {
    const int at = (tid + k * kThreads) * kVec, t0 = p0 + at;
    if (t0 + kVec <= p.vocab) {
      load8(in + t0, x[k]);
    } else {
#pragma unroll
      for (int e = 0; e < kVec; ++e) x[k][e] = t0 + e < p.vocab ? as_float(in[t0 + e]) : -INFINITY;
    }
  }
#pragma unroll
  for (int k = 0; k < kVecs; ++k) {
    const int at = (tid + k * kThreads) * kVec, t0 = p0 + at;
    const uint32_t bits = !allowed ? 0xffu : t0 < p.vocab ? allowed[t0 >> 5] >> (t0 & 31) & 0xffu : 0u;
    uint32_t said[kVec], bias[kVec];
    *reinterpret_cast<uint4*>(said) = *reinterpret_cast<const uint4*>(said_l + at);
    *reinterpret_cast<uint4*>(said + 4) = *reinterpret_cast<const uint4*>(said_l + at + 4);
    if (kBias) {
      *reinterpret_cast<uint4*>(bias) = *reinterpret_cast<const uint4*>(bias_l + at);
      *reinterpret_cast<uint4*>(bias + 4) = *reinterpret_cast<const uint4*>(bias_l + at + 4);
    }
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
      float z = x[k][e];
      if (said[e]) {
        const float c = (float)(said[e] >> 1);
        z = z > 0.f ? z / rep : z * rep;
        z = fmaf(-freq, c, z);
        if (c > 0.f) z -= pres;
      }
      if (kBias && bias[e]) z += p.bias_value[bias0 + bias[e] - 1];
      if (!(bits >> e & 1) || t0 + e >= p.vocab) z = -INFINITY;
      x[k][e] = kMode == kLogits ? z : z * inv_t;
    }
  }
  auto store = [&](int k) {
    const int t0 = p0 + (tid + k * kThreads) * kVec;
    if (t0 + kVec <= p.vocab) {
      store8(out + t0, x[k]);
    } else {
#pragma unroll
      for (int e = 0; e < kVec; ++e)
        if (t0 + e < p.vocab) put(out + t0 + e, x[k][e]);
    }
  };
  if (kMode == kLogits) {
#pragma unroll
    for (int k = 0; k < kVecs; ++k) store(k);
    return;
  }
  Stat all;
  if (kMode != kWrite) {
    float m = -INFINITY;
#pragma unroll
    for (int k = 0; k < kVecs; ++k)
#pragma unroll
      for (int e = 0; e < kVec; ++e) m = fmaxf(m, x[k][e]);
    m = max_f(m);
    int at = INT32_MAX;
    float s = 0.f;
    if (cold) {
#pragma unroll
      for (int k = 0; k < kVecs; ++k)
#pragma unroll
        for (int e = 0; e < kVec; ++e)
          if (x[k][e] == m && m > -INFINITY) at = min(at, p0 + (tid + k * kThreads) * kVec + e);
      at = min_i(at);
    } else {
      const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
      for (int k = 0; k < kVecs; ++k)
#pragma unroll
        for (int e = 0; e < kVec; ++e) s += exp_of(x[k][e] - ref);
      s = sum_f(s);
    }
    all = Stat{m, s, at, 0};
    if (kMode == kStats) {
      if (tid == 0) stats[r * pieces + piece] = all;
      return;
    }
  } else {
    // the row's: pieces in their order, 64 at a time
    const Stat* st = stats + r * pieces;
    all = Stat{-INFINITY, 0.f, INT32_MAX, 0};
    for (int i0 = 0; i0 < pieces; i0 += 64) {
      const Stat one = st[min(i0 + lane, pieces - 1)];
      const bool there = i0 + lane < pieces;
      const float m = wave_max(there ? one.m : -INFINITY), mn = fmaxf(all.m, m);
      if (cold) {
        const int at = wave_min_i(there && one.m == mn ? one.at : INT32_MAX);
        all.at = all.m == mn ? min(all.at, at) : at;
      } else {
        const float ref = mn == -INFINITY ? 0.f : mn;
        all.s = all.s * exp_of(all.m - ref) + wave_sum(there ? one.s * exp_of(one.m - ref) : 0.f);
      }
      all.m = mn;
    }
  }
  if (cold) {
#pragma unroll
    for (int k = 0; k < kVecs; ++k)
#pragma unroll
      for (int e = 0; e < kVec; ++e) x[k][e] = p0 + (tid + k * kThreads) * kVec + e == all.at ? 1.f : 0.f;
  } else {
    const float ref = all.m == -INFINITY ? 0.f : all.m;
    const float inv = all.s == 0.f ? 0.f : 1.f / all.s;
#pragma unroll
    for (int k = 0; k < kVecs; ++k)
#pragma unroll
      for (int e = 0; e < kVec; ++e) x[k][e] = exp_of(x[k][e] - ref) * inv;
  }
#pragma unroll
  for (int k = 0; k < kVecs; ++k) store(k);
}

inline int pieces_of(int vocab) { return (vocab + kPiece - 1) / kPiece; }

template <typename In, typename Out, bool kBias>
hipError_t launch_t(const ShapeLogits& p, bool probabilities, void* ws, hipStream_t stream) {
  const int pieces = pieces_of(p.vocab);
  const dim3 grid = grid_of(p.n_rows * pieces);
  Stat* stats = static_cast<Stat*>(ws);
  if (!probabilities) {
    shape_kernel<In, Out, kLogits, kBias><<<grid, kThreads, 0, stream>>>(p, stats, pieces);
  } else if (pieces == 1) {
    shape_kernel<In, Out, kWhole, kBias><<<grid, kThreads, 0, stream>>>(p, stats, pieces);
  } else {
    shape_kernel<In, Out, kStats, kBias><<<grid, kThreads, 0, stream>>>(p, stats, pieces);
    shape_kernel<In, Out, kWrite, kBias><<<grid, kThreads, 0, stream>>>(p, stats, pieces);
  }
  return hipGetLastError();
}

template <typename In, typename Out>
hipError_t launch_b(const ShapeLogits& p, bool probabilities, void* ws, hipStream_t stream) {
  return p.bias_start ? launch_t<In, Out, true>(p, probabilities, ws, stream)
                      : launch_t<In, Out, false>(p, probabilities, ws, stream);
}

}  // namespace

size_t shape_logits_workspace(int64_t n_rows, int vocab) {
  return pieces_of(vocab) > 1 ? (size_t)n_rows * pieces_of(vocab) * sizeof(Stat) : 0;
}

hipError_t launch_shape_logits(const ShapeLogits& p, bool in_bf16, bool out_bf16, bool probabilities, void* ws,
                               hipStream_t stream) {
  if (in_bf16)
    return out_bf16 ? launch_b<uint16_t, uint16_t>(p, probabilities, ws, stream)
                    : launch_b<uint16_t, float>(p, probabilities, ws, stream);
  return out_bf16 ? launch_b<float, uint16_t>(p, probabilities, ws, stream)
                  : launch_b<float, float>(p, probabilities, ws, stream);
}

}  // namespace qcf
