// Logits with penalties for what was said, biases and masks, as logits or as probabilities (qcf_shape_logits).
//
// A block takes a piece of a few consecutive rows.  How often each of the piece's tokens was said is counted in LDS
// from the request's history, once, and the drafted tokens that a row follows (32 bits per token: the count in the
// answer, and whether the prompt has it; whole numbers, so the order of the additions is of no account), with the
// entry of the bias list that is a token's last in the same word.  Probabilities take two launches: a piece's
// maximum and its sum of exponentials, then the row's from all of them (in the pieces' order) and the values; a row
// of one piece takes one.  z is formed the same way both times, so nothing is stored in between.
// Bound: instructions in the first launch (about 13 vector instructions per token where its vector has a token
// that was said), HBM in the second.  64 rows of 128000 tokens in float32 31.7 us (2.1 TB/s of logits read once and
// probabilities written once), 288 rows of 150001 tokens of drafted trees, bf16 to float32, with biases and masks 132 us
// (2.0 TB/s), without them 108 us (2.4 TB/s).
#include <float.h>

#include <algorithm>
#include <type_traits>

#include "qcf_device.h"
#include "qcf_turns_launch.h"

namespace qcf {
namespace {

constexpr int kThreads = 256;
constexpr int kVec = 8;  // tokens of a thread at a time
constexpr int kWaves = kThreads / 64;
// Where the biases' entries are kept: nowhere, in the upper half of the tokens' counts, or, for long lists and histories
// whose counts could pass 15 bits, beside them (pieces are half as long then: the trees above 149 us in place of 132)
enum Bias { kNone, kPacked, kBeside };
// Tokens of a block's piece: 32 KB of LDS for what is looked up of them
constexpr int piece_of(int bias) { return bias == kBeside ? 4096 : 8192; }
constexpr int64_t kShapeBlocks = 1024;

// Of a token's word: it was said in the prompt; its count; where its bias begins (kPacked)
constexpr uint32_t said_bit(int bias) { return bias == kPacked ? 1u << 15 : 1u << 31; }

enum Mode { kLogits, kStats, kWrite, kWhole };

// Of a part of a row.  With c = log2(e) / T in float32, exp(z / T) is exp2(z c) but for c's rounding, and exp2(z c - m) with
// one fused multiply-add keeps that product exact, so that a token near the maximum is hardly off at all.  The rounding of
// m, up to 2^-24 of it, is the same for all of a part and falls out of the quotient; beyond 2^22 (small temperatures) it
// would be too much to be an exponent, and such a part's z are taken less the largest first (where z c may pass float32).
struct Stat {
  float m, s;  // the maximum times c, sum of exp2(z c - m), of a big one exp2((z - max) c); T = 0: the maximum
  int at;      // lowest token with the maximum (T = 0)
  float z;     // the maximum
};

// a value that is the same in every lane, in scalar registers
__device__ __forceinline__ int uni(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ float uni(float x) { return __int_as_float(uni(__float_as_int(x))); }

__device__ __forceinline__ float finite(float m) { return m == -INFINITY ? 0.f : m; }
__device__ __forceinline__ bool is_big(float m) { return fabsf(finite(m)) > 0x1p22f; }

// What a part's sum counts for in one with the maximum r.m (r.z).  Where one of them may be big (they need not both be) the
// difference of what the sums are taken of is formed in float64, which holds the products.
template <bool kBig>
__device__ __forceinline__ float share_of(float m, float z, const Stat& r, float c) {
  if (!kBig) return __builtin_amdgcn_exp2f(m - finite(r.m));
  const double a = is_big(m) ? (double)z * c : m, ref = is_big(r.m) ? (double)r.z * c : finite(r.m);
  return __builtin_amdgcn_exp2f((float)(a - ref));
}

// two parts of a row, the first's tokens before the second's
template <bool kBig>
__device__ __forceinline__ Stat both(const Stat& a, const Stat& b, bool cold, float c) {
  Stat r{fmaxf(a.m, b.m), 0.f, INT32_MAX, fmaxf(a.z, b.z)};
  if (cold) r.at = min(a.m == r.m ? a.at : INT32_MAX, b.m == r.m ? b.at : INT32_MAX);
  else r.s = a.s * share_of<kBig>(a.m, a.z, r, c) + b.s * share_of<kBig>(b.m, b.z, r, c);
  return r;
}

// Between the phases of a row only LDS is handed on: loads of the next ones stay in flight
__device__ __forceinline__ void meet() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

__device__ __forceinline__ void put(uint16_t* p, float x) { *p = f2bf(x); }
__device__ __forceinline__ void put(float* p, float x) { *p = x; }

// 16 bytes at an address that is aligned as its elements are
typedef uint32_t v4_at2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t v4_at4 __attribute__((ext_vector_type(4), aligned(4)));
template <typename T> struct Loose { typedef v4_at4 V; };
template <> struct Loose<uint16_t> { typedef v4_at2 V; };
template <typename T>
__device__ __forceinline__ uint4 load16(const T* p) {
  const typename Loose<T>::V x = *reinterpret_cast<const typename Loose<T>::V*>(p);
  return make_uint4(x[0], x[1], x[2], x[3]);
}
template <typename T>
__device__ __forceinline__ void store16(T* p, const uint4& x) {
  *reinterpret_cast<typename Loose<T>::V*>(p) = typename Loose<T>::V{x.x, x.y, x.z, x.w};
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&x)[kVec]) {
#pragma unroll
  for (int i = 0; i < kVec; i += Vec16<T>::N) store16(p + i, Vec16<T>::pack(x + i));
}

// One piece of `per` consecutive rows.  A row's loads go out while the row before it is still worked on.
template <typename In, typename Out, int kMode, int kBias>
__global__ __launch_bounds__(kThreads, 4) void shape_kernel(ShapeLogits p, Stat* stats, int pieces, int per) {
  constexpr int kPiece = piece_of(kBias), kVecs = kPiece / (kThreads * kVec);
  __shared__ __attribute__((aligned(16))) uint32_t said_l[kPiece];
  __shared__ __attribute__((aligned(16))) uint32_t bias_l[kBias == kBeside ? kPiece : 4];
  constexpr uint32_t kSaid = said_bit(kBias), kCount = kSaid - 1;
  __shared__ Stat red_l[kWaves];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int64_t block = (int64_t)blockIdx.y << kGridLog2 | blockIdx.x;
  const int64_t group = (uint64_t)block >> 32 ? block / pieces : (int64_t)((uint32_t)block / (uint32_t)pieces);
  const int64_t r_first = group * per, r_end = min(r_first + per, p.n_rows);
  if (r_first >= r_end) return;
  const int piece = (int)(block - group * pieces), p0 = piece * kPiece;
  const bool inside = p0 + kPiece <= p.vocab;

  auto clear = [&]() {
    for (int i = tid; i < kPiece / 4; i += kThreads) {
      reinterpret_cast<uint4*>(said_l)[i] = make_uint4(0, 0, 0, 0);
      if (kBias == kBeside) reinterpret_cast<uint4*>(bias_l)[i] = make_uint4(0, 0, 0, 0);
    }
  };
  clear();
  // the first row's request: as many end at or before it (every wave looks for itself)
  int b = 0;
  for (int i0 = 0; i0 < p.batch; i0 += 256) {
    int end[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) end[k] = p.cu_rows[min(i0 + 64 * k + lane, p.batch - 1) + 1];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      b += __builtin_popcountll(__ballot(i0 + 64 * k + lane < p.batch && (int64_t)end[k] <= r_first));
  }
  // everything that is one number per request comes by one load, a lane each
  const int32_t* param = p.cu_rows;  // lane 0: where the request begins; 1: and ends
  int instead = 0;
  const auto lane_is = [&](int i, const void* x, int none) {
    if (lane == i) {
      param = static_cast<const int32_t*>(x);
      instead = none;
    }
  };
  lane_is(2, p.hist_len, 0);
  lane_is(3, p.prompt_len, 0);
  lane_is(4, p.repetition, __float_as_int(1.f));
  lane_is(5, p.presence, 0);
  lane_is(6, p.frequency, 0);
  lane_is(7, p.temperature, __float_as_int(1.f));
  lane_is(8, p.bias_start, 0);
  lane_is(9, p.bias_start, 0);
  const int second = lane == 1 || lane == 9 ? 1 : 0;

  int counted = -1;             // the request whose history is counted
  int64_t first = 0, last = 0;  // its rows
  float rep = 1.f, inv_rep = 1.f, pres = 0.f, freq = 0.f, c = 1.f;
  bool cold = false;
  int64_t bias0 = 0;
  // adds (1) or takes back (-1) the drafted tokens that row r follows, of the request's from the given one on
  auto drafts = [&](int64_t r, int64_t from, uint32_t what) {
    const uint32_t* m = p.tree_mask ? p.tree_mask + r * p.mask_words : nullptr;
    const uint32_t end = (uint32_t)max(m ? min(last - first, (int64_t)p.mask_words * 32) : r - first + 1, (int64_t)0);
    for (uint32_t j = (uint32_t)from + tid; j < end; j += kThreads) {
      const uint32_t at = (uint32_t)p.tokens[first + j] - (uint32_t)p0;
      if (at < (uint32_t)kPiece && (!m || (m[j >> 5] >> (j & 31) & 1))) atomicAdd(&said_l[at], what);
    }
  };
  // the history's tokens from .. to - 1: `count` is given the place of each that lies in the piece
  auto scan = [&](const int32_t* h, int from, int to, auto count) {
    if (to - from < 4) {
      if (tid < to - from) {
        const uint32_t at = (uint32_t)h[from + tid] - (uint32_t)p0;
        if (at < (uint32_t)kPiece) count(at);
      }
      return;
    }
    constexpr int U = 4;
#pragma unroll 1
    for (int i0 = from + tid * 4; i0 < to; i0 += kThreads * 4 * U) {
      uint4 t[U];
#pragma unroll
      for (int k = 0; k < U; ++k) t[k] = load16(h + min(i0 + k * kThreads * 4, to - 4));
#pragma unroll
      for (int k = 0; k < U; ++k) {
        // (the last four overlap the four before: those are left out)
        const int i = i0 + k * kThreads * 4, over = i - min(i, to - 4);
        const uint32_t a0 = t[k].x - p0, a1 = t[k].y - p0, a2 = t[k].z - p0, a3 = t[k].w - p0;
        if (a0 < (uint32_t)kPiece && over < 1) count(a0);
        if (a1 < (uint32_t)kPiece && over < 2) count(a1);
        if (a2 < (uint32_t)kPiece && over < 3) count(a2);
        if (a3 < (uint32_t)kPiece && over < 4) count(a3);
      }
    }
  };
  // vector k of a row's tokens, as they are stored (behind the vocabulary its last one), and its word of the mask
  struct Raw {
    uint4 q[sizeof(In) * kVec / 16];
    uint32_t allowed;
  };
  // (the thread's number, formed anew: offsets that are kept from row to row would be a register each)
  auto self = [&]() {
    int i = threadIdx.x;
    asm volatile("" : "+v"(i));
    return i;
  };
  auto load = [&](int64_t r, int k) {
    const In* in = static_cast<const In*>(p.logits) + r * p.logits_stride;
    const int t0 = p0 + (self() + k * kThreads) * kVec;
    Raw x;
    if (p.vocab >= kVec) {
      // (aligned as its elements are; behind the vocabulary's last vector that one stands in, and the one that
      // it ends in is read again by elements)
      const int over = max(t0 + kVec - p.vocab, 0);
#pragma unroll
      for (int i = 0; i < (int)(sizeof x.q / 16); ++i) x.q[i] = load16(in + t0 - over + i * Vec16<In>::N);
      if (!inside && over > 0 && over < kVec) {
        In v[kVec];
#pragma unroll
        for (int e = 0; e < kVec; ++e) v[e] = in[min(t0 + e, p.vocab - 1)];
        __builtin_memcpy(x.q, v, sizeof x.q);
      }
    } else {
      In v[kVec];
#pragma unroll
      for (int e = 0; e < kVec; ++e) v[e] = in[min(t0 + e, p.vocab - 1)];
      __builtin_memcpy(x.q, v, sizeof x.q);
    }
    x.allowed = p.allowed ? p.allowed[r * p.allowed_words + (min(t0, p.vocab - 1) >> 5)] : ~0u;
    return x;
  };
  // its z; -infinity behind the vocabulary
  const bool masked = !inside || p.allowed;
  auto shaped = [&](const Raw& raw, int k, float (&x)[kVec]) {
    const int at = (self() + k * kThreads) * kVec, t0 = p0 + at;
    uint32_t said[kVec];
    *reinterpret_cast<uint4*>(said) = *reinterpret_cast<const uint4*>(said_l + at);
    *reinterpret_cast<uint4*>(said + 4) = *reinterpret_cast<const uint4*>(said_l + at + 4);
#pragma unroll
    for (int i = 0; i < (int)(sizeof raw.q / 16); ++i) Vec16<In>::unpack(raw.q[i], &x[i * Vec16<In>::N]);
    const uint32_t any = (said[0] | said[1]) | (said[2] | said[3]) | (said[4] | said[5]) | (said[6] | said[7]);
    if (any & (kSaid | kCount)) {
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        const float n = (float)(said[e] & kCount), z = x[e];
        const float by = said[e] & (kSaid | kCount) ? z > 0.f ? inv_rep : rep : 1.f;
        x[e] = fmaf(z, by, n > 0.f ? -fmaf(freq, n, pres) : 0.f);
      }
    }
    if (kBias == kPacked && any >> 16) {
#pragma unroll
      for (int e = 0; e < kVec; ++e)
        if (said[e] >> 16) x[e] += p.bias_value[bias0 + (said[e] >> 16) - 1];
    }
    if (kBias == kBeside) {
      uint32_t bias[kVec];
      *reinterpret_cast<uint4*>(bias) = *reinterpret_cast<const uint4*>(bias_l + at);
      *reinterpret_cast<uint4*>(bias + 4) = *reinterpret_cast<const uint4*>(bias_l + at + 4);
      if ((bias[0] | bias[1]) | (bias[2] | bias[3]) | (bias[4] | bias[5]) | (bias[6] | bias[7])) {
#pragma unroll
        for (int e = 0; e < kVec; ++e)
          if (bias[e]) x[e] += p.bias_value[bias0 + bias[e] - 1];
      }
    }
    if (masked) {
      uint32_t bits = raw.allowed >> (t0 & 31) & 0xffu;
      bits &= t0 + kVec <= p.vocab ? 0xffu : t0 < p.vocab ? (1u << (p.vocab - t0)) - 1u : 0u;
#pragma unroll
      for (int e = 0; e < kVec; ++e) x[e] = bits >> e & 1 ? x[e] : -INFINITY;
    }
  };

  Raw raw[kVecs], next[kVecs];
#pragma unroll
  for (int k = 0; k < kVecs; ++k) next[k] = load(r_first, k);
  for (int64_t r = r_first; r < r_end; ++r) {
#pragma unroll
    for (int k = 0; k < kVecs; ++k) raw[k] = next[k];
    if (r > r_first) {
      if (r >= last)
        while (b < p.batch && (int64_t)p.cu_rows[b + 1] <= r) ++b;
      meet();  // the last row's counts have been read
    }
    if (b >= p.batch) return;
    int64_t chained = 0;
    if (b != counted) {
      const int x = *(param ? param + b + second : p.cu_rows);
      const auto of = [&](int i) { return __builtin_amdgcn_readlane(param ? x : instead, i); };
      if (counted >= 0) clear();
      counted = b;
      first = of(0);
      last = min((int64_t)of(1), p.n_rows);
      rep = __int_as_float(of(4));
      inv_rep = 1.f / rep;
      pres = __int_as_float(of(5));
      freq = __int_as_float(of(6));
      const float temp = kMode == kLogits ? 1.f : __int_as_float(of(7));
      cold = temp == 0.f;
      c = cold ? 1.f : kLog2e / temp;
      if (c == INFINITY) c = FLT_MAX;  // (a T below 2^-127 counts as that)
      if (c == 0.f) c = 0x1p-149f;     // (infinite: -infinity times c has to stay that, and no finite z counts)
      meet();  // (the counts are zero)
      if (kBias != kNone) {
        bias0 = max(of(8), 0);
        const int64_t bias1 = min((int64_t)of(9), p.n_bias);
        for (int64_t e = bias0 + tid; e < bias1; e += kThreads) {
          const uint32_t at = (uint32_t)p.bias_token[e] - (uint32_t)p0, entry = (uint32_t)(e - bias0) + 1u;
          if (at < (uint32_t)kPiece) {
            if (kBias == kPacked) atomicMax(&said_l[at], entry << 16);
            else atomicMax(&bias_l[at], entry);
          }
        }
        if (kBias == kPacked) meet();  // (the words are not compared any more)
      }
      if (p.history) {
        const int n = min(max(of(2), 0), p.max_history), prompt = min(max(of(3), 0), n);
        const int32_t* h = p.history + (int64_t)b * p.history_stride;
        scan(h, 0, prompt, [&](uint32_t at) { atomicOr(&said_l[at], kSaid); });
        scan(h, prompt, n, [&](uint32_t at) { atomicAdd(&said_l[at], 1u); });
      }
    } else if (p.tree_mask) {
      drafts(r - 1, 0, (uint32_t)-1);
    } else {
      chained = r - first;  // (a chain's next row follows one token more)
    }
    if (p.tokens) drafts(r, chained, 1u);
    meet();
    if (r + 1 < r_end)
#pragma unroll
      for (int k = 0; k < kVecs; ++k) next[k] = load(r + 1, k);

    Stat all{-INFINITY, 0.f, INT32_MAX, -INFINITY};
    if (kMode == kStats || kMode == kWhole) {
      // the waves', each with its own maximum, then the block's in the waves' order
      float x[kVecs][kVec], m = -INFINITY;
#pragma unroll
      for (int k = 0; k < kVecs; ++k) {
        shaped(raw[k], k, x[k]);
#pragma unroll
        for (int e = 0; e < kVec; ++e) m = fmaxf(m, x[k][e]);
      }
      m = uni(wave_max(m));
      // (-infinity is kept for a part without a z above it)
      Stat wave{cold || m == -INFINITY ? m : fmaxf(m * c, -FLT_MAX), 0.f, INT32_MAX, m};
      if (cold) {
        const int id = self();
#pragma unroll
        for (int k = kVecs - 1; k >= 0; --k)
#pragma unroll
          for (int e = kVec - 1; e >= 0; --e)
            if (x[k][e] == m && m > -INFINITY) wave.at = p0 + (id + k * kThreads) * kVec + e;
        wave.at = wave_min_i(wave.at);
      } else {
        const auto sum = [&](auto exponent) {
#pragma unroll
          for (int k = 0; k < kVecs; ++k) {
            float s = 0.f;
#pragma unroll
            for (int e = 0; e < kVec; ++e) s += __builtin_amdgcn_exp2f(exponent(x[k][e]));
            wave.s += s;
          }
        };
        const float ref = finite(wave.m);
        if (is_big(wave.m)) sum([&](float z) { return (z - m) * c; });
        else sum([&](float z) { return fmaf(z, c, -ref); });
        wave.s = wave_sum(wave.s);
      }
      if (lane == 0) red_l[w] = wave;
      meet();
      const auto join = [&](auto big) {
#pragma unroll 1
        for (int i = 0; i < kWaves; ++i) all = both<decltype(big)::value>(all, red_l[i], cold, c);
      };
      // (two loops: the test within one 137 us for the trees above in place of 132)
      if (__ballot(is_big(red_l[lane % kWaves].m))) join(std::true_type{});
      else join(std::false_type{});
      if (kMode == kStats && tid == 0) stats[r * pieces + piece] = all;
    } else if (kMode == kWrite) {
      // the row's: pieces in their order, 64 at a time
      const Stat* st = stats + r * pieces;
#pragma unroll 1
      for (int i0 = 0; i0 < pieces; i0 += 64) {
        Stat one = st[min(i0 + lane, pieces - 1)];
        const bool there = i0 + lane < pieces;
        // (a row whose maximum is big has it in a part that is)
        const bool big = __ballot(is_big(one.m)) != 0;
        Stat some{uni(wave_max(there ? one.m : -INFINITY)), 0.f, INT32_MAX, -INFINITY};
        if (big) some.z = uni(wave_max(there ? one.z : -INFINITY));
        if (cold) {
          some.at = wave_min_i(there && one.m == some.m ? one.at : INT32_MAX);
        } else {
          float share = share_of<false>(one.m, one.z, some, c);
          if (big) share = share_of<true>(one.m, one.z, some, c);
          some.s = wave_sum(there ? one.s * share : 0.f);
        }
        if (i0 == 0) all = some;
        else all = both<true>(all, some, cold, c);
      }
    }
    if (kMode != kStats) {
      const bool big = uni(is_big(all.m) && !cold ? 1 : 0);
      const float ref = uni(big ? 0.f : finite(all.m)), inv = uni(all.s == 0.f ? 0.f : 1.f / all.s), top = uni(all.z);
      Out* out = static_cast<Out*>(p.out) + r * p.out_stride;
#pragma unroll
      for (int k = 0; k < kVecs; ++k) {
        const int t0 = p0 + (self() + k * kThreads) * kVec;
        float x[kVec];
        shaped(raw[k], k, x);
        if (kMode != kLogits) {
          if (big) {
#pragma unroll
            for (int e = 0; e < kVec; ++e) x[e] -= top;
          }
#pragma unroll
          for (int e = 0; e < kVec; ++e) x[e] = cold ? (t0 + e == all.at ? 1.f : 0.f) : __builtin_amdgcn_exp2f(fmaf(x[e], c, -ref)) * inv;
        }
        if (t0 + kVec <= p.vocab) {
          store8(out + t0, x);
        } else if (!inside) {
#pragma unroll
          for (int e = 0; e < kVec; ++e)
            if (t0 + e < p.vocab) put(out + t0 + e, x[e]);
        }
      }
    }
  }
}

inline int pieces_of(int vocab, int bias) { return (vocab + piece_of(bias) - 1) / piece_of(bias); }

template <typename In, typename Out, int kBias>
hipError_t launch_t(const ShapeLogits& p, bool probabilities, void* ws, hipStream_t stream) {
  const int pieces = pieces_of(p.vocab, kBias);
  const int per = (int)std::min<int64_t>((p.n_rows * pieces + kShapeBlocks - 1) / kShapeBlocks, 16);
  const dim3 grid = grid_of((p.n_rows + per - 1) / per * pieces);
  Stat* stats = static_cast<Stat*>(ws);
  if (!probabilities) {
    shape_kernel<In, Out, kLogits, kBias><<<grid, kThreads, 0, stream>>>(p, stats, pieces, per);
  } else if (pieces == 1) {
    shape_kernel<In, Out, kWhole, kBias><<<grid, kThreads, 0, stream>>>(p, stats, pieces, per);
  } else {
    shape_kernel<In, Out, kStats, kBias><<<grid, kThreads, 0, stream>>>(p, stats, pieces, per);
    shape_kernel<In, Out, kWrite, kBias><<<grid, kThreads, 0, stream>>>(p, stats, pieces, per);
  }
  return hipGetLastError();
}

template <typename In, typename Out>
hipError_t launch_b(const ShapeLogits& p, bool probabilities, void* ws, hipStream_t stream) {
  if (!p.bias_start) return launch_t<In, Out, kNone>(p, probabilities, ws, stream);
  // a token is counted once for each place of the history and for each row at most
  if ((p.history ? p.max_history : 0) + (p.tokens ? p.n_rows : 0) < 1 << 15 && p.n_bias < 1 << 16)
    return launch_t<In, Out, kPacked>(p, probabilities, ws, stream);
  return launch_t<In, Out, kBeside>(p, probabilities, ws, stream);
}

}  // namespace

size_t shape_logits_workspace(int64_t n_rows, int vocab) {
  const int pieces = pieces_of(vocab, kBeside);  // (the smaller pieces)
  return pieces > 1 ? (size_t)n_rows * pieces * sizeof(Stat) : 0;
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
