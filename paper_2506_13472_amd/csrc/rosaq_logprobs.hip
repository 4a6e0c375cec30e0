// Log probabilities of given tokens, the entropy and the largest alternatives, from rows of logits.
//
// A workgroup takes a row and reads it once: every thread keeps the largest logit that it has seen, m, and over what it has seen the sums
// S = sum 2^d and T = sum 2^d d, d = a (x - m) log2 e, brought to a new m when one comes.  Of the whole row then
//   log p(x) = a (x - m) - ln S        H = ln S - ln 2 T / S
// in which no large numbers cancel: both terms of H are positive, and x - m is taken before it is multiplied.
//
// The alternatives need no second look at the row but at a few pieces of it.  Every thread also keeps the largest logit of its share (every
// THREADS-th piece of 16 bytes) and where that was.  Of 256 groups of threads the top-th largest (or some of those next to it) is a bound that at least
// `top` logits reach, and only in the shares of threads whose largest does: about `top` shares of a THREADS-th of the row.  Those are read
// again (from a cache, mostly), what reaches the bound goes to a list in LDS, and every member counts how many are before it.
// A bound that lets three times as many logits through (the least of `top` groups' largest) cost more on the list than it saved (64 rows of 32000, five
// of each: 2.7 us more); a search for it, bit by bit, in place of the count that up to 32 alternatives take, 0.7 more.
//
// Order is by value and of equal values by the lower index, so that the answer does not depend on who finds what when.  The bound is of the same order: a
// value, and the last piece in which that value counts.  A row of one value throughout (or of few logits and -inf besides) so has a short list too.
// Where the list would be longer than its place, which takes a row whose largest logits nearly all lie in few threads' shares, the bound is
// found by bisection over the whole row.
//
// Many rows are bound by memory (inputs beyond the last-level cache: 4095 x 32000 fp16 54 us = 4.9 TB/s, with five, twenty and fifty alternatives 58, 66 and 80;
// 40000 rows 442 = 5.8 TB/s): a logit takes some nine vector operations and an exponential (four more), over half of the time that it takes to come.  Few rows are
// bound by the same arithmetic in one compute unit each: 64 rows of 32000 take 5.3 us (6.0 with the conversion apart), and with five alternatives 8.0: bound,
// shares, list and ranks, one after the other, a few hundred ns of latency each; from 33 alternatives on the search for the bound too (9.2 us with 32, 9.7 with
// 33, 11.5 with 64).  Built and no faster: the next pieces fetched ahead (one row of 262144, not shared, 2 us more); d as one product and difference, with a whole
// number in place of m a log2 e and the other way where that is too large for it (7.9 and 5.2, but 4096 rows of 1000 19.4 against 18.0); every wave looking
// through its own threads' shares, without a list of those (0.2 more).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <string>

#include "rosaq_gemm.h"
#include "rosaq_reduce.h"
#include "rosaq_rows.h"

namespace rosaq {

constexpr int kGroups = 256;        // of threads, over which the bound is found
constexpr int kList = 1024;         // logits on the list, at most

// One type of logits: elements of a 16-byte piece, the low bits of a key (below) that say nothing, and words of -inf.
struct Half {
  static constexpr int kEach = 8, kShift = 13;
  static constexpr uint32_t kNone = 0xfc00fc00u;
  typedef _Float16 type;
};
struct Brain {
  static constexpr int kEach = 8, kShift = 16;
  static constexpr uint32_t kNone = 0xff80ff80u;
  typedef __bf16 type;
};
struct Single {
  static constexpr int kEach = 4, kShift = 0;
  static constexpr uint32_t kNone = 0xff800000u;
  typedef float type;
};

__device__ __forceinline__ float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }     // NaN where one is NaN

// A number that orders as the logits do, NaN above all, zeros alike.
__device__ __forceinline__ uint32_t key_of(float x) {      // of -inf above 0, without its low bits too
  const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.f);
  return x != x ? 0xffffffffu : (b >> 31 ? ~b : b | 0x80000000u);
}
__device__ __forceinline__ float of_key(uint32_t k) {
  return k == 0xffffffffu ? NAN : __builtin_bit_cast(float, k >> 31 ? k & 0x7fffffffu : ~k);
}

// The sums over some logits, 2^d for d below -200 being nothing.
struct Sums { float m, s, t; };
constexpr float kLeast = -200.f, kLowest = -3.402823466e38f;
__device__ __forceinline__ Sums moved(const Sums& a, float m, float c) {
  const float d = larger((a.m - m) * c, kLeast), f = __builtin_amdgcn_exp2f(d);
  return Sums{m, a.s * f, f * __builtin_fmaf(a.s, d, a.t)};
}

// A row, cut into pieces of 16 bytes at 16-byte addresses; the first and last may be partly of the row.
template <class K> struct Row {
  const typename K::type* first;      // of its first element
  int before;                         // elements of the first piece in front of it
  int length, pieces;
  __device__ Row(const LogprobArgs& a, int64_t row) {
    first = static_cast<const typename K::type*>(a.logits) + row * a.ld;
    before = static_cast<int>((reinterpret_cast<uintptr_t>(first) & 15) / sizeof(typename K::type));
    length = a.V;
    pieces = (before + length + K::kEach - 1) / K::kEach;
  }
  __device__ __forceinline__ int index(int piece, int j) const { return piece * K::kEach + j - before; }
  __device__ __forceinline__ bool whole(int piece) const { return index(piece, 0) >= 0 && index(piece, K::kEach) <= length; }
  __device__ __forceinline__ uint4 load(int piece) const { return *reinterpret_cast<const uint4*>(first + index(piece, 0)); }
  static __device__ __forceinline__ float element(const uint4& w, int j) {
    if constexpr (K::kShift == 13) return static_cast<float>(as_h8(w)[j]);
    else if constexpr (K::kShift == 16) return __builtin_bit_cast(float, j % 2 ? (&w.x)[j / 2] & 0xffff0000u : (&w.x)[j / 2] << 16);
    else return __builtin_bit_cast(float, (&w.x)[j]);
  }
  // The largest element of a piece, NaN where one is NaN.
  static __device__ __forceinline__ float most(const uint4& w) {
    if constexpr (K::kShift == 13) {
      typedef _Float16 half2 __attribute__((ext_vector_type(2)));
      auto two = [](uint32_t v) { return __builtin_bit_cast(half2, v); };
      const half2 a = __builtin_elementwise_maximum(__builtin_elementwise_maximum(two(w.x), two(w.y)), __builtin_elementwise_maximum(two(w.z), two(w.w)));
      return larger(static_cast<float>(a[0]), static_cast<float>(a[1]));
    } else {
      float top = element(w, 0);
#pragma unroll
      for (int j = 1; j < K::kEach; ++j) top = larger(top, element(w, j));
      return top;
    }
  }
  // Of any piece: -inf in place of what is not the row's; the places (bits) of those that are.
  __device__ __forceinline__ uint32_t load_any(int piece, uint4* w) const {
    if (whole(piece)) {
      *w = load(piece);
      return (1u << K::kEach) - 1;
    }
    uint32_t to[4] = {K::kNone, K::kNone, K::kNone, K::kNone}, there = 0;
#pragma unroll
    for (int j = 0; j < K::kEach; ++j) {
      const int at = index(piece, j);
      if (at < 0 || at >= length) continue;
      there |= 1u << j;
      if constexpr (K::kEach == 4) to[j] = __builtin_bit_cast(uint32_t, first[at]);
      else to[j / 2] = j % 2 ? (to[j / 2] & 0xffffu) | static_cast<uint32_t>(__builtin_bit_cast(uint16_t, first[at])) << 16
                             : (to[j / 2] & 0xffff0000u) | __builtin_bit_cast(uint16_t, first[at]);
    }
    *w = make_uint4(to[0], to[1], to[2], to[3]);
    return there;
  }
};

// A bound: a key without its low bits, and of logits of that key the last piece that counts.  As one number, the larger the fewer reach it.
typedef uint64_t Bound;
__device__ __forceinline__ Bound bound_of(uint32_t key, int piece) { return static_cast<uint64_t>(key) << 32 | ~static_cast<uint32_t>(piece); }

// A number of BITS bits that, as `count` says, at least n reach and no more than n + slack, or, where equal numbers leave none, the largest that n reach.
template <int BITS, class F> __device__ __forceinline__ uint32_t reached_by(int n, int slack, F count) {
  uint32_t v = 0;
#pragma unroll 1
  for (int bit = BITS - 1; bit >= 0; --bit) {
    const int reach = count(v | 1u << bit);
    if (reach >= n) v |= 1u << bit;
    if (reach >= n && reach <= n + slack) break;
  }
  return v;
}

// A logit and where it is, ordered as the alternatives are.
__device__ __forceinline__ uint64_t member_of(uint32_t key, int at) { return static_cast<uint64_t>(key) << 32 | ~static_cast<uint32_t>(at); }
__device__ __forceinline__ int index_of(uint64_t member) { return static_cast<int>(~static_cast<uint32_t>(member)); }

// How many of a list in LDS (in pairs, behind its n members zeros up to a multiple of eight) are before this one.
__device__ __forceinline__ int rank_of(uint64_t member, const ulonglong2* list, int n) {
  int before = 0;
#pragma unroll 1
  for (int o = 0; o < n; o += 8) {
    ulonglong2 w[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) w[u] = list[o / 2 + u];
#pragma unroll
    for (int u = 0; u < 4; ++u) before += (w[u].x > member) + (w[u].y > member);
  }
  return before;
}

// The sums of a workgroup's waves, from LDS to all threads.
template <int N> __device__ __forceinline__ Sums sums_of(const float (&m)[N], const float (&s)[N], const float (&t)[N], float c) {
  const int w = threadIdx.x % N;
  Sums a = moved(Sums{m[w], s[w], t[w]}, row_all<N>(m[w], larger), c);
  a.s = row_all<N>(a.s, added<float>);
  a.t = row_all<N>(a.t, added<float>);
  return a;
}

// What a row's sums say.
struct Answer {
  float m, scale, log2_s, share;       // share: T / S
  __device__ Answer(const Sums& a, float scale) : m(a.m), scale(scale), log2_s(log2f(a.s)), share(a.t / a.s) {}
  // The difference by halves, exact but for subnormal numbers: that of logits at both ends of fp32's range is beyond it, its product with the scale need not be.
  __device__ __forceinline__ float log_p(float x) const { return (0.5f * x - 0.5f * m) * (2.f * scale) - log2_s * 0.6931471805599453f; }
  __device__ __forceinline__ float entropy() const { return (log2_s - share) * 0.6931471805599453f; }
};
// The given tokens of a row, in two steps, so that nothing waits for them: `step` threads take them in turn, and the first round's are fetched ahead.
template <class K> __device__ __forceinline__ int64_t token_of(const LogprobArgs& a, int64_t row, int g) { return g < a.given ? a.tokens[row * a.given + g] : -1; }
template <class K> __device__ __forceinline__ float logit_of(const LogprobArgs& a, const Row<K>& x, int64_t token) {
  return token >= 0 && token < a.V ? static_cast<float>(x.first[token]) : NAN;
}
template <class K>
__device__ __forceinline__ void give(const LogprobArgs& a, int64_t row, const Row<K>& x, const Answer& y, int g, int step, int64_t token, float logit) {
  while (g < a.given) {
    a.given_out[row * a.given + g] = token < 0 ? 0.f : y.log_p(logit);
    g += step;
    token = token_of<K>(a, row, g);
    logit = logit_of(a, x, token);
  }
}

// Results of the parts of a row (SPLIT), of part p of row r at r parts + p: sums, then the alternatives' members, largest first, 0 behind them.
struct Parts {
  float4* sums;
  uint64_t* members;
  __device__ Parts(const LogprobArgs& a) : sums(static_cast<float4*>(a.ws)), members(reinterpret_cast<uint64_t*>(sums + static_cast<int64_t>(a.M) * a.parts)) {}
};

template <class K, int THREADS, bool TOP, bool SPLIT>
__global__ __launch_bounds__(THREADS) void logprobs_kernel(LogprobArgs a) {
  constexpr int E = K::kEach, kWaves = THREADS / 64, kAhead = 4, kBits = 32 - K::kShift;
  __shared__ float lds_m[kWaves], lds_s[kWaves], lds_t[kWaves];
  __shared__ Bound group[TOP ? kGroups : 1], lds_bound;
  __shared__ int share[TOP ? THREADS : 1];   // threads whose share holds logits that reach the bound
  __shared__ ulonglong2 list[TOP ? kList / 2 + 4 : 1];
  __shared__ int shares, members, count;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const float c = a.scale * 1.4426950408889634f;
  uint64_t* const member = reinterpret_cast<uint64_t*>(list);
  const int64_t tasks = SPLIT ? static_cast<int64_t>(a.M) * a.parts : a.M;
  for (int64_t task = blockIdx.x; task < tasks; task += gridDim.x) {
    const int64_t row = SPLIT ? task / a.parts : task;
    const Row<K> x(a, row);
    // the pieces of this workgroup, and those of them that are whole
    const int each = SPLIT ? (x.pieces + a.parts - 1) / a.parts : x.pieces, lo = SPLIT ? static_cast<int>(task % a.parts) * each : 0;
    const int hi = min(lo + each, x.pieces), turns = (each + THREADS - 1) / THREADS;
    const int first = lo == 0 && !x.whole(0) ? 1 : lo, end = hi == x.pieces && first < hi && !x.whole(hi - 1) ? hi - 1 : hi;
    Sums sums{kLowest, 0.f, 0.f};
    uint32_t best_key = 0;                   // of this thread's share: the largest, 0 without one, and the first piece that holds it
    int best_piece = lo + tid;
    Bound best = 0;                          // the two as one
    // v - m of an fp16 v as a product with a one that the compiler does not know: an instruction with the conversion in it
    float one = 1.f;
    asm("" : "+s"(one));
    auto add = [&](float v) {
      const float d = fmaxf((K::kShift == 13 ? __builtin_fmaf(v, one, -sums.m) : v - sums.m) * c, kLeast), e = __builtin_amdgcn_exp2f(d);
      sums.s += e;
      sums.t = __builtin_fmaf(e, d, sums.t);
    };
    const int g = tid - (THREADS - 64);      // the last wave answers for the given tokens
    const int64_t token = !SPLIT && g >= 0 ? token_of<K>(a, row, g) : -1;
    for (int p0 = lo + tid < first ? lo + tid + THREADS : lo + tid; p0 < end; p0 += kAhead * THREADS) {
      uint4 w[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int p = p0 + u * THREADS;
        w[u] = p < end ? x.load(p) : make_uint4(K::kNone, K::kNone, K::kNone, K::kNone);
      }
      float most = sums.m;
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const float top = x.most(w[u]);
        if constexpr (TOP) {
          const uint32_t k = key_of(top);
          if (k > best_key && p0 + u * THREADS < end) { best_key = k; best_piece = p0 + u * THREADS; }
        }
        most = larger(most, top);
      }
      sums = moved(sums, most, c);
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
#pragma unroll
        for (int j = 0; j < E; ++j) add(x.element(w[u], j));
    }
    // pieces that are partly of the row: its first and its last
#pragma unroll 1
    for (int p = lo; p < hi; p = p < hi - 1 ? hi - 1 : hi) {
      if (x.whole(p) || tid != (p - lo) % THREADS) continue;
      uint4 w;
      x.load_any(p, &w);
      const float top = x.most(w);
      if constexpr (TOP) {
        const uint32_t k = key_of(top);
        if (k > best_key || (k == best_key && p < best_piece)) { best_key = k; best_piece = p; }
      }
      sums = moved(sums, larger(sums.m, top), c);
#pragma unroll
      for (int j = 0; j < E; ++j) add(x.element(w, j));
    }
    const float logit = logit_of(a, x, token);
    sums = moved(sums, wave_all(sums.m, larger), c);
    sums.s = wave_all(sums.s, added<float>);
    sums.t = wave_all(sums.t, added<float>);
    if (lane == 0) { lds_m[wave] = sums.m; lds_s[wave] = sums.s; lds_t[wave] = sums.t; }
    if constexpr (TOP) {
      best = best_key ? bound_of(best_key >> K::kShift, best_piece) : 0;
      Bound most = best;
#pragma unroll
      for (int n = 1; n < THREADS / kGroups; n *= 2) most = max(most, __shfl_xor(most, n, 64));
      if (tid % (THREADS / kGroups) == 0) group[tid / (THREADS / kGroups)] = most;
      if (tid == 0) { shares = 0; members = 0; }
    }
    __syncthreads();
    sums = sums_of(lds_m, lds_s, lds_t, c);
    const Answer answer(sums, a.scale);
    if constexpr (SPLIT) {
      if (tid == 0) Parts(a).sums[task] = make_float4(sums.m, sums.s, sums.t, 0.f);
    }
    if constexpr (TOP) {
      if (wave == 0) {
        uint32_t k[kGroups / 64], p[kGroups / 64];
#pragma unroll
        for (int i = 0; i < kGroups / 64; ++i) {
          const Bound g = group[i * 64 + lane];
          k[i] = static_cast<uint32_t>(g >> 32);
          p[i] = static_cast<uint32_t>(g);
        }
        uint32_t lane_most = k[0];
#pragma unroll
        for (int i = 1; i < kGroups / 64; ++i) lane_most = max(lane_most, k[i]);
        // groups that reach a key
        auto at_least = [&](uint32_t v) {
          int n = 0;
#pragma unroll
          for (int i = 0; i < kGroups / 64; ++i) n += __popcll(__ballot(k[i] >= v));
          return n;
        };
        // For few alternatives a lane's four groups are one, which lets hardly more through, and each lane counts the lanes above it; else a search.  A row of few
        // pieces has fewer groups than alternatives: all of it is on the list.  In the search a few groups too many cost less than to tell them apart
        uint32_t key;
        if (a.top <= 32) {
          int above = 0;
#pragma unroll
          for (int o = 0; o < 64; ++o) above += lane_of(lane_most, o) > lane_most ? 1 : 0;
          key = wave_all(above < a.top ? lane_most : 0xffffffffu, [](uint32_t a, uint32_t b) { return min(a, b); });
        } else {
          key = reached_by<kBits>(a.top, 16, at_least);
        }
        uint32_t last = 0;
        if (key != 0 && at_least(key) > a.top + 24)
          last = reached_by<32>(a.top, 16, [&](uint32_t v) {
            int n = 0;
#pragma unroll
            for (int i = 0; i < kGroups / 64; ++i) n += __popcll(__ballot(k[i] > key || (k[i] == key && p[i] >= v)));
            return n;
          });
        if (lane == 0) lds_bound = static_cast<uint64_t>(key) << 32 | last;
      }
      __syncthreads();
      Bound b = lds_bound;
      if (best >= b && best) share[atomicAdd(&shares, 1)] = tid;
      __syncthreads();
      int n_shares = shares, log_lanes = turns > 8 ? 4 : 3;     // threads of a share
#pragma unroll 1
      while (true) {
        const uint32_t least = static_cast<uint32_t>(b >> 32);
        const int lanes = 1 << log_lanes;
#pragma unroll 1
        for (int s = tid >> log_lanes; s < n_shares; s += THREADS >> log_lanes) {
#pragma unroll 1
          for (int p = lo + share[s] + (tid & (lanes - 1)) * THREADS; p < hi; p += lanes * THREADS) {
            // all of a piece's logits that reach the bound take their places on the list at once
            const bool with = bound_of(least, p) >= b;          // those of that key too
            uint4 w;
            const uint32_t there = x.load_any(p, &w);
            uint32_t key[E], hits = 0;
#pragma unroll
            for (int j = 0; j < E; ++j) {
              key[j] = key_of(x.element(w, j));
              const uint32_t k = key[j] >> K::kShift;
              hits |= (k > least || (k == least && with) ? 1u : 0u) << j;
            }
            hits &= there;
            if (hits == 0) continue;
            int m = atomicAdd(&members, __popc(hits));
#pragma unroll
            for (int j = 0; j < E; ++j)
              if (hits >> j & 1) {
                if (m < kList) member[m] = member_of(key[j], x.index(p, j));
                ++m;
              }
          }
        }
        __syncthreads();
        if (members <= kList) break;
        // counts over all pieces, of logits that reach a bound
        auto count_of = [&](Bound o) {
          __syncthreads();
          if (tid == 0) count = 0;
          __syncthreads();
          int n = 0;
#pragma unroll 1
          for (int p = lo + tid; p < hi; p += THREADS) {
            uint4 w;
            const uint32_t there = x.load_any(p, &w);
#pragma unroll
            for (int j = 0; j < E; ++j) n += (there >> j & 1) && bound_of(key_of(x.element(w, j)) >> K::kShift, p) >= o;
          }
          n = wave_all(n, [](int a, int b) { return a + b; });
          if (lane == 0) atomicAdd(&count, n);
          __syncthreads();
          return count;
        };
        const uint32_t key = reached_by<kBits>(a.top, 64, [&](uint32_t v) { return count_of(bound_of(v, -1)); });
        b = static_cast<uint64_t>(key) << 32 | reached_by<32>(a.top, 64, [&](uint32_t v) { return count_of(static_cast<uint64_t>(key) << 32 | v); });
        __syncthreads();
        if (tid == 0) members = 0;
        share[tid] = tid;
        n_shares = THREADS;
        __syncthreads();
      }
      const int n = min(members, kList);
      if (tid < 8) member[n + tid] = 0;
      __syncthreads();
      for (int i = tid; i < n; i += THREADS) {
        const uint64_t mine = member[i];
        const int before = rank_of(mine, list, n);
        if (before >= a.top) continue;
        if constexpr (SPLIT) {
          Parts(a).members[task * a.top + before] = mine;
        } else {
          a.top_ids[row * a.top + before] = index_of(mine);
          a.top_out[row * a.top + before] = answer.log_p(of_key(static_cast<uint32_t>(mine >> 32)));
        }
      }
      if constexpr (SPLIT)
        for (int i = n + tid; i < a.top; i += THREADS) Parts(a).members[task * a.top + i] = 0;
    }
    if constexpr (!SPLIT) {
      if (a.entropy && g == 0) a.entropy[row] = answer.entropy();
      if (g >= 0) give(a, row, x, answer, g, 64, token, logit);
    }
    __syncthreads();                         // the next row uses the same LDS
  }
}

// Joins the parts of a row, a workgroup each: the sums in their order, and the alternatives from those of the parts.
template <class K> __global__ __launch_bounds__(256) void logprobs_join_kernel(LogprobArgs a) {
  __shared__ float lds_m[kMaxParts], lds_s[kMaxParts], lds_t[kMaxParts];
  __shared__ ulonglong2 list[kMaxTop * kMaxParts / 2 + 4];
  uint64_t* const member = reinterpret_cast<uint64_t*>(list);
  const int tid = threadIdx.x, n = a.parts * a.top;
  const int64_t row = blockIdx.x;
  const Parts in(a);
  const float c = a.scale * 1.4426950408889634f;
  const Row<K> x(a, row);
  const int64_t token = token_of<K>(a, row, tid);
  for (int i = tid; i < n; i += 256) member[i] = in.members[row * n + i];
  if (tid < 8) member[n + tid] = 0;
  if (tid < kMaxParts) {
    const float4 s = tid < a.parts ? in.sums[row * a.parts + tid] : make_float4(kLowest, 0.f, 0.f, 0.f);
    lds_m[tid] = s.x; lds_s[tid] = s.y; lds_t[tid] = s.z;
  }
  const float logit = logit_of(a, x, token);
  __syncthreads();
  const Answer answer(sums_of(lds_m, lds_s, lds_t, c), a.scale);
  if (a.entropy && tid == 0) a.entropy[row] = answer.entropy();
  give(a, row, x, answer, tid, 256, token, logit);
  for (int i = tid; i < n; i += 256) {
    const uint64_t mine = member[i];
    if (mine == 0) continue;
    const int before = rank_of(mine, list, n);
    if (before >= a.top) continue;
    a.top_ids[row * a.top + before] = index_of(mine);
    a.top_out[row * a.top + before] = answer.log_p(of_key(static_cast<uint32_t>(mine >> 32)));
  }
}

template <class K, int THREADS, bool SPLIT> static void run(const LogprobArgs& a, hipStream_t st) {
  const unsigned grid = static_cast<unsigned>(std::min<int64_t>(static_cast<int64_t>(a.M) * (SPLIT ? a.parts : 1), 1 << 20));
  if (a.top) logprobs_kernel<K, THREADS, true, SPLIT><<<grid, THREADS, 0, st>>>(a);
  else logprobs_kernel<K, THREADS, false, SPLIT><<<grid, THREADS, 0, st>>>(a);
}

// Threads of a workgroup.  Few lanes go idle in a row of few pieces, and more workgroups of 256 than of 512 run beside each other, of which some read while
// others look for alternatives; long rows want more loads under way.  us with 512 / 256 threads, fp16, five alternatives: 64 rows of 8000 6.5 / 5.7, of
// 32000 8.1 / 8.9, of 131072 18.0 / 23.1; 4096 rows of 8000 39.8 / 24.2, of 32000 62.3 / 56.4; fp32, twenty: 64 of 8000 6.0 / 6.3, 4096 of 32000 102 / 121.
static bool wide(const LogprobArgs& a) {
  const int64_t bytes = static_cast<int64_t>(a.V) * (a.type == ROSAQ_F32 ? 4 : 2);
  return bytes > (a.M > 640 ? 65536 : 32768);
}

// A compute unit alone takes some ten logits a ns, so that few long rows are better shared by several, at the price of another launch.  us in 1 / 2 / 4 / 8 / 16
// parts, fp16, five alternatives: one row of 65536 9.5 / 9.8 / 8.8 / 9.0 / 9.6, of 262144 26.2 / 18.3 / 12.6 / 10.5 / 9.8; 64 of 131072 17.9 / 14.8 / 12.0 / 12.7 / 16.6;
// 128 of 65536 11.4 / 11.9 / 12.7 / 16.1 / 24.1 (four here), of 262144 32.2 / 23.7 / 21.9 / 23.0 / 27.0; 257 of 32000 11.0 / 13.7 / 17.8 / 25.6 / 34.3.
int parts_of_logprobs(const LogprobArgs& a) {
  if (a.V < 65536) return 1;
  return std::max(1, std::min({kMaxParts, a.V / 16384, 512 / a.M}));
}

template <class K> static void run(const LogprobArgs& a, hipStream_t st) {
  if (a.parts > 1) {
    run<K, 512, true>(a, st);
    logprobs_join_kernel<K><<<static_cast<unsigned>(a.M), 256, 0, st>>>(a);
  } else if (wide(a)) {
    run<K, 512, false>(a, st);
  } else {
    run<K, 256, false>(a, st);
  }
}

int launch_logprobs(const LogprobArgs& a, void* stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (a.type == ROSAQ_F16) run<Half>(a, st);
  else if (a.type == ROSAQ_BF16) run<Brain>(a, st);
  else run<Single>(a, st);
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return ROSAQ_OK;
  try { set_error(std::string("logprobs: ") + hipGetErrorString(e)); } catch (...) {}     // no memory for the text
  return ROSAQ_ERR_HIP;
}

}  // namespace rosaq
