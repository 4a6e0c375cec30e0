// Log probabilities of given tokens, the entropy and the largest alternatives, from rows of logits.
//
// A workgroup takes a row and reads it once: every thread keeps the largest logit that it has seen, m, and over what it has seen the sums
// S = sum 2^d and T = sum 2^d d, d = a (x - m) log2 e, brought to a new m when one comes.  Of the whole row then
//   log p(x) = a (x - m) - ln S        H = ln S - ln 2 T / S
// in which no large numbers cancel: both terms of H are positive, and x - m is taken before it is multiplied.
//
// The alternatives need no second look at the row but at a few pieces of it.  Every thread also keeps the largest logit of its share (every
// THREADS-th piece of 16 bytes) and where that was.  Of 256 groups of threads the top-th largest is a bound that at least `top` logits
// reach, and logits that reach it lie only in the shares of threads whose largest does: about `top` shares of a THREADS-th of the row.  Those are read
// again (from a cache, mostly), what reaches the bound goes to a list in LDS, and every member counts how many are before it.
//
// Order is by value and of equal values by the lower index, so that the answer does not depend on who finds what when.  The bound is of the same order: a
// value, and the last piece in which that value counts.  A row of one value throughout (or of few logits and -inf besides) so has a short list too.
// Where the list would be longer than its place, which takes a row whose largest logits all lie in few threads' shares, the bound is
// found by bisection over the whole row.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <string>

#include "rosaq_gemm.h"
#include "rosaq_rows.h"

namespace rosaq {

constexpr int kGroups = 256;        // of threads, over which the bound is found
constexpr int kList = 1024;         // logits that reach it, at most

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
__device__ __forceinline__ Sums joined(const Sums& a, const Sums& b, float c) {
  const float m = larger(a.m, b.m);
  const Sums x = moved(a, m, c), y = moved(b, m, c);
  return Sums{m, x.s + y.s, x.t + y.t};
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
  // f(element, index) for those of a piece that are the row's
  template <class F> __device__ __forceinline__ void each(int piece, F f) const {
    if (whole(piece)) {
      const uint4 w = load(piece);
#pragma unroll
      for (int j = 0; j < K::kEach; ++j) f(element(w, j), index(piece, j));
    } else {
      for (int j = 0; j < K::kEach; ++j) {
        const int at = index(piece, j);
        if (at >= 0 && at < length) f(static_cast<float>(first[at]), at);
      }
    }
  }
};

// What a bound is: logits of a larger key, and those of its key in pieces up to `piece`.  Keys without their low bits.
struct Bound {
  uint32_t key;
  int piece;
  __device__ __forceinline__ bool reached(uint32_t k, int p) const { return k > key || (k == key && p <= piece); }
};

// The largest number of BITS bits that, as `count` says, at least n reach; or one that n reach and no more.
template <int BITS, class F> __device__ __forceinline__ uint32_t largest(int n, F count) {
  uint32_t v = 0;
  for (int bit = BITS - 1; bit >= 0; --bit) {
    const int reach = count(v | 1u << bit);
    if (reach >= n) v |= 1u << bit;
    if (reach == n) break;
  }
  return v;
}

__device__ __forceinline__ int wave_sum(int v) {
#pragma unroll
  for (int n = 1; n < 64; n *= 2) v += __shfl_xor(v, n, 64);
  return v;
}

template <class K, int THREADS, bool TOP>
__global__ __launch_bounds__(THREADS) void logprobs_kernel(LogprobArgs a) {
  constexpr int E = K::kEach, kWaves = THREADS / 64, kAhead = 4, kBits = 32 - K::kShift, kLanes = THREADS / kGroups;
  constexpr int kMember = TOP ? kList : 1, kGroup = TOP ? kGroups : 1, kShare = TOP ? THREADS : 1;
  __shared__ float lds_m[kWaves], lds_s[kWaves], lds_t[kWaves];
  __shared__ uint32_t group_key[kGroup];
  __shared__ int group_piece[kGroup];
  __shared__ int share[kShare];              // threads whose share holds logits that reach the bound
  __shared__ uint32_t member_key[kMember];
  __shared__ int member_at[kMember];
  __shared__ Bound bound;
  __shared__ int shares, members, count;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const float c = a.scale * 1.4426950408889634f;
  for (int64_t row = blockIdx.x; row < a.M; row += gridDim.x) {
    const Row<K> x(a, row);
    Sums sums{kLowest, 0.f, 0.f};
    uint32_t best_key = 0;                   // of this thread's share: the largest, 0 without one, and the first piece that holds it
    int best_piece = tid;
    auto seen = [&](float most, int piece) {
      if constexpr (TOP) {
        const uint32_t k = key_of(most);
        if (k > best_key) { best_key = k; best_piece = piece; }
      }
    };
    auto add = [&](float v) {
      const float d = larger((v - sums.m) * c, kLeast), e = __builtin_amdgcn_exp2f(d);
      sums.s += e;
      sums.t = __builtin_fmaf(e, d, sums.t);
    };
    auto part = [&](int piece) {             // one that is partly of the row
      x.each(piece, [&](float v, int) {
        seen(v, piece);
        sums = moved(sums, larger(sums.m, v), c);
        add(v);
      });
    };
    const int last = x.pieces - 1, end = x.whole(last) ? x.pieces : last;
    if (tid == 0 && !x.whole(0)) part(0);
    for (int p0 = tid ? tid : (x.whole(0) ? 0 : THREADS); p0 < end; p0 += kAhead * THREADS) {
      uint4 w[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int p = p0 + u * THREADS;
        w[u] = p < end ? x.load(p) : make_uint4(K::kNone, K::kNone, K::kNone, K::kNone);
      }
      float most = sums.m;
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        float top = x.element(w[u], 0);
#pragma unroll
        for (int j = 1; j < E; ++j) top = larger(top, x.element(w[u], j));
        if (p0 + u * THREADS < end) seen(top, p0 + u * THREADS);
        most = larger(most, top);
      }
      sums = moved(sums, most, c);
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
#pragma unroll
        for (int j = 0; j < E; ++j) add(x.element(w[u], j));
    }
    if (end == last && last > 0 && tid == last % THREADS) part(last);
#pragma unroll
    for (int n = 1; n < 64; n *= 2)
      sums = joined(sums, Sums{__shfl_xor(sums.m, n, 64), __shfl_xor(sums.s, n, 64), __shfl_xor(sums.t, n, 64)}, c);
    if (lane == 0) { lds_m[wave] = sums.m; lds_s[wave] = sums.s; lds_t[wave] = sums.t; }
    if constexpr (TOP) {
      best_key >>= K::kShift;
      uint32_t k = best_key;
      int p = best_piece;
#pragma unroll
      for (int n = 1; n < kLanes; n *= 2) {
        const uint32_t ok = __shfl_xor(k, n, 64);
        const int op = __shfl_xor(p, n, 64);
        if (ok > k || (ok == k && op < p)) { k = ok; p = op; }
      }
      if (tid % kLanes == 0) { group_key[tid / kLanes] = k; group_piece[tid / kLanes] = p; }
      if (tid == 0) { shares = 0; members = 0; }
    }
    __syncthreads();
    sums = Sums{lds_m[0], lds_s[0], lds_t[0]};
#pragma unroll
    for (int w = 1; w < kWaves; ++w) sums = joined(sums, Sums{lds_m[w], lds_s[w], lds_t[w]}, c);
    const float log2_s = log2f(sums.s);
    const float ln_s = log2_s * 0.6931471805599453f;
    auto log_p = [&](float v) { return (v - sums.m) * a.scale - ln_s; };
    if (a.entropy && tid == 0) a.entropy[row] = (log2_s - sums.t / sums.s) * 0.6931471805599453f;
    for (int g = tid; g < a.given; g += THREADS) {
      const int64_t token = a.tokens[row * a.given + g];
      a.given_out[row * a.given + g] = token < 0 ? 0.f : (token >= a.V ? NAN : log_p(static_cast<float>(x.first[token])));
    }
    if constexpr (TOP) {
      if (wave == 0) {
        uint32_t k[kGroups / 64];
        int p[kGroups / 64];
#pragma unroll
        for (int i = 0; i < kGroups / 64; ++i) { k[i] = group_key[i * 64 + lane]; p[i] = group_piece[i * 64 + lane]; }
        auto at_least = [&](uint32_t v) {
          int n = 0;
#pragma unroll
          for (int i = 0; i < kGroups / 64; ++i) n += __popcll(__ballot(k[i] >= v));
          return n;
        };
        // a row of few pieces has fewer groups than alternatives: all of it is on the list
        const uint32_t key = largest<kBits>(a.top, at_least);
        auto up_to = [&](uint32_t last) {    // groups that reach (key, last)
          int n = 0;
#pragma unroll
          for (int i = 0; i < kGroups / 64; ++i) n += __popcll(__ballot(k[i] > key || (k[i] == key && static_cast<uint32_t>(p[i]) <= last)));
          return n;
        };
        int piece = 0x7fffffff;
        // some more than `top` cost less on the list than here
        if (key != 0 && at_least(key) > a.top + 64) piece = 0x7fffffff - static_cast<int>(largest<31>(a.top, [&](uint32_t v) { return up_to(0x7fffffffu - v); }));
        if (lane == 0) bound = Bound{key, piece};
      }
      __syncthreads();
      Bound b = bound;
      const int turns = (x.pieces + THREADS - 1) / THREADS;
      if (tid < x.pieces && b.reached(best_key, best_piece)) share[atomicAdd(&shares, 1)] = tid;
      __syncthreads();
      const int n_shares = shares;
      auto gather = [&](int s, int turn) {
        const int piece = share[s] + turn * THREADS;
        if (piece >= x.pieces) return;
        x.each(piece, [&](float v, int at) {
          const uint32_t k = key_of(v);
          if (!b.reached(k >> K::kShift, piece)) return;
          const int m = atomicAdd(&members, 1);
          if (m < kList) { member_key[m] = k; member_at[m] = at; }
        });
      };
      for (int i = tid; i < n_shares * turns; i += THREADS) gather(i % n_shares, i / n_shares);
      __syncthreads();
      if (members > kList) {
        // counts over the whole row, of logits that reach a bound
        auto count_of = [&](Bound o) {
          __syncthreads();
          if (tid == 0) count = 0;
          __syncthreads();
          int n = 0;
          for (int p = tid; p < x.pieces; p += THREADS) x.each(p, [&](float v, int) { n += o.reached(key_of(v) >> K::kShift, p); });
          n = wave_sum(n);
          if (lane == 0) atomicAdd(&count, n);
          __syncthreads();
          return count;
        };
        b.key = largest<kBits>(a.top, [&](uint32_t v) { return count_of(Bound{v, 0x7fffffff}); });
        b.piece = 0x7fffffff - static_cast<int>(largest<31>(a.top, [&](uint32_t v) { return count_of(Bound{b.key, static_cast<int>(0x7fffffffu - v)}); }));
        __syncthreads();
        if (tid == 0) { members = 0; shares = 0; }
        __syncthreads();
        if (tid < x.pieces) share[atomicAdd(&shares, 1)] = tid;
        __syncthreads();
        const int all = shares;
        for (int i = tid; i < all * turns; i += THREADS) gather(i % all, i / all);
        __syncthreads();
      }
      const int n = min(members, kList);
      for (int i = tid; i < n; i += THREADS) {
        const uint32_t k = member_key[i];
        const int at = member_at[i];
        int before = 0;
        for (int o = 0; o < n; ++o) before += member_key[o] > k || (member_key[o] == k && member_at[o] < at);
        if (before < a.top) {
          a.top_ids[row * a.top + before] = at;
          a.top_out[row * a.top + before] = log_p(of_key(k));
        }
      }
    }
    __syncthreads();                         // the next row uses the same LDS
  }
}

template <class K, int THREADS> static void run(const LogprobArgs& a, hipStream_t st) {
  const unsigned grid = static_cast<unsigned>(std::min(a.M, 1 << 20));
  if (a.top) logprobs_kernel<K, THREADS, true><<<grid, THREADS, 0, st>>>(a);
  else logprobs_kernel<K, THREADS, false><<<grid, THREADS, 0, st>>>(a);
}

template <class K> static void run(const LogprobArgs& a, hipStream_t st) {
  run<K, 1024>(a, st);
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
