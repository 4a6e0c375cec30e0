// Root-mean-square norm of rows, with the addition to the residual stream in front of it: h = x + residual, y = h / sqrt(mean h^2 + eps) * weight.
//
// A row is held by a team of threads, sixteen to 1024, in pieces of eight channels: read once, added up over the team, written once.  So it is bound
// by memory (65536 x 4096 with an fp16 residual, 2.1 GB, 388 us = 5.5 TB/s, where a copy reaches 5.0), or by a launch where there are few rows (64 of them 2.9 us).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <string>
#include <type_traits>

#include "rosaq_gemm.h"
#include "rosaq_reduce.h"
#include "rosaq_rows.h"

namespace rosaq {

// Eight channels of a row as they lie in memory; F32: those of the residual are fp32.
template <bool F32> struct Residual { uint4 w; };
template <> struct Residual<true> { float4 w[2]; };
template <bool F32> __device__ __forceinline__ float channel(const Residual<F32>& r, int j) {
  if constexpr (F32) return j < 4 ? (&r.w[0].x)[j] : (&r.w[1].x)[j - 4];
  else return static_cast<float>(as_h8(r.w)[j]);
}

// f over the values of a team's threads (f(a, b) and f(b, a) the same), in one order whatever runs when.
template <int TEAM, class T, class F> __device__ __forceinline__ T reduce(T v, T* lds, F f) {
  if constexpr (TEAM == 16) return row_all<16>(v, f);
  v = wave_all(v, f);
  if constexpr (TEAM > 64) {
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x / 64] = v;
    __syncthreads();
    v = row_all<TEAM / 64>(lds[threadIdx.x % (TEAM / 64)], f);
  }
  return v;
}

// A team of more than a wave is a workgroup, whose LDS and barriers it has alone.
constexpr int threads_of(int team) { return team > 64 ? team : 256; }

// ADD 0: no residual, 1: fp16, 2: fp32.  The sum of squares is fp32, of rows whose residual is fp32 in fp64: those may hold numbers whose squares
// fp32 does not.  CODES: all in fp64, because a code next to a border is a whole step off when it falls to the other side; a step is a 127th of the largest
// value.  The vector units bound it then: the conversions to fp64, and a row's own part (reductions, root, quotients), which every wave of it pays (1003 x 5120
// with an fp32 residual 15.8 us, 11.5 at a copy's rate; 8192 x 4096 with an fp16 one 51 and 48, without one 32 and 20).  Built and slower: fp32, and fp64 again
// for what fp32 cannot decide (22 and 61 us for the first two: a branch a channel).
template <int TEAM, int CH, int ADD, bool CODES>
__global__ __launch_bounds__(threads_of(TEAM)) void rmsnorm_kernel(NormArgs a) {
  constexpr int kThreads = threads_of(TEAM), kTeams = kThreads / TEAM;
  constexpr bool F32 = ADD == 2, kHold = CODES && !(TEAM == 1024 && CH > 2);      // there the registers are too few
  using Sum = std::conditional_t<F32 || CODES, double, float>;
  using Value = std::conditional_t<CODES, double, float>;
  __shared__ Sum lds_sum[TEAM > 64 ? TEAM / 64 : 1];
  __shared__ Value lds_most[TEAM > 64 ? TEAM / 64 : 1];
  const int t = threadIdx.x % TEAM, pieces = a.D / 8;
  for (int64_t row = static_cast<int64_t>(blockIdx.x) * kTeams + threadIdx.x / TEAM; row < a.M; row += static_cast<int64_t>(gridDim.x) * kTeams) {
    uint4 x[CH];
    Residual<F32> r[CH];
    uint4 w[CH];
    const uint4* xs = reinterpret_cast<const uint4*>(static_cast<const _Float16*>(a.x) + row * a.ldx);
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int p = t + i * TEAM;
      if (p >= pieces) continue;
      x[i] = xs[p];
      if constexpr (ADD == 1) r[i].w = reinterpret_cast<const uint4*>(static_cast<const _Float16*>(a.residual) + row * a.ld_residual)[p];
      if constexpr (ADD == 2) {
        const float4* rs = reinterpret_cast<const float4*>(static_cast<const float*>(a.residual) + row * a.ld_residual) + 2 * p;
        r[i].w[0] = rs[0];
        r[i].w[1] = rs[1];
      }
    }
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int p = t + i * TEAM;
      if (p >= pieces) continue;
      if (a.weight) w[i] = static_cast<const uint4*>(a.weight)[p];
    }
    auto h = [&](int i, int j) {
      const Value v = static_cast<Value>(static_cast<float>(as_h8(x[i])[j]));
      if constexpr (ADD) return v + static_cast<Value>(channel<F32>(r[i], j));
      else return v;
    };
    Sum sum = 0;
    double wide[kHold ? CH : 1][8];        // h, then y
#pragma unroll
    for (int i = 0; i < CH; ++i)
      if (t + i * TEAM < pieces)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const Sum v = static_cast<Sum>(h(i, j));
          sum += v * v;
          if constexpr (kHold) wide[i][j] = v;
        }
    auto held = [&](int i, int j) {
      if constexpr (kHold) return wide[i][j];
      else return h(i, j);
    };
    // the sum rounded to fp32 is the same from fp32 operands as from fp64's; of an fp32 residual it is at hand in fp64 (8192 x 4096 to codes 70 us, 5 more from fp32)
    if constexpr (ADD != 0) {
      if (a.residual_out) {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
          const int p = t + i * TEAM;
          if (p >= pieces) continue;
          if constexpr (F32) {
            float4 o[2];
#pragma unroll
            for (int j = 0; j < 8; ++j) (&o[j / 4].x)[j % 4] = static_cast<float>(held(i, j));
            float4* to = reinterpret_cast<float4*>(static_cast<float*>(a.residual_out) + row * a.ld_residual_out) + 2 * p;
            to[0] = o[0];
            to[1] = o[1];
          } else {
            half8 o;
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = static_cast<_Float16>(static_cast<float>(as_h8(x[i])[j]) + channel<F32>(r[i], j));
            reinterpret_cast<uint4*>(static_cast<_Float16*>(a.residual_out) + row * a.ld_residual_out)[p] = __builtin_bit_cast(uint4, o);
          }
        }
      }
    }
    sum = reduce<TEAM>(sum, lds_sum, added<Sum>);
    // of rows whose residual is fp32 the factor may be beyond fp32, and its power of two goes to h first
    Value factor;
    int power = 0;
    if constexpr (CODES) factor = rsqrt(sum / a.D + a.eps);
    else if constexpr (F32) factor = static_cast<float>(frexp(rsqrt(sum / a.D + a.eps), &power));
    else factor = 1.f / sqrtf(sum / static_cast<float>(a.D) + static_cast<float>(a.eps));
    auto formed = [&](int i, int j) {
      Value v = held(i, j);
      if constexpr (F32 && !CODES) v = __builtin_ldexpf(v, power);
      v *= factor;
      return a.weight ? v * static_cast<Value>(static_cast<float>(as_h8(w[i])[j])) : v;
    };
    if constexpr (kHold)
#pragma unroll
      for (int i = 0; i < CH; ++i)
        if (t + i * TEAM < pieces)
#pragma unroll
          for (int j = 0; j < 8; ++j) wide[i][j] = formed(i, j);
    auto value = [&](int i, int j) {
      if constexpr (kHold) return wide[i][j];
      else return formed(i, j);
    };
    if (a.y) {
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        const int p = t + i * TEAM;
        if (p >= pieces) continue;
        half8 o;
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] = static_cast<_Float16>(static_cast<float>(value(i, j)));
        reinterpret_cast<uint4*>(static_cast<_Float16*>(a.y) + row * a.ldy)[p] = __builtin_bit_cast(uint4, o);
      }
    }
    if constexpr (CODES) {
      // the maximum passes over NaN, which a product with zero does not, and neither over infinities
      double most = 0.0, none = 0.0;
#pragma unroll
      for (int i = 0; i < CH; ++i)
        if (t + i * TEAM < pieces)
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const double v = value(i, j);
            most = __builtin_fmax(most, __builtin_fabs(v));
            none = __builtin_fma(v, 0.0, none);
          }
      most = reduce<TEAM>(none == 0.0 ? most : INFINITY, lds_most, [](double a, double b) { return __builtin_fmax(a, b); });
      const float scale = static_cast<float>(most / 127.0);
      // a scale that is no positive number has no codes: zero's, or those of NaN
      const bool some = scale > 0.f && scale < INFINITY;
      const double inverse = some ? 1.0 / static_cast<double>(scale) : 0.0;
      if (t == 0) a.scales[row] = scale < INFINITY ? scale : NAN;
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        const int p = t + i * TEAM;
        if (p >= pieces) continue;
        uint32_t o[2] = {0u, 0u};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          // to the nearest whole number, which is the low word of 1.5 x 2^52 and it.  A scale among fp32's subnormals is far from its 127th, so codes are kept to
          // their range
          const double whole = __builtin_fma(value(i, j), inverse, 0x1.8p52);
          const int c = min(max(static_cast<int>(__builtin_bit_cast(uint64_t, whole)), -127), 127);
          o[j / 4] |= (static_cast<uint32_t>(c) & 0xffu) << (j % 4 * 8);
        }
        reinterpret_cast<uint2*>(static_cast<char*>(a.codes) + row * a.ld_codes)[p] = some ? make_uint2(o[0], o[1]) : make_uint2(0u, 0u);
      }
    }
    if constexpr (TEAM > 64) __syncthreads();       // the next row's sums go to the same place
  }
}

template <int TEAM, int CH, int ADD, bool CODES> static void run(const NormArgs& a, hipStream_t st) {
  constexpr int kThreads = threads_of(TEAM), kTeams = kThreads / TEAM;
  const int64_t groups = (static_cast<int64_t>(a.M) + kTeams - 1) / kTeams;
  rmsnorm_kernel<TEAM, CH, ADD, CODES><<<static_cast<unsigned>(std::min<int64_t>(groups, 1 << 20)), kThreads, 0, st>>>(a);
}

template <int TEAM, int CH, bool CODES> static void run(const NormArgs& a, hipStream_t st) {
  if (!a.residual) run<TEAM, CH, 0, CODES>(a, st);
  else if (!a.residual_f32) run<TEAM, CH, 1, CODES>(a, st);
  else run<TEAM, CH, 2, CODES>(a, st);
}

template <int TEAM, int CH> static void run(const NormArgs& a, hipStream_t st) {
  if (a.codes) run<TEAM, CH, true>(a, st);
  else run<TEAM, CH, false>(a, st);
}

// The smallest team whose threads hold one or two pieces each: more loads under way beside each other, fewer registers.  us with 256 threads / 512 / 1024, inputs
// and outputs beyond the last-level cache: 8192 x 4096 with an fp16 residual 51.1 / 46.8 / 51.0, 64 of them 3.4 / 2.9 / 3.1; 8192 x 5120 66.1 / 61.9 / 66.8, 64 of
// them 4.0 / 3.4 / 3.3; a wave a row is slower still (8192 x 4096 58.0, 64 of them 6.6).  To codes of up to 4096 channels two pieces each, which halve the waves
// that a row's own part is paid in: 8192 x 4096 without a residual 40.5 us in 512 threads, 32.1 in 256, 8192 x 2048 with an fp16 one 26.9 in 256, 27.4 in 128;
// 1003 x 5120 15.8 in 512, 16.4 in 256.
int launch_rmsnorm(const NormArgs& a, void* stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  const int pieces = a.D / 8;
  if (pieces <= 16) run<16, 1>(a, st);
  else if (pieces <= 64) run<64, 1>(a, st);
  else if (pieces <= 256 && a.codes) run<128, 2, true>(a, st);
  else if (pieces <= 256) run<256, 1, false>(a, st);
  else if (pieces <= 512 && a.codes) run<256, 2, true>(a, st);
  else if (pieces <= 512) run<512, 1, false>(a, st);
  else if (pieces <= 1024) run<512, 2>(a, st);
  else if (pieces <= 2048) run<1024, 2>(a, st);
  else run<1024, 4>(a, st);
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return ROSAQ_OK;
  try { set_error(std::string("rmsnorm: ") + hipGetErrorString(e)); } catch (...) {}     // no memory for the text
  return ROSAQ_ERR_HIP;
}

}  // namespace rosaq
