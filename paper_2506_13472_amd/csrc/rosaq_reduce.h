// Reductions over the lanes of a wave and the waves of a workgroup, by moves between registers (DPP), which take a few cycles where
// a shuffle through LDS takes some fifty.  Every lane gets the same bits, where f(a, b) and f(b, a) are the same: so sums go by added(), whose addition the
// compiler must not make one operation with a product in front of it, which rounds one of the two summands and not the other.
#pragma once
#include <hip/hip_runtime.h>

namespace rosaq {

template <class T> __device__ __forceinline__ T added(T a, T b) {
#pragma clang fp contract(off)
  return a + b;
}

// The value N lanes on, round a row of 16.
template <int N, class T> __device__ __forceinline__ T lane_round_row(T v) {
  static_assert(sizeof(T) == 4 || sizeof(T) == 8, "");
  if constexpr (sizeof(T) == 4) {
    const int i = __builtin_bit_cast(int, v);
    return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(i, i, 0x120 + N, 0xf, 0xf, false));
  } else {
    int2 i = __builtin_bit_cast(int2, v);
    i.x = __builtin_amdgcn_update_dpp(i.x, i.x, 0x120 + N, 0xf, 0xf, false);
    i.y = __builtin_amdgcn_update_dpp(i.y, i.y, 0x120 + N, 0xf, 0xf, false);
    return __builtin_bit_cast(T, i);
  }
}

template <class T> __device__ __forceinline__ T lane_of(T v, int lane) {
  if constexpr (sizeof(T) == 4) {
    return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
  } else {
    const int2 i = __builtin_bit_cast(int2, v);
    return __builtin_bit_cast(T, make_int2(__builtin_amdgcn_readlane(i.x, lane), __builtin_amdgcn_readlane(i.y, lane)));
  }
}

// f over a row of 16 lanes that hold the same N values again and again (16: as many values as lanes).
template <int N, class T, class F> __device__ __forceinline__ T row_all(T v, F f) {
  if constexpr (N > 8) v = f(v, lane_round_row<8>(v));
  if constexpr (N > 4) v = f(v, lane_round_row<4>(v));
  if constexpr (N > 2) v = f(v, lane_round_row<2>(v));
  if constexpr (N > 1) v = f(v, lane_round_row<1>(v));
  return v;
}

// f over a wave whose lanes are all there.
template <class T, class F> __device__ __forceinline__ T wave_all(T v, F f) {
  v = row_all<16>(v, f);
  return f(f(lane_of(v, 0), lane_of(v, 16)), f(lane_of(v, 32), lane_of(v, 48)));
}

}  // namespace rosaq
