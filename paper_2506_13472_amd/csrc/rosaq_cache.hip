// Rotary positions, and the quantised cache as it is written and read back.
//
// All three kernels move data: 16 lanes take one head of one token, a lane its dim / 16 channels, which is one load of
// 16 bytes (dim 128), and a row of 16 lanes reduces over the head with DPP moves.  Measured, against 5.2 TB/s of a copy: rope of 8191 rows x 40 heads
// 33 us (170 MB, 5.1 TB/s); append of 4096 tokens x 40 heads of 8 bits with the queries 58 us (211 MB, 3.6 TB/s: the quantiser's and
// the rotation's vector operations), reading them back 24 (127 MB, 5.3 TB/s); calls of one decode step 3 to 4 us, which is a launch.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <string>

#include "rosaq_attention.h"
#include "rosaq_gemm.h"

namespace rosaq {

static int launched(const char* what) {
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return ROSAQ_OK;
  try { set_error(std::string(what) + ": " + hipGetErrorString(e)); } catch (...) {}     // no memory for the text
  return ROSAQ_ERR_HIP;
}

// U fp16 values of one lane, as dwords.
template <int U> struct Lane { uint32_t w[U / 2]; };

template <int U> __device__ __forceinline__ Lane<U> load_lane(const void* p) {
  return *static_cast<const Lane<U>*>(__builtin_assume_aligned(p, U * 2));
}
template <int U> __device__ __forceinline__ void store_lane(void* p, const Lane<U>& v) {
  *static_cast<Lane<U>*>(__builtin_assume_aligned(p, U * 2)) = v;
}
template <int U> __device__ __forceinline__ _Float16 half_of(const Lane<U>& v, int j) { return as_h2(v.w[j / 2])[j % 2]; }

__device__ __forceinline__ uint32_t pack2(_Float16 a, _Float16 b) { return __builtin_bit_cast(uint32_t, half2v{a, b}); }

// fp64 -> fp32 -> fp16, each to nearest even: what a user's own fp64 rotation gives, so that a rotated key has the same
// code from either.  The compiler would make one rounding of the two, in integer arithmetic; it is kept from seeing both.
__device__ __forceinline__ _Float16 narrow(double v) {
  float f = static_cast<float>(v);
  asm("" : "+v"(f));
  return static_cast<_Float16>(f);
}

// The angles of a lane's channels: cos and sin of the pair that channel j belongs to, the sign of the second product with the sine.
template <int U> struct Angles { double c[U], s[U]; };

template <int U> __device__ __forceinline__ Angles<U> load_angles(const RopeDev& r, int row, int c0) {
  Angles<U> a;
  const float2* t = reinterpret_cast<const float2*>(r.table) + static_cast<int64_t>(r.at[row]) * (r.rot / 2);
  const int half = r.rot / 2;
  const int i0 = c0 >= r.rot ? 0 : (r.interleaved ? c0 / 2 : (c0 < half ? c0 : c0 - half));
#pragma unroll
  for (int j = 0; j < U; ++j) {
    const float2 cs = t[i0 + (r.interleaved ? j / 2 : j)];
    a.c[j] = cs.x;
    a.s[j] = (r.interleaved ? j % 2 == 0 : c0 < half) ? -cs.y : cs.y;
  }
  return a;
}

// Minimum / maximum over the 16 lanes of a row (rotations by 8, 4, 2 and 1 lanes).
template <int N, class T> __device__ __forceinline__ T row_ror(T v) {
  const int i = __builtin_bit_cast(int, v);
  return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(i, i, 0x120 + N, 0xf, 0xf, false));
}
__device__ __forceinline__ float row_min(float v) {
  v = fminf(v, row_ror<8>(v)); v = fminf(v, row_ror<4>(v)); v = fminf(v, row_ror<2>(v));
  return fminf(v, row_ror<1>(v));
}
__device__ __forceinline__ float row_max(float v) {
  v = fmaxf(v, row_ror<8>(v)); v = fmaxf(v, row_ror<4>(v)); v = fmaxf(v, row_ror<2>(v));
  return fmaxf(v, row_ror<1>(v));
}

// The rotated values of a lane.  Products of fp16 and fp32 are exact in fp64, so the only error is the sum's rounding, 2^-53, and the two of
// narrow().  rot is a multiple of 2 U, so a lane lies within one half of the rotated part.
template <int U>
__device__ __forceinline__ Lane<U> rotate_lane(const Lane<U>& x, const Angles<U>& a, const RopeDev& r, int c0, int lane) {
  Lane<U> other = x, y;
  if (!r.interleaved) {
    const int lanes = r.rot / 2 / U;              // lanes from a channel to its partner
    if (lanes == 8) {                             // the whole head turns: a move within the row of 16 lanes
#pragma unroll
      for (int j = 0; j < U / 2; ++j) other.w[j] = row_ror<8>(x.w[j]);
    } else {
      const int from = c0 >= r.rot ? lane : (c0 < r.rot / 2 ? lane + lanes : lane - lanes);
#pragma unroll
      for (int j = 0; j < U / 2; ++j) other.w[j] = __shfl(static_cast<int>(x.w[j]), from, 64);
    }
  }
  if (c0 >= r.rot) return x;
#pragma unroll
  for (int j = 0; j < U; j += 2) {
    _Float16 out[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const double mine = half_of<U>(x, j + e), pair = r.interleaved ? half_of<U>(x, j + (e ^ 1)) : half_of<U>(other, j + e);
      out[e] = narrow(__builtin_fma(mine, a.c[j + e], pair * a.s[j + e]));
    }
    y.w[j / 2] = pack2(out[0], out[1]);
  }
  return y;
}

// Codes and parameters of one head of one token, spread over its 16 lanes.
template <int U> struct Coded { uint32_t code[U]; uint32_t sz; };

// x / s for fp16 numbers, r = 1 / s to an ulp or two: right to an ulp, and exact where the quotient is a number of few bits.  A
// division takes three times as long.
__device__ __forceinline__ float quotient(float x, float s, float r) {
  const float q = x * r;
  return __builtin_fmaf(__builtin_fmaf(-q, s, x), r, q);
}

// The library's asymmetric quantiser with a range that always holds zero, in fp32, so that codes do not depend on who
// computes them: quotients of two fp16 numbers up to 256 keep 2^-12 from a whole or half-way number or lie on it, where fp32
// resolves 2^-16.  A group with NaN or Inf gets the scale NaN.
template <int U, int BITS>
__device__ __forceinline__ Coded<U> quantise(const Lane<U>& x, int lane) {
  constexpr float top = (1 << BITS) - 1;
  float f[U], lo = 0.f, hi = 0.f;
  bool odd = false;
#pragma unroll
  for (int j = 0; j < U; ++j) {
    const _Float16 h = half_of<U>(x, j);
    odd |= (__builtin_bit_cast(uint16_t, h) & 0x7c00u) == 0x7c00u;
    f[j] = static_cast<float>(h);
    lo = fminf(lo, f[j]);
    hi = fmaxf(hi, f[j]);
  }
  const bool bad = (__ballot(odd) >> (lane & 48)) & 0xffffu;
  lo = row_min(lo);
  hi = row_max(hi);
  const _Float16 s16 = static_cast<_Float16>(fmaxf((hi - lo) / top, 0x1p-14f));
  const float s = static_cast<float>(s16);
  const float rcp = __builtin_amdgcn_rcpf(s);
  const float z = fminf(rintf(quotient(-lo, s, rcp)), top);
  const float far = floorf(quotient(65504.f, s, rcp));   // codes further from z stand for more than fp16 holds
  const float least = fmaxf(0.f, z - far), most = fminf(top, z + far);
  Coded<U> c;
#pragma unroll
  for (int j = 0; j < U; ++j)
    c.code[j] = bad ? 0u : static_cast<uint32_t>(fminf(fmaxf(rintf(quotient(f[j], s, rcp)) + z, least), most));
  c.sz = bad ? 0x7e00u : __builtin_bit_cast(uint16_t, s16) | (static_cast<uint32_t>(__builtin_bit_cast(uint16_t, static_cast<_Float16>(z))) << 16);
  return c;
}

// Where a lane's codes of a token lie in a record.  keys: `key_offset` and contiguous; values: units of 16 bits, the
// i-th of a lane at value_offset(.., i).
template <int D, int BITS> __device__ __forceinline__ int key_offset(int token, int r) {
  constexpr int U = D / 16;
  constexpr int lane_bytes = D / 4 * BITS / 8;                          // of an MFMA lane: 8, 16 or 32
  constexpr int planes = lane_bytes > 16 ? lane_bytes / 16 : 1, width = lane_bytes / planes;
  const int g = r / 4, at = r % 4 * U * BITS / 8;                       // byte within the MFMA lane
  return at / width * (64 * width) + token * (4 * width) + g * width + at % width;
}
template <int D, int BITS> __device__ __forceinline__ int value_offset(int token, int r, int i) {
  constexpr int units = D / 16 * BITS / 16;                             // of a token and lane: 1, 2 or 4
  constexpr int per_plane = units > 2 ? 2 : units;
  return cache_code_bytes(D, BITS) + i / per_plane * (64 * per_plane * 8) + (token / 4 * 16 + r) * (per_plane * 8) +
         i % per_plane * 8 + token % 4 * 2;
}

// Record of a slot and head; null where the slot is none of the cache's.
__device__ __forceinline__ char* record_of(const CacheDev& c, int64_t slot, int head, int record_bytes) {
  const int64_t page = slot >> c.page_shift;
  if (slot < 0 || page >= c.num_pages) return nullptr;
  const int in_page = static_cast<int>(slot & ((int64_t{1} << c.page_shift) - 1));
  return c.base + page * c.page_bytes + head * c.head_bytes + static_cast<int64_t>(in_page / kCacheBlock) * record_bytes;
}

constexpr int kTasksPerBlock = 16;      // of a workgroup of 256 threads
constexpr int kRun = 8;                 // heads of a task, where there are many

// Tasks are numbered kind by kind (keys, values, queries), and a task is RUN heads of one token: their angles are loaded and widened once,
// and their loads do not wait for each other.  Four tokens in a row, whose values lie side by side in a record, are one wave's.
struct Task { int row, first; };
__device__ __forceinline__ Task task_of(uint32_t task, int runs, int run) {
  const uint32_t four = task / 4;
  return Task{static_cast<int>(four / runs * 4 + task % 4), static_cast<int>(four % runs) * run};
}

template <int D, int BITS, int RUN>
__global__ __launch_bounds__(256) void cache_append_kernel(AppendArgs a) {
  constexpr int U = D / 16;
  const int lane = threadIdx.x & 63, r = threadIdx.x & 15, c0 = r * U;
  const int kv = a.cache.kv_heads;
  const int kv_runs = (kv + RUN - 1) / RUN, q_runs = a.q ? (a.q_heads + RUN - 1) / RUN : 0;
  uint32_t task = blockIdx.x * kTasksPerBlock + threadIdx.x / 16;       // < 2^28
  const uint32_t kv_tasks = (static_cast<uint32_t>(a.M) + 3) / 4 * 4 * kv_runs;
  const int kind = task < kv_tasks ? 0 : (task < 2 * kv_tasks ? 1 : 2);
  task -= kind * kv_tasks;
  const int runs = kind == 2 ? q_runs : kv_runs;
  // a row of 16 lanes is all in or all out; the shuffles and ballots below stay within one
  if (runs == 0) return;
  const Task t = task_of(task, runs, RUN);
  const int row = t.row, first = t.first;
  if (row >= a.M) return;
  const int heads = kind == 2 ? a.q_heads : kv;
  const int64_t slot = a.slots[row];
  const bool rotated = a.rope.table != nullptr && kind != 1;
  if (slot < 0 || (slot >> a.cache.page_shift) >= a.cache.num_pages) return;
  if (a.rope.table != nullptr && (a.rope.at[row] < 0 || a.rope.at[row] >= a.rope.positions)) return;
  const _Float16* src = static_cast<const _Float16*>(kind == 0 ? a.k : (kind == 1 ? a.v : a.q)) +
                        row * (kind == 0 ? a.ldk : (kind == 1 ? a.ldv : a.ldq)) + c0;
  Lane<U> x[RUN];
#pragma unroll
  for (int i = 0; i < RUN; ++i)
    if (first + i < heads) x[i] = load_lane<U>(src + (first + i) * D);
  if (rotated) {
    const Angles<U> angles = load_angles<U>(a.rope, row, c0);
#pragma unroll
    for (int i = 0; i < RUN; ++i) x[i] = rotate_lane<U>(x[i], angles, a.rope, c0, lane);
  }
  const int token = static_cast<int>(slot & (kCacheBlock - 1));
#pragma unroll
  for (int i = 0; i < RUN; ++i) {
    const int h = first + i;
    if (h >= heads) return;
    if (kind == 2) {
      store_lane<U>(static_cast<_Float16*>(a.q_out) + row * a.ldq_out + h * D + c0, x[i]);
      continue;
    }
    const Coded<U> c = quantise<U, BITS>(x[i], lane);
    char* rec = record_of(a.cache, slot, h, cache_record_bytes(D, BITS));
    constexpr int per_unit = 16 / BITS, units = U / per_unit;
    uint32_t unit[units];
#pragma unroll
    for (int e = 0; e < units; ++e) {
      unit[e] = 0;
#pragma unroll
      for (int j = 0; j < per_unit; ++j) unit[e] |= c.code[e * per_unit + j] << (j * BITS);
    }
    if (kind == 0) {
      char* dst = rec + key_offset<D, BITS>(token, r);
      if constexpr (units == 4) *reinterpret_cast<uint2*>(dst) = make_uint2(unit[0] | unit[1] << 16, unit[2] | unit[3] << 16);
      else if constexpr (units == 2) *reinterpret_cast<uint32_t*>(dst) = unit[0] | unit[1] << 16;
      else *reinterpret_cast<uint16_t*>(dst) = static_cast<uint16_t>(unit[0]);
    } else {
#pragma unroll
      for (int e = 0; e < units; ++e)
        *reinterpret_cast<uint16_t*>(rec + value_offset<D, BITS>(token, r, e)) = static_cast<uint16_t>(unit[e]);
    }
    if (r == 0)
      *reinterpret_cast<uint32_t*>(rec + 2 * cache_code_bytes(D, BITS) + kind * kCacheBlock * 4 + token * 4) = c.sz;
  }
}

template <int D, int BITS, int RUN>
__global__ __launch_bounds__(256) void cache_read_kernel(ReadArgs a) {
  constexpr int U = D / 16, per_unit = 16 / BITS, units = U / per_unit;
  const int r = threadIdx.x & 15;
  const int kv = a.cache.kv_heads, kinds = (a.k ? 1 : 0) + (a.v ? 1 : 0), runs = (kv + RUN - 1) / RUN;
  uint32_t task = blockIdx.x * kTasksPerBlock + threadIdx.x / 16;
  const uint32_t of_kind = (static_cast<uint32_t>(a.M) + 3) / 4 * 4 * runs;
  if (task >= kinds * of_kind) return;
  const bool key = a.k && task < of_kind;                      // keys first, where both are wanted
  if (!key && a.k) task -= of_kind;
  const Task t = task_of(task, runs, RUN);
  const int row = t.row, first = t.first;
  if (row >= a.M) return;
  const int64_t slot = a.slots[row];
  if (slot < 0 || (slot >> a.cache.page_shift) >= a.cache.num_pages) return;
  const int token = static_cast<int>(slot & (kCacheBlock - 1));
  uint32_t unit[RUN][units], sz[RUN];
#pragma unroll
  for (int i = 0; i < RUN; ++i) {
    const char* rec = record_of(a.cache, slot, min(first + i, kv - 1), cache_record_bytes(D, BITS));
    if (key) {
      const char* at = rec + key_offset<D, BITS>(token, r);
      uint32_t w[2];
      if constexpr (units == 4) { const uint2 t = *reinterpret_cast<const uint2*>(at); w[0] = t.x; w[1] = t.y; }
      else if constexpr (units == 2) w[0] = *reinterpret_cast<const uint32_t*>(at);
      else w[0] = *reinterpret_cast<const uint16_t*>(at);
#pragma unroll
      for (int e = 0; e < units; ++e) unit[i][e] = w[e / 2] >> (e % 2 * 16);
    } else {
#pragma unroll
      for (int e = 0; e < units; ++e) unit[i][e] = *reinterpret_cast<const uint16_t*>(rec + value_offset<D, BITS>(token, r, e));
    }
    sz[i] = *reinterpret_cast<const uint32_t*>(rec + 2 * cache_code_bytes(D, BITS) + (key ? 0 : kCacheBlock * 4) + token * 4);
  }
  _Float16* dst = (key ? static_cast<_Float16*>(a.k) + row * a.ldk : static_cast<_Float16*>(a.v) + row * a.ldv) + r * U;
#pragma unroll
  for (int i = 0; i < RUN; ++i) {
    if (first + i >= kv) return;
    const float s = static_cast<float>(as_h2(sz[i]).x), z = static_cast<float>(as_h2(sz[i]).y);
    Lane<U> y;
#pragma unroll
    for (int j = 0; j < U; j += 2) {
      _Float16 v[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const uint32_t code = (unit[i][(j + e) / per_unit] >> ((j + e) % per_unit * BITS)) & ((1u << BITS) - 1);
        v[e] = static_cast<_Float16>((static_cast<float>(code) - z) * s);     // exact in fp32, rounded once
      }
      y.w[j / 2] = pack2(v[0], v[1]);
    }
    store_lane<U>(dst + (first + i) * D, y);
  }
}

template <int D, int RUN>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a) {
  constexpr int U = D / 16;
  const int lane = threadIdx.x & 63, c0 = (threadIdx.x & 15) * U;
  const int runs = (a.heads + RUN - 1) / RUN;
  const uint32_t task = blockIdx.x * kTasksPerBlock + threadIdx.x / 16;
  const int row = static_cast<int>(task / runs), first = static_cast<int>(task % runs) * RUN;
  if (row >= a.M) return;
  const int at = a.rope.at[row];
  if (at < 0 || at >= a.rope.positions) return;
  const _Float16* src = static_cast<const _Float16*>(a.x) + row * a.ldx + c0;
  Lane<U> x[RUN];
#pragma unroll
  for (int i = 0; i < RUN; ++i)
    if (first + i < a.heads) x[i] = load_lane<U>(src + (first + i) * D);
  const Angles<U> angles = load_angles<U>(a.rope, row, c0);
#pragma unroll
  for (int i = 0; i < RUN; ++i) {
    const Lane<U> y = rotate_lane<U>(x[i], angles, a.rope, c0, lane);
    if (first + i < a.heads) store_lane<U>(static_cast<_Float16*>(a.y) + row * a.ldy + (first + i) * D + c0, y);
  }
}

// One thread a pair, everything in fp64: a table is made once for as long as a model is served.
__global__ __launch_bounds__(256) void rope_table_kernel(rosaq_rope_desc d, float2* table, int32_t positions) {
  const int half = d.rot_dim / 2;
  const int64_t n = static_cast<int64_t>(positions) * half;
  const int64_t id = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (id >= n) return;
  const int i = static_cast<int>(id % half);
  double f = pow(d.base, -2.0 * i / d.rot_dim);
  if (d.scaling == ROSAQ_ROPE_SCALE_LINEAR) f /= d.factor;
  if (d.scaling == ROSAQ_ROPE_SCALE_WAVELENGTH) {
    // turns of the pair over the trained length: few -> divided, many -> kept, blended between
    const double turns = d.trained_positions * f / 6.283185307179586476925;
    double keep = (turns - d.low) / (d.high - d.low);
    keep = keep < 0.0 ? 0.0 : (keep > 1.0 ? 1.0 : keep);
    f = (1.0 - keep) * (f / d.factor) + keep * f;
  }
  double s, c;
  sincos(static_cast<double>(id / half) * f, &s, &c);
  table[id] = make_float2(static_cast<float>(c), static_cast<float>(s));
}

static unsigned blocks_of(int64_t tasks) { return static_cast<unsigned>((tasks + kTasksPerBlock - 1) / kTasksPerBlock); }
static int64_t runs_of(int64_t heads, int run) { return (heads + run - 1) / run; }

// Whether tasks of kRun heads still fill the card: with 512 workgroups of them.  us with one head a task / with eight, heads of 128 channels:
// rope of 1024 rows x 32 heads 8.8 / 8.8 (as fast as it is issued), of 2048 12.8 / 10.6, of 4096 21.5 / 13.6; append and read
// of 512 tokens x 96 heads (4 bits) 19.7 / 20.4, of 1024 25.6 / 24.0, of 2048 46.1 / 37.3.
static bool many(int64_t rows_heads) { return rows_heads >= 1 << 16; }

int launch_rope_table(const rosaq_rope_desc& d, float* table, int32_t positions, void* stream) {
  const int64_t n = static_cast<int64_t>(positions) * (d.rot_dim / 2);
  rope_table_kernel<<<static_cast<unsigned>((n + 255) / 256), 256, 0, static_cast<hipStream_t>(stream)>>>(
      d, reinterpret_cast<float2*>(table), positions);
  return launched("rope table");
}

int launch_rope(const RopeArgs& a, void* stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  const int run = many(static_cast<int64_t>(a.M) * a.heads) ? kRun : 1;
  const unsigned grid = blocks_of(a.M * runs_of(a.heads, run));
  if (a.dim == 128 && run == 1) rope_kernel<128, 1><<<grid, 256, 0, st>>>(a);
  else if (a.dim == 128) rope_kernel<128, kRun><<<grid, 256, 0, st>>>(a);
  else if (run == 1) rope_kernel<64, 1><<<grid, 256, 0, st>>>(a);
  else rope_kernel<64, kRun><<<grid, 256, 0, st>>>(a);
  return launched("rope");
}

template <int D, int BITS> static void append(const AppendArgs& a, hipStream_t st) {
  const int run = many(static_cast<int64_t>(a.M) * (2 * a.cache.kv_heads + a.q_heads)) ? kRun : 1;
  const unsigned grid = blocks_of(runs_of(a.M, 4) * 4 * (2 * runs_of(a.cache.kv_heads, run) + (a.q ? runs_of(a.q_heads, run) : 0)));
  if (run == 1) cache_append_kernel<D, BITS, 1><<<grid, 256, 0, st>>>(a);
  else cache_append_kernel<D, BITS, kRun><<<grid, 256, 0, st>>>(a);
}

int launch_cache_append(const AppendArgs& a, void* stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (a.dim == 128) a.bits == 4 ? append<128, 4>(a, st) : append<128, 8>(a, st);
  else a.bits == 4 ? append<64, 4>(a, st) : append<64, 8>(a, st);
  return launched("cache append");
}

template <int D, int BITS> static void read(const ReadArgs& a, hipStream_t st) {
  const int kinds = (a.k ? 1 : 0) + (a.v ? 1 : 0);
  const int run = many(static_cast<int64_t>(a.M) * kinds * a.cache.kv_heads) ? kRun : 1;
  const unsigned grid = blocks_of(runs_of(a.M, 4) * 4 * kinds * runs_of(a.cache.kv_heads, run));
  if (run == 1) cache_read_kernel<D, BITS, 1><<<grid, 256, 0, st>>>(a);
  else cache_read_kernel<D, BITS, kRun><<<grid, 256, 0, st>>>(a);
}

int launch_cache_read(const ReadArgs& a, void* stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (a.dim == 128) a.bits == 4 ? read<128, 4>(a, st) : read<128, 8>(a, st);
  else a.bits == 4 ? read<64, 4>(a, st) : read<64, 8>(a, st);
  return launched("cache read");
}

}  // namespace rosaq
