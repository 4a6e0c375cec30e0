// Attention over the quantised cache: y = softmax(scale q K^T) V with the keys and values as codes.
//
// One pass over the cache with the running reference and sum of a softmax.  A wave multiplies 16 query rows with 32 tokens a
// step.  Both products run with the tokens on the rows of the MFMA's result, S^T = K Q^T and Y^T = V^T P^T:
// lane (g, r) of S^T holds query row r's scores of tokens 4 g .. 4 g + 3 of each 16, which is, as it stands, the operand P^T of
// the second product if V's lanes bring the same tokens in the same order, and the cache's layout sees to that.  So the
// probabilities go from one product to the other without leaving their registers, a row's reference and sum live in the
// lane that needs them, and codes become factors in the registers they were loaded to.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <string>

#include "rosaq_attention.h"
#include "rosaq_gemm.h"

namespace rosaq {

constexpr int kStep = 2 * kCacheBlock;      // tokens of a step: the depth of one MFMA over the values
constexpr int kWaves = 4;
constexpr int kRows = 16;                   // query rows of a workgroup
constexpr float kNoScore = -1e30f;          // the reference before any score: finite, so that exp2(x - reference) is 0 or huge, never NaN, for hidden tokens

// Probabilities are 2^(score - reference), kept in fp16 for the MFMA.  The reference is kLead below the largest score of
// the step that set it, and moves only when a score passes it by kRoom: moving it costs shuffles and a pass over the sums, and hardly any
// step needs it.  2^15 is in fp16's range, and what is 2^-24 below the reference (29 below the maximum, as powers of two) is lost.
constexpr float kLead = 5.f, kRoom = 15.f;

// A sequence's rows in the call.
struct Rows { int start, count; };
__device__ __forceinline__ Rows rows_of(const AttendArgs& a, int seq) {
  if (!a.row_start) return Rows{seq, 1};
  const int s = min(max(a.row_start[seq], 0), a.M), e = min(max(a.row_start[seq + 1], s), a.M);
  return Rows{s, e - s};
}
__device__ __forceinline__ int own_tokens(const AttendArgs& a, int seq) { return min(max(a.kv_len[seq], 0), a.capacity); }
// tokens of its sequence that row i of `count` sees
__device__ __forceinline__ int visible(const AttendArgs& a, int tokens, int count, int i) {
  return a.causal ? max(tokens - count + i + 1, 0) : tokens;
}
// steps over the prefix, and all steps that the rows of one tile take, the last of which is row i of its sequence
__device__ __forceinline__ int prefix_steps_of(const AttendArgs& a, int over, int step) {
  return over == kOwn ? 0 : (a.prefix_len + step - 1) / step;
}
__device__ __forceinline__ int steps_of(const AttendArgs& a, int over, int step, int tokens, int count, int i) {
  return prefix_steps_of(a, over, step) + (over == kPrefix ? 0 : (visible(a, tokens, count, i) + step - 1) / step);
}

// A workgroup's share of a launch.  Workgroups go to the XCDs in turn; with by_xcd, those of one sequence and kv head, which read
// the same codes, stay on one XCD and its L2.  Tiles go from the last to the first, which under the causal mask is from the longest.
struct Share { int seq, kv_head, tile, part; bool any; };
__device__ __forceinline__ Share share_of(const AttendArgs& a, const AttendLaunch& n) {
  const int heads = a.cache.kv_heads, seqs = n.over == kPrefix ? 1 : a.seqs, each = n.tiles * n.parts;
  int id = blockIdx.x, pair, rest;
  if (n.by_xcd) {
    pair = (id >> 3) / each * 8 + (id & 7);
    rest = (id >> 3) % each;
  } else {
    pair = id / each;
    rest = id % each;
  }
  return Share{pair / heads, pair % heads, n.tiles - 1 - rest / n.parts, rest % n.parts, pair < seqs * heads};
}

// rows of a launch's sequence: with kPrefix all rows of the call are one
__device__ __forceinline__ Rows launch_rows(const AttendArgs& a, int over, int seq) {
  if (over != kPrefix) return rows_of(a, seq);
  return Rows{0, a.row_start ? min(max(a.row_start[a.seqs], 0), a.M) : a.seqs};
}

// What a lane holds of one step: codes of two records and the scales and zeros it needs of them.
template <int D, int BITS> struct Step {
  static constexpr int kDwords = D / 4 * BITS / 32;     // of a lane, keys or values of one record: 2, 4 or 8
  uint32_t k[2][kDwords], v[2][kDwords];
  uint32_t k_own[2];        // scale | zero of the key token that the lane multiplies
  uint4 k_sz[2], v_sz[2];   // of tokens 4 g .. 4 g + 3
};

// `place`: the lane's place among the 64 of a plane
template <int N> __device__ __forceinline__ void load_codes(uint32_t (&to)[N], const char* plane0, int place) {
  if constexpr (N == 2) {
    const uint2 t = reinterpret_cast<const uint2*>(plane0)[place];
    to[0] = t.x; to[1] = t.y;
  } else {
#pragma unroll
    for (int p = 0; p < N / 4; ++p) {
      const uint4 t = reinterpret_cast<const uint4*>(plane0)[p * 64 + place];
      to[4 * p] = t.x; to[4 * p + 1] = t.y; to[4 * p + 2] = t.z; to[4 * p + 3] = t.w;
    }
  }
}

// Eight channels of one key token, as whole numbers code - z.  Four-bit codes come out in the order 0 4 1 5 2 6 3 7.
template <int BITS> __device__ __forceinline__ half8 key_factor(const uint32_t* w, half2v c_lo, half2v c_hi) {
  if constexpr (BITS == 4) {
    return dequant4(w[0], c_lo, c_hi);
  } else {
    const uint32_t magic = 0x64646464u;      // a byte b under 0x64 is the fp16 number 1024 + b
    const half2v h0 = as_h2(__builtin_amdgcn_perm(magic, w[0], 0x04010400u)) + c_lo;
    const half2v h1 = as_h2(__builtin_amdgcn_perm(magic, w[0], 0x04030402u)) + c_lo;
    const half2v h2 = as_h2(__builtin_amdgcn_perm(magic, w[1], 0x04010400u)) + c_lo;
    const half2v h3 = as_h2(__builtin_amdgcn_perm(magic, w[1], 0x04030402u)) + c_lo;
    return half8{h0.x, h0.y, h1.x, h1.y, h2.x, h2.y, h3.x, h3.y};
  }
}

// Channel j (of a lane's D / 16) of two tokens of a record as values (code - z) s, rounded to fp16 as reading the cache rounds them.  `w`: the
// lane's dwords, dword 2 i + t = unit i of the tokens 2 t and 2 t + 1.
template <int BITS> __device__ __forceinline__ half2v value_pair(const uint32_t* w, int j, int t, half2v c_lo, half2v c_hi, half2v s) {
  const half2v sixteenth = {(_Float16)0.0625f, (_Float16)0.0625f};
  if constexpr (BITS == 4) {
    const uint32_t d = w[2 * (j / 4) + t] >> (j % 4 / 2 * 8);
    if (j % 2 == 0) return (as_h2(and_or<false>(d, 0x000f000fu, 0x64006400u)) + c_lo) * s;
    return __builtin_elementwise_fma(as_h2(and_or<false>(d, 0x00f000f0u, 0x64006400u)), sixteenth, c_hi) * s;
  } else {
    const uint32_t d = w[2 * (j / 2) + t];
    return (as_h2(__builtin_amdgcn_perm(0x64646464u, d, j % 2 == 0 ? 0x04020400u : 0x04030401u)) + c_lo) * s;
  }
}

__device__ __forceinline__ half2v minus(float bias, half2v z) {
  const half2v b = {(_Float16)bias, (_Float16)bias};
  return -(z + b);
}

// fp32 partial results: [part][row][head][D] sums, then [part][row][head] (reference, sum of probabilities).
template <int D> struct Part {
  float* sums;
  float2* stats;
  __device__ Part(const AttendArgs& a, int parts)
      : sums(a.part), stats(reinterpret_cast<float2*>(a.part + static_cast<int64_t>(parts) * a.M * a.q_heads * D)) {}
};

template <int D, int BITS>
__global__ __launch_bounds__(64 * kWaves) void attend_kernel(AttendArgs a, AttendLaunch n, int parts) {
  constexpr int U = D / 16, KS = D / 32;
  __shared__ float lds_sum[kWaves][kRows][D + 4];
  __shared__ float lds_ref[kWaves][kRows], lds_l[kWaves][kRows];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, g = lane >> 4;
  const Share w = share_of(a, n);
  if (!w.any) return;
  const int kv_head = w.kv_head, seq = w.seq, tile = w.tile;
  const Rows rows = rows_of(a, seq);
  const int used = min(rows.count, a.max_rows) * a.group;         // rows of this kv head: (token, query head of the group)
  if (tile * kRows >= used) return;
  const int tokens = own_tokens(a, seq);
  const int last = (min(tile * kRows + kRows, used) - 1) / a.group;
  const int prefix_steps = prefix_steps_of(a, n.over, kStep);
  const int all = steps_of(a, n.over, kStep, tokens, rows.count, last);
  const int begin = w.part * n.steps, end = min(begin + n.steps, all);
  if (w.part > 0 && begin >= all) return;                         // part 0 always answers, if only that there is nothing

  // rows of the tile: (token, head) of this lane's column, clamped into the sequence's
  const int my = min(tile * kRows + r, used - 1);
  const int my_token = my / a.group, my_head = kv_head * a.group + my % a.group;
  const int limit = visible(a, tokens, rows.count, my_token);

  half8 q[KS];
  {
    const _Float16* src = static_cast<const _Float16*>(a.q) + static_cast<int64_t>(rows.start + my_token) * a.ldq + my_head * D + g * (D / 4);
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const half8 h = as_h8(reinterpret_cast<const uint4*>(src)[s]);
      q[s] = BITS == 4 ? half8{h[0], h[4], h[1], h[5], h[2], h[6], h[3], h[7]} : h;
    }
  }

  const CacheDev& c = a.cache;
  const int block_shift = c.page_shift - 4;
  constexpr int kRecord = cache_record_bytes(D, BITS), kCodes = cache_code_bytes(D, BITS);
  const char* head_base = c.base + kv_head * c.head_bytes;

  // loads a step; `hidden` says which of its records have no page
  auto load = [&](int step, Step<D, BITS>& x, int& hidden) {
    const bool own = step >= prefix_steps;
    const int block0 = (own ? step - prefix_steps : step) * 2;
    const int32_t* table = own ? a.pages + static_cast<int64_t>(seq) * a.page_stride : a.prefix_pages;
    const int blocks = ((own ? tokens : a.prefix_len) + kCacheBlock - 1) / kCacheBlock;
    hidden = 0;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const int block = block0 + b;
      int page = block < blocks ? table[block >> block_shift] : -1;
      page = __builtin_amdgcn_readfirstlane(page);
      const bool bad = page < 0 || page >= c.num_pages;
      hidden |= bad ? 1 << b : 0;
      // a record without a page is hidden below; the loads then take the cache's first one
      const char* rec = head_base + (bad ? 0 : page * c.page_bytes + static_cast<int64_t>(block & ((1 << block_shift) - 1)) * kRecord);
      load_codes(x.k[b], rec, r * 4 + g);
      load_codes(x.v[b], rec + kCodes, lane);
      const uint32_t* sz = reinterpret_cast<const uint32_t*>(rec + 2 * kCodes);
      x.k_own[b] = sz[r];
      x.k_sz[b] = reinterpret_cast<const uint4*>(sz)[g];
      x.v_sz[b] = reinterpret_cast<const uint4*>(sz)[4 + g];
    }
  };

  floatx4 sum[U];
#pragma unroll
  for (int j = 0; j < U; ++j) sum[j] = floatx4{0.f, 0.f, 0.f, 0.f};
  float ref = kNoScore, l = 0.f;

  for (int step = begin + wave; step < end; step += kWaves) {
    Step<D, BITS> x;
    int hidden;
    load(step, x, hidden);
    const bool own = step >= prefix_steps;
    const int t0 = (own ? step - prefix_steps : step) * kStep;
    const int lim = (own ? limit : a.prefix_len) - t0;               // of the step's 32 tokens, this row sees those below it
    const int held = (own ? tokens : a.prefix_len) - t0;             // and those below this are written at all

    float score[2][4];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const half2v own_sz = as_h2(x.k_own[b]);
      const half2v z = {own_sz.y, own_sz.y}, c_lo = minus(1024.f, z), c_hi = minus(64.f, z);
      floatx4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < KS; ++k) s = mfma16(key_factor<BITS>(&x.k[b][k * BITS / 4], c_lo, c_hi), q[k], s);
      const uint32_t sz[4] = {x.k_sz[b].x, x.k_sz[b].y, x.k_sz[b].z, x.k_sz[b].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float scale = static_cast<float>(as_h2(sz[i]).x) * a.scale_log2;
        const bool seen = b * kCacheBlock + 4 * g + i < lim && !(hidden >> b & 1);
        score[b][i] = seen ? s[i] * scale : -INFINITY;
      }
    }
    float most = score[0][0];
#pragma unroll
    for (int i = 1; i < 8; ++i) most = fmaxf(most, score[i / 4][i % 4]);
    if (__any(most > ref + kRoom)) {
      most = fmaxf(most, __shfl_xor(most, 16, 64));
      most = fmaxf(most, __shfl_xor(most, 32, 64));
      const float next = fmaxf(ref, most - kLead);
      const float down = __builtin_amdgcn_exp2f(ref - next);
      l *= down;
#pragma unroll
      for (int j = 0; j < U; ++j) sum[j] *= floatx4{down, down, down, down};
      ref = next;
    }
    half8 p;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      p[i] = static_cast<_Float16>(__builtin_amdgcn_exp2f(score[i / 4][i % 4] - ref));
      l += static_cast<float>(p[i]);            // what the product below adds up, so that its rounding cancels
    }
    half2v s2[2][2], c_lo[2][2], c_hi[2][2];
    uint32_t worst = 0;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const uint32_t sz[4] = {x.v_sz[b].x, x.v_sz[b].y, x.v_sz[b].z, x.v_sz[b].w};
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        half2v pair[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          // what no one has written may be NaN, and 0 x NaN is not 0
          const bool there = b * kCacheBlock + 4 * g + 2 * t + e < held && !(hidden >> b & 1);
          pair[e] = as_h2(there ? sz[2 * t + e] : 0u);
          worst = max(worst, __builtin_bit_cast(uint32_t, pair[e]) & 0x7fffu);
        }
        s2[b][t] = half2v{pair[0].x, pair[1].x};
        const half2v z = {pair[0].y, pair[1].y};
        c_lo[b][t] = minus(1024.f, z);
        c_hi[b][t] = minus(64.f, z);
      }
    }
    // A value that is NaN belongs to the rows that see it and to no other, but 0 x NaN is NaN: it goes to their sums of
    // probabilities, and into the product as zero.
    if (__any(worst >= 0x7c00u)) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const _Float16 s = s2[i / 4][i % 4 / 2][i % 2];
        if ((__builtin_bit_cast(uint16_t, s) & 0x7c00u) != 0x7c00u) continue;
        s2[i / 4][i % 4 / 2][i % 2] = (_Float16)0.f;
        if (i / 4 * kCacheBlock + 4 * g + i % 4 < lim) l = NAN;
      }
    }
#pragma unroll
    for (int j = 0; j < U; ++j) {
      half2v v[4];
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int t = 0; t < 2; ++t) v[2 * b + t] = value_pair<BITS>(x.v[b], j, t, c_lo[b][t], c_hi[b][t], s2[b][t]);
      const half8 f = {v[0].x, v[0].y, v[1].x, v[1].y, v[2].x, v[2].y, v[3].x, v[3].y};
      sum[j] = mfma16(f, p, sum[j]);
    }
  }

  // the waves' shares, brought to one reference and added
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  if (g == 0) { lds_ref[wave][r] = ref; lds_l[wave][r] = l; }
  __syncthreads();
  float top = lds_ref[0][r];
#pragma unroll
  for (int o = 1; o < kWaves; ++o) top = fmaxf(top, lds_ref[o][r]);
  const float down = __builtin_amdgcn_exp2f(ref - top);
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < U; ++j) lds_sum[wave][r][(4 * g + i) * U + j] = sum[j][i] * down;
  __syncthreads();
  const Part<D> out(a, parts);
  for (int e = threadIdx.x; e < kRows * D / 2; e += 64 * kWaves) {
    const int row = e / (D / 2), ch = e % (D / 2) * 2, at_row = tile * kRows + row;
    if (at_row >= used) break;
    float t = lds_ref[0][row], total = 0.f, y0 = 0.f, y1 = 0.f;
#pragma unroll
    for (int o = 1; o < kWaves; ++o) t = fmaxf(t, lds_ref[o][row]);
#pragma unroll
    for (int o = 0; o < kWaves; ++o) {
      total += lds_l[o][row] * __builtin_amdgcn_exp2f(lds_ref[o][row] - t);
      y0 += lds_sum[o][row][ch];
      y1 += lds_sum[o][row][ch + 1];
    }
    const int64_t token = rows.start + at_row / a.group;
    const int head = kv_head * a.group + at_row % a.group;
    if (parts == 1) {
      const float inv = total == 0.f ? 0.f : 1.f / total;
      *reinterpret_cast<half2v*>(static_cast<_Float16*>(a.y) + token * a.ldy + head * D + ch) =
          half2v{static_cast<_Float16>(y0 * inv), static_cast<_Float16>(y1 * inv)};
    } else {
      const int64_t at = (static_cast<int64_t>(n.first_part + w.part) * a.M + token) * a.q_heads + head;
      *reinterpret_cast<float2*>(out.sums + at * D + ch) = make_float2(y0, y1);
      if (ch == 0) out.stats[at] = make_float2(t, total);
    }
  }
}

// ---- many rows ----------------------------------------------------------------------------------
//
// A workgroup of four waves takes 64 RT query rows of one sequence and kv head (of all rows of the call, over the prefix) and
// stages of 64 tokens.  The codes become fp16 factors once a stage, a record's keys and half of two records' values a wave, and go to LDS as whole MFMA
// operands (1 KiB, lane order), which all waves read; two stages' worth of LDS, so that one barrier a stage is enough.  Keys are multiplied as the whole numbers
// code - z and their scale acts on the scores, in fp32.  The sum of the probabilities is one more MFMA, against ones.
constexpr int kStage = 4 * kCacheBlock;

template <int D, int BITS> struct StageCodes {
  static constexpr int kKey = D / 4 * BITS / 32;                          // dwords of a lane, keys of one record
  static constexpr int kUnits = D / 32 * BITS / 16 > 0 ? D / 32 * BITS / 16 : 1;   // 16-bit units of half a lane's value channels
  uint32_t k[kKey], v[2][2 * kUnits];
  uint32_t k_own, v_own;      // scale | zero of the token the lane multiplies
  uint4 v_sz[2];
};

template <int D> struct alignas(16) StageLds {
  uint4 k[4][D / 32][64];
  uint4 v[2][D / 16][64];
  float scale[kStage];        // of the keys, times scale_log2; NaN where a value is NaN
};

// Workgroup barrier that orders LDS traffic only: the next stage's codes stay in flight across it.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

template <int D, int BITS, int RT>
__global__ __launch_bounds__(64 * kWaves, 2) void attend_tile_kernel(AttendArgs a, AttendLaunch n, int parts) {
  constexpr int U = D / 16, KS = D / 32, kTileRows = 16 * RT * kWaves;
  constexpr int kRecord = cache_record_bytes(D, BITS), kCodes = cache_code_bytes(D, BITS);
  using Codes = StageCodes<D, BITS>;
  __shared__ StageLds<D> lds[2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, g = lane >> 4;
  const Share w = share_of(a, n);
  if (!w.any) return;
  const Rows rows = launch_rows(a, n.over, w.seq);
  const int used = (n.over == kPrefix ? rows.count : min(rows.count, a.max_rows)) * a.group;
  const int row0 = w.tile * kTileRows;
  if (row0 >= used) return;
  const int tokens = n.over == kPrefix ? 0 : own_tokens(a, w.seq);
  const int last = (min(row0 + kTileRows, used) - 1) / a.group;
  const int prefix_stages = prefix_steps_of(a, n.over, kStage);
  const int all = steps_of(a, n.over, kStage, tokens, rows.count, last);
  const int begin = w.part * n.steps, end = min(begin + n.steps, all);
  if (w.part > 0 && begin >= all) return;

  const int first_row = row0 + wave * 16 * RT;                    // of the wave
  const bool idle = first_row >= used;                            // it still brings its share of the codes
  const int least = visible(a, tokens, rows.count, min(first_row, used - 1) / a.group);
  const int most_seen = visible(a, tokens, rows.count, min(first_row + 16 * RT - 1, used - 1) / a.group);
  half8 q[RT][KS];
  int limit[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int my = min(first_row + 16 * t + r, used - 1), my_token = my / a.group;
    limit[t] = visible(a, tokens, rows.count, my_token);
    const _Float16* src = static_cast<const _Float16*>(a.q) + static_cast<int64_t>(rows.start + my_token) * a.ldq +
                          (w.kv_head * a.group + my % a.group) * D + g * (D / 4);
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const half8 h = as_h8(reinterpret_cast<const uint4*>(src)[s]);
      q[t][s] = BITS == 4 ? half8{h[0], h[4], h[1], h[5], h[2], h[6], h[3], h[7]} : h;
    }
  }

  const CacheDev& c = a.cache;
  const int block_shift = c.page_shift - 4;
  const char* head_base = c.base + w.kv_head * c.head_bytes;

  // loads this wave's share of a stage; `hidden`: which of the stage's four records have no page
  auto load = [&](int stage, Codes& x, int& hidden) {
    const bool own = stage >= prefix_stages;
    const int block0 = (own ? stage - prefix_stages : stage) * 4;
    const int32_t* table = own ? a.pages + static_cast<int64_t>(w.seq) * a.page_stride : a.prefix_pages;
    const int blocks = ((own ? tokens : a.prefix_len) + kCacheBlock - 1) / kCacheBlock;
    const char* rec[4];
    hidden = 0;
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      const int block = block0 + b;
      int page = block < blocks ? table[block >> block_shift] : -1;
      page = __builtin_amdgcn_readfirstlane(page);
      const bool bad = page < 0 || page >= c.num_pages;
      hidden |= bad ? 1 << b : 0;
      rec[b] = head_base + (bad ? 0 : page * c.page_bytes + static_cast<int64_t>(block & ((1 << block_shift) - 1)) * kRecord);
    }
    const char* mine = wave == 0 ? rec[0] : (wave == 1 ? rec[1] : (wave == 2 ? rec[2] : rec[3]));
    load_codes(x.k, mine, r * 4 + g);
    const uint32_t* sz = reinterpret_cast<const uint32_t*>(mine + 2 * kCodes);
    x.k_own = sz[r];
    x.v_own = sz[kCacheBlock + r];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const char* of = wave < 2 ? rec[b] : rec[2 + b];
      // the lane's units of channels (wave & 1) * U / 2 .. + U / 2 - 1
      constexpr int all_units = D / 16 * BITS / 16;
      const int half = wave & 1;
      const char* at = of + kCodes + (all_units == 4 ? half * 1024 + lane * 16 : (all_units == 2 ? lane * 16 + half * 8 : lane * 8));
      if constexpr (Codes::kUnits == 2) {
        const uint4 v = *reinterpret_cast<const uint4*>(at);
        x.v[b][0] = v.x; x.v[b][1] = v.y; x.v[b][2] = v.z; x.v[b][3] = v.w;
      } else {
        const uint2 v = *reinterpret_cast<const uint2*>(at);
        x.v[b][0] = v.x; x.v[b][1] = v.y;
      }
      x.v_sz[b] = reinterpret_cast<const uint4*>(of + 2 * kCodes)[4 + g];
    }
  };

  // codes -> factors in LDS
  auto store = [&](int stage, const Codes& x, int hidden, StageLds<D>& to) {
    const bool own = stage >= prefix_stages;
    const int t0 = (own ? stage - prefix_stages : stage) * kStage;
    const int held = (own ? tokens : a.prefix_len) - t0;
    const half2v own_sz = as_h2(x.k_own);
    const half2v z = {own_sz.y, own_sz.y}, k_lo = minus(1024.f, z), k_hi = minus(64.f, z);
#pragma unroll
    for (int s = 0; s < KS; ++s) to.k[wave][s][lane] = __builtin_bit_cast(uint4, key_factor<BITS>(&x.k[s * BITS / 4], k_lo, k_hi));
    if (g == 0) {
      // a value that is NaN reaches the rows that see it through their scores (the product has zero for it)
      const bool odd = (x.v_own & 0x7c00u) == 0x7c00u;
      to.scale[wave * kCacheBlock + r] = odd ? NAN : static_cast<float>(own_sz.x) * a.scale_log2;
    }
    half2v s2[2][2], c_lo[2][2], c_hi[2][2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const int record = (wave & 2) + b;
      const uint32_t sz[4] = {x.v_sz[b].x, x.v_sz[b].y, x.v_sz[b].z, x.v_sz[b].w};
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        half2v pair[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const bool there = record * kCacheBlock + 4 * g + 2 * t + e < held && !(hidden >> record & 1) &&
                             (sz[2 * t + e] & 0x7c00u) != 0x7c00u;
          pair[e] = as_h2(there ? sz[2 * t + e] : 0u);
        }
        s2[b][t] = half2v{pair[0].x, pair[1].x};
        const half2v vz = {pair[0].y, pair[1].y};
        c_lo[b][t] = minus(1024.f, vz);
        c_hi[b][t] = minus(64.f, vz);
      }
    }
#pragma unroll
    for (int j = 0; j < U / 2; ++j) {
      half2v v[4];
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          if constexpr (D == 64 && BITS == 4) {      // one unit holds all four channels
            const uint32_t mine[2] = {x.v[b][0] >> ((wave & 1) * 8), x.v[b][1] >> ((wave & 1) * 8)};
            v[2 * b + t] = value_pair<BITS>(mine, j, t, c_lo[b][t], c_hi[b][t], s2[b][t]);
          } else {
            v[2 * b + t] = value_pair<BITS>(x.v[b], j, t, c_lo[b][t], c_hi[b][t], s2[b][t]);
          }
        }
      const half8 f = {v[0].x, v[0].y, v[1].x, v[1].y, v[2].x, v[2].y, v[3].x, v[3].y};
      to.v[wave >> 1][(wave & 1) * (U / 2) + j][lane] = __builtin_bit_cast(uint4, f);
    }
  };

  floatx4 sum[RT][U], l[RT];
  float ref[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    l[t] = floatx4{0.f, 0.f, 0.f, 0.f};
    ref[t] = kNoScore;
#pragma unroll
    for (int j = 0; j < U; ++j) sum[t][j] = floatx4{0.f, 0.f, 0.f, 0.f};
  }
  const _Float16 one = (_Float16)1.f;
  const half8 ones = {one, one, one, one, one, one, one, one};

  auto multiply = [&](int stage, int hidden, const StageLds<D>& from) {
    const bool own = stage >= prefix_stages;
    const int t0 = (own ? stage - prefix_stages : stage) * kStage;
    if (own && t0 >= most_seen) return;
    const bool masked = hidden != 0 || t0 + kStage > (own ? least : a.prefix_len);
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      floatx4 score[2][RT];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
#pragma unroll
        for (int t = 0; t < RT; ++t) score[b][t] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          const half8 f = as_h8(from.k[2 * p + b][s][lane]);
#pragma unroll
          for (int t = 0; t < RT; ++t) score[b][t] = mfma16(f, q[t][s], score[b][t]);
        }
        const floatx4 scale = *reinterpret_cast<const floatx4*>(&from.scale[(2 * p + b) * kCacheBlock + 4 * g]);
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) score[b][t][i] *= scale[i];
        if (masked) {
#pragma unroll
          for (int t = 0; t < RT; ++t) {
            const int lim = (own ? limit[t] : a.prefix_len) - t0 - (2 * p + b) * kCacheBlock - 4 * g;
#pragma unroll
            for (int i = 0; i < 4; ++i) score[b][t][i] = i < lim && !(hidden >> (2 * p + b) & 1) ? score[b][t][i] : -INFINITY;
          }
        }
      }
      float most[RT];
      bool over = false;
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        most[t] = score[0][t][0];
#pragma unroll
        for (int i = 1; i < 8; ++i) most[t] = fmaxf(most[t], score[i / 4][t][i % 4]);
        over |= most[t] > ref[t] + kRoom;
      }
      if (__any(over)) {
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          most[t] = fmaxf(most[t], __shfl_xor(most[t], 16, 64));
          most[t] = fmaxf(most[t], __shfl_xor(most[t], 32, 64));
          const float next = fmaxf(ref[t], most[t] - kLead);
          const float down = __builtin_amdgcn_exp2f(ref[t] - next);
          l[t] *= floatx4{down, down, down, down};
#pragma unroll
          for (int j = 0; j < U; ++j) sum[t][j] *= floatx4{down, down, down, down};
          ref[t] = next;
        }
      }
      half8 prob[RT];
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        uint32_t pk[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
          pk[i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(__builtin_amdgcn_exp2f(score[i / 2][t][i % 2 * 2] - ref[t]),
                                                                        __builtin_amdgcn_exp2f(score[i / 2][t][i % 2 * 2 + 1] - ref[t])));
        prob[t] = as_h8(uint4{pk[0], pk[1], pk[2], pk[3]});
        l[t] = mfma16(ones, prob[t], l[t]);
      }
#pragma unroll
      for (int j = 0; j < U; ++j) {
        const half8 f = as_h8(from.v[p][j][lane]);
#pragma unroll
        for (int t = 0; t < RT; ++t) sum[t][j] = mfma16(f, prob[t], sum[t][j]);
      }
    }
  };

  if (begin < end) {
    Codes x;
    int hidden, next_hidden = 0;
    load(begin, x, hidden);
    store(begin, x, hidden, lds[0]);
    lds_barrier();
    for (int stage = begin, cur = 0; stage < end; ++stage, cur ^= 1) {
      if (stage + 1 < end) load(stage + 1, x, next_hidden);
      if (!idle) multiply(stage, hidden, lds[cur]);
      if (stage + 1 < end) store(stage + 1, x, next_hidden, lds[cur ^ 1]);
      hidden = next_hidden;
      lds_barrier();
    }
  }

  const Part<D> out(a, parts);
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int my = first_row + 16 * t + r;
    if (my >= used) continue;
    const int64_t token = rows.start + my / a.group;
    const int head = w.kv_head * a.group + my % a.group;
    if (parts == 1) {
      const float inv = l[t][0] == 0.f ? 0.f : 1.f / l[t][0];
      _Float16* y = static_cast<_Float16*>(a.y) + token * a.ldy + head * D + 4 * g * U;
#pragma unroll
      for (int e = 0; e < 4 * U / 8; ++e) {
        half8 h;
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] = static_cast<_Float16>(sum[t][(8 * e + i) % U][(8 * e + i) / U] * inv);
        reinterpret_cast<uint4*>(y)[e] = __builtin_bit_cast(uint4, h);
      }
    } else {
      const int64_t at = (static_cast<int64_t>(n.first_part + w.part) * a.M + token) * a.q_heads + head;
      float* y = out.sums + at * D + 4 * g * U;
#pragma unroll
      for (int e = 0; e < 4 * U / 4; ++e) {
        floatx4 h;
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = sum[t][(4 * e + i) % U][(4 * e + i) / U];
        reinterpret_cast<floatx4*>(y)[e] = h;
      }
      if (g == 0) out.stats[at] = make_float2(ref[t], l[t][0]);
    }
  }
}

// One wave adds up the parts of one (row, head): those of its own tokens that its sequence is long enough for, and all of the prefix.
template <int D>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendArgs a, AttendPlan plan) {
  const int lane = threadIdx.x & 63;
  const int64_t task = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
  const int row = static_cast<int>(task / a.q_heads), head = static_cast<int>(task % a.q_heads);
  if (row >= a.M) return;
  int seq = row;
  if (a.row_start) {            // the last sequence that starts at or before the row
    int lo = 0, hi = a.seqs;
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (a.row_start[mid] <= row) lo = mid; else hi = mid;
    }
    seq = lo;
  } else if (row >= a.seqs) {
    return;
  }
  const Rows rows = rows_of(a, seq);
  const int i = row - rows.start;
  const int count = min(rows.count, a.max_rows);
  if (i < 0 || i >= count) return;
  const int tile_rows = plan.own.row_tiles ? 16 * plan.own.row_tiles * kWaves : kRows;
  const int tile = (i * a.group + head % a.group) / tile_rows;
  const int last = (min((tile + 1) * tile_rows, count * a.group) - 1) / a.group;
  const int steps = steps_of(a, plan.own.over, plan.own.row_tiles ? kStage : kStep, own_tokens(a, seq), rows.count, last);
  const int filled = max(1, (steps + plan.own.steps - 1) / plan.own.steps);
  const int apart = plan.prefix.grid ? plan.prefix.parts : 0;
  const Part<D> in(a, plan.parts);
  float ref = kNoScore, l = 0.f, y[D / 64] = {};
  for (int k = 0; k < filled + apart; ++k) {
    const int p = k < filled ? plan.own.first_part + k : plan.prefix.first_part + k - filled;
    const int64_t at = (static_cast<int64_t>(p) * a.M + row) * a.q_heads + head;
    const float2 s = in.stats[at];
    const float top = fmaxf(ref, s.x), mine = __builtin_amdgcn_exp2f(ref - top), theirs = __builtin_amdgcn_exp2f(s.x - top);
    l = l * mine + s.y * theirs;
#pragma unroll
    for (int e = 0; e < D / 64; ++e) y[e] = y[e] * mine + in.sums[at * D + lane * (D / 64) + e] * theirs;
    ref = top;
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int e = 0; e < D / 64; ++e)
    static_cast<_Float16*>(a.y)[row * a.ldy + head * D + lane * (D / 64) + e] = static_cast<_Float16>(y[e] * inv);
}

static int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Shapes a launch over `rows` rows and `tokens` tokens of each of `seqs` sequences.
static AttendLaunch shape_launch(const AttendArgs& a, int over, int64_t rows, int64_t tokens_prefix, int64_t tokens_own, int64_t seqs) {
  AttendLaunch n;
  n.over = over;
  n.row_tiles = rows <= kRows && over != kPrefix ? 0 : (rows <= 64 ? 1 : 2);
  n.tiles = static_cast<int>(ceil_div(rows, n.row_tiles ? 16 * n.row_tiles * kWaves : kRows));
  const int step = n.row_tiles ? kStage : kStep;
  const int64_t all = std::max<int64_t>(1, ceil_div(tokens_prefix, step) + ceil_div(tokens_own, step));
  const int64_t pairs = seqs * a.cache.kv_heads, groups = pairs * n.tiles;
  const int64_t parts = std::clamp<int64_t>((n.row_tiles ? 512 : 2048) / groups, 1, std::max<int64_t>(1, all / (n.row_tiles ? 2 : 8)));
  n.steps = static_cast<int>(ceil_div(all, parts));
  n.parts = static_cast<int>(ceil_div(all, n.steps));
  n.by_xcd = pairs >= 8 && (pairs % 8 == 0 || pairs >= 64);
  n.grid = (n.by_xcd ? ceil_div(pairs, 8) * 8 : pairs) * n.tiles * n.parts;
  return n;
}

AttendPlan plan_attention(const AttendArgs& a) {
  AttendPlan p;
  const int64_t rows = static_cast<int64_t>(a.max_rows) * a.group;
  const bool apart = a.prefix_len > 0 && a.seqs > 1 && rows < 64;
  p.own = shape_launch(a, apart ? kOwn : kPrefixAndOwn, rows, apart ? 0 : a.prefix_len, a.max_kv, a.seqs);
  p.parts = p.own.parts;
  if (apart) {
    p.prefix = shape_launch(a, kPrefix, static_cast<int64_t>(a.M) * a.group, a.prefix_len, 0, 1);
    p.prefix.first_part = p.own.parts;
    p.parts += p.prefix.parts;
  }
  if (p.parts > 1) p.ws_bytes = static_cast<size_t>(p.parts) * a.M * a.q_heads * (a.dim + 2) * sizeof(float);
  return p;
}

template <int D, int BITS> static void launch_one(const AttendArgs& a, const AttendLaunch& n, int parts, hipStream_t st) {
  const dim3 grid(static_cast<unsigned>(n.grid)), block(64 * kWaves);
  if (n.row_tiles == 0) attend_kernel<D, BITS><<<grid, block, 0, st>>>(a, n, parts);
  else if (n.row_tiles == 1) attend_tile_kernel<D, BITS, 1><<<grid, block, 0, st>>>(a, n, parts);
  else attend_tile_kernel<D, BITS, 2><<<grid, block, 0, st>>>(a, n, parts);
}

template <int D, int BITS> static int run(const AttendArgs& a, const AttendPlan& p, hipStream_t st) {
  if (p.prefix.grid) launch_one<D, BITS>(a, p.prefix, p.parts, st);
  launch_one<D, BITS>(a, p.own, p.parts, st);
  if (p.parts > 1)
    attend_join_kernel<D><<<static_cast<unsigned>(ceil_div(static_cast<int64_t>(a.M) * a.q_heads, 4)), 256, 0, st>>>(a, p);
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return ROSAQ_OK;
  set_error(std::string("attention: ") + hipGetErrorString(e));
  return ROSAQ_ERR_HIP;
}

int launch_attention(const AttendArgs& a, const AttendPlan& p, void* stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (a.dim == 128) return a.bits == 4 ? run<128, 4>(a, p, st) : run<128, 8>(a, p, st);
  return a.bits == 4 ? run<64, 4>(a, p, st) : run<64, 8>(a, p, st);
}

}  // namespace rosaq
