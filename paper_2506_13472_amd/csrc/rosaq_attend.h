// Attention over the quantised cache: y = softmax(scale q K^T) V with the keys and values as codes.
//
// One pass over the cache with the running reference and sum of a softmax, in two kernels: attend_rows for up to 16 rows of a sequence and
// kv head (decode, drafted tokens), bound by the codes' way from memory, and attend_tile for more (prompts, a prefix under a whole
// batch), bound by arithmetic.  Both products of both run with the tokens on the rows of the MFMA's result, S^T = K Q^T and Y^T = V^T P^T:
// lane (g, r) of S^T holds query row r's scores of tokens 4 g .. 4 g + 3 of each 16, which is, as it stands, the operand P^T of
// the second product if V's lanes bring the same tokens in the same order, and the cache's layout sees to that.  So the
// probabilities go from one product to the other without leaving their registers, a row's reference and sum live in the
// lane that needs them, and codes become factors in the registers they were loaded to.
#pragma once
#include <hip/hip_runtime.h>

#include <type_traits>

#include "rosaq_attention.h"
#include "rosaq_gemm.h"

namespace rosaq {

constexpr int kStep = 2 * kCacheBlock;      // tokens of a step: the depth of one MFMA over the values
constexpr int kWaves = 4;
constexpr int kRows = 16;                   // query rows of a tile of attend_rows
constexpr float kNoScore = -1e30f;          // the reference before any score: finite, so that exp2(x - reference) is 0 or huge, never NaN, for hidden tokens

// What the second product multiplies are P' = fp16(2^(score - reference) s), with s the scale of the token's values: one rounding, to nearest, for a
// product of three numbers, and no operation for the scale on each of the values.  The reference is of the same numbers: kLead
// below the largest exponent of the step that set it, and it moves only when one passes it by kRoom, because moving it costs shuffles and a pass
// over the sums and hardly any step needs it.  2^15 is in fp16's range.  Below 2^-24 of the largest P' one loses bits, at most 2^-35 of the largest,
// and only to the product: the sums of the probabilities are fp32, from before the rounding.  As a token's largest value is at least half its scale times the
// codes' range, n tokens of one part cost at most n 2^-34 of the largest value.  A lead of 5, with 32 times that, is no faster; of 12
// the reference moves oftener (a chunk of 3 x 509 rows 242 us against 236, 32 x 3 rows behind a prefix 67.5 against 65.5).
constexpr float kLead = 10.f, kRoom = 15.f;

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

// With a window (W) row i, at position p = tokens - count + i, sees token j <= p if j > p - window or j < sinks.  A tile's steps then go from the whole step
// that the first row's window begins in to the last row, and then over the sinks, where a gap lies behind them.  Tokens that no row of the tile
// sees are neither counted on to be in the cache nor their pages to be the sequence's: of those that lie in the same step nothing is used.
// Measured: 64 x 32 heads, window 1024, 4 bits 63 us (287 MB, 4.6 TB/s), heads of 64 channels 49: half of the bytes, but three quarters of the vector operations,
// which are 60 % of its cycles; one row's 32 heads, window 8191, 8 bits 20.5; four prompts of 2048 rows x 32 heads, window 512, 8 bits 121 us = 500 TFLOP/s of
// what the mask leaves, where the whole triangle runs at 750: a tile has 11 stages then, not 17 on average, and of its 30 us some 5 go until the first codes are
// in LDS, 1.3 to the end, and the stages that some row does not see all of cost a third more than others.
// Built and slower: steps over records of 16 tokens wherever they lie, which spares up to one in eleven stages but looks up four pages a stage (prompts 139 us
// against 131, one row 21.9 against 20.7; odd windows 103 against 113), the sinks in free records of the first stage (136), their own records alone multiplied
// within the loop (spills, 188), one comparison a score for each side's mask (as fast as two), one row tile a wave (144), the second and third stage's codes touched
// ahead (139 against 136); a wave's priority raised for its products (137 against 123, 4 bits).  The sinks first cost a stage and the wait for its codes (131 against 127).
__device__ __forceinline__ int lowest(const AttendArgs& a, int tokens, int count, int i) { return max(tokens - count + i + 1 - a.window, 0); }
struct Walk {
  int start = 0;           // token that the steps begin with
  int low = 0;             // token that the first row's window begins with
  int to_sinks = 0;        // steps in front of those over the sinks
  int all = 0;             // steps
};
__device__ __forceinline__ Walk walk_of(const AttendArgs& a, int step, int tokens, int count, int first, int last) {
  Walk w;
  w.low = lowest(a, tokens, count, first);
  w.start = w.low / step * step;
  if (a.sinks >= w.start) w.start = 0;
  w.to_sinks = (max(visible(a, tokens, count, last) - w.start, 0) + step - 1) / step;
  w.all = w.to_sinks + (w.start ? (a.sinks + step - 1) / step : 0);
  return w;
}
__device__ __forceinline__ int token_of(const Walk& w, int step, int tokens) {
  return step < w.to_sinks ? w.start + step * tokens : (step - w.to_sinks) * tokens;
}

// A workgroup's share of a launch.  Workgroups go to the XCDs in turn; with by_xcd, those of one sequence and kv head, which read
// the same codes, stay on one XCD and its L2.  They are handed out from the last tile of all sequences to the first, which
// under the causal mask is from the longest: what runs last is short.  The parts of a tile run side by side: the heads of a
// sequence, on their XCDs, so read the same pages at a time (16 sequences of 8192 to 32768 tokens, 8 kv heads: 89 us, part by part 95).
struct Share { int seq, kv_head, tile, part; bool any; };
__device__ __forceinline__ Share share_of(const AttendArgs& a, const AttendLaunch& n, int id) {
  const int heads = a.cache.kv_heads, pairs = (n.over == kPrefix ? 1 : a.seqs) * heads;
  const int xcds = n.by_xcd ? 8 : 1, each = (pairs + xcds - 1) / xcds, turn = id / xcds;
  const int part = turn % n.parts, rest = turn / n.parts;
  const int pair = rest % each * xcds + id % xcds, tile = n.tiles - 1 - rest / each;
  return Share{pair / heads, pair % heads, tile, part, pair < pairs && tile >= 0};
}

// rows of a launch's sequence: with kPrefix all rows of the call are one
__device__ __forceinline__ Rows launch_rows(const AttendArgs& a, int over, int seq) {
  if (over != kPrefix) return rows_of(a, seq);
  return Rows{0, a.row_start ? min(max(a.row_start[a.seqs], 0), a.M) : a.seqs};
}

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

// Channel j (of a lane's D / 16) of two tokens of a record, as whole numbers code - z.  `w`: the lane's dwords, dword 2 i + t = unit
// i of the tokens 2 t and 2 t + 1.
template <int BITS> __device__ __forceinline__ half2v value_pair(const uint32_t* w, int j, int t, half2v c_lo, half2v c_hi) {
  const half2v sixteenth = {(_Float16)0.0625f, (_Float16)0.0625f};
  if constexpr (BITS == 4) {
    const uint32_t d = w[2 * (j / 4) + t] >> (j % 4 / 2 * 8);
    if (j % 2 == 0) return as_h2(and_or<false>(d, 0x000f000fu, 0x64006400u)) + c_lo;
    return __builtin_elementwise_fma(as_h2(and_or<false>(d, 0x00f000f0u, 0x64006400u)), sixteenth, c_hi);
  } else {
    const uint32_t d = w[2 * (j / 2) + t];
    return as_h2(__builtin_amdgcn_perm(0x64646464u, d, j % 2 == 0 ? 0x04020400u : 0x04030401u)) + c_lo;
  }
}

// The records of a step over one sequence's tokens or the prefix: N of them, from record block0 on.  look_up fetches the pages, a
// step ahead of their use; place turns them into offsets and says which records have no page (those read the cache's first, and are hidden).
// Where a page holds whole steps, one entry is enough, and records behind the last token are in the same page.
template <int N> struct Pages { int page[N]; };
template <int N> __device__ __forceinline__ Pages<N> look_up(const int32_t* table, int block0, int blocks, int block_shift) {
  Pages<N> p;
  if ((1 << block_shift) >= N) {
    p.page[0] = block0 < blocks ? table[block0 >> block_shift] : -1;
  } else {
#pragma unroll
    for (int b = 0; b < N; ++b) p.page[b] = block0 + b < blocks ? table[(block0 + b) >> block_shift] : -1;
  }
  return p;
}
template <int N>
__device__ __forceinline__ int place(const CacheDev& c, const Pages<N>& p, int block0, int block_shift, int record, int64_t (&at)[N]) {
  int hidden = 0;
  if ((1 << block_shift) >= N) {
    const int page = __builtin_amdgcn_readfirstlane(p.page[0]);
    const bool bad = static_cast<unsigned>(page) >= static_cast<unsigned>(c.num_pages);
    if (bad) hidden = (1 << N) - 1;
    const int64_t first = (bad ? 0 : page) * c.page_bytes + (block0 & ((1 << block_shift) - 1)) * record;
#pragma unroll
    for (int b = 0; b < N; ++b) at[b] = first + b * record;
  } else {
#pragma unroll
    for (int b = 0; b < N; ++b) {
      const int page = __builtin_amdgcn_readfirstlane(p.page[b]);
      const bool bad = static_cast<unsigned>(page) >= static_cast<unsigned>(c.num_pages);
      if (bad) hidden |= 1 << b;
      at[b] = (bad ? 0 : page) * c.page_bytes + ((block0 + b) & ((1 << block_shift) - 1)) * record;
    }
  }
  return hidden;
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

// Eight channels of a query, infinities as NaN (inf * 0 + inf).  A channel that is no number makes every score of its row one: infinite in one
// sign or both, or NaN, and the softmax of each is NaN.  Scores of -inf alone would look like a row that sees nothing, which is zero.
__device__ __forceinline__ half8 load_query(const _Float16* p) {
  const half8 h = as_h8(*reinterpret_cast<const uint4*>(p)), zero = {0, 0, 0, 0, 0, 0, 0, 0};
  return __builtin_elementwise_fma(h, zero, h);
}

// The power of two above a scale | zero's scale: s < 2^exponent_of <= 2 s.  (Of 0 -14, of NaN 17.)
__device__ __forceinline__ float exponent_of(uint32_t sz) { return static_cast<float>(static_cast<int>(sz >> 10 & 0x1fu) - 14); }

// Two channels of a row's answer: means of values that fp16 holds, times what the probabilities' rounding makes of them, at most 1 + 2^-11.  Above 65520
// that would be infinite, and stays at the largest number instead.  NaN passes (minimum and maximum keep it, unlike min and max).
__device__ __forceinline__ half2v answer(float a, float b) {
  const half2v most = {(_Float16)65504.f, (_Float16)65504.f};
  return __builtin_elementwise_maximum(__builtin_elementwise_minimum(half2v{static_cast<_Float16>(a), static_cast<_Float16>(b)}, most), -most);
}

// A lane's share of a row, channels 4 g U .. + 4 U - 1, to y or to the row's partial results.
template <int D>
__device__ __forceinline__ void store_row(const AttendArgs& a, const Part<D>& out, int parts, int part, int64_t token, int head, int g,
                                          float ref, float l, const floatx4 (&sum)[D / 16]) {
  constexpr int U = D / 16;
  if (parts == 1) {
    const float inv = l == 0.f ? 0.f : 1.f / l;
    _Float16* y = static_cast<_Float16*>(a.y) + token * a.ldy + head * D + 4 * g * U;
#pragma unroll
    for (int e = 0; e < 4 * U / 8; ++e) {
      half2v h[4];
#pragma unroll
      for (int i = 0; i < 8; i += 2) h[i / 2] = answer(sum[(8 * e + i) % U][(8 * e + i) / U] * inv, sum[(8 * e + i + 1) % U][(8 * e + i + 1) / U] * inv);
      reinterpret_cast<uint4*>(y)[e] = __builtin_bit_cast(uint4, h);
    }
  } else {
    const int64_t at = (static_cast<int64_t>(part) * a.M + token) * a.q_heads + head;
    float* y = out.sums + at * D + 4 * g * U;
#pragma unroll
    for (int e = 0; e < 4 * U / 4; ++e) {
      floatx4 h;
#pragma unroll
      for (int i = 0; i < 4; ++i) h[i] = sum[(4 * e + i) % U][(4 * e + i) / U];
      reinterpret_cast<floatx4*>(y)[e] = h;
    }
    if (g == 0) out.stats[at] = make_float2(ref, l);
  }
}

// What a lane holds of one step: codes of two records and the scales and zeros it needs of them.
template <int D, int BITS> struct Step {
  static constexpr int kDwords = D / 4 * BITS / 32;     // of a lane, keys or values of one record: 2, 4 or 8
  uint32_t k[2][kDwords], v[2][kDwords];
  uint32_t k_own[2];        // scale | zero of the key token that the lane multiplies
  uint4 k_sz[2], v_sz[2];   // of tokens 4 g .. 4 g + 3
  int hidden;               // which of the two records have no page
};

// ---- few rows -----------------------------------------------------------------------------------
//
// A wave takes one tile of up to 16 rows and steps of 32 tokens, alone (SPLIT 1: four tiles a workgroup) or as one of the four of a workgroup
// that take its steps in turn (SPLIT 4) and add up what they have in LDS.  Codes become factors in the registers they were loaded to, a step ahead,
// their pages two.  Besides the stream of codes (5.3 TB/s of 5.2 that a copy reaches: 98 us for 65537 tokens x 32 heads of 8 bits)
// the vector units bound it: some 270 operations a step and wave, of which those on 4-bit codes are as many as on 8-bit ones,
// so that 4 bits reach 4.3 TB/s (88 us, 16 sequences of 8192 to 32768 tokens x 8 kv heads).  Short sequences are bound by the way to the
// first codes (arguments, lengths, pages): 64 x 32 heads of up to 256 tokens take 16 us for 54 MB.
template <int D> struct RowsLds {
  float sum[kWaves][kRows][D + 4];
  float ref[kWaves][kRows], l[kWaves][kRows];
};
template <int D, int BITS, int SPLIT, bool W = false>
__device__ __forceinline__ void attend_rows(const AttendArgs& a, const AttendLaunch& n, int parts, int block, RowsLds<D>& lds) {
  constexpr int U = D / 16, KS = D / 32;
  constexpr int kRecord = cache_record_bytes(D, BITS), kCodes = cache_code_bytes(D, BITS);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, g = lane >> 4;
  const Share w = share_of(a, n, SPLIT == 1 ? block * kWaves + wave : block);
  if (!w.any) return;
  const int kv_head = w.kv_head, seq = w.seq, tile = w.tile;
  const CacheDev& c = a.cache;
  const int block_shift = c.page_shift - 4;
  const char* head_base = c.base + kv_head * c.head_bytes;
  const int32_t* own_pages = a.pages + static_cast<int64_t>(seq) * a.page_stride;
  const int prefix_steps = prefix_steps_of(a, n.over, kStep);
  Walk walk;
  // pages of a step, given how many tokens the sequence has
  auto pages_of = [&](int step, int tokens) {
    if constexpr (W) {
      const int held = step < walk.to_sinks ? tokens : min(a.sinks, tokens);
      return look_up<2>(own_pages, token_of(walk, step, kStep) / kCacheBlock, (held + kCacheBlock - 1) / kCacheBlock, block_shift);
    }
    const bool own = step >= prefix_steps;
    return look_up<2>(own ? own_pages : a.prefix_pages, (own ? step - prefix_steps : step) * 2,
                      ((own ? tokens : a.prefix_len) + kCacheBlock - 1) / kCacheBlock, block_shift);
  };
  // those of the first step are fetched beside the sequence's length, for as many tokens as it may have
  Pages<2> first_pages;
  if constexpr (!W) first_pages = pages_of(w.part * n.steps + (SPLIT == 1 ? 0 : wave), a.capacity);
  const Rows rows = rows_of(a, seq);
  const int used = min(rows.count, a.max_rows) * a.group;         // rows of this kv head: (token, query head of the group)
  if (tile * kRows >= used) return;
  const int tokens = own_tokens(a, seq);
  const int first = tile * kRows / a.group, last = (min(tile * kRows + kRows, used) - 1) / a.group;
  if constexpr (W) walk = walk_of(a, kStep, tokens, rows.count, first, last);
  const int all = W ? walk.all : steps_of(a, n.over, kStep, tokens, rows.count, last);
  const int begin = w.part * n.steps, end = min(begin + n.steps, all);
  if (w.part > 0 && begin >= all) return;                         // part 0 always answers, if only that there is nothing

  // rows of the tile: (token, head) of this lane's column, clamped into the sequence's
  const int my = min(tile * kRows + r, used - 1);
  const int my_token = my / a.group;
  const int limit = visible(a, tokens, rows.count, my_token), least = visible(a, tokens, rows.count, first);
  const int low = W ? lowest(a, tokens, rows.count, my_token) : 0, most_low = W ? lowest(a, tokens, rows.count, last) : 0;

  auto load = [&](int step, const Pages<2>& pages, Step<D, BITS>& x) {
    int64_t at[2];
    const int block0 = W ? token_of(walk, step, kStep) / kCacheBlock : (step >= prefix_steps ? step - prefix_steps : step) * 2;
    x.hidden = place<2>(c, pages, block0, block_shift, kRecord, at);
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const char* rec = head_base + at[b];
      load_codes(x.k[b], rec, r * 4 + g);
      load_codes(x.v[b], rec + kCodes, lane);
      const uint32_t* sz = reinterpret_cast<const uint32_t*>(rec + 2 * kCodes);
      x.k_own[b] = sz[r];
      x.k_sz[b] = reinterpret_cast<const uint4*>(sz)[g];
      x.v_sz[b] = reinterpret_cast<const uint4*>(sz)[4 + g];
    }
  };

  // The first codes are asked for first: the queries' way is as long.
  constexpr int kTurn = SPLIT == 1 ? 1 : kWaves;
  int step = begin + (SPLIT == 1 ? 0 : wave);
  Step<D, BITS> x, y;
  if (step < end) {
    if constexpr (W) first_pages = pages_of(step, tokens);
    load(step, first_pages, x);
  }
  auto tokens_to = [&](int step) { return step < end ? tokens : 0; };

  half8 q[KS];
  {
    const _Float16* src = static_cast<const _Float16*>(a.q) + static_cast<int64_t>(rows.start + my_token) * a.ldq +
                          (kv_head * a.group + my % a.group) * D + g * (D / 4);
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const half8 h = load_query(src + 8 * s);
      q[s] = BITS == 4 ? half8{h[0], h[4], h[1], h[5], h[2], h[6], h[3], h[7]} : h;
    }
  }

  floatx4 sum[U];
#pragma unroll
  for (int j = 0; j < U; ++j) sum[j] = floatx4{0.f, 0.f, 0.f, 0.f};
  float ref = kNoScore, l = 0.f;

  auto multiply = [&](int step, const Step<D, BITS>& x) {
    const bool own = W || step >= prefix_steps;
    const int t0 = W ? token_of(walk, step, kStep) : (own ? step - prefix_steps : step) * kStep;
    float score[8];
    uint32_t v_sz[8], v_z[8];     // scales that the lane's row takes, zeros that its channels take: of the same tokens
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const half2v own_sz = as_h2(x.k_own[b]);
      const half2v z = {own_sz.y, own_sz.y}, c_lo = minus(1024.f, z), c_hi = minus(64.f, z);
      floatx4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < KS; ++k) s = mfma16(key_factor<BITS>(&x.k[b][k * BITS / 4], c_lo, c_hi), q[k], s);
      const uint32_t ks[4] = {x.k_sz[b].x, x.k_sz[b].y, x.k_sz[b].z, x.k_sz[b].w};
      const uint32_t vs[4] = {x.v_sz[b].x, x.v_sz[b].y, x.v_sz[b].z, x.v_sz[b].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        score[4 * b + i] = s[i] * (static_cast<float>(as_h2(ks[i]).x) * a.scale_log2);
        v_sz[4 * b + i] = v_z[4 * b + i] = vs[i];
      }
    }
    if (x.hidden != 0 || t0 + kStep > (own ? least : a.prefix_len) || (W && t0 < most_low && t0 + kStep > a.sinks)) {
      // what a row does not see weighs nothing, and what no one has written may be NaN: its scale and zero are not used either
      const int lim = (own ? limit : a.prefix_len) - t0 - 4 * g, held = (own ? tokens : a.prefix_len) - t0 - 4 * g;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int at = i / 4 * kCacheBlock + i % 4;
        const bool there = !(x.hidden >> (i / 4) & 1);
        const int token = t0 + 4 * g + at;
        const bool seen = there && at < lim && (!W || token >= low || token < a.sinks);
        score[i] = seen ? score[i] : -INFINITY;
        v_sz[i] = seen ? v_sz[i] : 0u;
        v_z[i] = there && at < held && (!W || token >= walk.low || token < a.sinks) ? v_z[i] : 0u;
      }
    }
    float most = score[0] + exponent_of(v_sz[0]);
#pragma unroll
    for (int i = 1; i < 8; ++i) most = fmaxf(most, score[i] + exponent_of(v_sz[i]));
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
      const float e = __builtin_amdgcn_exp2f(score[i] - ref);
      l += e;
      p[i] = static_cast<_Float16>(e * static_cast<float>(as_h2(v_sz[i]).x));
    }
    half2v c_lo[4], c_hi[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const half2v z = {as_h2(v_z[2 * t]).y, as_h2(v_z[2 * t + 1]).y};
      c_lo[t] = minus(1024.f, z);
      c_hi[t] = minus(64.f, z);
    }
#pragma unroll
    for (int j = 0; j < U; ++j) {
      half2v v[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) v[t] = value_pair<BITS>(x.v[t / 2], j, t % 2, c_lo[t], c_hi[t]);
      const half8 f = {v[0].x, v[0].y, v[1].x, v[1].y, v[2].x, v[2].y, v[3].x, v[3].y};
      sum[j] = mfma16(f, p, sum[j]);
    }
  };

  if (step < end) {
    // two steps' codes: one is multiplied while the next is on its way, and the pages of the one after
    Pages<2> next = pages_of(step + kTurn, tokens_to(step + kTurn));
    while (true) {
      if (step + kTurn < end) {
        load(step + kTurn, next, y);
        next = pages_of(step + 2 * kTurn, tokens_to(step + 2 * kTurn));
      }
      multiply(step, x);
      step += kTurn;
      if (step >= end) break;
      if (step + kTurn < end) {
        load(step + kTurn, next, x);
        next = pages_of(step + 2 * kTurn, tokens_to(step + 2 * kTurn));
      }
      multiply(step, y);
      step += kTurn;
      if (step >= end) break;
    }
  }
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  const Part<D> out(a, parts);
  const int part = n.first_part + w.part;

  if constexpr (SPLIT == 1) {
    if (tile * kRows + r < used)
      store_row<D>(a, out, parts, part, rows.start + my_token, kv_head * a.group + my % a.group, g, ref, l, sum);
  } else {
    // the waves' shares, brought to one reference and added
    if (g == 0) { lds.ref[wave][r] = ref; lds.l[wave][r] = l; }
    __syncthreads();
    float top = lds.ref[0][r];
#pragma unroll
    for (int o = 1; o < kWaves; ++o) top = fmaxf(top, lds.ref[o][r]);
    const float down = __builtin_amdgcn_exp2f(ref - top);
    if (tile * kRows + r < used) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < U; ++j) lds.sum[wave][r][(4 * g + i) * U + j] = sum[j][i] * down;
    }
    __syncthreads();
    for (int e = threadIdx.x; e < kRows * D / 2; e += 64 * kWaves) {
      const int row = e / (D / 2), ch = e % (D / 2) * 2, at_row = tile * kRows + row;
      if (at_row >= used) break;
      float t = lds.ref[0][row], total = 0.f, y0 = 0.f, y1 = 0.f;
#pragma unroll
      for (int o = 1; o < kWaves; ++o) t = fmaxf(t, lds.ref[o][row]);
#pragma unroll
      for (int o = 0; o < kWaves; ++o) {
        total += lds.l[o][row] * __builtin_amdgcn_exp2f(lds.ref[o][row] - t);
        y0 += lds.sum[o][row][ch];
        y1 += lds.sum[o][row][ch + 1];
      }
      const int64_t token = rows.start + at_row / a.group;
      const int head = kv_head * a.group + at_row % a.group;
      if (parts == 1) {
        const float inv = total == 0.f ? 0.f : 1.f / total;
        *reinterpret_cast<half2v*>(static_cast<_Float16*>(a.y) + token * a.ldy + head * D + ch) =
            answer(y0 * inv, y1 * inv);
      } else {
        const int64_t at = (static_cast<int64_t>(part) * a.M + token) * a.q_heads + head;
        *reinterpret_cast<float2*>(out.sums + at * D + ch) = make_float2(y0, y1);
        if (ch == 0) out.stats[at] = make_float2(t, total);
      }
    }
  }
}

// ---- many rows ----------------------------------------------------------------------------------
//
// A workgroup of four waves takes 64 RT query rows (RT 1 for up to 64 rows, else 2) of one sequence and kv head (of all rows of the call, over the prefix) and
// stages of 64 tokens.  The codes become fp16 factors once a stage, a record's keys and half of two records' values a wave, and go to LDS as whole MFMA
// operands (1 KiB, lane order), which all waves read.
// Both are the whole numbers code - z.  The keys' scale acts on the scores, in fp32: rounded factors would be off by 2^-11 of a
// score that may be in the hundreds.  The values' scale is in the other factor, as in attend_rows, here through the exponent: P' = 2^(score + log2 s - reference),
// with log2 s over the keys' scale as what the sum of a score starts from.
// The sum of the probabilities, P' / s in fp32, takes P' before it is rounded: next to a token of large values, those of others may round to nothing,
// which the product does not notice, but their weights would be missing here.
//
// Measured: four prompts of 2048 tokens x 32 heads (8 bits) 180 to 186 us = 740 to 766 TFLOP/s of the products that the mask leaves (a product of two
// 8192 x 8192 fp16 matrices: 1133).  A stage of a wave takes 62 MFMAs of 16 cycles and some 285 vector operations (four cycles, eight for each of its 32
// exponentials), 31 % and 39 % of a SIMD's 442 thousand cycles.  One after the other they would take 70 %, so its two waves (240 registers) fill
// none of each other's gaps on the whole: each waits for data or the barrier in 28 % of its cycles, and to issue in 28 %.
// Built and slower: eight waves a workgroup with half of them half a stage behind (233 against 189 us: the barriers
// cost more than the sharing saves), the factors of the next stage between the MFMAs by the scheduler's groups (spills; 260
// against 239 on the 4-bit chunk), three and four row tiles a wave (spills), half a stage at a time and one stage's LDS for three workgroups
// a unit (spills), priorities around either product (none or worse).
constexpr int kStage = 4 * kCacheBlock;

template <int D, int BITS> struct StageCodes {
  static constexpr int kKey = D / 4 * BITS / 32;                          // dwords of a lane, keys of one record
  static constexpr int kUnits = D / 32 * BITS / 16 > 0 ? D / 32 * BITS / 16 : 1;   // 16-bit units of half a lane's value channels
  uint32_t k[kKey], v[2][2 * kUnits];
  uint32_t k_own, v_own;      // scale | zero of the token the lane multiplies
  uint4 v_sz[2];
  int hidden;                 // which of the stage's four records have no page
};

// Two stages' factors, so that one barrier a stage is enough; with one row tile a wave one stage's, which leaves room for three workgroups on a compute unit.
constexpr int stage_buffers(int row_tiles) { return row_tiles == 1 ? 1 : 2; }

template <int D> struct alignas(16) StageLds {
  uint4 k[4][D / 32][64];
  uint4 v[2][D / 16][64];
  float scale[kStage];        // of the keys, times scale_log2
  float start[kStage];        // log2 of the values' scales, over `scale`; NaN where a value is NaN
  float inverse[kStage];      // of the values' scales, 0 where that is no number
};

// Workgroup barrier that orders LDS traffic only: the next stage's codes stay in flight across it.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// The bits of 64 from this one on.
__device__ __forceinline__ uint64_t from_bit(int n) {
  const int m = min(max(n, 0), 64);
  return ~uint64_t{0} << m / 2 << (m - m / 2);
}

template <int D, int BITS, int RT, bool W = false>
__device__ __forceinline__ void attend_tile(const AttendArgs& a, const AttendLaunch& n, int parts, int block, StageLds<D> (&lds)[stage_buffers(RT)]) {
  constexpr int U = D / 16, KS = D / 32, kTileRows = 16 * RT * kWaves;
  constexpr int kRecord = cache_record_bytes(D, BITS), kCodes = cache_code_bytes(D, BITS);
  constexpr int kBuffers = stage_buffers(RT);
  using Codes = StageCodes<D, BITS>;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, g = lane >> 4;
  const Share w = share_of(a, n, block);
  if (!w.any) return;
  const Rows rows = launch_rows(a, n.over, w.seq);
  const int used = (n.over == kPrefix ? rows.count : min(rows.count, a.max_rows)) * a.group;
  const int row0 = w.tile * kTileRows;
  if (row0 >= used) return;
  const int tokens = n.over == kPrefix ? 0 : own_tokens(a, w.seq);
  const int last = (min(row0 + kTileRows, used) - 1) / a.group;
  const int prefix_stages = prefix_steps_of(a, n.over, kStage);
  Walk walk;
  if constexpr (W) walk = walk_of(a, kStage, tokens, rows.count, row0 / a.group, last);
  const int all = W ? walk.all : steps_of(a, n.over, kStage, tokens, rows.count, last);
  const int begin = w.part * n.steps, end = min(begin + n.steps, all);
  if (w.part > 0 && begin >= all) return;

  const int first_row = row0 + wave * 16 * RT;                    // of the wave
  const bool idle = first_row >= used;                            // it still brings its share of the codes
  const int least = visible(a, tokens, rows.count, min(first_row, used - 1) / a.group);
  const int most_seen = visible(a, tokens, rows.count, min(first_row + 16 * RT - 1, used - 1) / a.group);
  const int least_low = W ? lowest(a, tokens, rows.count, min(first_row, used - 1) / a.group) : 0;
  const int most_low = W ? lowest(a, tokens, rows.count, min(first_row + 16 * RT - 1, used - 1) / a.group) : 0;
  half8 q[RT][KS];
  int limit[RT];
  auto load_queries = [&]() {
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const int my = min(first_row + 16 * t + r, used - 1), my_token = my / a.group;
      limit[t] = visible(a, tokens, rows.count, my_token);
      const _Float16* src = static_cast<const _Float16*>(a.q) + static_cast<int64_t>(rows.start + my_token) * a.ldq +
                            (w.kv_head * a.group + my % a.group) * D + g * (D / 4);
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const half8 h = load_query(src + 8 * s);
        q[t][s] = BITS == 4 ? half8{h[0], h[4], h[1], h[5], h[2], h[6], h[3], h[7]} : h;
      }
    }
  };

  const CacheDev& c = a.cache;
  const int block_shift = c.page_shift - 4;
  const char* head_base = c.base + w.kv_head * c.head_bytes;
  const int32_t* own_pages = a.pages + static_cast<int64_t>(w.seq) * a.page_stride;
  // of a lane: its codes within a record
  constexpr int kAllUnits = D / 16 * BITS / 16;
  const uint32_t k_at = (r * 4 + g) * (Codes::kKey == 2 ? 8 : 16);
  const uint32_t v_at = kCodes + (kAllUnits == 4 ? (wave & 1) * 1024 + lane * 16 : (kAllUnits == 2 ? lane * 16 + (wave & 1) * 8 : lane * 8));

  auto pages_of = [&](int stage) {
    if constexpr (W) {
      const int held = stage < walk.to_sinks ? tokens : min(a.sinks, tokens);
      return look_up<4>(own_pages, token_of(walk, stage, kStage) / kCacheBlock, stage < end ? (held + kCacheBlock - 1) / kCacheBlock : 0, block_shift);
    }
    const bool own = stage >= prefix_stages;
    return look_up<4>(own ? own_pages : a.prefix_pages, (own ? stage - prefix_stages : stage) * 4,
                      stage < end ? ((own ? tokens : a.prefix_len) + kCacheBlock - 1) / kCacheBlock : 0, block_shift);
  };
  // loads this wave's share of a stage
  auto load = [&](int stage, const Pages<4>& pages, Codes& x) {
    int64_t at[4];
    const int block0 = W ? token_of(walk, stage, kStage) / kCacheBlock : (stage >= prefix_stages ? stage - prefix_stages : stage) * 4;
    x.hidden = place<4>(c, pages, block0, block_shift, kRecord, at);
    const int64_t pair[2] = {wave < 2 ? at[0] : at[2], wave < 2 ? at[1] : at[3]};
    const char* mine = head_base + (wave & 1 ? pair[1] : pair[0]);
#pragma unroll
    for (int p = 0; p < (Codes::kKey + 3) / 4; ++p) {
      if constexpr (Codes::kKey == 2) {
        const uint2 t = *reinterpret_cast<const uint2*>(mine + k_at);
        x.k[0] = t.x; x.k[1] = t.y;
      } else {
        const uint4 t = *reinterpret_cast<const uint4*>(mine + k_at + p * 1024);
        x.k[4 * p] = t.x; x.k[4 * p + 1] = t.y; x.k[4 * p + 2] = t.z; x.k[4 * p + 3] = t.w;
      }
    }
    x.k_own = *reinterpret_cast<const uint32_t*>(mine + 2 * kCodes + 4u * r);
    x.v_own = *reinterpret_cast<const uint32_t*>(mine + 2 * kCodes + kCacheBlock * 4 + 4u * r);
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const char* of = head_base + pair[b];
      if constexpr (Codes::kUnits == 2) {
        const uint4 v = *reinterpret_cast<const uint4*>(of + v_at);
        x.v[b][0] = v.x; x.v[b][1] = v.y; x.v[b][2] = v.z; x.v[b][3] = v.w;
      } else {
        const uint2 v = *reinterpret_cast<const uint2*>(of + v_at);
        x.v[b][0] = v.x; x.v[b][1] = v.y;
      }
      x.v_sz[b] = *reinterpret_cast<const uint4*>(of + 2 * kCodes + kCacheBlock * 4 + 16u * g);
    }
  };

  // codes -> factors in LDS
  auto store = [&](int stage, const Codes& x, StageLds<D>& to) {
    const bool own = W || stage >= prefix_stages;
    const int t0 = W ? token_of(walk, stage, kStage) : (own ? stage - prefix_stages : stage) * kStage;
    const int held = (own ? tokens : a.prefix_len) - t0;
    const half2v own_sz = as_h2(x.k_own);
    const half2v z = {own_sz.y, own_sz.y}, k_lo = minus(1024.f, z), k_hi = minus(64.f, z);
    if (g == 0) {
      // a value that is NaN reaches the rows that see it through their scores, and no other row
      const int at = wave * kCacheBlock + r;
      const float s = static_cast<float>(as_h2(x.v_own).x);
      const float ks = static_cast<float>(own_sz.x) * a.scale_log2;
      to.scale[at] = ks;
      to.start[at] = __builtin_amdgcn_logf(s) * __builtin_amdgcn_rcpf(ks);
      // what a row does not see weighs 0 there, and 0 x NaN is NaN
      to.inverse[at] = s > 0.f && s < INFINITY ? __builtin_amdgcn_rcpf(s) : 0.f;
    }
#pragma unroll
    for (int s = 0; s < KS; ++s)
      to.k[wave][s][lane] = __builtin_bit_cast(uint4, key_factor<BITS>(&x.k[s * BITS / 4], k_lo, k_hi));
    uint32_t sz[2][4];
#pragma unroll
    for (int b = 0; b < 2; ++b) { sz[b][0] = x.v_sz[b].x; sz[b][1] = x.v_sz[b].y; sz[b][2] = x.v_sz[b].z; sz[b][3] = x.v_sz[b].w; }
    if (held < kStage || x.hidden || (W && t0 < walk.low && t0 + kStage > a.sinks)) {       // what no one has written, or another sequence
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int record = (wave & 2) + b;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int at = record * kCacheBlock + 4 * g + i;
          const bool away = (at >= held) | ((x.hidden >> record & 1) != 0) | (W && ((t0 + at < walk.low) & (t0 + at >= a.sinks)));
          sz[b][i] = away ? 0u : sz[b][i];
        }
      }
    }
    half2v c_lo[2][2], c_hi[2][2];
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const half2v vz = as_h2(__builtin_amdgcn_perm(sz[b][2 * t + 1], sz[b][2 * t], 0x07060302u));
        c_lo[b][t] = minus(1024.f, vz);
        c_hi[b][t] = minus(64.f, vz);
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
            v[2 * b + t] = value_pair<BITS>(mine, j, t, c_lo[b][t], c_hi[b][t]);
          } else {
            v[2 * b + t] = value_pair<BITS>(x.v[b], j, t, c_lo[b][t], c_hi[b][t]);
          }
        }
      const half8 f = {v[0].x, v[0].y, v[1].x, v[1].y, v[2].x, v[2].y, v[3].x, v[3].y};
      to.v[wave >> 1][(wave & 1) * (U / 2) + j][lane] = __builtin_bit_cast(uint4, f);
    }
  };

  floatx4 sum[RT][U];
  float ref[RT], l[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    l[t] = 0.f;
    ref[t] = kNoScore;
#pragma unroll
    for (int j = 0; j < U; ++j) sum[t][j] = floatx4{0.f, 0.f, 0.f, 0.f};
  }

  // NB: records of the stage that count
  auto multiply = [&](auto records, int stage, int hidden, const StageLds<D>& from) {
    constexpr int NB = decltype(records)::value;
    const bool own = W || stage >= prefix_stages;
    const int t0 = W ? token_of(walk, stage, kStage) : (own ? stage - prefix_stages : stage) * kStage;
    if (own && t0 >= most_seen) return;
    if (W && t0 + kStage <= least_low && t0 >= a.sinks) return;
    const bool masked = hidden != 0 || t0 + kStage > (own ? least : a.prefix_len) || (W && t0 < most_low && t0 + kStage > a.sinks);
    floatx4 score[4][RT];                // products, then scores less the reference
    float base[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) base[t] = ref[t] == kNoScore ? 0.f : ref[t];
    floatx4 start[4];
#pragma unroll
    for (int b = 0; b < NB; ++b) start[b] = *reinterpret_cast<const floatx4*>(&from.start[b * kCacheBlock + 4 * g]);
#pragma unroll
    for (int s = 0; s < KS; ++s)         // a product never waits for the sum of the one before
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const half8 f = as_h8(from.k[b][s][lane]);
#pragma unroll
        for (int t = 0; t < RT; ++t) score[b][t] = mfma16(f, q[t][s], s ? score[b][t] : start[b]);
      }
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const floatx4 scale = *reinterpret_cast<const floatx4*>(&from.scale[b * kCacheBlock + 4 * g]);
#pragma unroll
      for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) score[b][t][i] = __builtin_fmaf(score[b][t][i], scale[i], -base[t]);
    }
    if (W && masked) {
      // a bit for each token of the stage that a row does not see.  With two borders and the sinks faster than comparisons for each score (119.3 us against
      // 123, 4 x 2048 rows x 32 heads, window 512, 4 bits), with one border slower
      const uint64_t no_sinks = from_bit(a.sinks - t0);
      uint64_t absent = 0;
#pragma unroll
      for (int b = 0; b < NB; ++b) absent |= (hidden >> b & 1) ? uint64_t{0xffff} << 16 * b : 0;
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        const int lim = limit[t] - t0;         // a row's window begins `window` tokens before its limit
        const uint64_t away = (from_bit(lim) | (no_sinks & ~from_bit(lim - a.window)) | absent) >> 4 * g;
        const uint32_t half[2] = {static_cast<uint32_t>(away), static_cast<uint32_t>(away >> 32)};
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const bool off = half[b / 2] >> (16 * (b % 2) + i) & 1;
            score[b][t][i] = off ? -INFINITY : score[b][t][i];
          }
      }
    } else if (masked) {
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          const int lim = (own ? limit[t] : a.prefix_len) - t0 - b * kCacheBlock - 4 * g;
#pragma unroll
          for (int i = 0; i < 4; ++i)
            score[b][t][i] = i < lim && !(hidden >> b & 1) ? score[b][t][i] : -INFINITY;
        }
    }
    float most[RT];
    bool over = false;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      most[t] = score[0][t][0];
#pragma unroll
      for (int i = 1; i < 4 * NB; ++i) most[t] = fmaxf(most[t], score[i / 4][t][i % 4]);
      over |= most[t] > (ref[t] == kNoScore ? kNoScore : kRoom);
    }
    if (__any(over)) {
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        most[t] = fmaxf(most[t], __shfl_xor(most[t], 16, 64));
        most[t] = fmaxf(most[t], __shfl_xor(most[t], 32, 64));
        const bool first = ref[t] == kNoScore;       // the reference goes to the first scores, up or down
        if (first && !(most[t] > kNoScore)) continue;
        const float up = first ? most[t] - kLead : fmaxf(0.f, most[t] - kLead), down = first ? 0.f : __builtin_amdgcn_exp2f(-up);
        l[t] *= down;
#pragma unroll
        for (int j = 0; j < U; ++j) sum[t][j] *= floatx4{down, down, down, down};
#pragma unroll
        for (int i = 0; i < 4 * NB; ++i) score[i / 4][t][i % 4] -= up;
        ref[t] = base[t] + up;
      }
    }
#pragma unroll
    for (int p = 0; p < (NB + 1) / 2; ++p) {
      half8 prob[RT];
      floatx4 inverse[2];
#pragma unroll
      for (int b = 0; b < 2; ++b) inverse[b] = *reinterpret_cast<const floatx4*>(&from.inverse[(2 * p + b) * kCacheBlock + 4 * g]);
#pragma unroll
      for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (2 * p + i / 4 >= NB) { prob[t][i] = static_cast<_Float16>(0.f); continue; }
          const float e = __builtin_amdgcn_exp2f(score[2 * p + i / 4][t][i % 4]);
          l[t] = __builtin_fmaf(e, inverse[i / 4][i % 4], l[t]);
          prob[t][i] = static_cast<_Float16>(e);
        }
#pragma unroll
      for (int j = 0; j < U; ++j) {
        const half8 f = as_h8(from.v[p][j][lane]);
#pragma unroll
        for (int t = 0; t < RT; ++t) sum[t][j] = mfma16(f, prob[t], sum[t][j]);
      }
    }
  };

  // few sinks are one record, which takes a third of a stage's products, behind the loop
  const int short_one = W && end > begin && end > walk.to_sinks && a.sinks <= kCacheBlock ? 1 : 0;
  if (begin < end) {
    Codes x;
    int hidden;
    Pages<4> next = pages_of(begin);
    load(begin, next, x);
    next = pages_of(begin + 1);
    load_queries();           // behind the codes, which are waited for first: four prompts as above without a window 184 to 190 us, queries first 188 to 190
    store(begin, x, lds[0]);
    hidden = x.hidden;
    lds_barrier();
    for (int stage = begin, cur = 0; stage < end - short_one; ++stage, cur ^= 1) {
      if (stage + 1 < end) {
        load(stage + 1, next, x);
        next = pages_of(stage + 2);
      }
      if (!idle) multiply(std::integral_constant<int, 4>{}, stage, hidden, lds[kBuffers == 1 ? 0 : cur]);
      if (kBuffers == 1) lds_barrier();
      if (stage + 1 < end) store(stage + 1, x, lds[kBuffers == 1 ? 0 : cur ^ 1]);
      hidden = x.hidden;
      lds_barrier();
    }
    if (W && short_one && !idle) multiply(std::integral_constant<int, 1>{}, end - 1, hidden, lds[kBuffers == 1 ? 0 : (end - 1 - begin) & 1]);
  }

  const Part<D> out(a, parts);
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int my = first_row + 16 * t + r;
    l[t] += __shfl_xor(l[t], 16, 64);
    l[t] += __shfl_xor(l[t], 32, 64);
    if (my >= used) continue;
    store_row<D>(a, out, parts, n.first_part + w.part, rows.start + my / a.group, w.kv_head * a.group + my % a.group, g, ref[t],
                 l[t], sum[t]);
  }
}

template <int D, int BITS, int SPLIT, bool W>
__global__ __launch_bounds__(64 * kWaves, D == 128 && BITS == 8 ? 2 : 3) void attend_rows_kernel(AttendArgs a, AttendLaunch n, int parts) {
  __shared__ RowsLds<D> lds;
  attend_rows<D, BITS, SPLIT, W>(a, n, parts, blockIdx.x, lds);
}

template <int D, int BITS, int RT, bool W>
__global__ __launch_bounds__(64 * kWaves, 2) void attend_tile_kernel(AttendArgs a, AttendLaunch n, int parts) {
  __shared__ StageLds<D> lds[stage_buffers(RT)];
  attend_tile<D, BITS, RT, W>(a, n, parts, blockIdx.x, lds);
}

// Adds up the parts of one (row, head): those of its own tokens that its sequence is long enough for, and all of the prefix.  WAVES of a workgroup of
// four take one: parts go to its half waves in turn, 4 (D 64: 2) channels a lane, and a half wave's loads do not wait for each other.
// A call may have 2^27 outputs, and a dimension of a grid ends at 2^32 threads, beyond which a launch runs a part of them without an error: the
// workgroups lie in rows of kJoinRow.
constexpr int kJoinRow = 1 << 20;
template <int D, int WAVES, bool W>
__global__ __launch_bounds__(64 * kWaves) void attend_join_kernel(AttendArgs a, AttendPlan plan) {
  constexpr int C = D / 32, kHalves = 2 * WAVES;
  typedef float vec __attribute__((ext_vector_type(C)));
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t block = static_cast<int64_t>(blockIdx.y) * kJoinRow + blockIdx.x, task = WAVES == 1 ? block * kWaves + wave : block;
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
  const int step = plan.own.row_tiles ? kStage : kStep;
  const int steps = W ? walk_of(a, step, own_tokens(a, seq), rows.count, tile * tile_rows / a.group, last).all
                      : steps_of(a, plan.own.over, step, own_tokens(a, seq), rows.count, last);
  const int filled = max(1, (steps + plan.own.steps - 1) / plan.own.steps);
  const int total = filled + (plan.prefix.grid ? plan.prefix.parts : 0);
  const Part<D> in(a, plan.parts);
  const int half = WAVES == 1 ? lane >> 5 : threadIdx.x >> 5, ch = (lane & 31) * C;
  auto place = [&](int k) {
    const int p = k < filled ? plan.own.first_part + k : plan.prefix.first_part + k - filled;
    return (static_cast<int64_t>(p) * a.M + row) * a.q_heads + head;
  };
  float ref = kNoScore, l = 0.f;
  vec y = {};
  for (int k0 = half; k0 < total; k0 += 4 * kHalves) {
    float2 s[4];
    vec v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int k = k0 + u * kHalves;
      const int64_t at = place(min(k, total - 1));
      s[u] = in.stats[at];
      v[u] = *reinterpret_cast<const vec*>(in.sums + at * D + ch);
      if (k >= total) s[u] = make_float2(kNoScore, 0.f);
    }
    float top = ref;
#pragma unroll
    for (int u = 0; u < 4; ++u) top = fmaxf(top, s[u].x);
    const float mine = __builtin_amdgcn_exp2f(ref - top);
    l *= mine;
    y *= mine;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (k0 + u * kHalves >= total) continue;
      const float theirs = __builtin_amdgcn_exp2f(s[u].x - top);
      l += s[u].y * theirs;
      y += v[u] * theirs;
    }
    ref = top;
  }
  // the half waves' shares, in their order
  __shared__ float lds_sum[WAVES == 1 ? 1 : kHalves][D], lds_ref[kHalves], lds_l[kHalves];
  if constexpr (WAVES == 1) {
    const float other = __shfl_xor(ref, 32, 64), top = fmaxf(ref, other), mine = __builtin_amdgcn_exp2f(ref - top);
    l *= mine;
    l += __shfl_xor(l, 32, 64);
#pragma unroll
    for (int e = 0; e < C; ++e) {
      y[e] *= mine;
      y[e] += __shfl_xor(y[e], 32, 64);
    }
  } else {
    if ((lane & 31) == 0) { lds_ref[half] = ref; lds_l[half] = l; }
#pragma unroll
    for (int e = 0; e < C; ++e) lds_sum[half][ch + e] = y[e];
    __syncthreads();
    if (wave != 0) return;
    float top = kNoScore;
    for (int h = 0; h < kHalves; ++h) top = fmaxf(top, lds_ref[h]);
    l = 0.f;
    y = vec{};
    for (int h = 0; h < kHalves; ++h) {
      const float theirs = __builtin_amdgcn_exp2f(lds_ref[h] - top);
      l += lds_l[h] * theirs;
#pragma unroll
      for (int e = 0; e < C; ++e) y[e] += lds_sum[h][ch + e] * theirs;
    }
  }
  if (lane >= 32) return;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  _Float16* to = static_cast<_Float16*>(a.y) + row * a.ldy + head * D + ch;
#pragma unroll
  for (int e = 0; e < C; e += 2)
    *reinterpret_cast<half2v*>(to + e) = answer(y[e] * inv, y[e + 1] * inv);
}

template <int D, bool W> static void launch_join(const AttendArgs& a, const AttendPlan& p, hipStream_t st) {
  const int64_t outputs = static_cast<int64_t>(a.M) * a.q_heads, blocks = p.parts > 16 ? outputs : (outputs + kWaves - 1) / kWaves;
  const dim3 join(static_cast<unsigned>(blocks < kJoinRow ? blocks : kJoinRow), static_cast<unsigned>((blocks + kJoinRow - 1) / kJoinRow)), block(64 * kWaves);
  if (p.parts > 16) attend_join_kernel<D, 4, W><<<join, block, 0, st>>>(a, p);
  else attend_join_kernel<D, 1, W><<<join, block, 0, st>>>(a, p);
}

// The launches of a call without a prefix apart.
template <int D, int BITS, bool W> static void launch_own(const AttendArgs& a, const AttendPlan& p, hipStream_t st) {
  const AttendLaunch& n = p.own;
  const dim3 grid(static_cast<unsigned>(n.grid)), block(64 * kWaves);
  if (n.row_tiles == 0 && n.alone) attend_rows_kernel<D, BITS, 1, W><<<grid, block, 0, st>>>(a, n, p.parts);
  else if (n.row_tiles == 0) attend_rows_kernel<D, BITS, 4, W><<<grid, block, 0, st>>>(a, n, p.parts);
  else if (n.row_tiles == 1) attend_tile_kernel<D, BITS, 1, W><<<grid, block, 0, st>>>(a, n, p.parts);
  else attend_tile_kernel<D, BITS, 2, W><<<grid, block, 0, st>>>(a, n, p.parts);
}

}  // namespace rosaq
