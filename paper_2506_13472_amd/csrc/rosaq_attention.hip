// Attention over the quantised cache: the launches.  The kernels are in rosaq_attend.h; those of calls with a window are instantiated in
// rosaq_attention_window.hip.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <string>

#include "rosaq_attend.h"

namespace rosaq {

// Both halves of a call whose prefix is apart, beside each other: the prefix for all rows, and behind those workgroups the sequences'
// own tokens, of which there are too few to keep the card busy.
template <int D, int BITS, int RT, int SPLIT>
__global__ __launch_bounds__(64 * kWaves, RT == 1 && BITS == 4 ? 3 : 2) void attend_both_kernel(AttendArgs a, AttendLaunch prefix, AttendLaunch own, int parts) {
  __shared__ union { StageLds<D> stages[stage_buffers(RT)]; RowsLds<D> rows; } lds;
  if (blockIdx.x < prefix.grid) attend_tile<D, BITS, RT>(a, prefix, parts, blockIdx.x, lds.stages);
  else attend_rows<D, BITS, SPLIT>(a, own, parts, blockIdx.x - static_cast<int>(prefix.grid), lds.rows);
}

static int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// The fewest parts from `parts` on whose workgroups leave the compute units about evenly busy, the fullest with up to 1.15 times the average (`parts` themselves may
// leave it with `bearable` hundredths); `parts` where none do.
static int64_t even_parts(int64_t groups, int64_t steps, int64_t parts, int64_t most, int64_t bearable) {
  for (int64_t p = parts; p <= most; ++p) {
    const int64_t workgroups = groups * ceil_div(steps, ceil_div(steps, p));
    if (100 * 256 * ceil_div(workgroups, 256) <= (p == parts ? bearable : 115) * workgroups) return p;
  }
  return parts;
}

// Shapes a launch over `rows` rows and `tokens` tokens of each of `seqs` sequences.
//
// Kernel: up to 16 rows are one tile of attend_rows.  From 17 to 32 both are as fast (us, attend_tile / attend_rows: 8 sequences of up to 8192 tokens x 8
// kv heads, 32 rows, 4 bits 41 / 38; 32 of up to 1024, 8 bits 28 / 29; one of 32768 27 / 30), at 48 rows attend_tile is (43 / 45, 33 / 48, 30 / 49).
// Parts: enough workgroups for all compute units, eight steps or two stages in each at least.  More of them balance ragged lengths better and cost more
// partial results: 16 sequences of 8192 to 32768 tokens in 1536 / 2048 / 6144 workgroups 96 / 89 / 93 us; a chunk of 3 x 509 rows x 32 heads,
// 384 workgroups as they are 239 us, in 2, 3, 4 and 5 parts 292, 240, 286 and 224: which is best goes by the lengths, which the host does not
// know.  A prefix under 64 rows, 32 heads: 256 / 512 workgroups 27.6 / 32.2 us beside the sequences' own; under 384 rows, 8 heads, 16389 tokens:
// 256 / 384 / 512 74.9 / 69.9 / 66.8.
// With a window sequences that are longer take about the same number of steps, and one round of workgroups, as many as are resident at a time (512 or 768), is better than
// many: in 2048 / 768 / 512 workgroups 16 x (8 x 4) rows, window 4096, 4 bits 30.1 / 24.1 / 24.9 us, 128 x (8 x 4) heads of 64, window 1024 32.1 / 25.0 / 24.6;
// 8 bits, one row of 32 heads, window 8191 23.0 / 22.9 / 21.3, 32 x (8 x 4), window 2048 37.7 / 37.7 / 35.8.
// Where one round leaves some compute units with far more than others, more parts even that out: us in one round / as even_parts has it, 4 and 8 bits, 264
// workgroups a part, window 4096 45.0 / 41.5 and 78.9 / 68.0, 3000 35.4 / 32.8 and 58.9 / 52.8, 520 of them 81.5 / 75.7 and 138 / 124, 62.4 / 59.0 and 101 / 91.5,
// 776 116 / 106 and 179 / 173, 85.2 / 81.1 and 139 / 135.  In few steps they do not pay (520, window 1200 27.8 / 30.6 and 42.8 / 44.8, 2048 42.0 / 42.8 and 76.2 /
// 71.2, 2500 52.7 / 51.1 and 89.9 / 81.9; 392, 2048 32.2 / 33.2 and 48.4 / 51.7), and nor where two workgroups are resident a compute unit and it has one or two
// (8 bits, 392, window 4096 91.7 / 92.8, 3000 64.0 / 67.2; with 4 bits 61.5 / 58.7, 46.3 / 43.1).
// Under a window near max_kv it depends on the lengths, which are not known here: 128 workgroups a part in one round / in 2048, 4 and 8 bits, lengths of 1000 to
// 32768 under a window of 29491 93.4 / 81.0 and 123 / 119, under one of 21000 75.6 / 73.5 and 105 / 108, all of 4200 under 4096 23.1 / 28.0 and 30.2 / 38.3.
// A few steps are better left whole, as two or three parts save less than the launch that joins them: us in parts / whole, 16 x (8 x 4) rows, window 450
// 11.2 / 8.5, 900 14.0 / 13.0 (8 bits 15.3 / 13.3), 1024 13.9 / 14.3 (15.6 / 14.6), 1500 16.0 / 18.4; 32 x (8 x 4), 1024 17.6 / 15.0 (20.9 / 17.1); with fewer
// workgroups parts are worth more: 4 x (8 x 4), window 512 9.6 / 8.9, 640 10.1 / 9.7, 768 9.7 / 10.6.
// Waves alone: where there are 2048 tiles of up to 16 steps (64 x 32 heads, us together / alone: 256 tokens 20.6 / 19.3, 512 34.2 / 32.3, 1024
// 52.5 / 54.8).
static AttendLaunch shape_launch(const AttendArgs& a, int over, int64_t rows, int64_t tokens_prefix, int64_t tokens_own, int64_t seqs) {
  AttendLaunch n;
  n.over = over;
  n.row_tiles = rows <= kRows && over != kPrefix ? 0 : (rows <= 64 ? 1 : 2);
  n.tiles = static_cast<int>(ceil_div(rows, n.row_tiles ? 16 * n.row_tiles * kWaves : kRows));
  const int step = n.row_tiles ? kStage : kStep;
  const int64_t everything = std::max<int64_t>(1, ceil_div(tokens_prefix, step) + ceil_div(tokens_own, step));
  int64_t all = everything;
  if (a.window) {
    // the sinks, and from the step that the first row's window begins in to the last of a tile's rows
    const int64_t tile_rows = n.row_tiles ? 16 * n.row_tiles * kWaves : kRows;
    const int64_t apart = std::min<int64_t>(ceil_div(tile_rows - 1, a.group), a.max_rows - 1);
    all = std::min<int64_t>(all, ceil_div(a.sinks, step) + ceil_div(static_cast<int64_t>(a.window) + apart + step - 1, step));
  }
  const bool narrow = all < everything;      // a window over everything takes the parts, and so adds in the order, of a call without one
  const int64_t pairs = seqs * a.cache.kv_heads, groups = pairs * n.tiles;
  const int64_t resident = 256 * (a.dim == 128 && a.bits == 8 ? 2 : 3);      // workgroups of attend_rows, by its registers
  const int64_t fill = n.row_tiles == 0 ? (narrow ? resident : 2048) : (n.row_tiles == 1 && over == kPrefix ? 256 : 512);
  const bool whole = narrow && (all < 20 || (all < 36 && groups >= 96));
  const int64_t most = std::max<int64_t>(1, n.row_tiles ? all / 2 : (whole ? 1 : all / 8));
  int64_t parts = std::clamp<int64_t>(fill / groups, 1, most);
  if (narrow && n.row_tiles == 0 && all >= 72) parts = even_parts(groups, all, parts, most, resident == 512 ? 131 : 115);
  n.steps = static_cast<int>(ceil_div(all, parts));
  n.parts = static_cast<int>(ceil_div(all, n.steps));
  n.alone = n.row_tiles == 0 && groups * n.parts >= 2048 && n.steps <= 16;
  n.by_xcd = !n.alone && pairs >= 8 && (pairs % 8 == 0 || pairs >= 64);
  n.grid = (n.by_xcd ? ceil_div(pairs, 8) * 8 : pairs) * n.tiles * n.parts;
  if (n.alone) n.grid = ceil_div(n.grid, kWaves);
  return n;
}

// Whether the prefix is computed for all sequences at once, apart from their own tokens: where it saves enough steps of rereading it
// to pay for the partial results and the launch that joins them.  us, with every sequence / apart, own tokens up to 256:
//   64 sequences x 32 heads, 4 bits: prefix of 64 tokens 19.9 / 21.0, 128 22.8 / 22.1, 512 40.2 / 24.6
//   16 x 8 kv heads x 4, 8 bits: 512 tokens 12.5 / 12.6, 1024 15.5 / 13.5, 2048 21.3 / 14.2
//   4 x 32, 4 bits: 512 11.5 / 11.4, 2048 17.9 / 16.3;  2 x 8 x 4: 4096 12.0 / 12.4;  32 x 4 rows x 8 x 4: 512 18.3 / 20.1
// Rows that need more than one tile fill the matrix cores without their neighbours (16 x 12 rows x 8 x 4, 1024: 25.5 / 37.6).
static bool prefix_apart(const AttendArgs& a) {
  if (a.prefix_len == 0 || a.max_rows * static_cast<int64_t>(a.group) > kRows) return false;
  const int64_t saved = static_cast<int64_t>(a.seqs - 1) * a.cache.kv_heads * ceil_div(a.prefix_len, kStep);
  return saved >= 3000 + static_cast<int64_t>(a.M) * a.q_heads;
}

AttendPlan plan_attention(const AttendArgs& a) {
  AttendPlan p;
  const int64_t rows = static_cast<int64_t>(a.max_rows) * a.group;
  const bool apart = prefix_apart(a);
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

template <int D, int BITS, int RT> static void launch_both(const AttendArgs& a, const AttendPlan& p, hipStream_t st) {
  const dim3 grid(static_cast<unsigned>(p.prefix.grid + p.own.grid)), block(64 * kWaves);
  if (p.own.alone) attend_both_kernel<D, BITS, RT, 1><<<grid, block, 0, st>>>(a, p.prefix, p.own, p.parts);
  else attend_both_kernel<D, BITS, RT, 4><<<grid, block, 0, st>>>(a, p.prefix, p.own, p.parts);
}

template <int D, int BITS> static void run(const AttendArgs& a, const AttendPlan& p, hipStream_t st) {
  if (p.prefix.grid && p.prefix.row_tiles == 1) launch_both<D, BITS, 1>(a, p, st);
  else if (p.prefix.grid) launch_both<D, BITS, 2>(a, p, st);
  else launch_own<D, BITS, false>(a, p, st);
  if (p.parts > 1) launch_join<D, false>(a, p, st);
}

int launch_attention(const AttendArgs& a, const AttendPlan& p, void* stream) {
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (a.window) launch_attention_window(a, p, stream);
  else if (a.dim == 128) a.bits == 4 ? run<128, 4>(a, p, st) : run<128, 8>(a, p, st);
  else a.bits == 4 ? run<64, 4>(a, p, st) : run<64, 8>(a, p, st);
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return ROSAQ_OK;
  try { set_error(std::string("attention: ") + hipGetErrorString(e)); } catch (...) {}     // no memory for the text
  return ROSAQ_ERR_HIP;
}

}  // namespace rosaq
