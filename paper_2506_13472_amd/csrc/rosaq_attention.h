// The quantised cache of keys and values: its layout, shared by the kernels that write, read and attend, and what the
// attention's launches are told.
#pragma once
#include <cstddef>
#include <cstdint>

#include "rosaq.h"

#ifdef __HIPCC__
#define ROSAQ_BOTH __host__ __device__
#else
#define ROSAQ_BOTH
#endif

namespace rosaq {

// A page holds, head after head, records of 16 tokens; a record is
//   [keys | values | 16 dwords of the keys | 16 dwords of the values],   dword = scale | zero << 16 (both fp16) of a token,
// with the codes where a wave's lanes want them for v_mfma_f32_16x16x32_f16 (lane = 16 g + r):
//   keys    lane (r, g) multiplies token r's channels g * D/4 .. + D/4 - 1: in planes of up to 16 bytes a lane,
//           [plane][token][g][bytes], channels ascending (4-bit codes: low nibble first), so that a load of a wave is one run
//           of 1 KiB.  A token's codes of one plane are contiguous.
//   values  lane (r, g) multiplies, for tokens 4 g .. 4 g + 3, channels r * D/16 .. + D/16 - 1: units of 16 bits (4 channels of
//           4 bits, 2 of 8), the four tokens' units side by side, so that a dword holds the same channels of two tokens and
//           one mask makes an fp16 pair along the contraction: [plane][g][r][unit of the plane][token - 4 g].
// Both are permutations in which a token owns whole 16-bit words: one token is written without reading any other's.
constexpr int kCacheBlock = 16;                     // tokens of a record
constexpr int kCacheParams = 2 * kCacheBlock * 4;   // bytes of scales and zeros behind the codes

ROSAQ_BOTH constexpr int cache_code_bytes(int dim, int bits) { return kCacheBlock * dim * bits / 8; }
ROSAQ_BOTH constexpr int cache_record_bytes(int dim, int bits) { return 2 * cache_code_bytes(dim, bits) + kCacheParams; }

// What the kernels are told of a cache.
struct CacheDev {
  char* base;
  int64_t page_bytes, head_bytes;   // a page, and one head's records in it
  int num_pages, kv_heads;
  int page_shift;                   // log2 of the tokens of a page
};

struct RopeDev {
  const float* table;       // [positions][rot / 2] pairs (cos, sin); null: no rotation
  const int32_t* at;        // position of every row
  int positions, rot, interleaved;
};

struct AppendArgs {
  CacheDev cache;
  const int64_t* slots;
  int M;
  const void* k; int64_t ldk;
  const void* v; int64_t ldv;
  RopeDev rope;
  const void* q; int64_t ldq; int q_heads;      // q null: keys and values only
  void* q_out; int64_t ldq_out;
  int dim, bits;
};
int launch_cache_append(const AppendArgs& a, void* stream);
struct ReadArgs {
  CacheDev cache;
  const int64_t* slots;
  int M;
  void* k; int64_t ldk;     // null: not wanted
  void* v; int64_t ldv;
  int dim, bits;
};
int launch_cache_read(const ReadArgs& a, void* stream);
struct RopeArgs {
  RopeDev rope;
  const void* x; int64_t ldx;
  void* y; int64_t ldy;
  int M, heads, dim;
};
int launch_rope(const RopeArgs& a, void* stream);
int launch_rope_table(const rosaq_rope_desc& d, float* table, int32_t positions, void* stream);

struct AttendArgs {
  CacheDev cache;
  const void* q; int64_t ldq;
  void* y; int64_t ldy;
  int M, seqs, q_heads, group;              // group: query heads of one kv head
  const int32_t* row_start;                 // null: one row each
  const int32_t* kv_len;
  const int32_t* pages; int64_t page_stride;
  const int32_t* prefix_pages; int prefix_len;
  int max_rows, max_kv;
  int capacity;                             // tokens of a sequence that are looked at: of max_kv, those that `pages` has room for
  int causal;
  int window, sinks;                        // window 0: none
  float scale_log2;                         // scale * log2(e)
  int dim, bits;
  float* part;                              // partial results (AttendPlan::parts > 1)
};
// One launch of a call: the rows of every sequence over their own tokens, behind the prefix or not, or all rows of the call
// over the prefix.
enum AttendOver { kOwn, kPrefixAndOwn, kPrefix };
struct AttendLaunch {
  int over = kPrefixAndOwn;
  int row_tiles = 0;        // 16-row tiles of a wave, 0: the kernel for up to 16 rows
  int tiles = 1;            // workgroups that share the rows of a sequence and kv head
  int steps = 0, parts = 1; // steps of kStep or kStage tokens that a workgroup takes; workgroups that share all of them
  int first_part = 0;       // number of the first of them among the parts of a row
  int alone = 0;            // up to 16 rows: a wave takes all steps of its part, four of them a workgroup
  int by_xcd = 0;           // workgroups of one sequence and kv head on one XCD
  int64_t grid = 0;         // workgroups
};
// How a call runs.  Every row is computed in own.parts (+ prefix.parts) parts; one alone is stored directly, more go through
// the workspace and are joined by another launch.
struct AttendPlan {
  AttendLaunch own, prefix; // prefix.grid 0: not apart
  int parts = 1;            // of all launches
  size_t ws_bytes = 0;
};
AttendPlan plan_attention(const AttendArgs& a);
int launch_attention(const AttendArgs& a, const AttendPlan& plan, void* stream);
void launch_attention_window(const AttendArgs& a, const AttendPlan& plan, void* stream);

}  // namespace rosaq
