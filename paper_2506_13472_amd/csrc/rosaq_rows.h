// What the kernels of whole rows are told: the norm in front of the projections, the log probabilities behind the last.
#pragma once
#include <cstddef>
#include <cstdint>

#include "rosaq.h"

namespace rosaq {

constexpr int kNormMaxWidth = 32768;

struct NormArgs {
  int M, D;
  double eps;
  const void* x; int64_t ldx;
  const void* residual; int64_t ld_residual;      // null: none
  void* residual_out; int64_t ld_residual_out;    // null: not wanted
  int residual_f32;
  const void* weight;                             // null: ones
  void* y; int64_t ldy;                           // null: not wanted
  void* codes; int64_t ld_codes; float* scales;   // null: not wanted
};
int launch_rmsnorm(const NormArgs& a, void* stream);

constexpr int kMaxTop = 64, kMaxGiven = 4096, kMaxParts = 8;

struct LogprobArgs {
  int M, V, type;                                 // ROSAQ_F16, _BF16, _F32
  const void* logits; int64_t ld;
  float scale;
  int given; const int64_t* tokens; float* given_out;
  float* entropy;                                 // null: not wanted
  int top; int64_t* top_ids; float* top_out;
  int parts; void* ws;                            // workgroups that share a row; more than one, with room for their results
};
// Workgroups that would best share a row (at most kMaxParts), and the workspace that they take.
int parts_of_logprobs(const LogprobArgs& a);
inline size_t workspace_of_logprobs(const LogprobArgs& a, int parts) {
  return parts == 1 ? 0 : static_cast<size_t>(a.M) * parts * (16 + 8 * static_cast<size_t>(a.top));
}
int launch_logprobs(const LogprobArgs& a, void* stream);

}  // namespace rosaq
