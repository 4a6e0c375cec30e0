// C ABI of the operators over whole rows: argument checks of the norm and of the log probabilities.  No arithmetic of the method happens here.
#include "rosaq_rows.h"

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <string>

#include "rosaq_checks.h"

namespace rosaq {

// A matrix of M rows, in bytes.
struct Matrix {
  const char* name;
  const void* p;
  int64_t ld, width;
  bool same(const Matrix& o) const { return p == o.p && ld == o.ld && width == o.width; }
};

// ld and width in elements of `size` bytes; rows are read in pieces of eight elements.
static int check_matrix(const char* name, const void* p, int64_t ld, int64_t width, int size, Matrix* out) {
  try {
    if (!p) { set_error(std::string(name) + " is NULL"); return ROSAQ_ERR_NULL; }
    if (ld < width) { set_error(std::string(name) + ": leading dimension smaller than width"); return ROSAQ_ERR_SHAPE; }
    if (ld > (int64_t{1} << 40)) { set_error(std::string(name) + ": leading dimension above 2^40"); return ROSAQ_ERR_SHAPE; }
    const int align = size == 1 ? 8 : 16;
    if (misaligned(p, align) || ld * size % align) {
      set_error(std::string(name) + ": base and rows must be " + std::to_string(align) + "-byte aligned");
      return ROSAQ_ERR_ALIGN;
    }
  } catch (...) { return ROSAQ_ERR_NOMEM; }
  *out = Matrix{name, p, ld * size, width * size};
  return ROSAQ_OK;
}

static bool overlap(const Matrix& a, const Matrix& b, int M) { return overlap_bytes(a.p, a.ld, a.width, b.p, b.ld, b.width, M); }

static int overlapping(const Matrix& a, const Matrix& b) {
  try { set_error(std::string(a.name) + " must not overlap " + b.name); } catch (...) {}
  return ROSAQ_ERR_ARG;
}

static int check_rmsnorm(const rosaq_rmsnorm_desc* d, NormArgs* a) {
  if (!d) return fail(ROSAQ_ERR_NULL, "desc is NULL");
  if (d->M < 1) return fail(ROSAQ_ERR_SHAPE, "M must be at least 1");
  if (d->D < 8 || d->D > kNormMaxWidth || d->D % 8) return fail(ROSAQ_ERR_SHAPE, "D must be a multiple of 8 in [8, 32768]");
  if (!(d->eps >= 0.0) || !std::isfinite(d->eps)) return fail(ROSAQ_ERR_ARG, "eps must be finite and not negative");
  if (d->residual_type != ROSAQ_F16 && d->residual_type != ROSAQ_F32) return fail(ROSAQ_ERR_ARG, "residual_type must be ROSAQ_F16 or ROSAQ_F32");
  if (d->residual_out_dev && !d->residual_dev) return fail(ROSAQ_ERR_NULL, "residual_out without a residual");
  if (!d->y_dev && !d->codes_dev) return fail(ROSAQ_ERR_NULL, "y and codes are NULL");
  if (!d->codes_dev != !d->scales_dev) return fail(ROSAQ_ERR_NULL, "codes and scales go together");
  const int stream = d->residual_type == ROSAQ_F32 ? 4 : 2;
  Matrix in[3], out[4];
  int ins = 0, outs = 0, rc;
  if ((rc = check_matrix("x", d->x_dev, d->ldx, d->D, 2, &in[ins++])) != ROSAQ_OK) return rc;
  if (d->residual_dev && (rc = check_matrix("residual", d->residual_dev, d->ld_residual, d->D, stream, &in[ins++])) != ROSAQ_OK) return rc;
  if (d->residual_out_dev &&
      (rc = check_matrix("residual_out", d->residual_out_dev, d->ld_residual_out, d->D, stream, &out[outs++])) != ROSAQ_OK) return rc;
  if (d->y_dev && (rc = check_matrix("y", d->y_dev, d->ldy, d->D, 2, &out[outs++])) != ROSAQ_OK) return rc;
  const int whole = outs;                   // of these a row may take the place of the row of an input
  if (d->codes_dev) {
    if ((rc = check_matrix("codes", d->codes_dev, d->ld_codes, d->D, 1, &out[outs++])) != ROSAQ_OK) return rc;
    if (misaligned(d->scales_dev, 4)) return fail(ROSAQ_ERR_ALIGN, "scales must be 4-byte aligned");
    out[outs++] = Matrix{"scales", d->scales_dev, 4, 4};
  }
  if (misaligned(d->weight_dev, 16)) return fail(ROSAQ_ERR_ALIGN, "weight must be 16-byte aligned");
  for (int o = 0; o < outs; ++o) {
    for (int i = 0; i < ins; ++i)
      if (!(o < whole && out[o].same(in[i])) && overlap(out[o], in[i], d->M)) return overlapping(out[o], in[i]);
    for (int i = 0; i < o; ++i)
      if (overlap(out[o], out[i], d->M)) return overlapping(out[o], out[i]);
    // the weights are one row for all: M rows of them, none behind the other
    if (d->weight_dev && overlap(out[o], Matrix{"weight", d->weight_dev, 0, 2 * static_cast<int64_t>(d->D)}, d->M))
      return overlapping(out[o], Matrix{"weight", nullptr, 0, 0});
  }
  a->M = d->M; a->D = d->D; a->eps = d->eps;
  a->x = d->x_dev; a->ldx = d->ldx;
  a->residual = d->residual_dev; a->ld_residual = d->ld_residual;
  a->residual_out = d->residual_out_dev; a->ld_residual_out = d->ld_residual_out;
  a->residual_f32 = d->residual_dev && d->residual_type == ROSAQ_F32;
  // Where the kernel adds eps in fp32 it is kept to that type's normal numbers.  2^-126 is nothing beside the least mean square of fp16 numbers, 2^-48 / D, and
  // keeps a row of zeros from 0 / 0 as a smaller eps does; with the largest one, as with any beyond it, every y is zero but an infinite weight's
  if (!a->residual_f32 && !d->codes_dev && d->eps > 0.0) a->eps = std::clamp<double>(d->eps, FLT_MIN, FLT_MAX);
  a->weight = d->weight_dev;
  a->y = d->y_dev; a->ldy = d->ldy;
  a->codes = d->codes_dev; a->ld_codes = d->ld_codes; a->scales = d->scales_dev;
  return ROSAQ_OK;
}

static int check_logprobs(const rosaq_logprobs_desc* d, LogprobArgs* a, bool pointers) {
  if (!d) return fail(ROSAQ_ERR_NULL, "desc is NULL");
  if (d->M < 1) return fail(ROSAQ_ERR_SHAPE, "M must be at least 1");
  if (d->V < 1 || d->V > (1 << 30)) return fail(ROSAQ_ERR_SHAPE, "V must be in [1, 2^30]");
  if (d->type != ROSAQ_F16 && d->type != ROSAQ_BF16 && d->type != ROSAQ_F32) return fail(ROSAQ_ERR_ARG, "type is not one of ROSAQ_F16, _BF16, _F32");
  if (!(d->scale >= 0x1p-60f && d->scale <= 0x1p60f)) return fail(ROSAQ_ERR_ARG, "scale must be a number of 2^-60 to 2^60");
  if (d->given < 0 || d->given > kMaxGiven) return fail(ROSAQ_ERR_SHAPE, "given must be in [0, 4096]");
  if (d->top < 0 || d->top > kMaxTop || d->top > d->V) return fail(ROSAQ_ERR_SHAPE, "top must be in [0, 64] and at most V");
  a->M = d->M; a->V = d->V; a->type = d->type; a->scale = d->scale; a->given = d->given; a->top = d->top;
  a->parts = 1; a->ws = nullptr;
  if (!pointers) return ROSAQ_OK;
  if (!d->given && !d->top && !d->entropy_dev) return fail(ROSAQ_ERR_NULL, "no output is wanted");
  if (!d->logits_dev || (d->given && (!d->tokens_dev || !d->given_out_dev)) || (d->top && (!d->top_ids_dev || !d->top_out_dev)))
    return fail(ROSAQ_ERR_NULL, "logits, or what `given` or `top` need, is NULL");
  const int size = d->type == ROSAQ_F32 ? 4 : 2;
  if (d->ld < d->V) return fail(ROSAQ_ERR_SHAPE, "logits: leading dimension smaller than width");
  if (d->ld > (int64_t{1} << 40)) return fail(ROSAQ_ERR_SHAPE, "logits: leading dimension above 2^40");
  if (misaligned(d->logits_dev, size) || misaligned(d->tokens_dev, 8) || misaligned(d->given_out_dev, 4) || misaligned(d->entropy_dev, 4) ||
      misaligned(d->top_ids_dev, 8) || misaligned(d->top_out_dev, 4))
    return fail(ROSAQ_ERR_ALIGN, "logits, tokens and outputs must be aligned to their elements");
  const Matrix in[2] = {{"logits", d->logits_dev, d->ld * size, static_cast<int64_t>(d->V) * size},
                        {"tokens", d->given ? d->tokens_dev : nullptr, 8 * d->given, 8 * d->given}};
  const Matrix out[4] = {{"given_out", d->given ? d->given_out_dev : nullptr, 4 * d->given, 4 * d->given},
                         {"entropy", d->entropy_dev, 4, 4},
                         {"top_ids", d->top ? d->top_ids_dev : nullptr, 8 * d->top, 8 * d->top},
                         {"top_out", d->top ? d->top_out_dev : nullptr, 4 * d->top, 4 * d->top}};
  for (int o = 0; o < 4; ++o) {
    if (!out[o].p) continue;
    for (const Matrix& i : in)
      if (i.p && overlap(out[o], i, d->M)) return overlapping(out[o], i);
    for (int i = 0; i < o; ++i)
      if (out[i].p && overlap(out[o], out[i], d->M)) return overlapping(out[o], out[i]);
  }
  a->logits = d->logits_dev; a->ld = d->ld;
  a->tokens = d->tokens_dev; a->given_out = d->given_out_dev;
  a->entropy = d->entropy_dev;
  a->top_ids = d->top_ids_dev; a->top_out = d->top_out_dev;
  return ROSAQ_OK;
}

}  // namespace rosaq

using namespace rosaq;

extern "C" {

int rosaq_rmsnorm(const rosaq_rmsnorm_desc* desc, void* hip_stream) {
  NormArgs a{};
  const int rc = check_rmsnorm(desc, &a);
  return rc != ROSAQ_OK ? rc : launch_rmsnorm(a, hip_stream);
}

size_t rosaq_workspace_bytes_logprobs(const rosaq_logprobs_desc* desc) {
  LogprobArgs a{};
  if (check_logprobs(desc, &a, false) != ROSAQ_OK) return 0;
  return std::max<size_t>(256, workspace_of_logprobs(a, parts_of_logprobs(a)));
}

int rosaq_logprobs(const rosaq_logprobs_desc* desc, void* ws_dev, size_t ws_bytes, void* hip_stream) {
  LogprobArgs a{};
  const int rc = check_logprobs(desc, &a, true);
  if (rc != ROSAQ_OK) return rc;
  if (misaligned(ws_dev, 256)) return fail(ROSAQ_ERR_ALIGN, "workspace must be 256-byte aligned");
  const int parts = parts_of_logprobs(a);
  if (parts > 1 && ws_dev && ws_bytes >= workspace_of_logprobs(a, parts)) {
    a.parts = parts;
    a.ws = ws_dev;
  }
  return launch_logprobs(a, hip_stream);
}

}  // extern "C"
