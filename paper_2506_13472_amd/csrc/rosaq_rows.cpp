// C ABI of the operators over whole rows: argument checks of the norm and of the log probabilities.  No arithmetic of the method happens here.
#include "rosaq_rows.h"

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
  a->weight = d->weight_dev;
  a->y = d->y_dev; a->ldy = d->ldy;
  a->codes = d->codes_dev; a->ld_codes = d->ld_codes; a->scales = d->scales_dev;
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

}  // extern "C"
