// C ABI of the attention between the q/k/v projections and the output projection: argument checks of the rotary positions,
// the quantised cache and the attention over it.  No arithmetic of the method happens here.
#include <climits>
#include <cmath>
#include <string>

#include "rosaq_attention.h"
#include "rosaq_checks.h"

namespace rosaq {

// Rows x heads: what the launches of rotary positions and cache, with 16 of them a workgroup of 256 threads, number in 32 bits.
constexpr int64_t kMaxTasks = int64_t{1} << 27;
constexpr int64_t kMaxGrid = int64_t{1} << 24;     // workgroups of 256 threads, of which a dimension of a grid has fewer than 2^32
constexpr int kMaxSequences = 1 << 20;

static int check_heads(int32_t heads, int32_t head_dim) {
  if (head_dim != 64 && head_dim != 128) return fail(ROSAQ_ERR_ARG, "head_dim must be 64 or 128");
  if (heads < 1 || heads > 4096) return fail(ROSAQ_ERR_SHAPE, "the number of heads must be in [1, 4096]");
  return ROSAQ_OK;
}

static int log2_of(int v) {
  int s = 0;
  while ((1 << s) < v) ++s;
  return s;
}

// Bytes of a cache, or -1 where its shape is wrong (the error text is set).
static int64_t cache_bytes(int32_t kv_heads, int32_t head_dim, int32_t bits, int32_t page_tokens, int32_t num_pages, int* rc) {
  *rc = check_heads(kv_heads, head_dim);
  if (*rc != ROSAQ_OK) return -1;
  if (bits != 4 && bits != 8) *rc = fail(ROSAQ_ERR_ARG, "bits of a cache must be 4 or 8");
  else if (page_tokens < 16 || page_tokens > 4096 || (page_tokens & (page_tokens - 1)))
    *rc = fail(ROSAQ_ERR_SHAPE, "page_tokens must be a power of two in [16, 4096]");
  else if (num_pages < 1) *rc = fail(ROSAQ_ERR_SHAPE, "num_pages must be at least 1");
  if (*rc != ROSAQ_OK) return -1;
  const int64_t page = static_cast<int64_t>(kv_heads) * (page_tokens / kCacheBlock) * cache_record_bytes(head_dim, bits);   // < 2^34
  if (num_pages > (int64_t{1} << 46) / page) {
    *rc = fail(ROSAQ_ERR_SHAPE, "a cache of more than 2^46 bytes");
    return -1;
  }
  return page * num_pages;
}

static int check_cache(const rosaq_cache* c, CacheDev* out) {
  if (!c) return fail(ROSAQ_ERR_NULL, "cache is NULL");
  int rc;
  const int64_t need = cache_bytes(c->kv_heads, c->head_dim, c->bits, c->page_tokens, c->num_pages, &rc);
  if (need < 0) return rc;
  if (!c->data) return fail(ROSAQ_ERR_NULL, "cache data is NULL");
  if (misaligned(c->data, 256)) return fail(ROSAQ_ERR_ALIGN, "cache data must be 256-byte aligned");
  out->base = static_cast<char*>(c->data);
  out->page_bytes = need / c->num_pages;
  out->head_bytes = out->page_bytes / c->kv_heads;
  out->num_pages = c->num_pages;
  out->kv_heads = c->kv_heads;
  out->page_shift = log2_of(c->page_tokens);
  return ROSAQ_OK;
}

// One fp16 matrix of M rows of heads.
static int check_matrix(const char* name, const void* p, int64_t ld, int64_t width) {
  try {
    if (!p) { set_error(std::string(name) + " is NULL"); return ROSAQ_ERR_NULL; }
    if (ld < width) { set_error(std::string(name) + ": leading dimension smaller than width"); return ROSAQ_ERR_SHAPE; }
    if (ld > (int64_t{1} << 40)) { set_error(std::string(name) + ": leading dimension above 2^40"); return ROSAQ_ERR_SHAPE; }
    if (misaligned(p, 16) || ld % 8) {
      set_error(std::string(name) + " must be 16-byte aligned and its leading dimension a multiple of 8");
      return ROSAQ_ERR_ALIGN;
    }
  } catch (...) { return ROSAQ_ERR_NOMEM; }
  return ROSAQ_OK;
}

static int check_rows(int32_t M, int64_t heads) {
  if (M < 1) return fail(ROSAQ_ERR_SHAPE, "M must be at least 1");
  if (static_cast<int64_t>(M) * heads > kMaxTasks) return fail(ROSAQ_ERR_SHAPE, "M x heads above 2^27: split the call");
  return ROSAQ_OK;
}

static int check_rope(const rosaq_rope_angles* r, const int32_t* positions, int32_t head_dim, RopeDev* out) {
  if (!r || !r->table || !positions) return fail(ROSAQ_ERR_NULL, "rope, its table or positions is NULL");
  if (r->layout != ROSAQ_ROPE_HALF && r->layout != ROSAQ_ROPE_INTERLEAVED)
    return fail(ROSAQ_ERR_ARG, "layout is not one of ROSAQ_ROPE_*");
  if (r->positions < 1) return fail(ROSAQ_ERR_SHAPE, "the table must have at least one position");
  if (r->rot_dim < 16 || r->rot_dim > head_dim || r->rot_dim % 16)
    return fail(ROSAQ_ERR_SHAPE, "rot_dim must be a multiple of 16 in [16, head_dim]");
  if (misaligned(r->table, 8) || misaligned(positions, 4)) return fail(ROSAQ_ERR_ALIGN, "table must be 8-byte aligned, positions 4-byte");
  *out = RopeDev{static_cast<const float*>(r->table), positions, r->positions, r->rot_dim, r->layout == ROSAQ_ROPE_INTERLEAVED};
  return ROSAQ_OK;
}

// The same of fp16 matrices, in elements.
static bool overlap(const void* x, int64_t ldx, int64_t wx, const void* y, int64_t ldy, int64_t wy, int M) {
  return overlap_bytes(x, 2 * ldx, 2 * wx, y, 2 * ldy, 2 * wy, M);
}
static int check_in_place(const void* x, int64_t ldx, const void* y, int64_t ldy, int M, int64_t width) {
  if (x == y && ldx == ldy) return ROSAQ_OK;
  return overlap(x, ldx, width, y, ldy, width, M) ? fail(ROSAQ_ERR_ARG, "the output overlaps the input without being the same matrix") : ROSAQ_OK;
}

static int check_attention(const rosaq_attention_desc* d, AttendArgs* a, bool pointers) {
  if (!d) return fail(ROSAQ_ERR_NULL, "desc is NULL");
  if (!d->cache) return fail(ROSAQ_ERR_NULL, "cache is NULL");
  rosaq_cache shape = *d->cache;
  if (!pointers && !shape.data) shape.data = reinterpret_cast<void*>(256);     // a question about sizes
  int rc = check_cache(&shape, &a->cache);
  if (rc != ROSAQ_OK) return rc;
  rc = check_heads(d->q_heads, shape.head_dim);
  if (rc != ROSAQ_OK) return rc;
  if (d->q_heads % shape.kv_heads) return fail(ROSAQ_ERR_SHAPE, "q_heads must be a multiple of the cache's kv_heads");
  rc = check_rows(d->M, d->q_heads);
  if (rc != ROSAQ_OK) return rc;
  if (d->sequences < 1 || d->sequences > kMaxSequences) return fail(ROSAQ_ERR_SHAPE, "sequences must be in [1, 2^20]");
  if (d->max_rows < 1 || d->max_rows > d->M) return fail(ROSAQ_ERR_SHAPE, "max_rows must be in [1, M]");
  if (d->max_kv < 0 || d->prefix_len < 0) return fail(ROSAQ_ERR_SHAPE, "max_kv and prefix_len must not be negative");
  if (d->max_kv > (1 << 30) || d->prefix_len > (1 << 30)) return fail(ROSAQ_ERR_SHAPE, "max_kv and prefix_len go up to 2^30");
  if (!(std::fabs(d->scale) <= 0x1p60f)) return fail(ROSAQ_ERR_ARG, "scale must be a number of at most 2^60");
  if (d->causal != 0 && d->causal != 1) return fail(ROSAQ_ERR_ARG, "causal must be 0 or 1");
  if (!pointers || !d->row_start_dev) {
    // without row starts every sequence has one row
    if (pointers && (d->max_rows != 1 || d->M < d->sequences))
      return fail(ROSAQ_ERR_SHAPE, "without row_start_dev every sequence has one row: max_rows 1 and M of at least `sequences`");
  }
  const int64_t width = static_cast<int64_t>(d->q_heads) * shape.head_dim;
  if (pointers) {
    if ((rc = check_matrix("q", d->q_dev, d->ldq, width)) != ROSAQ_OK) return rc;
    if ((rc = check_matrix("y", d->y_dev, d->ldy, width)) != ROSAQ_OK) return rc;
    if (overlap(d->q_dev, d->ldq, width, d->y_dev, d->ldy, width, d->M)) return fail(ROSAQ_ERR_ARG, "y must not overlap q");
    if (!d->kv_len_dev) return fail(ROSAQ_ERR_NULL, "kv_len_dev is NULL");
    if (d->page_stride < 0) return fail(ROSAQ_ERR_SHAPE, "page_stride must not be negative");
    // a table of no columns has no address: no sequence has tokens then
    if (d->max_kv > 0 && d->page_stride > 0 && !d->pages_dev) return fail(ROSAQ_ERR_NULL, "pages_dev is NULL");
    if (d->prefix_len > 0 && !d->prefix_pages_dev) return fail(ROSAQ_ERR_NULL, "prefix_pages_dev is NULL");
    if (misaligned(d->kv_len_dev, 4) || misaligned(d->row_start_dev, 4) || misaligned(d->pages_dev, 4) || misaligned(d->prefix_pages_dev, 4))
      return fail(ROSAQ_ERR_ALIGN, "the integer arrays must be 4-byte aligned");
  }
  a->q = d->q_dev; a->ldq = d->ldq; a->y = d->y_dev; a->ldy = d->ldy;
  a->M = d->M; a->seqs = d->sequences; a->q_heads = d->q_heads; a->group = d->q_heads / shape.kv_heads;
  a->row_start = d->row_start_dev; a->kv_len = d->kv_len_dev;
  a->pages = d->pages_dev; a->page_stride = d->page_stride;
  a->prefix_pages = d->prefix_pages_dev; a->prefix_len = d->prefix_len;
  // a plan for max_kv tokens serves a table cut to the pages that are in use
  const int64_t room = pointers ? static_cast<int64_t>(d->page_stride) * shape.page_tokens : d->max_kv;
  a->max_rows = d->max_rows; a->max_kv = d->max_kv; a->capacity = static_cast<int>(room < d->max_kv ? room : d->max_kv); a->causal = d->causal;
  // The kernels divide by the keys' scales times this.  Below 2^-60 it makes every score 0 to the last bit that counts (|q.k| < 2^40).
  const double scale = static_cast<double>(d->scale) * 1.4426950408889634;
  a->scale_log2 = static_cast<float>(std::fabs(scale) < 0x1p-60 ? 0x1p-60 : scale);
  a->dim = shape.head_dim; a->bits = shape.bits;
  a->part = nullptr;
  return ROSAQ_OK;
}

static int check_window(const rosaq_attention_desc& d, int32_t window, int32_t sinks, AttendArgs* a) {
  if (window < 1 || window > (1 << 30)) return fail(ROSAQ_ERR_SHAPE, "window must be in [1, 2^30]");
  if (sinks < 0 || sinks > (1 << 30)) return fail(ROSAQ_ERR_SHAPE, "sinks must be in [0, 2^30]");
  if (d.causal != 1) return fail(ROSAQ_ERR_ARG, "a window is counted back from a row's own position: causal must be 1");
  if (d.prefix_len != 0) return fail(ROSAQ_ERR_ARG, "with a window a shared prefix is part of every sequence's pages: prefix_len must be 0");
  a->window = window;
  a->sinks = sinks;
  return ROSAQ_OK;
}

static size_t workspace_of(const AttendArgs& a) {
  const AttendPlan p = plan_attention(a);
  return p.ws_bytes < 256 ? 256 : p.ws_bytes;
}

static int attend(AttendArgs& a, void* ws_dev, size_t ws_bytes, void* hip_stream) {
  const AttendPlan p = plan_attention(a);
  if (p.own.grid + p.prefix.grid >= kMaxGrid) return fail(ROSAQ_ERR_SHAPE, "sequences x max_rows x q_heads too large: split the call");
  if (p.ws_bytes) {
    if (!ws_dev || ws_bytes < p.ws_bytes) return fail(ROSAQ_ERR_WORKSPACE, "workspace missing or too small");
    if (misaligned(ws_dev, 256)) return fail(ROSAQ_ERR_ALIGN, "workspace must be 256-byte aligned");
    a.part = static_cast<float*>(ws_dev);
  }
  return launch_attention(a, p, hip_stream);
}

}  // namespace rosaq

using namespace rosaq;

extern "C" {

size_t rosaq_cache_bytes(int32_t kv_heads, int32_t head_dim, int32_t bits, int32_t page_tokens, int32_t num_pages) {
  int rc;
  const int64_t n = cache_bytes(kv_heads, head_dim, bits, page_tokens, num_pages, &rc);
  return n < 0 ? 0 : static_cast<size_t>(n);
}

int rosaq_rope_table(const rosaq_rope_desc* desc, void* table_dev, int32_t positions, void* hip_stream) {
  if (!desc || !table_dev) return fail(ROSAQ_ERR_NULL, "desc or table_dev is NULL");
  if (desc->rot_dim < 16 || desc->rot_dim > 128 || desc->rot_dim % 16)
    return fail(ROSAQ_ERR_SHAPE, "rot_dim must be a multiple of 16 in [16, 128]");
  if (positions < 1 || positions > (1 << 24)) return fail(ROSAQ_ERR_SHAPE, "positions must be in [1, 2^24]");
  if (!(desc->base > 1.0) || !std::isfinite(desc->base)) return fail(ROSAQ_ERR_ARG, "base must be finite and above 1");
  if (desc->scaling < ROSAQ_ROPE_SCALE_NONE || desc->scaling > ROSAQ_ROPE_SCALE_WAVELENGTH)
    return fail(ROSAQ_ERR_ARG, "scaling is not one of ROSAQ_ROPE_SCALE_*");
  if (desc->scaling != ROSAQ_ROPE_SCALE_NONE && (!(desc->factor > 0.0) || !std::isfinite(desc->factor)))
    return fail(ROSAQ_ERR_ARG, "factor must be finite and positive");
  if (desc->scaling == ROSAQ_ROPE_SCALE_WAVELENGTH &&
      (!(desc->low >= 0.0) || !(desc->high > desc->low) || !std::isfinite(desc->high) || !(desc->trained_positions > 0.0) ||
       !std::isfinite(desc->trained_positions)))
    return fail(ROSAQ_ERR_ARG, "scaling by wavelength needs 0 <= low < high and trained_positions > 0");
  if (misaligned(table_dev, 8)) return fail(ROSAQ_ERR_ALIGN, "table must be 8-byte aligned");
  return launch_rope_table(*desc, static_cast<float*>(table_dev), positions, hip_stream);
}

int rosaq_rope(const rosaq_rope_angles* rope, const int32_t* positions_dev, const void* x_dev, int32_t M, int64_t ldx,
               int32_t heads, int32_t head_dim, void* y_dev, int64_t ldy, void* hip_stream) {
  RopeArgs a{};
  int rc = check_heads(heads, head_dim);
  if (rc == ROSAQ_OK) rc = check_rows(M, heads);
  if (rc == ROSAQ_OK) rc = check_rope(rope, positions_dev, head_dim, &a.rope);
  const int64_t width = static_cast<int64_t>(heads) * head_dim;
  if (rc == ROSAQ_OK) rc = check_matrix("x", x_dev, ldx, width);
  if (rc == ROSAQ_OK) rc = check_matrix("y", y_dev, ldy, width);
  if (rc == ROSAQ_OK) rc = check_in_place(x_dev, ldx, y_dev, ldy, M, width);
  if (rc != ROSAQ_OK) return rc;
  a.x = x_dev; a.ldx = ldx; a.y = y_dev; a.ldy = ldy; a.M = M; a.heads = heads; a.dim = head_dim;
  return launch_rope(a, hip_stream);
}

int rosaq_cache_append(const rosaq_cache* cache, const int64_t* slots_dev, int32_t M, const void* k_dev, int64_t ldk,
                       const void* v_dev, int64_t ldv, const rosaq_rope_angles* rope, const int32_t* positions_dev,
                       const void* q_dev, int64_t ldq, int32_t q_heads, void* q_out_dev, int64_t ldq_out, void* hip_stream) {
  AppendArgs a{};
  int rc = check_cache(cache, &a.cache);
  if (rc != ROSAQ_OK) return rc;
  if (!slots_dev) return fail(ROSAQ_ERR_NULL, "slots_dev is NULL");
  if (misaligned(slots_dev, 8)) return fail(ROSAQ_ERR_ALIGN, "slots_dev must be 8-byte aligned");
  const int64_t width = static_cast<int64_t>(cache->kv_heads) * cache->head_dim;
  if ((rc = check_matrix("k", k_dev, ldk, width)) != ROSAQ_OK || (rc = check_matrix("v", v_dev, ldv, width)) != ROSAQ_OK) return rc;
  int64_t heads = 2 * static_cast<int64_t>(cache->kv_heads);
  if (rope && (rc = check_rope(rope, positions_dev, cache->head_dim, &a.rope)) != ROSAQ_OK) return rc;
  if (q_dev) {
    if (!rope) return fail(ROSAQ_ERR_NULL, "q is only read to be rotated: rope is NULL");
    if ((rc = check_heads(q_heads, cache->head_dim)) != ROSAQ_OK) return rc;
    const int64_t q_width = static_cast<int64_t>(q_heads) * cache->head_dim;
    if ((rc = check_matrix("q", q_dev, ldq, q_width)) != ROSAQ_OK || (rc = check_matrix("q_out", q_out_dev, ldq_out, q_width)) != ROSAQ_OK)
      return rc;
    heads += q_heads;
  }
  if ((rc = check_rows(M, heads)) != ROSAQ_OK) return rc;
  if (q_dev) {
    const int64_t q_width = static_cast<int64_t>(q_heads) * cache->head_dim;
    if ((rc = check_in_place(q_dev, ldq, q_out_dev, ldq_out, M, q_width)) != ROSAQ_OK) return rc;
    if (overlap(k_dev, ldk, width, q_out_dev, ldq_out, q_width, M) || overlap(v_dev, ldv, width, q_out_dev, ldq_out, q_width, M))
      return fail(ROSAQ_ERR_ARG, "q_out must not overlap k or v");
  }
  a.slots = slots_dev; a.M = M; a.k = k_dev; a.ldk = ldk; a.v = v_dev; a.ldv = ldv;
  a.q = q_dev; a.ldq = ldq; a.q_heads = q_dev ? q_heads : 0; a.q_out = q_out_dev; a.ldq_out = ldq_out;
  a.dim = cache->head_dim; a.bits = cache->bits;
  return launch_cache_append(a, hip_stream);
}

int rosaq_cache_read(const rosaq_cache* cache, const int64_t* slots_dev, int32_t M, void* k_dev, int64_t ldk, void* v_dev,
                     int64_t ldv, void* hip_stream) {
  ReadArgs a{};
  int rc = check_cache(cache, &a.cache);
  if (rc != ROSAQ_OK) return rc;
  if (!slots_dev || (!k_dev && !v_dev)) return fail(ROSAQ_ERR_NULL, "slots_dev, or both k_dev and v_dev, are NULL");
  if (misaligned(slots_dev, 8)) return fail(ROSAQ_ERR_ALIGN, "slots_dev must be 8-byte aligned");
  const int64_t width = static_cast<int64_t>(cache->kv_heads) * cache->head_dim;
  if ((k_dev && (rc = check_matrix("k", k_dev, ldk, width)) != ROSAQ_OK) || (v_dev && (rc = check_matrix("v", v_dev, ldv, width)) != ROSAQ_OK))
    return rc;
  if ((rc = check_rows(M, 2 * static_cast<int64_t>(cache->kv_heads))) != ROSAQ_OK) return rc;
  if (k_dev && v_dev && overlap(k_dev, ldk, width, v_dev, ldv, width, M)) return fail(ROSAQ_ERR_ARG, "k and v must not overlap");
  a.slots = slots_dev; a.M = M; a.k = k_dev; a.ldk = ldk; a.v = v_dev; a.ldv = ldv; a.dim = cache->head_dim; a.bits = cache->bits;
  return launch_cache_read(a, hip_stream);
}

size_t rosaq_workspace_bytes_attention(const rosaq_attention_desc* desc) {
  AttendArgs a{};
  return check_attention(desc, &a, false) != ROSAQ_OK ? 0 : workspace_of(a);
}

int rosaq_attention(const rosaq_attention_desc* desc, void* ws_dev, size_t ws_bytes, void* hip_stream) {
  AttendArgs a{};
  const int rc = check_attention(desc, &a, true);
  return rc != ROSAQ_OK ? rc : attend(a, ws_dev, ws_bytes, hip_stream);
}

size_t rosaq_workspace_bytes_attention_window(const rosaq_attention_desc* desc, int32_t window, int32_t sinks) {
  AttendArgs a{};
  return check_attention(desc, &a, false) != ROSAQ_OK || check_window(*desc, window, sinks, &a) != ROSAQ_OK ? 0 : workspace_of(a);
}

int rosaq_attention_window(const rosaq_attention_desc* desc, int32_t window, int32_t sinks, void* ws_dev, size_t ws_bytes, void* hip_stream) {
  AttendArgs a{};
  int rc = check_attention(desc, &a, true);
  if (rc == ROSAQ_OK) rc = check_window(*desc, window, sinks, &a);
  return rc != ROSAQ_OK ? rc : attend(a, ws_dev, ws_bytes, hip_stream);
}

}  // extern "C"
