// C ABI entry points of the operators beside the layers: argument checks, then the launch.
#include "ops.h"

#include <cmath>
#include <limits>

using namespace pgcn;

namespace {

constexpr int64_t kMaxRows = std::numeric_limits<int32_t>::max();

bool aligned16(const void *q) { return ((uintptr_t)q & 15u) == 0; }
size_t elem_size(int32_t dtype) { return dtype == PGCN_BF16 ? 2 : 4; }
bool stride_ok(int32_t dtype, int64_t ld, int64_t cols) {
  return ld >= cols && ld % (dtype == PGCN_BF16 ? 8 : 4) == 0 && ld <= (int64_t(1) << 40);
}

// A buffer's byte range: rows of `cols` elements at a stride of ld.
struct Range {
  const void *p;
  size_t bytes;
};
Range matrix(const void *p, int64_t rows, int64_t cols, int64_t ld, size_t elem) {
  return Range{p, rows > 0 ? ((size_t)(rows - 1) * (size_t)ld + (size_t)cols) * elem : 0};
}
bool overlap(const Range &a, const Range &b) {
  const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
  return a.p && b.p && a.bytes && b.bytes && x < y + b.bytes && y < x + a.bytes;
}
// Whether one of the first `outs` ranges overlaps any other one.
template <size_t n>
bool outputs_overlap(const Range (&r)[n], size_t outs) {
  for (size_t i = 0; i < outs; ++i)
    for (size_t j = 0; j < n; ++j)
      if (j != i && overlap(r[i], r[j])) return true;
  return false;
}

// The stream has to belong to the current device (a null stream does).
int check_stream(hipStream_t s, const char *fn) {
  if (!s) return PGCN_OK;
  int dev = -1;
  PGCN_HIP(hipGetDevice(&dev));
  hipDevice_t own = -1;
  PGCN_HIP(hipStreamGetDevice(s, &own));
  if (own != dev) return set_error(PGCN_EINVAL, std::string(fn) + ": the stream belongs to another device than the current one");
  return PGCN_OK;
}

int check_workspace(const void *ws, size_t bytes, size_t need, const char *fn) {
  if (need == 0) return PGCN_OK;
  if (!ws || bytes < need)
    return set_error(PGCN_EWORKSPACE, std::string(fn) + ": workspace too small, " + std::to_string(need) + " bytes needed");
  PGCN_REQUIRE(aligned16(ws), std::string(fn) + ": workspace must be 16-byte aligned");
  return PGCN_OK;
}

bool top_sizes_ok(int32_t dtype, int64_t rows, int32_t classes, int32_t top) {
  return (dtype == PGCN_F32 || dtype == PGCN_BF16) && rows >= 0 && rows <= kMaxRows && classes >= 1 &&
         classes <= PGCN_MAX_CLASSES && top >= 1 && top <= PGCN_MAX_TOP && top <= classes;
}

int check_top(int32_t dtype, int64_t rows, int32_t classes, int32_t top, int64_t ld, int64_t ld_top, float temperature,
              const char *fn) {
  const std::string f(fn);
  PGCN_REQUIRE(dtype == PGCN_F32 || dtype == PGCN_BF16, f + ": bad dtype");
  PGCN_REQUIRE(rows >= 0 && rows <= kMaxRows, f + ": rows out of range");
  PGCN_REQUIRE(classes >= 1 && classes <= PGCN_MAX_CLASSES, f + ": classes must be in [1, PGCN_MAX_CLASSES]");
  PGCN_REQUIRE(top >= 1 && top <= PGCN_MAX_TOP && top <= classes, f + ": top must be in [1, min(classes, PGCN_MAX_TOP)]");
  PGCN_REQUIRE(stride_ok(dtype, ld, classes), f + ": ld must be >= classes and a multiple of 4 (fp32) or 8 (bf16)");
  PGCN_REQUIRE(ld_top >= top && ld_top <= (int64_t(1) << 40), f + ": ld_top must be >= top");
  PGCN_REQUIRE(temperature >= 1e-4f && temperature <= 1e4f, f + ": temperature must be in [1e-4, 1e4]");
  return PGCN_OK;
}

bool norm_sizes_ok(int32_t dtype, int32_t channels, int32_t groups, int64_t samples, int64_t sample_rows) {
  return (dtype == PGCN_F32 || dtype == PGCN_BF16) && channels >= 1 && channels <= PGCN_MAX_CHANNELS && groups >= 1 &&
         channels % groups == 0 && samples >= 0 && sample_rows >= 1 && samples <= kMaxRows && sample_rows <= kMaxRows &&
         samples * sample_rows <= kMaxRows;
}

int check_norm(int32_t dtype, int32_t act, int32_t channels, int32_t groups, int64_t samples, int64_t sample_rows, const char *fn) {
  const std::string f(fn);
  PGCN_REQUIRE(dtype == PGCN_F32 || dtype == PGCN_BF16, f + ": bad dtype");
  PGCN_REQUIRE(act >= PGCN_ACT_NONE && act <= PGCN_ACT_GELU, f + ": bad act");
  PGCN_REQUIRE(channels >= 1 && channels <= PGCN_MAX_CHANNELS, f + ": channels must be in [1, PGCN_MAX_CHANNELS]");
  PGCN_REQUIRE(groups >= 1 && channels % groups == 0, f + ": groups must divide channels");
  PGCN_REQUIRE(norm_sizes_ok(dtype, channels, groups, samples, sample_rows), f + ": samples or sample_rows out of range");
  return PGCN_OK;
}

bool mx_format_ok(int32_t format) { return format == PGCN_MX_INT8 || format == PGCN_MX_FP4; }
bool aligned4(const void *q) { return ((uintptr_t)q & 3u) == 0; }

// Elements and scales of rows in 8 or 4 bits.
int check_mx(int32_t format, int64_t cols, int64_t ld_q, int64_t ld_s, const std::string &f, const char *q, const char *s) {
  PGCN_REQUIRE(ld_q >= mx_row_bytes(format, cols) && ld_q % 16 == 0 && ld_q <= (int64_t(1) << 40),
               f + ": the stride of " + q + " must hold a row's blocks and be a multiple of 16");
  PGCN_REQUIRE(ld_s >= mx_blocks(cols) && ld_s % 4 == 0 && ld_s <= (int64_t(1) << 40),
               f + ": the stride of " + s + " must hold a row's blocks and be a multiple of 4");
  return PGCN_OK;
}
Range mx_elements(const void *p, int32_t format, int64_t rows, int64_t cols, int64_t ld) {
  return matrix(p, rows, mx_row_bytes(format, cols), ld, 1);
}

bool mx_wgrad_sizes_ok(int32_t dtype, int64_t rows, int32_t f_in, int32_t f_out) {
  return (dtype == PGCN_F32 || dtype == PGCN_BF16) && rows >= 0 && rows <= kMaxRows && f_in >= 1 && f_in <= PGCN_MAX_WIDTH &&
         f_out >= 1 && f_out <= PGCN_MAX_WIDTH;
}
bool mx_matmul_sizes_ok(int32_t dtype, int64_t m, int32_t n, int32_t k) {
  return (dtype == PGCN_F32 || dtype == PGCN_BF16) && m >= 0 && m <= kMaxRows && n >= 1 && n <= PGCN_MAX_MX_COLS && k >= 1 &&
         k <= PGCN_MAX_MX_COLS;
}

}  // namespace

extern "C" size_t pgcn_top_logits_workspace_size(int32_t dtype, int64_t rows, int32_t classes, int32_t top) try {
  return top_sizes_ok(dtype, rows, classes, top) ? top_logits_workspace(dtype, rows, classes, top) : 0;
} catch (...) {
  (void)exception_status("pgcn_top_logits_workspace_size");
  return 0;
}

extern "C" int pgcn_top_logits(const pgcn_top_logits_args *a, hipStream_t s) try {
  const char *fn = "pgcn_top_logits";
  PGCN_REQUIRE(a, "pgcn_top_logits: null args");
  int rc = check_top(a->dtype, a->rows, a->classes, a->top, a->ld, a->ld_top, a->temperature, fn);
  if (rc || a->rows == 0) return rc;
  PGCN_REQUIRE(a->Z && a->top_values && a->top_ids, "pgcn_top_logits: null Z, top_values or top_ids");
  PGCN_REQUIRE(aligned16(a->Z), "pgcn_top_logits: Z must be 16-byte aligned");
  rc = check_workspace(a->workspace, a->workspace_bytes, top_logits_workspace(a->dtype, a->rows, a->classes, a->top), fn);
  if (rc) return rc;
  const Range r[] = {matrix(a->top_values, a->rows, a->top, a->ld_top, 4), matrix(a->top_ids, a->rows, a->top, a->ld_top, 4),
                     matrix(a->tail_lse, 1, a->rows, a->rows, 4), Range{a->workspace, a->workspace_bytes},
                     matrix(a->Z, a->rows, a->classes, a->ld, elem_size(a->dtype))};
  PGCN_REQUIRE(!outputs_overlap(r, 4), "pgcn_top_logits: an output or the workspace overlaps another buffer");
  rc = check_stream(s, fn);
  return rc ? rc : launch_top_logits(*a, s);
} catch (...) {
  return exception_status("pgcn_top_logits");
}

extern "C" size_t pgcn_distill_workspace_size(int32_t dtype, int64_t rows, int32_t classes, int32_t top) try {
  return top_sizes_ok(dtype, rows, classes, top) ? distill_workspace(dtype, rows, classes, top) : 0;
} catch (...) {
  (void)exception_status("pgcn_distill_workspace_size");
  return 0;
}

extern "C" int pgcn_distill_loss_fwd_bwd(const pgcn_distill_args *a, hipStream_t s) try {
  const char *fn = "pgcn_distill_loss_fwd_bwd";
  PGCN_REQUIRE(a, "pgcn_distill_loss_fwd_bwd: null args");
  int rc = check_top(a->dtype, a->rows, a->classes, a->top, a->ld, a->ld_top, a->temperature, fn);
  if (rc) return rc;
  PGCN_REQUIRE(std::isfinite(a->soft_scale) && std::isfinite(a->hard_scale), "pgcn_distill_loss_fwd_bwd: a scale is not finite");
  PGCN_REQUIRE(a->loss_out, "pgcn_distill_loss_fwd_bwd: null loss_out");
  if (a->rows > 0) {
    PGCN_REQUIRE(a->Z && a->J && a->top_values && a->top_ids, "pgcn_distill_loss_fwd_bwd: null Z, J, top_values or top_ids");
    PGCN_REQUIRE(aligned16(a->Z) && aligned16(a->J), "pgcn_distill_loss_fwd_bwd: Z and J must be 16-byte aligned");
    rc = check_workspace(a->workspace, a->workspace_bytes, distill_workspace(a->dtype, a->rows, a->classes, a->top), fn);
    if (rc) return rc;
    const size_t e = elem_size(a->dtype);
    const Range r[] = {matrix(a->J, a->rows, a->classes, a->ld, e), Range{a->loss_out, 4},
                       Range{a->workspace, a->workspace_bytes}, matrix(a->Z, a->rows, a->classes, a->ld, e),
                       matrix(a->top_values, a->rows, a->top, a->ld_top, 4), matrix(a->top_ids, a->rows, a->top, a->ld_top, 4),
                       matrix(a->tail_lse, 1, a->rows, a->rows, 4), matrix(a->labels, 1, a->rows, a->rows, 4)};
    PGCN_REQUIRE(!outputs_overlap(r, 3), "pgcn_distill_loss_fwd_bwd: an output or the workspace overlaps another buffer");
  }
  rc = check_stream(s, fn);
  return rc ? rc : launch_distill(*a, s);
} catch (...) {
  return exception_status("pgcn_distill_loss_fwd_bwd");
}

extern "C" size_t pgcn_group_norm_workspace_size(int32_t dtype, int32_t channels, int32_t groups, int64_t samples,
                                                 int64_t sample_rows) try {
  return norm_sizes_ok(dtype, channels, groups, samples, sample_rows)
             ? group_norm_workspace(dtype, channels, groups, samples, sample_rows) : 0;
} catch (...) {
  (void)exception_status("pgcn_group_norm_workspace_size");
  return 0;
}

extern "C" int pgcn_group_norm_fwd(const pgcn_group_norm_fwd_args *a, hipStream_t s) try {
  const char *fn = "pgcn_group_norm_fwd";
  PGCN_REQUIRE(a, "pgcn_group_norm_fwd: null args");
  int rc = check_norm(a->dtype, a->act, a->channels, a->groups, a->samples, a->sample_rows, fn);
  if (rc) return rc;
  PGCN_REQUIRE(stride_ok(a->dtype, a->ld_x, a->channels) && stride_ok(a->dtype, a->ld_y, a->channels),
               "pgcn_group_norm_fwd: strides must be >= channels and multiples of 4 (fp32) or 8 (bf16)");
  PGCN_REQUIRE(a->eps > 0.f && std::isfinite(a->eps), "pgcn_group_norm_fwd: eps must be positive and finite");
  if (a->samples == 0) return PGCN_OK;
  PGCN_REQUIRE(a->X && a->Y && aligned16(a->X) && aligned16(a->Y), "pgcn_group_norm_fwd: null or unaligned X or Y");
  rc = check_workspace(a->workspace, a->workspace_bytes,
                       group_norm_workspace(a->dtype, a->channels, a->groups, a->samples, a->sample_rows), fn);
  if (rc) return rc;
  const int64_t rows = a->samples * a->sample_rows, stats = a->samples * a->groups;
  const size_t e = elem_size(a->dtype);
  const Range r[] = {matrix(a->Y, rows, a->channels, a->ld_y, e), matrix(a->mean, 1, stats, stats, 4),
                     matrix(a->rstd, 1, stats, stats, 4), Range{a->workspace, a->workspace_bytes},
                     matrix(a->X, rows, a->channels, a->ld_x, e), matrix(a->gamma, 1, a->channels, a->channels, 4),
                     matrix(a->beta, 1, a->channels, a->channels, 4)};
  PGCN_REQUIRE(!outputs_overlap(r, 4), "pgcn_group_norm_fwd: an output or the workspace overlaps another buffer");
  rc = check_stream(s, fn);
  return rc ? rc : launch_group_norm_fwd(*a, s);
} catch (...) {
  return exception_status("pgcn_group_norm_fwd");
}

extern "C" int pgcn_group_norm_bwd(const pgcn_group_norm_bwd_args *a, hipStream_t s) try {
  const char *fn = "pgcn_group_norm_bwd";
  PGCN_REQUIRE(a, "pgcn_group_norm_bwd: null args");
  int rc = check_norm(a->dtype, a->act, a->channels, a->groups, a->samples, a->sample_rows, fn);
  if (rc) return rc;
  PGCN_REQUIRE(stride_ok(a->dtype, a->ld_x, a->channels) && stride_ok(a->dtype, a->ld_j_out, a->channels) &&
                   (!a->J_in || stride_ok(a->dtype, a->ld_j_in, a->channels)),
               "pgcn_group_norm_bwd: strides must be >= channels and multiples of 4 (fp32) or 8 (bf16)");
  if (a->samples > 0) {
    PGCN_REQUIRE(a->X && a->J_out && aligned16(a->X) && aligned16(a->J_out) && aligned16(a->J_in),
                 "pgcn_group_norm_bwd: null or unaligned X, J_out or J_in");
    PGCN_REQUIRE(a->mean && a->rstd, "pgcn_group_norm_bwd: null mean or rstd");
    rc = check_workspace(a->workspace, a->workspace_bytes,
                         group_norm_workspace(a->dtype, a->channels, a->groups, a->samples, a->sample_rows), fn);
    if (rc) return rc;
    const int64_t rows = a->samples * a->sample_rows, stats = a->samples * a->groups;
    const size_t e = elem_size(a->dtype);
    const Range r[] = {matrix(a->J_in, rows, a->channels, a->ld_j_in, e), matrix(a->dgamma, 1, a->channels, a->channels, 4),
                       matrix(a->dbeta, 1, a->channels, a->channels, 4), Range{a->workspace, a->workspace_bytes},
                       matrix(a->X, rows, a->channels, a->ld_x, e), matrix(a->J_out, rows, a->channels, a->ld_j_out, e),
                       matrix(a->gamma, 1, a->channels, a->channels, 4), matrix(a->beta, 1, a->channels, a->channels, 4),
                       matrix(a->mean, 1, stats, stats, 4), matrix(a->rstd, 1, stats, stats, 4)};
    PGCN_REQUIRE(!outputs_overlap(r, 4), "pgcn_group_norm_bwd: an output or the workspace overlaps another buffer");
  }
  rc = check_stream(s, fn);
  return rc ? rc : launch_group_norm_bwd(*a, s);
} catch (...) {
  return exception_status("pgcn_group_norm_bwd");
}

extern "C" int pgcn_mx_quantize(const pgcn_mx_quantize_args *a, hipStream_t s) try {
  const char *fn = "pgcn_mx_quantize";
  PGCN_REQUIRE(a, "pgcn_mx_quantize: null args");
  PGCN_REQUIRE(mx_format_ok(a->format), "pgcn_mx_quantize: bad format");
  PGCN_REQUIRE(a->dtype == PGCN_F32 || a->dtype == PGCN_BF16, "pgcn_mx_quantize: bad dtype");
  PGCN_REQUIRE(a->transpose == 0 || a->transpose == 1, "pgcn_mx_quantize: transpose must be 0 or 1");
  PGCN_REQUIRE(a->cols >= 1 && a->cols <= PGCN_MAX_MX_COLS, "pgcn_mx_quantize: cols must be in [1, PGCN_MAX_MX_COLS]");
  PGCN_REQUIRE(a->rows >= 0 && a->rows <= kMaxRows && a->src_rows >= 0 && a->src_rows <= kMaxRows,
               "pgcn_mx_quantize: rows or src_rows out of range");
  if (a->transpose) {
    PGCN_REQUIRE(!a->index && a->rows == a->src_rows, "pgcn_mx_quantize: a transpose takes every row of X, and no index");
    PGCN_REQUIRE(a->rows <= PGCN_MAX_MX_COLS, "pgcn_mx_quantize: a transpose takes up to PGCN_MAX_MX_COLS rows");
  } else {
    PGCN_REQUIRE(a->index || a->rows <= a->src_rows, "pgcn_mx_quantize: more rows than X has need an index");
  }
  PGCN_REQUIRE(stride_ok(a->dtype, a->ld_x, a->cols), "pgcn_mx_quantize: ld_x must be >= cols and a multiple of 4 (fp32) or 8 (bf16)");
  const int64_t q_rows = a->transpose ? a->cols : a->rows, q_cols = a->transpose ? a->rows : a->cols;
  int rc = check_mx(a->format, q_cols, a->ld_q, a->ld_s, fn, "Q", "S");
  if (rc || a->rows == 0) return rc;
  PGCN_REQUIRE((a->X || a->src_rows == 0) && a->Q && a->S, "pgcn_mx_quantize: null X, Q or S");
  PGCN_REQUIRE(aligned16(a->X) && aligned16(a->Q) && aligned4(a->S) && aligned4(a->index),
               "pgcn_mx_quantize: X and Q must be 16-byte aligned, S and index 4-byte");
  const Range r[] = {mx_elements(a->Q, a->format, q_rows, q_cols, a->ld_q), matrix(a->S, q_rows, mx_blocks(q_cols), a->ld_s, 1),
                     matrix(a->X, a->src_rows, a->cols, a->ld_x, elem_size(a->dtype)), matrix(a->index, 1, a->rows, a->rows, 4)};
  PGCN_REQUIRE(!outputs_overlap(r, 2), "pgcn_mx_quantize: an output overlaps another buffer");
  rc = check_stream(s, fn);
  return rc ? rc : launch_mx_quantize(*a, s);
} catch (...) {
  return exception_status("pgcn_mx_quantize");
}

extern "C" int pgcn_mx_dequantize(const pgcn_mx_dequantize_args *a, hipStream_t s) try {
  const char *fn = "pgcn_mx_dequantize";
  PGCN_REQUIRE(a, "pgcn_mx_dequantize: null args");
  PGCN_REQUIRE(mx_format_ok(a->format), "pgcn_mx_dequantize: bad format");
  PGCN_REQUIRE(a->dtype == PGCN_F32 || a->dtype == PGCN_BF16, "pgcn_mx_dequantize: bad dtype");
  PGCN_REQUIRE(a->cols >= 1 && a->cols <= PGCN_MAX_MX_COLS, "pgcn_mx_dequantize: cols must be in [1, PGCN_MAX_MX_COLS]");
  PGCN_REQUIRE(a->rows >= 0 && a->rows <= kMaxRows, "pgcn_mx_dequantize: rows out of range");
  PGCN_REQUIRE(a->gamma >= 0.f && a->gamma <= 1.f, "pgcn_mx_dequantize: gamma must be in [0, 1]");
  PGCN_REQUIRE(a->gamma == 0.f || a->dtype == PGCN_F32, "pgcn_mx_dequantize: a moving average is kept in fp32");
  PGCN_REQUIRE(stride_ok(a->dtype, a->ld_out, a->cols), "pgcn_mx_dequantize: ld_out must be >= cols and a multiple of 4 (fp32) or 8 (bf16)");
  int rc = check_mx(a->format, a->cols, a->ld_q, a->ld_s, fn, "Q", "S");
  if (rc || a->rows == 0) return rc;
  PGCN_REQUIRE(a->Q && a->S && a->out, "pgcn_mx_dequantize: null Q, S or out");
  PGCN_REQUIRE(aligned16(a->out) && aligned16(a->Q) && aligned4(a->S), "pgcn_mx_dequantize: out and Q must be 16-byte aligned, S 4-byte");
  const Range r[] = {matrix(a->out, a->rows, a->cols, a->ld_out, elem_size(a->dtype)),
                     mx_elements(a->Q, a->format, a->rows, a->cols, a->ld_q), matrix(a->S, a->rows, mx_blocks(a->cols), a->ld_s, 1)};
  PGCN_REQUIRE(!outputs_overlap(r, 1), "pgcn_mx_dequantize: the output overlaps another buffer");
  rc = check_stream(s, fn);
  return rc ? rc : launch_mx_dequantize(*a, s);
} catch (...) {
  return exception_status("pgcn_mx_dequantize");
}

extern "C" size_t pgcn_mx_wgrad_workspace_size(int32_t dtype, int64_t rows, int32_t f_in, int32_t f_out) try {
  return mx_wgrad_sizes_ok(dtype, rows, f_in, f_out) ? mx_wgrad_workspace(dtype, rows, f_in, f_out) : 0;
} catch (...) {
  (void)exception_status("pgcn_mx_wgrad_workspace_size");
  return 0;
}

extern "C" int pgcn_mx_wgrad(const pgcn_mx_wgrad_args *a, hipStream_t s) try {
  const char *fn = "pgcn_mx_wgrad";
  PGCN_REQUIRE(a, "pgcn_mx_wgrad: null args");
  PGCN_REQUIRE(a->dtype == PGCN_F32 || a->dtype == PGCN_BF16, "pgcn_mx_wgrad: bad dtype");
  PGCN_REQUIRE(a->f_in >= 1 && a->f_in <= PGCN_MAX_WIDTH && a->f_out >= 1 && a->f_out <= PGCN_MAX_WIDTH,
               "pgcn_mx_wgrad: widths must be in [1, PGCN_MAX_WIDTH]");
  PGCN_REQUIRE(a->rows >= 0 && a->rows <= kMaxRows, "pgcn_mx_wgrad: rows out of range");
  PGCN_REQUIRE(stride_ok(PGCN_F32, a->ld_j, a->f_out) && (!a->H || stride_ok(PGCN_F32, a->ld_h, a->f_out)),
               "pgcn_mx_wgrad: ld_j and ld_h must be >= f_out and multiples of 4");
  int rc = check_mx(PGCN_MX_INT8, a->f_in, a->ld_q, a->ld_s, fn, "Q", "S");
  if (rc) return rc;
  PGCN_REQUIRE(a->dW && aligned4(a->dW), "pgcn_mx_wgrad: null or unaligned dW");
  if (a->rows > 0) {
    PGCN_REQUIRE(a->Q && a->S && a->J, "pgcn_mx_wgrad: null Q, S or J");
    PGCN_REQUIRE(aligned16(a->Q) && aligned4(a->S) && aligned16(a->J) && aligned16(a->H),
                 "pgcn_mx_wgrad: Q, J and H must be 16-byte aligned, S 4-byte");
  }
  rc = check_workspace(a->workspace, a->workspace_bytes, mx_wgrad_workspace(a->dtype, a->rows, a->f_in, a->f_out), fn);
  if (rc) return rc;
  const Range r[] = {matrix(a->dW, 1, (int64_t)a->f_in * a->f_out, (int64_t)a->f_in * a->f_out, 4),
                     Range{a->workspace, a->workspace_bytes}, mx_elements(a->Q, PGCN_MX_INT8, a->rows, a->f_in, a->ld_q),
                     matrix(a->S, a->rows, mx_blocks(a->f_in), a->ld_s, 1), matrix(a->J, a->rows, a->f_out, a->ld_j, 4),
                     matrix(a->H, a->rows, a->f_out, a->ld_h, 4)};
  PGCN_REQUIRE(!outputs_overlap(r, 2), "pgcn_mx_wgrad: dW or the workspace overlaps another buffer");
  rc = check_stream(s, fn);
  return rc ? rc : launch_mx_wgrad(*a, s);
} catch (...) {
  return exception_status("pgcn_mx_wgrad");
}

extern "C" size_t pgcn_mx_matmul_workspace_size(int32_t dtype, int64_t m, int32_t n, int32_t k) try {
  return mx_matmul_sizes_ok(dtype, m, n, k) ? mx_matmul_workspace(dtype, m, n, k) : 0;
} catch (...) {
  (void)exception_status("pgcn_mx_matmul_workspace_size");
  return 0;
}

extern "C" int pgcn_mx_matmul(const pgcn_mx_matmul_args *a, hipStream_t s) try {
  const char *fn = "pgcn_mx_matmul";
  PGCN_REQUIRE(a, "pgcn_mx_matmul: null args");
  PGCN_REQUIRE(a->dtype == PGCN_F32 || a->dtype == PGCN_BF16, "pgcn_mx_matmul: bad dtype");
  PGCN_REQUIRE(a->relu == 0 || a->relu == 1, "pgcn_mx_matmul: relu must be 0 or 1");
  PGCN_REQUIRE(a->m >= 0 && a->m <= kMaxRows, "pgcn_mx_matmul: m out of range");
  PGCN_REQUIRE(a->n >= 1 && a->n <= PGCN_MAX_MX_COLS && a->k >= 1 && a->k <= PGCN_MAX_MX_COLS,
               "pgcn_mx_matmul: n and k must be in [1, PGCN_MAX_MX_COLS]");
  PGCN_REQUIRE(stride_ok(a->dtype, a->ld_c, a->n), "pgcn_mx_matmul: ld_c must be >= n and a multiple of 4 (fp32) or 8 (bf16)");
  int rc = check_mx(PGCN_MX_FP4, a->k, a->ld_a, a->ld_a_scales, fn, "A", "A_scales");
  if (!rc) rc = check_mx(PGCN_MX_FP4, a->k, a->ld_b, a->ld_b_scales, fn, "B", "B_scales");
  if (rc || a->m == 0) return rc;
  PGCN_REQUIRE(a->A && a->A_scales && a->B && a->B_scales && a->C, "pgcn_mx_matmul: null A, B, scales or C");
  PGCN_REQUIRE(aligned16(a->A) && aligned16(a->B) && aligned16(a->C) && aligned4(a->A_scales) && aligned4(a->B_scales),
               "pgcn_mx_matmul: A, B and C must be 16-byte aligned, scales 4-byte");
  rc = check_workspace(a->workspace, a->workspace_bytes, mx_matmul_workspace(a->dtype, a->m, a->n, a->k), fn);
  if (rc) return rc;
  const Range r[] = {matrix(a->C, a->m, a->n, a->ld_c, elem_size(a->dtype)), Range{a->workspace, a->workspace_bytes},
                     mx_elements(a->A, PGCN_MX_FP4, a->m, a->k, a->ld_a), matrix(a->A_scales, a->m, mx_blocks(a->k), a->ld_a_scales, 1),
                     mx_elements(a->B, PGCN_MX_FP4, a->n, a->k, a->ld_b), matrix(a->B_scales, a->n, mx_blocks(a->k), a->ld_b_scales, 1)};
  PGCN_REQUIRE(!outputs_overlap(r, 2), "pgcn_mx_matmul: C or the workspace overlaps another buffer");
  rc = check_stream(s, fn);
  return rc ? rc : launch_mx_matmul(*a, s);
} catch (...) {
  return exception_status("pgcn_mx_matmul");
}
