// Host side of the layer norm entry points: argument checks and the launches.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <cstring>

#include "layer_norm_device.h"
#include "microadam.h"
#include "ops_host.h"

using namespace microadam;

namespace {

constexpr int64_t kMaxCols = (int64_t)1 << 24;
constexpr int64_t kMaxRows = (int64_t)1 << 31;
constexpr int64_t kMaxLd = (int64_t)1 << 40;
constexpr int64_t kMaxReach = (int64_t)1 << 60;

int64_t size_of(int32_t dtype) { return dtype == MICROADAM_BF16 ? 2 : 4; }
bool is_dtype(int32_t d) { return d == MICROADAM_F32 || d == MICROADAM_BF16; }

int check_size(const microadam_rows* r) {
  if (!r) return report(MICROADAM_ERR_INVALID_ARG, "rows is NULL");
  if (!is_dtype(r->dtype) || !is_dtype(r->weight_dtype))
    return report(MICROADAM_ERR_INVALID_ARG, "dtype and weight_dtype must be F32 or BF16");
  if (r->rows < 0 || r->cols < 1) return report(MICROADAM_ERR_INVALID_ARG, "rows must be >= 0 and cols >= 1");
  if (r->cols > kMaxCols) return report(MICROADAM_ERR_UNSUPPORTED, "cols above 2^24");
  if (r->rows > kMaxRows) return report(MICROADAM_ERR_UNSUPPORTED, "more than 2^31 rows");
  return MICROADAM_OK;
}

int check(const microadam_rows* r, LayerNormArgs& a) {
  const int rc = check_size(r);
  if (rc) return rc;
  if (!(r->eps >= 0.0) || !std::isfinite((float)r->eps))
    return report(MICROADAM_ERR_INVALID_ARG, "eps must be >= 0 and finite in binary32");
  if (r->rows > 0 && !r->x) return report(MICROADAM_ERR_INVALID_ARG, "x is NULL");
  if ((uintptr_t)r->x % size_of(r->dtype)) return report(MICROADAM_ERR_INVALID_ARG, "x is not aligned to its element type");
  if ((uintptr_t)r->weight % size_of(r->weight_dtype) || (uintptr_t)r->bias % size_of(r->weight_dtype))
    return report(MICROADAM_ERR_INVALID_ARG, "weight or bias is not aligned to its element type");
  std::memset(&a, 0, sizeof(a));
  a.x = r->x;
  a.weight = r->weight;
  a.bias = r->bias;
  a.rows = r->rows;
  a.cols = (int32_t)r->cols;
  a.x_ld = r->ld;
  a.bf16 = r->dtype == MICROADAM_BF16;
  a.weight_bf16 = r->weight_dtype == MICROADAM_BF16;
  a.eps = (float)r->eps;
  return MICROADAM_OK;
}

int check_ld(int64_t ld, const microadam_rows* r) {
  if (ld < r->cols && r->rows > 1) return report(MICROADAM_ERR_INVALID_ARG, "a row stride is below cols");
  if (ld > kMaxLd) return report(MICROADAM_ERR_UNSUPPORTED, "a row stride is above 2^40");
  if (r->rows > 1 && ld > kMaxReach / r->rows)
    return report(MICROADAM_ERR_UNSUPPORTED, "a matrix reaches over more than 2^60 elements");
  return MICROADAM_OK;
}

struct Range {
  uintptr_t at, end;
};

Range matrix(const void* p, int64_t ld, const microadam_rows* r) {
  const uintptr_t at = (uintptr_t)p;
  return {at, p && r->rows ? at + (uintptr_t)(((r->rows - 1) * ld + r->cols) * size_of(r->dtype)) : at};
}

Range run(const void* p, int64_t bytes) { return {(uintptr_t)p, p ? (uintptr_t)p + (uintptr_t)bytes : (uintptr_t)p}; }

// What is written shares no byte with what is read, nor with what else is
// written: workgroups take rows in any order.
int check_apart(const Range* written, int n_written, const Range* read, int n_read) {
  for (int i = 0; i < n_written; ++i) {
    for (int j = 0; j < i + n_read; ++j) {
      const Range& o = j < i ? written[j] : read[j - i];
      if (written[i].at < o.end && o.at < written[i].end)
        return report(MICROADAM_ERR_INVALID_ARG, "an output overlaps an input or another output");
    }
  }
  return MICROADAM_OK;
}

uint64_t workspace_of(const microadam_rows* r) {
  const LayerNormSums n = layer_norm_sums(r->rows, r->cols, r->dtype == MICROADAM_BF16);
  return n.parts > 1 ? (uint64_t)n.parts * 2 * (uint64_t)n.sums * sizeof(float) : 0;
}

}  // namespace

extern "C" {

int microadam_layer_norm(const microadam_rows* rows, void* y, int64_t y_ld, float* mean, float* rstd, void* stream) {
  LayerNormArgs a;
  int rc = check(rows, a);
  if (rc) return rc;
  if (!mean != !rstd) return report(MICROADAM_ERR_INVALID_ARG, "mean and rstd: both or neither");
  if ((uintptr_t)mean % 4 || (uintptr_t)rstd % 4 || (uintptr_t)y % size_of(rows->dtype))
    return report(MICROADAM_ERR_INVALID_ARG, "an output is not aligned to its element type");
  if (a.rows > 0) {
    if (!y) return report(MICROADAM_ERR_INVALID_ARG, "y is NULL");
    if ((rc = check_ld(rows->ld, rows)) || (rc = check_ld(y_ld, rows))) return rc;
    const int64_t side = rows->cols * size_of(rows->weight_dtype);
    const Range written[] = {matrix(y, y_ld, rows), run(mean, 4 * rows->rows), run(rstd, 4 * rows->rows)};
    const Range read[] = {matrix(rows->x, rows->ld, rows), run(rows->weight, side), run(rows->bias, side)};
    if ((rc = check_apart(written, 3, read, 3))) return rc;
    a.y = y;
    a.y_ld = y_ld;
    a.mean = mean;
    a.rstd = rstd;
    const hipError_t e = launch_layer_norm(a, (hipStream_t)stream);
    if (e != hipSuccess) return report_hip(e, "launching layer norm");
  }
  clear_report();
  return MICROADAM_OK;
}

int microadam_layer_norm_workspace(const microadam_rows* rows, uint64_t* bytes) {
  const int rc = check_size(rows);
  if (rc) return rc;
  if (!bytes) return report(MICROADAM_ERR_INVALID_ARG, "bytes is NULL");
  *bytes = workspace_of(rows);
  clear_report();
  return MICROADAM_OK;
}

int microadam_layer_norm_grad(const microadam_rows* rows, const float* mean, const float* rstd, const void* dy,
                              int64_t dy_ld, void* dx, int64_t dx_ld, void* dweight, void* dbias, void* workspace,
                              uint64_t workspace_bytes, void* stream) {
  LayerNormArgs a;
  int rc = check(rows, a);
  if (rc) return rc;
  if (a.rows > 0) {
    if (!mean || !rstd || !dy) return report(MICROADAM_ERR_INVALID_ARG, "mean, rstd or dy is NULL");
    if ((rc = check_ld(rows->ld, rows)) || (rc = check_ld(dy_ld, rows))) return rc;
    if (dx && (rc = check_ld(dx_ld, rows))) return rc;
  }
  if ((uintptr_t)mean % 4 || (uintptr_t)rstd % 4 || (uintptr_t)dy % size_of(rows->dtype) ||
      (uintptr_t)dx % size_of(rows->dtype) || (uintptr_t)dweight % size_of(rows->weight_dtype) ||
      (uintptr_t)dbias % size_of(rows->weight_dtype))
    return report(MICROADAM_ERR_INVALID_ARG, "an argument is not aligned to its element type");
  const bool sides = dweight || dbias;
  const uint64_t need = sides ? workspace_of(rows) : 0;
  if (workspace_bytes < need)
    return report(MICROADAM_ERR_STATE_SIZE, "workspace smaller than microadam_layer_norm_workspace's");
  if (need && !workspace) return report(MICROADAM_ERR_INVALID_ARG, "workspace is NULL");
  if (need && (uintptr_t)workspace % 16)
    return report(MICROADAM_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
  const int64_t side = rows->cols * size_of(rows->weight_dtype);
  const Range written[] = {matrix(dx, dx_ld, rows), run(dweight, side), run(dbias, side),
                           run(need ? workspace : nullptr, (int64_t)need)};
  const Range read[] = {matrix(rows->x, rows->ld, rows), matrix(dy, dy_ld, rows), run(rows->weight, side),
                        run(mean, 4 * rows->rows), run(rstd, 4 * rows->rows)};
  if ((rc = check_apart(written, 4, read, 5))) return rc;
  a.mean = const_cast<float*>(mean);
  a.rstd = const_cast<float*>(rstd);
  a.dy = dy;
  a.dy_ld = dy_ld;
  a.dx = dx;
  a.dx_ld = dx_ld;
  a.dweight = dweight;
  a.dbias = dbias;
  a.partial = (float*)workspace;
  const LayerNormSums n = layer_norm_sums(rows->rows, rows->cols, a.bf16);
  a.parts = n.parts;
  a.sums = n.sums;
  a.group_bits = n.group_bits;
  a.per_bits = n.per_bits;
  // (no rows: the sums are zeros)
  if (sides || (dx && a.rows > 0)) {
    const hipError_t e = launch_layer_norm_grad(a, (hipStream_t)stream);
    if (e != hipSuccess) return report_hip(e, "launching layer norm's backward pass");
  }
  clear_report();
  return MICROADAM_OK;
}

}  // extern "C"
