// Host side of the token log-probability entry points: argument checks and
// the launch.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <cstring>

#include "logprobs_device.h"
#include "microadam.h"
#include "ops_host.h"

using namespace microadam;

namespace {

constexpr int64_t kMaxVocab = (int64_t)1 << 24;
constexpr int64_t kMaxRows = (int64_t)1 << 20;

int check(const microadam_logits* l, LogprobArgs& a) {
  if (!l) return report(MICROADAM_ERR_INVALID_ARG, "logits is NULL");
  if (l->dtype != MICROADAM_F32 && l->dtype != MICROADAM_BF16)
    return report(MICROADAM_ERR_INVALID_ARG, "dtype must be F32 or BF16");
  if (l->reserved != 0) return report(MICROADAM_ERR_INVALID_ARG, "reserved must be 0");
  if (l->rows < 0 || l->vocab < 1) return report(MICROADAM_ERR_INVALID_ARG, "rows must be >= 0 and vocab >= 1");
  if (l->vocab > kMaxVocab) return report(MICROADAM_ERR_UNSUPPORTED, "vocab above 2^24");
  if (l->rows > kMaxRows) return report(MICROADAM_ERR_UNSUPPORTED, "more than 2^20 rows");
  if (l->ld < l->vocab && l->rows > 1) return report(MICROADAM_ERR_INVALID_ARG, "the row stride is below vocab");
  if (l->ld > ((int64_t)1 << 40)) return report(MICROADAM_ERR_UNSUPPORTED, "the row stride is above 2^40");
  if (l->group_rows < 0 || (l->group_rows > 0 && l->rows % l->group_rows) || l->group_stride < 0 ||
      (l->group_rows == 0 && l->group_stride != 0))
    return report(MICROADAM_ERR_INVALID_ARG, "group_rows must divide rows, and group_stride be 0 without it");
  if (l->group_stride > ((int64_t)1 << 40))
    return report(MICROADAM_ERR_UNSUPPORTED, "the stride of groups is above 2^40");
  if (!(l->temperature > 0.0) || !std::isfinite(l->temperature))
    return report(MICROADAM_ERR_INVALID_ARG, "temperature must be finite and > 0");
  const double c = 1.4426950408889634 / l->temperature;
  if (!((float)c > 0.0f) || !std::isfinite((float)c) || !std::isfinite((float)(1.0 / l->temperature)))
    return report(MICROADAM_ERR_INVALID_ARG, "temperature is out of the range of binary32");
  if (l->rows > 0) {
    if (!l->data) return report(MICROADAM_ERR_INVALID_ARG, "the logits pointer is NULL");
    if (!l->targets) return report(MICROADAM_ERR_INVALID_ARG, "targets is NULL");
    if ((uintptr_t)l->data % (l->dtype == MICROADAM_BF16 ? 2 : 4) || (uintptr_t)l->targets % 8)
      return report(MICROADAM_ERR_INVALID_ARG, "logits or targets are not aligned to their element type");
  }
  std::memset(&a, 0, sizeof(a));
  a.logits = l->data;
  a.targets = l->targets;
  a.ld = l->ld;
  a.ignore_index = l->ignore_index;
  a.rows = l->rows;
  a.vocab = (int32_t)l->vocab;
  a.group_rows = l->rows > 0 ? (int32_t)l->group_rows : 0;
  a.group_stride = l->group_stride;
  a.c = (float)c;
  a.inv_t = (float)(1.0 / l->temperature);
  return MICROADAM_OK;
}

// Whether the rows of logits and gradient share bytes: rows at the same
// stride, the places within it decide; else the ranges do.
bool share_bytes(const LogprobArgs& l, const void* g, int64_t grad_ld, int64_t size) {
  const uintptr_t a = (uintptr_t)l.logits, b = (uintptr_t)g;
  const int64_t width = l.vocab * size, stride_x = l.ld * size, stride_g = grad_ld * size;
  const int64_t inner = l.group_rows ? l.group_rows : l.rows;
  const uint64_t reach_x =
      (uint64_t)((l.rows / inner - 1) * l.group_stride * size + (inner - 1) * stride_x + width);
  const uint64_t reach_g = (uint64_t)((l.rows - 1) * stride_g + width);
  if (a <= b ? b - a >= reach_x : a - b >= reach_g) return false;
  if (l.rows == 1 || l.group_rows || stride_x != stride_g) return true;
  const int64_t place = (int64_t)((a <= b ? b - a : a - b) % (uint64_t)stride_x);
  return place < width || place > stride_x - width;
}

bool aligned4(const void* p) { return (uintptr_t)p % 4 == 0; }

int launch(const LogprobArgs& a, int32_t dtype, void* stream) {
  if (a.rows > 0) {
    const hipError_t e = launch_token_logprobs(a, dtype == MICROADAM_BF16, (hipStream_t)stream);
    if (e != hipSuccess) return report_hip(e, "launching the log-probability kernel");
  }
  clear_report();
  return MICROADAM_OK;
}

}  // namespace

extern "C" {

int microadam_token_logprobs(const microadam_logits* logits, int32_t top_k, float* logp, float* entropy,
                             float* top_logprobs, int64_t* top_indices, void* stream) {
  LogprobArgs a;
  const int rc = check(logits, a);
  if (rc) return rc;
  if (top_k < 0 || top_k > logits->vocab) return report(MICROADAM_ERR_INVALID_ARG, "top_k must be in [0, vocab]");
  if (top_k > kMaxTopK) return report(MICROADAM_ERR_UNSUPPORTED, "top_k above 64");
  if (top_k > 0 && a.rows > 0 && (!top_logprobs || !top_indices))
    return report(MICROADAM_ERR_INVALID_ARG, "top_logprobs / top_indices is NULL");
  if (!aligned4(logp) || !aligned4(entropy) || !aligned4(top_logprobs) || (uintptr_t)top_indices % 8)
    return report(MICROADAM_ERR_INVALID_ARG, "an output is not aligned to its element type");
  a.top_k = top_k;
  a.logp = logp;
  a.entropy = entropy;
  a.top_logprobs = top_logprobs;
  a.top_indices = top_indices;
  return launch(a, logits->dtype, stream);
}

int microadam_token_logprobs_grad(const microadam_logits* logits, const float* grad_logp, const float* grad_entropy,
                                  float* logp, float* entropy, void* grad, int64_t grad_ld, void* stream) {
  LogprobArgs a;
  const int rc = check(logits, a);
  if (rc) return rc;
  if (a.rows > 0) {
    if (!grad_logp || !grad) return report(MICROADAM_ERR_INVALID_ARG, "grad_logp / grad is NULL");
    if (grad_ld < logits->vocab && a.rows > 1)
      return report(MICROADAM_ERR_INVALID_ARG, "the gradient's row stride is below vocab");
    if (grad_ld > ((int64_t)1 << 40)) return report(MICROADAM_ERR_UNSUPPORTED, "the gradient's row stride is above 2^40");
    if (grad == logits->data && (grad_ld != logits->ld || a.group_rows))
      return report(MICROADAM_ERR_INVALID_ARG, "in place, the rows must have one stride, the same one");
    const int64_t size = logits->dtype == MICROADAM_BF16 ? 2 : 4;
    if (grad != logits->data && share_bytes(a, grad, grad_ld, size))
      return report(MICROADAM_ERR_INVALID_ARG, "the gradient overlaps the logits without being in place");
    if (!aligned4(grad_logp) || !aligned4(grad_entropy) || !aligned4(logp) || !aligned4(entropy) ||
        (uintptr_t)grad % (logits->dtype == MICROADAM_BF16 ? 2 : 4))
      return report(MICROADAM_ERR_INVALID_ARG, "an argument is not aligned to its element type");
  }
  a.grad_logp = grad_logp;
  a.grad_entropy = grad_entropy;
  a.logp = logp;
  a.entropy = entropy;
  a.grad = grad;
  a.grad_ld = grad_ld;
  return launch(a, logits->dtype, stream);
}

}  // extern "C"
