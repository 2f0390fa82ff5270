// Host side of the gradient norm and clipping entry points: argument checks,
// the cutting of the list into launches, and the launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstring>
#include <new>
#include <utility>
#include <vector>

#include "clip_device.h"
#include "microadam.h"
#include "ops_host.h"

using namespace microadam;

namespace {

constexpr uint64_t kWorkspace = (uint64_t)(kClipSlots + 1) * sizeof(double);
// The last-level cache's 256 MiB: beyond it reads past the caches take 549 instead
// of 652 us for 3.8 GB, and the scaling 1440 instead of 1510; a list of 53 MB is
// scaled in 21 instead of 18 us.
constexpr int64_t kCached = (int64_t)256 << 20;
constexpr int64_t kMaxNumel = (int64_t)1 << 40;
static_assert(sizeof(ClipArgs) <= 4096, "kernel arguments");

int check(const void* const* grads, const int64_t* numels, const int32_t* dtypes, int32_t n, const float* norm,
          const void* workspace, uint64_t workspace_bytes) {
  if (n < 0) return report(MICROADAM_ERR_INVALID_ARG, "n_grads must be >= 0");
  if (n > 0 && (!grads || !numels || !dtypes))
    return report(MICROADAM_ERR_INVALID_ARG, "grads, numels or dtypes is NULL");
  for (int32_t i = 0; i < n; ++i) {
    if (dtypes[i] != MICROADAM_F32 && dtypes[i] != MICROADAM_BF16)
      return report(MICROADAM_ERR_INVALID_ARG, "dtypes must be F32 or BF16");
    if (numels[i] < 0) return report(MICROADAM_ERR_INVALID_ARG, "numels must be >= 0");
    if (numels[i] > kMaxNumel) return report(MICROADAM_ERR_UNSUPPORTED, "a gradient of more than 2^40 elements");
    if (numels[i] > 0 && !grads[i]) return report(MICROADAM_ERR_INVALID_ARG, "a gradient pointer is NULL");
    if ((uintptr_t)grads[i] % (dtypes[i] == MICROADAM_BF16 ? 2 : 4))
      return report(MICROADAM_ERR_INVALID_ARG, "a gradient is not aligned to its element type");
  }
  if (!norm || (uintptr_t)norm % 4) return report(MICROADAM_ERR_INVALID_ARG, "norm is NULL or not aligned");
  if (workspace_bytes < kWorkspace)
    return report(MICROADAM_ERR_STATE_SIZE, "workspace smaller than microadam_clip_workspace's");
  if (!workspace) return report(MICROADAM_ERR_INVALID_ARG, "workspace is NULL");
  if ((uintptr_t)workspace % 8) return report(MICROADAM_ERR_INVALID_ARG, "workspace must be 8-byte aligned");
  return MICROADAM_OK;
}

// Gradients that are scaled lie apart, from each other (one that shares bytes
// with another would be scaled twice, or by halves) and from the norm and the
// workspace.
int check_apart(const void* const* grads, const int64_t* numels, const int32_t* dtypes, int32_t n, const float* norm,
                const void* workspace) {
  std::vector<std::pair<uint64_t, uint64_t>> all;
  all.reserve((size_t)n + 2);
  bool sorted = true;
  for (int32_t i = 0; i < n; ++i)
    if (numels[i] > 0) {
      const uint64_t at = (uint64_t)(uintptr_t)grads[i];
      all.emplace_back(at, at + (uint64_t)numels[i] * (dtypes[i] == MICROADAM_BF16 ? 2 : 4));
      sorted = sorted && (all.size() < 2 || all[all.size() - 2].first <= at);
    }
  const uint64_t other[2][2] = {{(uint64_t)(uintptr_t)norm, 4}, {(uint64_t)(uintptr_t)workspace, kWorkspace}};
  for (const auto& o : other) {
    sorted = sorted && (all.empty() || all.back().first <= o[0]);
    all.emplace_back(o[0], o[0] + o[1]);
  }
  if (!sorted) std::sort(all.begin(), all.end());
  for (size_t i = 1; i < all.size(); ++i)
    if (all[i].first < all[i - 1].second)
      return report(MICROADAM_ERR_INVALID_ARG, "gradients overlap (or one is listed twice), or the norm or workspace lies in one");
  return MICROADAM_OK;
}

// The list from entry `i` on into a launch's table; the entry after the last
// that fitted.
int32_t fill(ClipArgs& a, const void* const* grads, const int64_t* numels, const int32_t* dtypes, int32_t n,
             int32_t i) {
  a.n = 0;
  int64_t chunks = 0;
  for (; i < n; ++i) {
    if (numels[i] == 0) continue;
    const bool bf16 = dtypes[i] == MICROADAM_BF16;
    const uint64_t at = (uint64_t)(uintptr_t)grads[i], end = at + (uint64_t)numels[i] * (bf16 ? 2 : 4);
    const int64_t own = (int64_t)((end - (at & ~(uint64_t)15) + kClipChunk - 1) / kClipChunk);
    if (a.n == kClipTensors || (a.n > 0 && chunks + own > kClipMost)) break;
    a.at[a.n] = at | (bf16 ? 1 : 0);
    a.end[a.n] = end;
    a.first[a.n] = (int32_t)chunks;
    chunks += own;
    ++a.n;
  }
  a.first[a.n] = (int32_t)chunks;
  return i;
}

int queue(const void* const* grads, const int64_t* numels, const int32_t* dtypes, int32_t n, bool scale,
          double max_norm, double eps, float* norm, void* workspace, hipStream_t s) {
  ClipArgs a;
  std::memset(&a, 0, sizeof(a));
  a.partial = (double*)workspace;
  a.max_norm = max_norm;
  a.eps = eps;
  // one number of slots for all launches of the call
  int64_t most = 1, bytes = 0;  // (bytes: a small gradient's chunk is nearly empty)
  for (int32_t i = 0; i < n;) {
    i = fill(a, grads, numels, dtypes, n, i);
    for (int32_t k = 0; k < a.n; ++k) bytes += (int64_t)(a.end[k] - (a.at[k] & ~(uint64_t)1));
    most = std::max(most, (int64_t)a.first[a.n]);
  }
  a.past = bytes > kCached ? 1 : 0;
  a.slots = (int32_t)std::min<int64_t>(kClipSlots, most);
  hipError_t e;
  std::vector<int32_t> starts;
  int32_t i = 0;
  do {
    starts.push_back(i);
    i = fill(a, grads, numels, dtypes, n, i);
    if ((e = launch_square_sums(a, s)) != hipSuccess) return report_hip(e, "launching the sums of squares");
    a.add = 1;
  } while (i < n);
  if (!scale || a.past) {
    a.norm = norm;
    if ((e = launch_grad_norm(a, s)) != hipSuccess) return report_hip(e, "launching the norm");
    if (!scale) return MICROADAM_OK;
  }
  // the last launch's tensors first, as they were read last
  for (size_t k = starts.size(); k-- > 0;) {
    if (k + 1 < starts.size()) fill(a, grads, numels, dtypes, n, starts[k]);
    a.norm = k + 1 == starts.size() ? norm : nullptr;
    if ((e = launch_scale_grads(a, s)) != hipSuccess) return report_hip(e, "launching the scaling");
  }
  return MICROADAM_OK;
}

}  // namespace

extern "C" {

int microadam_clip_workspace(uint64_t* bytes) {
  if (!bytes) return report(MICROADAM_ERR_INVALID_ARG, "bytes is NULL");
  *bytes = kWorkspace;
  clear_report();
  return MICROADAM_OK;
}

int microadam_grad_norm(const void* const* grads, const int64_t* numels, const int32_t* dtypes, int32_t n_grads,
                        float* norm, void* workspace, uint64_t workspace_bytes, void* stream) {
  int rc = check(grads, numels, dtypes, n_grads, norm, workspace, workspace_bytes);
  if (rc) return rc;
  try {
    rc = queue(grads, numels, dtypes, n_grads, false, 0.0, 0.0, norm, workspace, (hipStream_t)stream);
  } catch (const std::bad_alloc&) {
    return report(MICROADAM_ERR_NO_MEMORY, "host allocation failed");
  }
  if (!rc) clear_report();
  return rc;
}

int microadam_clip_grads(void* const* grads, const int64_t* numels, const int32_t* dtypes, int32_t n_grads,
                         double max_norm, double eps, float* norm, void* workspace, uint64_t workspace_bytes,
                         void* stream) {
  int rc = check(grads, numels, dtypes, n_grads, norm, workspace, workspace_bytes);
  if (rc) return rc;
  if (!(max_norm >= 0.0)) return report(MICROADAM_ERR_INVALID_ARG, "max_norm must be >= 0");
  if (!(eps >= 0.0) || !std::isfinite(eps)) return report(MICROADAM_ERR_INVALID_ARG, "eps must be finite and >= 0");
  try {
    rc = check_apart(grads, numels, dtypes, n_grads, norm, workspace);
    if (!rc)
      rc = queue(grads, numels, dtypes, n_grads, true, max_norm, eps, norm, workspace, (hipStream_t)stream);
  } catch (const std::bad_alloc&) {
    return report(MICROADAM_ERR_NO_MEMORY, "host allocation failed");
  }
  if (!rc) clear_report();
  return rc;
}

}  // extern "C"
