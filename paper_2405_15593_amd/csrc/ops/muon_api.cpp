// Host side of the Newton-Schulz entry points: argument checks, the grouping
// of a matrix list by working shape, the workspace plan and the launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstring>
#include <new>
#include <vector>

#include "microadam.h"
#include "ops_host.h"
#include "schulz_device.h"

using namespace microadam;

namespace {

constexpr uint64_t kAlign = 256;
constexpr uint64_t kPartialBytes = (uint64_t)kMaxMatrices * kNormParts * sizeof(double);
constexpr int64_t kMaxSide = (int64_t)1 << 20;
constexpr int64_t kMaxElements = (int64_t)1 << 33;
constexpr int32_t kMaxSteps = 16;
// A workspace beyond this buys nothing measurable: it holds enough matrices
// of any one size to fill the device.
constexpr uint64_t kUsefulWorkspace = (uint64_t)2 << 30;
constexpr double kDefaultCoefficients[3] = {3.4445, -4.7750, 2.0315};

int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

struct Item {
  int32_t index;
  int32_t m, n;
};

int check_schulz(const microadam_schulz_config* c) {
  if (!c) return report(MICROADAM_ERR_INVALID_ARG, "config is NULL");
  if (c->steps < 1 || c->steps > kMaxSteps) return report(MICROADAM_ERR_INVALID_ARG, "steps must be in [1, 16]");
  if (!(c->eps > 0.0) || !std::isfinite(c->eps))
    return report(MICROADAM_ERR_INVALID_ARG, "eps must be finite and > 0");
  if (c->precision != MICROADAM_PRECISION_AUTO && c->precision != MICROADAM_PRECISION_F16 &&
      c->precision != MICROADAM_PRECISION_SPLIT)
    return report(MICROADAM_ERR_INVALID_ARG, "precision must be AUTO, F16 or SPLIT");
  if (c->coefficients)
    for (int i = 0; i < 3 * c->steps; ++i)
      if (!std::isfinite(c->coefficients[i])) return report(MICROADAM_ERR_INVALID_ARG, "coefficients must be finite");
  return MICROADAM_OK;
}

bool is_dtype(int32_t d) { return d == MICROADAM_F32 || d == MICROADAM_BF16; }

int check_shapes(const microadam_matrix* mats, int32_t n) {
  if (n < 1) return report(MICROADAM_ERR_INVALID_ARG, "n_matrices must be >= 1");
  if (!mats) return report(MICROADAM_ERR_INVALID_ARG, "matrices is NULL");
  for (int32_t i = 0; i < n; ++i) {
    const microadam_matrix& a = mats[i];
    if (a.rows < 1 || a.cols < 1) return report(MICROADAM_ERR_INVALID_ARG, "rows and cols must be >= 1");
    if (a.rows > kMaxSide || a.cols > kMaxSide || up(a.rows, kPad) * up(a.cols, kPad) > kMaxElements)
      return report(MICROADAM_ERR_UNSUPPORTED, "matrix too large (2^20 a side, 2^33 elements)");
  }
  return MICROADAM_OK;
}

int check_operand(const void* p, int64_t ld, int64_t cols, int32_t dtype, const char* null_msg) {
  if (!p) return report(MICROADAM_ERR_INVALID_ARG, null_msg);
  if ((uintptr_t)p % (dtype == MICROADAM_BF16 ? 2 : 4))
    return report(MICROADAM_ERR_INVALID_ARG, "a matrix is not aligned to its element type");
  if (ld < cols) return report(MICROADAM_ERR_INVALID_ARG, "a row stride is below cols");
  if (ld >= ((int64_t)1 << 31)) return report(MICROADAM_ERR_UNSUPPORTED, "a row stride is 2^31 or more");
  return MICROADAM_OK;
}

// The bytes of a matrix: rows of `width` at `stride` (at least width).
struct Region {
  uint64_t at, end, width, stride;
  int64_t rows;
  int32_t matrix;
  enum Kind : int32_t { kGrad, kMomentum, kOut } kind;
};

Region region(const void* p, const microadam_matrix& a, int64_t ld, int32_t dtype, int32_t matrix,
              Region::Kind kind) {
  const uint64_t size = dtype == MICROADAM_BF16 ? 2 : 4;
  Region r;
  r.at = (uint64_t)(uintptr_t)p;
  r.rows = a.rows;
  r.width = (uint64_t)a.cols * size;
  r.stride = (uint64_t)ld * size;
  if (r.rows == 1 || r.width == r.stride) {  // one run of bytes
    r.width = r.stride = r.width * (uint64_t)r.rows;
    r.rows = 1;
  }
  r.end = r.at + (uint64_t)(r.rows - 1) * r.stride + r.width;
  r.matrix = matrix;
  r.kind = kind;
  return r;
}

// Whether [from, to) holds a byte of one of r's rows.
bool holds(const Region& r, uint64_t from, uint64_t to) {
  if (from >= r.end || to <= r.at) return false;
  // the first row that ends after `from`
  const uint64_t row = from < r.at + r.width ? 0 : (from - r.at - r.width) / r.stride + 1;
  return r.at + row * r.stride < to;
}

bool share_bytes(const Region& a, const Region& b) {
  if (a.at >= b.end || b.at >= a.end) return false;
  if (a.rows > 1 && b.rows > 1 && a.stride == b.stride) {
    // row i of the first and row i + k of the second are `apart` + k * stride
    // from each other, so that only the two k around 0 matter
    const Region &x = a.at <= b.at ? a : b, &y = a.at <= b.at ? b : a;
    const uint64_t apart = y.at - x.at, place = apart % x.stride;
    const int64_t rows = (int64_t)(apart / x.stride);  // of x before y's first
    return (place < x.width && rows < x.rows) || (place + y.width > x.stride && rows + 1 < x.rows);
  }
  const Region &few = a.rows <= b.rows ? a : b, &many = a.rows <= b.rows ? b : a;
  for (int64_t i = 0; i < few.rows; ++i) {
    const uint64_t from = few.at + (uint64_t)i * few.stride;
    if (holds(many, from, from + few.width)) return true;
  }
  return false;
}

// What is written shares no byte with anything else of the list: tiles would
// race, and whether a grad is read before it is overwritten would go by the
// batch.  Only a matrix's own grad, which its last product comes after, may lie
// where its output goes.
int check_apart(const microadam_matrix* mats, int32_t n, int32_t grad_dtype, int32_t momentum_dtype, int32_t out_dtype,
                bool momentum) {
  std::vector<Region> all;
  all.reserve((size_t)n * (momentum ? 3 : 2));
  for (int32_t i = 0; i < n; ++i) {
    const microadam_matrix& a = mats[i];
    all.push_back(region(a.grad, a, a.grad_ld, grad_dtype, i, Region::kGrad));
    if (momentum) all.push_back(region(a.momentum, a, a.momentum_ld, momentum_dtype, i, Region::kMomentum));
    all.push_back(region(a.out, a, a.out_ld, out_dtype, i, Region::kOut));
  }
  std::sort(all.begin(), all.end(), [](const Region& a, const Region& b) { return a.at < b.at; });
  std::vector<const Region*> open;  // those that end after the current one starts
  for (const Region& r : all) {
    size_t kept = 0;
    for (const Region* o : open) {
      if (o->end <= r.at) continue;
      open[kept++] = o;
      if (r.kind == Region::kGrad && o->kind == Region::kGrad) continue;
      if (r.matrix == o->matrix && r.kind != Region::kMomentum && o->kind != Region::kMomentum) continue;
      if (share_bytes(r, *o))
        return report(MICROADAM_ERR_INVALID_ARG,
                      "an output or momentum overlaps another of the list, or a grad that is not its own");
    }
    open.resize(kept);
    open.push_back(&r);
  }
  return MICROADAM_OK;
}

// Padded sizes and the offsets of a record of a group of m x n.
SchulzGroup group_of(int32_t m, int32_t n, bool split) {
  SchulzGroup g;
  std::memset(&g, 0, sizeof(g));
  g.m = m;
  g.n = n;
  g.mp = (int32_t)up(m, kPad);
  g.np = (int32_t)up(n, kPad);
  const uint64_t xb = (uint64_t)g.mp * g.np * 2 * (split ? 2 : 1);
  const uint64_t ab = (uint64_t)g.mp * g.mp * 2 * (split ? 2 : 1);
  g.xt = 0;  // every size is a multiple of 8192 bytes
  g.a = 2 * xb;
  g.b = 2 * xb + ab;
  g.record = 2 * xb + 2 * ab;
  return g;
}

bool use_split(const microadam_schulz_config* c, int32_t out_dtype) {
  return c->precision == MICROADAM_PRECISION_SPLIT ||
         (c->precision == MICROADAM_PRECISION_AUTO && out_dtype == MICROADAM_F32);
}

struct Call {
  const microadam_schulz_config* cfg;
  const microadam_matrix* mats;
  int32_t grad_dtype, momentum_dtype, out_dtype;
  bool momentum, update, nesterov;
  double mu, lr, decay;
  int32_t scale;
};

double update_scale(const Call& c, const microadam_matrix& a) {
  if (!c.update) return 1.0;
  switch (c.scale) {
    case MICROADAM_SCALE_MATCH_RMS: return c.lr * 0.2 * std::sqrt((double)std::max(a.rows, a.cols));
    case MICROADAM_SCALE_SPECTRAL: return c.lr * std::sqrt(std::max(1.0, (double)a.rows / (double)a.cols));
    default: return c.lr;
  }
}

// Queues the matrices items[0..count) (equal working shapes adjacent).
int queue_chunk(const Call& c, const Item* items, int32_t count, uint8_t* ws, hipStream_t s) {
  const bool split = use_split(c.cfg, c.out_dtype);
  PackArgs pa;
  GemmArgs ga;
  std::memset(&pa, 0, sizeof(pa));
  std::memset(&ga, 0, sizeof(ga));
  uint64_t at = kPartialBytes;
  int64_t most = 0;
  for (int32_t i = 0; i < count; ++i) {
    const Item& it = items[i];
    if (i == 0 || it.m != items[i - 1].m || it.n != items[i - 1].n) {
      SchulzGroup g = group_of(it.m, it.n, split);
      g.base = at;
      g.first = i;
      pa.group[pa.n_groups++] = g;
    }
    SchulzGroup& g = pa.group[pa.n_groups - 1];
    ++g.count;
    at += g.record;
    most = std::max(most, (int64_t)it.m * it.n);
    const microadam_matrix& a = c.mats[it.index];
    pa.mat[i].grad = a.grad;
    pa.mat[i].momentum = c.momentum ? a.momentum : nullptr;
    pa.mat[i].grad_ld = (int32_t)a.grad_ld;
    pa.mat[i].momentum_ld = c.momentum ? (int32_t)a.momentum_ld : 0;
    pa.tall[i] = ga.tall[i] = a.rows > a.cols;
    pa.of[i] = (uint8_t)(pa.n_groups - 1);
    ga.mat[i].out = a.out;
    ga.mat[i].out_ld = (int32_t)a.out_ld;
    ga.mat[i].scale = (float)update_scale(c, a);
  }
  pa.ws = ga.ws = ws;
  pa.partials = (double*)ws;
  pa.mu = (float)c.mu;
  pa.one_minus_mu = (float)(1.0 - c.mu);
  pa.eps = c.cfg->eps;
  pa.split = ga.split = split ? 1 : 0;
  pa.nesterov = c.nesterov ? 1 : 0;
  pa.grad_bf16 = c.grad_dtype == MICROADAM_BF16;
  pa.momentum_bf16 = c.momentum_dtype == MICROADAM_BF16;
  // parts of about 2048 elements, one read of each thread
  pa.n_parts = (int32_t)std::min<int64_t>(kNormParts, std::max<int64_t>(1, most / 2048));
  hipError_t e;
  if ((e = launch_schulz_norm(pa, count, s)) != hipSuccess) return report_hip(e, "launching the norm kernel");
  if ((e = launch_schulz_pack(pa, count, s)) != hipSuccess) return report_hip(e, "launching the pack kernel");

  ga.n_groups = pa.n_groups;
  std::memcpy(ga.group, pa.group, sizeof(ga.group));
  ga.decay = (float)c.decay;
  ga.out_bf16 = c.out_dtype == MICROADAM_BF16;
  ga.update = c.update ? 1 : 0;
  const int gram = choose_schulz_tile(ga, kGram), poly = choose_schulz_tile(ga, kPoly),
            full = choose_schulz_tile(ga, kApply);
  for (int32_t k = 0; k < c.cfg->steps; ++k) {
    const double* co = c.cfg->coefficients ? c.cfg->coefficients + 3 * k : kDefaultCoefficients;
    ga.ca = (float)(co[0] * kScaleA);
    ga.cb = (float)co[1];
    ga.cc = (float)(co[2] / kScaleA);
    ga.buffer = k & 1;
    if ((e = launch_schulz_gemm(ga, kGram, gram, s)) != hipSuccess ||
        (e = launch_schulz_gemm(ga, kPoly, poly, s)) != hipSuccess ||
        (e = launch_schulz_gemm(ga, k + 1 < c.cfg->steps ? kApply : kFinal, full, s)) != hipSuccess)
      return report_hip(e, "launching a product");
  }
  return MICROADAM_OK;
}

int make_items(const microadam_matrix* mats, int32_t n, std::vector<Item>& items) {
  items.resize((size_t)n);
  for (int32_t i = 0; i < n; ++i) {
    items[i].index = i;
    items[i].m = (int32_t)std::min(mats[i].rows, mats[i].cols);
    items[i].n = (int32_t)std::max(mats[i].rows, mats[i].cols);
  }
  // equal shapes adjacent, large ones first
  std::stable_sort(items.begin(), items.end(), [](const Item& a, const Item& b) {
    return a.n != b.n ? a.n > b.n : a.m > b.m;
  });
  return MICROADAM_OK;
}

int run(const Call& c, int32_t n, void* workspace, uint64_t workspace_bytes, hipStream_t s) {
  std::vector<Item> items;
  make_items(c.mats, n, items);
  const bool split = use_split(c.cfg, c.out_dtype);
  for (const Item& it : items)
    if (kPartialBytes + group_of(it.m, it.n, split).record > workspace_bytes)
      return report(MICROADAM_ERR_STATE_SIZE, "workspace smaller than microadam_matrix_workspace's minimum");
  const int shared = check_apart(c.mats, n, c.grad_dtype, c.momentum_dtype, c.out_dtype, c.momentum);
  if (shared) return shared;
  if (!workspace) return report(MICROADAM_ERR_INVALID_ARG, "workspace is NULL");
  if ((uintptr_t)workspace % kAlign) return report(MICROADAM_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
  int32_t begin = 0;
  while (begin < n) {
    uint64_t bytes = kPartialBytes;
    int32_t end = begin, groups = 0;
    while (end < n && end - begin < kMaxMatrices) {
      const Item& it = items[end];
      const bool fresh = end == begin || it.m != items[end - 1].m || it.n != items[end - 1].n;
      const uint64_t rec = group_of(it.m, it.n, split).record;
      if (bytes + rec > workspace_bytes || groups + (fresh ? 1 : 0) > kMaxGroups) break;
      bytes += rec;
      groups += fresh ? 1 : 0;
      ++end;
    }
    const int rc = queue_chunk(c, items.data() + begin, end - begin, (uint8_t*)workspace, s);
    if (rc) return rc;
    begin = end;
  }
  clear_report();
  return MICROADAM_OK;
}

}  // namespace

extern "C" {

int microadam_matrix_workspace(const microadam_schulz_config* cfg, const microadam_matrix* matrices,
                               int32_t n_matrices, int32_t out_dtype, uint64_t* min_bytes, uint64_t* useful_bytes) {
  int rc = check_schulz(cfg);
  if (rc) return rc;
  if (!min_bytes && !useful_bytes) return report(MICROADAM_ERR_INVALID_ARG, "min_bytes and useful_bytes are NULL");
  if (!is_dtype(out_dtype)) return report(MICROADAM_ERR_INVALID_ARG, "out_dtype must be F32 or BF16");
  rc = check_shapes(matrices, n_matrices);
  if (rc) return rc;
  const bool split = use_split(cfg, out_dtype);
  uint64_t most = 0, all = 0;
  for (int32_t i = 0; i < n_matrices; ++i) {
    const uint64_t r = group_of((int32_t)std::min(matrices[i].rows, matrices[i].cols),
                                (int32_t)std::max(matrices[i].rows, matrices[i].cols), split)
                           .record;
    most = std::max(most, r);
    all = std::min(all + r, kUsefulWorkspace);
  }
  if (min_bytes) *min_bytes = kPartialBytes + most;
  if (useful_bytes) *useful_bytes = kPartialBytes + std::max(most, all);
  clear_report();
  return MICROADAM_OK;
}

int microadam_orthogonalize(const microadam_schulz_config* cfg, const microadam_matrix* matrices, int32_t n_matrices,
                            int32_t grad_dtype, int32_t out_dtype, void* workspace, uint64_t workspace_bytes,
                            void* stream) {
  int rc = check_schulz(cfg);
  if (rc) return rc;
  if (!is_dtype(grad_dtype) || !is_dtype(out_dtype))
    return report(MICROADAM_ERR_INVALID_ARG, "grad_dtype / out_dtype must be F32 or BF16");
  rc = check_shapes(matrices, n_matrices);
  if (rc) return rc;
  for (int32_t i = 0; i < n_matrices; ++i) {
    const microadam_matrix& a = matrices[i];
    if ((rc = check_operand(a.grad, a.grad_ld, a.cols, grad_dtype, "a grad pointer is NULL"))) return rc;
    if ((rc = check_operand(a.out, a.out_ld, a.cols, out_dtype, "an out pointer is NULL"))) return rc;
    if (a.momentum) return report(MICROADAM_ERR_INVALID_ARG, "orthogonalize takes no momentum");
  }
  Call c;
  std::memset(&c, 0, sizeof(c));
  c.cfg = cfg;
  c.mats = matrices;
  c.grad_dtype = grad_dtype;
  c.out_dtype = out_dtype;
  c.decay = 1.0;
  try {
    return run(c, n_matrices, workspace, workspace_bytes, (hipStream_t)stream);
  } catch (const std::bad_alloc&) {
    return report(MICROADAM_ERR_NO_MEMORY, "host allocation failed");
  }
}

int microadam_muon_step(const microadam_muon_config* cfg, const microadam_matrix* matrices, int32_t n_matrices,
                        int32_t grad_dtype, int32_t momentum_dtype, int32_t param_dtype, double lr, void* workspace,
                        uint64_t workspace_bytes, void* stream) {
  if (!cfg) return report(MICROADAM_ERR_INVALID_ARG, "config is NULL");
  int rc = check_schulz(&cfg->schulz);
  if (rc) return rc;
  if (!(cfg->momentum >= 0.0 && cfg->momentum < 1.0))
    return report(MICROADAM_ERR_INVALID_ARG, "momentum must be in [0, 1)");
  if (!(cfg->weight_decay >= 0.0) || !std::isfinite(cfg->weight_decay))
    return report(MICROADAM_ERR_INVALID_ARG, "weight_decay must be finite and >= 0");
  if (cfg->nesterov != 0 && cfg->nesterov != 1)
    return report(MICROADAM_ERR_INVALID_ARG, "nesterov must be 0 or 1");
  if (cfg->scale != MICROADAM_SCALE_MATCH_RMS && cfg->scale != MICROADAM_SCALE_SPECTRAL &&
      cfg->scale != MICROADAM_SCALE_NONE)
    return report(MICROADAM_ERR_INVALID_ARG, "scale must be MATCH_RMS, SPECTRAL or NONE");
  if (!is_dtype(grad_dtype) || !is_dtype(momentum_dtype) || !is_dtype(param_dtype))
    return report(MICROADAM_ERR_INVALID_ARG, "grad_dtype / momentum_dtype / param_dtype must be F32 or BF16");
  if (!std::isfinite(lr)) return report(MICROADAM_ERR_INVALID_ARG, "lr must be finite");
  rc = check_shapes(matrices, n_matrices);
  if (rc) return rc;
  for (int32_t i = 0; i < n_matrices; ++i) {
    const microadam_matrix& a = matrices[i];
    if ((rc = check_operand(a.grad, a.grad_ld, a.cols, grad_dtype, "a grad pointer is NULL"))) return rc;
    if ((rc = check_operand(a.momentum, a.momentum_ld, a.cols, momentum_dtype, "a momentum pointer is NULL")))
      return rc;
    if ((rc = check_operand(a.out, a.out_ld, a.cols, param_dtype, "a parameter pointer is NULL"))) return rc;
  }
  Call c;
  std::memset(&c, 0, sizeof(c));
  c.cfg = &cfg->schulz;
  c.mats = matrices;
  c.grad_dtype = grad_dtype;
  c.momentum_dtype = momentum_dtype;
  c.out_dtype = param_dtype;
  c.momentum = c.update = true;
  c.nesterov = cfg->nesterov != 0;
  c.mu = cfg->momentum;
  c.lr = lr;
  c.decay = 1.0 - lr * cfg->weight_decay;
  c.scale = cfg->scale;
  try {
    return run(c, n_matrices, workspace, workspace_bytes, (hipStream_t)stream);
  } catch (const std::bad_alloc&) {
    return report(MICROADAM_ERR_NO_MEMORY, "host allocation failed");
  }
}

}  // extern "C"
