// Host side of the attention entry points: argument checks, workspace and the
// launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstring>
#include <utility>

#include "attention_device.h"
#include "microadam.h"
#include "ops_host.h"

using namespace microadam;

namespace {

constexpr int64_t kMaxSide = (int64_t)1 << 30;     // queries of a key head's query heads, keys
constexpr int64_t kMaxStride = (int64_t)1 << 40;
constexpr int64_t kMaxPosition = (int64_t)1 << 23;  // the rows that are loaded at once (64, of bfloat16 128) lie within 2^31 bytes
constexpr int64_t kMaxGroups = (int64_t)1 << 24;   // workgroups of 256: a launch has fewer than 2^32 threads
constexpr uint64_t kAlign = 256;

int64_t size_of(int32_t dtype) { return dtype == MICROADAM_BF16 ? 2 : 4; }

int check(const microadam_attention* t, AttentionArgs& a) {
  if (!t) return report(MICROADAM_ERR_INVALID_ARG, "attention is NULL");
  if (t->dtype != MICROADAM_F32 && t->dtype != MICROADAM_BF16)
    return report(MICROADAM_ERR_INVALID_ARG, "dtype must be F32 or BF16");
  if (t->causal != 0 && t->causal != 1) return report(MICROADAM_ERR_INVALID_ARG, "causal must be 0 or 1");
  if (t->batch < 0 || t->queries < 0 || t->keys < 0)
    return report(MICROADAM_ERR_INVALID_ARG, "batch, queries and keys must be >= 0");
  if (t->heads < 1 || t->kv_heads < 1 || t->heads % t->kv_heads)
    return report(MICROADAM_ERR_INVALID_ARG, "heads and kv_heads must be >= 1, and kv_heads divide heads");
  if (t->dim < 1) return report(MICROADAM_ERR_INVALID_ARG, "dim must be >= 1");
  if (t->dim > 128 || t->dim % 8) return report(MICROADAM_ERR_UNSUPPORTED, "dim must be a multiple of 8, at most 128");
  if (t->batch > kMaxSide || t->queries > kMaxSide || t->keys > kMaxSide || t->heads > kMaxSide ||
      (t->heads / t->kv_heads) * t->queries > kMaxSide)
    return report(MICROADAM_ERR_UNSUPPORTED, "more than 2^30 sequences, keys, or queries that share a key head");
  // (tiles of 32 are taken only where those of 128 are fewer than 512)
  const int64_t tiles = (std::max((t->heads / t->kv_heads) * t->queries, t->keys) + 127) / 128;
  if (t->batch > 0 && tiles > 0 && t->kv_heads > (kMaxGroups - 1) / t->batch / tiles)
    return report(MICROADAM_ERR_UNSUPPORTED, "sequences times key heads times tiles of 128 positions: 2^24 or more");
  const float c = (float)(t->scale * 1.4426950408889634);
  if (!(c > 0.0f) || !std::isfinite(c) || !((float)t->scale > 0.0f))
    return report(MICROADAM_ERR_INVALID_ARG, "scale must be > 0 and in the range of binary32");
  std::memset(&a, 0, sizeof(a));
  a.batch = (int32_t)t->batch;
  a.queries = (int32_t)t->queries;
  a.keys = (int32_t)t->keys;
  a.heads = (int32_t)t->heads;
  a.kv_heads = (int32_t)t->kv_heads;
  a.dim = (int32_t)t->dim;
  a.group = (int32_t)(t->heads / t->kv_heads);
  a.rows = a.group * a.queries;
  a.causal = t->causal;
  a.bf16 = t->dtype == MICROADAM_BF16;
  a.scale = (float)t->scale;
  a.c = c;
  a.lengths = t->key_lengths;
  a.parts = attention_parts(a);
  a.grad_parts = attention_grad_parts(a);
  return MICROADAM_OK;
}

struct Range {
  uintptr_t at, end;
};

// An operand's strides and address, and the bytes it reaches over.  Nothing is
// asked of one without elements.
int operand(const microadam_heads* h, int64_t batch, int64_t positions, int64_t heads, int64_t dim, int32_t dtype,
            bool written, HeadTensor& to, Range& r) {
  if (!h) return report(MICROADAM_ERR_INVALID_ARG, "an operand is NULL");
  r.at = r.end = (uintptr_t)h->data;
  to = {h->data, h->batch_stride, h->pos_stride, h->head_stride};
  if (batch == 0 || positions == 0) return MICROADAM_OK;
  if (!h->data) return report(MICROADAM_ERR_INVALID_ARG, "an operand's address is NULL");
  if ((uintptr_t)h->data % size_of(dtype))
    return report(MICROADAM_ERR_INVALID_ARG, "an operand is not aligned to its element type");
  if (positions == 1) to.pos = dim;
  std::pair<int64_t, int64_t> d[3] = {{h->batch_stride, batch}, {h->pos_stride, positions}, {h->head_stride, heads}};
  if (positions > 1 && h->pos_stride >= 0 && h->pos_stride < dim)
    return report(MICROADAM_ERR_INVALID_ARG, "a position stride is below dim");
  if (positions > 1 && h->pos_stride > kMaxPosition)
    return report(MICROADAM_ERR_UNSUPPORTED, "a position stride is above 2^23");
  int64_t reach = dim;
  for (const auto& s : d) {
    if (s.second == 1) continue;
    if (s.first < 0) return report(MICROADAM_ERR_INVALID_ARG, "strides must be >= 0");
    if (s.first > kMaxStride) return report(MICROADAM_ERR_UNSUPPORTED, "a stride is above 2^40");
    if (s.first > ((int64_t)1 << 60) / s.second)
      return report(MICROADAM_ERR_UNSUPPORTED, "an operand reaches over more than 2^60 elements");
    reach += (s.second - 1) * s.first;
  }
  if (reach > (int64_t)1 << 60) return report(MICROADAM_ERR_UNSUPPORTED, "an operand reaches over more than 2^60 elements");
  if (written) {
    std::sort(d, d + 3);
    int64_t used = dim;  // elements that what lies closer together takes
    for (const auto& s : d) {
      if (s.second == 1) continue;
      if (s.first < used) return report(MICROADAM_ERR_INVALID_ARG, "an output has elements in one place");
      used += (s.second - 1) * s.first;
    }
  }
  r.end = r.at + (uintptr_t)(reach * size_of(dtype));
  return MICROADAM_OK;
}

Range run(const void* p, int64_t bytes) { return {(uintptr_t)p, p ? (uintptr_t)p + (uintptr_t)bytes : (uintptr_t)p}; }

int check_apart(const Range* written, int n_written, const Range* read, int n_read) {
  for (int i = 0; i < n_written; ++i)
    for (int j = 0; j < i + n_read; ++j) {
      const Range& o = j < i ? written[j] : read[j - i];
      if (written[i].at < o.end && o.at < written[i].end)
        return report(MICROADAM_ERR_INVALID_ARG, "an output overlaps an input or another output");
    }
  return MICROADAM_OK;
}

uint64_t up(uint64_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

uint64_t stats_bytes(const AttentionArgs& a) { return (uint64_t)a.batch * a.heads * a.queries * sizeof(float); }

// The rows' log sums, and for bfloat16 what the rounding of out left over.
uint64_t saved_bytes(const AttentionArgs& a) {
  return up(stats_bytes(a)) + (a.bf16 ? up((uint64_t)a.batch * a.heads * a.queries * a.dim * 2) : 0);
}

void set_saved(AttentionArgs& a, const void* saved) {
  a.lse = (float*)const_cast<void*>(saved);
  a.rest = saved && a.bf16 ? (uint16_t*)((uint8_t*)const_cast<void*>(saved) + up(stats_bytes(a))) : nullptr;
}

uint64_t part_rows(const AttentionArgs& a) { return (uint64_t)a.batch * a.kv_heads * a.parts * a.rows; }

uint64_t workspace_of(const AttentionArgs& a, bool grad) {
  if (grad)
    return up(stats_bytes(a)) +
           up((uint64_t)a.grad_parts * 2 * a.batch * a.kv_heads * a.keys * a.dim * sizeof(float));
  return a.parts ? up(part_rows(a) * 2 * sizeof(float)) + up(part_rows(a) * a.dim * sizeof(float)) : 0;
}

int check_workspace(const AttentionArgs& a, bool grad, const void* workspace, uint64_t bytes) {
  const uint64_t need = workspace_of(a, grad);
  if (bytes < need) return report(MICROADAM_ERR_STATE_SIZE, "workspace smaller than microadam_attention_workspace's");
  if (need && !workspace) return report(MICROADAM_ERR_INVALID_ARG, "workspace is NULL");
  if (need && (uintptr_t)workspace % kAlign)
    return report(MICROADAM_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
  return MICROADAM_OK;
}

int check_saved(const AttentionArgs& a, const void* saved, uint64_t size) {
  if (size < saved_bytes(a)) return report(MICROADAM_ERR_STATE_SIZE, "saved is smaller than microadam_attention_saved's");
  if ((uintptr_t)saved % kAlign) return report(MICROADAM_ERR_INVALID_ARG, "saved must be 256-byte aligned");
  return MICROADAM_OK;
}

int inputs(const microadam_attention* t, AttentionArgs& a, Range* r) {
  int rc;
  const bool none = t->queries == 0;  // nothing is read
  if ((rc = operand(&t->q, t->batch, t->queries, t->heads, t->dim, t->dtype, false, a.q, r[0])) ||
      (rc = operand(&t->k, t->batch, none ? 0 : t->keys, t->kv_heads, t->dim, t->dtype, false, a.k, r[1])) ||
      (rc = operand(&t->v, t->batch, none ? 0 : t->keys, t->kv_heads, t->dim, t->dtype, false, a.v, r[2])))
    return rc;
  if ((uintptr_t)t->key_lengths % 4) return report(MICROADAM_ERR_INVALID_ARG, "key_lengths is not aligned");
  r[3] = run(t->key_lengths, t->batch * 4);
  return MICROADAM_OK;
}

}  // namespace

extern "C" {

int microadam_attention_workspace(const microadam_attention* attention, int32_t grad, uint64_t* bytes) {
  AttentionArgs a;
  const int rc = check(attention, a);
  if (rc) return rc;
  if (!bytes) return report(MICROADAM_ERR_INVALID_ARG, "bytes is NULL");
  *bytes = workspace_of(a, grad != 0);
  clear_report();
  return MICROADAM_OK;
}

int microadam_attention_saved(const microadam_attention* attention, uint64_t* bytes) {
  AttentionArgs a;
  const int rc = check(attention, a);
  if (rc) return rc;
  if (!bytes) return report(MICROADAM_ERR_INVALID_ARG, "bytes is NULL");
  *bytes = saved_bytes(a);
  clear_report();
  return MICROADAM_OK;
}

int microadam_attention_forward(const microadam_attention* attention, const microadam_heads* out, void* saved,
                                uint64_t saved_size, void* workspace, uint64_t workspace_bytes, void* stream) {
  AttentionArgs a;
  int rc = check(attention, a);
  if (rc) return rc;
  const microadam_attention& t = *attention;
  Range read[4], written[3];
  if ((rc = inputs(attention, a, read))) return rc;
  if ((rc = operand(out, t.batch, t.queries, t.heads, t.dim, t.dtype, true, a.out, written[0]))) return rc;
  if (saved && (rc = check_saved(a, saved, saved_size))) return rc;
  if ((rc = check_workspace(a, false, workspace, workspace_bytes))) return rc;
  written[1] = run(saved, (int64_t)saved_bytes(a));
  written[2] = run(workspace_of(a, false) ? workspace : nullptr, (int64_t)workspace_of(a, false));
  if ((rc = check_apart(written, 3, read, 4))) return rc;
  set_saved(a, saved);
  if (a.parts) {
    a.part_stats = (float*)workspace;
    a.part_out = (float*)((uint8_t*)workspace + up(part_rows(a) * 2 * sizeof(float)));
  }
  if (a.batch > 0 && a.rows > 0) {
    const hipError_t e = launch_attention(a, (hipStream_t)stream);
    if (e != hipSuccess) return report_hip(e, "launching attention");
  }
  clear_report();
  return MICROADAM_OK;
}

int microadam_attention_grad(const microadam_attention* attention, const microadam_heads* out, const void* saved,
                             uint64_t saved_size, const microadam_heads* dout, const microadam_heads* dq,
                             const microadam_heads* dk, const microadam_heads* dv, void* workspace,
                             uint64_t workspace_bytes, void* stream) {
  AttentionArgs a;
  int rc = check(attention, a);
  if (rc) return rc;
  const microadam_attention& t = *attention;
  Range read[7], written[4];
  if ((rc = inputs(attention, a, read)) ||
      (rc = operand(out, t.batch, t.queries, t.heads, t.dim, t.dtype, false, a.out, read[4])) ||
      (rc = operand(dout, t.batch, t.queries, t.heads, t.dim, t.dtype, false, a.dout, read[5])) ||
      (rc = operand(dq, t.batch, t.queries, t.heads, t.dim, t.dtype, true, a.dq, written[0])) ||
      (rc = operand(dk, t.batch, t.keys, t.kv_heads, t.dim, t.dtype, true, a.dk, written[1])) ||
      (rc = operand(dv, t.batch, t.keys, t.kv_heads, t.dim, t.dtype, true, a.dv, written[2])))
    return rc;
  if (saved_bytes(a) && !saved) return report(MICROADAM_ERR_INVALID_ARG, "saved is NULL");
  if ((rc = check_saved(a, saved, saved_size))) return rc;
  if ((rc = check_workspace(a, true, workspace, workspace_bytes))) return rc;
  read[6] = run(saved, (int64_t)saved_bytes(a));
  written[3] = run(workspace_of(a, true) ? workspace : nullptr, (int64_t)workspace_of(a, true));
  if ((rc = check_apart(written, 4, read, 7))) return rc;
  set_saved(a, saved);
  a.delta = (float*)workspace;
  a.grad_part = (float*)((uint8_t*)workspace + up(stats_bytes(a)));
  if (a.batch > 0) {
    const hipError_t e = launch_attention_grad(a, (hipStream_t)stream);
    if (e != hipSuccess) return report_hip(e, "launching attention's backward pass");
  }
  clear_report();
  return MICROADAM_OK;
}

}  // extern "C"
