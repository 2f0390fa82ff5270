// Launch interface of the attention kernels.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace microadam {

// A (batch, position, head, dim) operand: elements between neighbours; dim is
// contiguous.
struct HeadTensor {
  void* at;
  int64_t batch, pos, head;
};

struct AttentionArgs {
  HeadTensor q, k, v, out, dout, dq, dk, dv;
  const int32_t* lengths;  // NULL: all keys
  int32_t batch, queries, keys, heads, kv_heads, dim;
  int32_t group;  // query heads of a key head
  int32_t rows;   // group * queries: the rows that share a key head's keys
  int32_t causal, bf16;
  float scale;
  float c;       // scale * log2(e)
  float* lse;      // [batch][heads][queries], in units of ln 2; +inf: no key; NULL forward: not wanted
  uint16_t* rest;  // with lse and bfloat16, [batch][heads][queries][dim]: out before its rounding less out
  float* delta;    // backward: sum of dout out, as lse
  // forward, with the keys split over workgroups: per part and row (maximum,
  // sum) and the unnormalised output
  float* part_out;    // [batch][kv_heads][parts][rows][dim]
  float* part_stats;  // [batch][kv_heads][parts][rows][2]
  int32_t parts;      // 0: not split
};

constexpr int kMostParts = 256;

// How many parts a forward call's keys are split into; 0: not at all.
int32_t attention_parts(const AttentionArgs& a);

hipError_t launch_attention(const AttentionArgs& a, hipStream_t s);
hipError_t launch_attention_grad(const AttentionArgs& a, hipStream_t s);

}  // namespace microadam
