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
  // backward, with the rows that see a key split over workgroups: dk and dv of each
  // part, without dk's scale
  float* grad_part;    // [grad_parts][2][batch][kv_heads][keys][dim]
  int32_t grad_parts;  // 0: not split
};

constexpr int kMostParts = 256;

// Whether 128 rows (or keys) to a workgroup are too few workgroups for 256 CUs, so
// that its four waves had better share 32 of them and take every fourth tile of
// the others.  One workgroup to a CU, two for binary32, whose matrix instructions
// leave no time over, and some more for causal ones of short rows and many keys, of
// which the longest would be waited for.  Forward / backward in us, shared or not:
//   bfloat16  1 x 2048 x 8 heads of 128, causal  128 workgroups  29 / 117  48 / 163
//             2 x  512 x 32           "          256             26 / 104  20 / 60
//   binary32  4 x 1024 x 8 heads of 64, causal   256             54 / 193  86 / 267
//             32 x 512 x 4            "          512             64 / 257  60 / 196
//   bfloat16  1 x 2048 x 16 heads of 64, causal  256             30 / 77   35 / 103
//             1 x 4096 x 10           "          320             59 / 160  63 / 162
//             3 x 1024 x 16           "          384             25 / 72   22 / 64
//             4 x  512 x 16           "          256             16 / 38   13 / 36
// (Shared ones of bfloat16 multiply what the rounding of p and ds leaves over too, a
// tenth of their time.)
inline bool few_groups(const AttentionArgs& a, int positions) {
  const bool uneven = a.causal && a.dim <= 64 && a.keys >= 1024 && a.queries >= a.keys / 2;
  const int enough = !a.bf16 ? 512 : uneven ? 321 : 256;
  return (int64_t)((positions + 127) / 128) * a.kv_heads * a.batch < enough;
}

// Whether the rows go to the kernel without matrix products.
constexpr int kTokenRows = 8;
inline bool token_rows(const AttentionArgs& a) { return !a.bf16 && a.rows <= kTokenRows; }

// Whether keys and values, which a few rows' call reads once, are read past the
// caches: where they fill the last-level cache's 256 MiB alone (fewer may be there
// still from the call before) and a load takes whole lines of 128 bytes.  One query
// of 32 heads on 8, with / without, us:
//   bfloat16  64 x 2048 keys of 128 (537 MB)  88 / 99    131072 (537 MB)  94 / 104
//             8 x 4096, lengths (67 of 134 MB)  cold 23.0 / 24.8, else 24.6 / 20.8
//             8 x 8192 of 80 (lines shared with other heads)  40 / 38
//   binary32  32768 of 128 (268 MB)  51 / 56             4 x 16384, lengths  46 / 49
inline bool past_caches(const AttentionArgs& a) {
  const int size = a.bf16 ? 2 : 4;
  return a.dim >= 64 && a.dim * size % 128 == 0 &&
         (int64_t)a.batch * a.kv_heads * a.keys * a.dim * 2 * size >= (int64_t)256 << 20;
}

void launch_attention_token(const AttentionArgs& a, hipStream_t s);

// How many parts a forward call's keys are split into; 0: not at all.
int32_t attention_parts(const AttentionArgs& a);

// How many parts the backward call's rows are split into for dk and dv; 0: not at all.
int32_t attention_grad_parts(const AttentionArgs& a);

hipError_t launch_attention(const AttentionArgs& a, hipStream_t s);
hipError_t launch_attention_grad(const AttentionArgs& a, hipStream_t s);

}  // namespace microadam
