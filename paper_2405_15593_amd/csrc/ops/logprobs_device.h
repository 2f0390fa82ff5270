// Launch interface of the token log-probability kernels.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace microadam {

constexpr int kMaxTopK = 64;

struct LogprobArgs {
  const void* logits;
  const int64_t* targets;
  int64_t ld, grad_ld;  // elements
  int64_t group_stride;        // of the logits; elements
  int64_t ignore_index;
  int64_t rows;
  int32_t vocab;
  int32_t top_k;
  int32_t group_rows;          // 0: rows at one stride
  float c;              // log2(e) / temperature
  float inv_t;          // 1 / temperature
  float* logp;          // each of these may be NULL
  float* entropy;
  float* top_logprobs;  // [rows][top_k]
  int64_t* top_indices;
  const float* grad_logp;
  const float* grad_entropy;  // may be NULL
  void* grad;                 // NULL: values only
};

hipError_t launch_token_logprobs(const LogprobArgs& a, bool bf16, hipStream_t s);

}  // namespace microadam
