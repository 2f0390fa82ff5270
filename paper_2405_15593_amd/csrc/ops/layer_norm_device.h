// Launch interface of the layer norm kernels.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace microadam {

constexpr int kNormMostParts = 256;  // partial sums of the weight's and bias's gradients, at most

struct LayerNormArgs {
  const void* x;
  const void* weight;  // NULL: ones
  const void* bias;    // NULL: zeros
  int64_t rows, x_ld;
  int32_t cols;
  int32_t bf16, weight_bf16;
  float eps;
  // forward
  void* y;
  int64_t y_ld;
  float* mean;  // [rows]; NULL forward: not wanted
  float* rstd;
  // backward
  const void* dy;
  int64_t dy_ld;
  void* dx;
  int64_t dx_ld;
  void* dweight;  // NULL: not wanted
  void* dbias;
  float* partial;  // [parts][2][sums]
  int32_t parts, sums, group_bits, per_bits;
};

// The partial sums of dw and db that the backward pass of this size writes: how
// many, of how many places each, and where a column's is (k_layer_norm.hip).
struct LayerNormSums {
  int32_t parts, sums, group_bits, per_bits;
};
LayerNormSums layer_norm_sums(int64_t rows, int64_t cols, bool bf16);

hipError_t launch_layer_norm(const LayerNormArgs& a, hipStream_t s);
hipError_t launch_layer_norm_grad(const LayerNormArgs& a, hipStream_t s);

}  // namespace microadam
