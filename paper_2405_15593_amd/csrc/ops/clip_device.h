// Launch interface of the gradient norm and clipping kernels.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace microadam {

constexpr int kClipTensors = 160;             // of a launch, whose table is a kernel argument
constexpr int kClipSlots = 1024;              // partial sums: workgroups of a launch, at most
constexpr int64_t kClipChunk = 32768;         // bytes that a workgroup takes at a time
constexpr int64_t kClipMost = (int64_t)1 << 29;  // chunks of a launch

struct ClipArgs {
  // A tensor's address, with bit 0 set for bfloat16 (an address is even), its
  // last byte's successor, and its first chunk's number.  Chunks are counted
  // from the address rounded down to 16 bytes.
  uint64_t at[kClipTensors];
  uint64_t end[kClipTensors];
  int32_t first[kClipTensors + 1];
  int32_t n;
  double* partial;  // kClipSlots, then the norm where `past`
  int32_t slots;    // in use
  int32_t past;     // the whole list is more than the caches hold
  int32_t add;      // to what an earlier launch of the call left there
  double max_norm, eps;
  float* norm;  // NULL: not this launch's to write
};

hipError_t launch_square_sums(const ClipArgs& a, hipStream_t s);  // slots workgroups
hipError_t launch_grad_norm(const ClipArgs& a, hipStream_t s);
hipError_t launch_scale_grads(const ClipArgs& a, hipStream_t s);

}  // namespace microadam
