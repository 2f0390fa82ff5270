// Elements of binary32 or bfloat16 as the kernels beside the step take them:
// sixteen bytes at a time, in binary32 in the registers.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace microadam {

typedef uint32_t uint4v __attribute__((ext_vector_type(4)));
typedef float float2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Sixteen bytes at an address that is aligned to the element type alone (the
// memory system takes any alignment; a piece across a line costs one more).
struct __attribute__((packed, aligned(2))) Piece2 {
  uint4v q;
};
struct __attribute__((packed, aligned(4))) Piece4 {
  uint4v q;
};
typedef uint32_t piece2 __attribute__((ext_vector_type(4), aligned(2)));

// Two binary32 values as two bfloat16, rounded to nearest even.
__device__ inline uint32_t pack_bf16(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(float2v{a, b}, bf16x2));
}

template <bool BF16>
struct Elements {
  static constexpr int kPer = BF16 ? 8 : 4;  // in sixteen bytes
  static constexpr int kSize = BF16 ? 2 : 4;
  __device__ static float get(const uint4v& q, int i) {
    if (BF16) return __uint_as_float((i & 1) ? q[i / 2] & 0xffff0000u : q[i / 2] << 16);
    return __uint_as_float(q[i]);
  }
  __device__ static uint4v put(const float* v) {
    if (BF16) return uint4v{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
    return uint4v{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
  }
  __device__ static float load1(const void* p, int64_t i) {
    if (BF16) return __uint_as_float((uint32_t)((const uint16_t*)p)[i] << 16);
    return ((const float*)p)[i];
  }
  __device__ static void store1(void* p, int64_t i, float v) {
    if (BF16)
      ((uint16_t*)p)[i] = (uint16_t)pack_bf16(v, v);
    else
      ((float*)p)[i] = v;
  }
  // sixteen bytes from element i on
  __device__ static uint4v load(const void* p, int64_t i) {
    if (BF16) return ((const Piece2*)((const uint16_t*)p + i))->q;
    return ((const Piece4*)((const float*)p + i))->q;
  }
  // ... past the caches
  __device__ static uint4v load_past(const void* p, int64_t i) {
    return (uint4v)__builtin_nontemporal_load((const piece2*)((const uint8_t*)p + i * kSize));
  }
  __device__ static void store(void* p, int64_t i, const uint4v& q) {
    if (BF16)
      ((Piece2*)((uint16_t*)p + i))->q = q;
    else
      ((Piece4*)((float*)p + i))->q = q;
  }
};

}  // namespace microadam
