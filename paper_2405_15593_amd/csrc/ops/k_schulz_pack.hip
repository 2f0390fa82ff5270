// The two passes before the Newton-Schulz products: the Frobenius norm of
// each matrix's update, then the update itself, normalised, as the binary16
// iterate, transposed.
//
//   V' = mu V + (1 - mu) G;  U = mu V' + (1 - mu) G (Nesterov) or V';
//   without momentum U = G.      X = S_X U / (||U||_F + eps)
//
// Both passes are bound by memory: they read G and V twice and write V'
// and X^T once.  U is not kept between them (it would have to be written and
// read again), and the squares are summed in binary64, so neither tiny nor
// huge gradients leave the range.  Every sum has a fixed order.  72 matrices of
// BERT-base's shapes (85 M elements, bf16 gradients, binary32 momenta): 100 us
// for the norms (5.1 TB/s) and 174 us for the packing (5.9 TB/s).
#include "schulz_device.h"

namespace microadam {
namespace {

typedef _Float16 half_t;
typedef half_t half4 __attribute__((ext_vector_type(4)));
typedef half_t half8 __attribute__((ext_vector_type(8)));
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));
typedef float float4v __attribute__((ext_vector_type(4)));

__device__ inline float bf16_to_f32(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }

__device__ inline uint16_t f32_to_bf16(float x) {
  const uint32_t u = __float_as_uint(x);
  if ((u & 0x7fffffffu) > 0x7f800000u) return (uint16_t)((u >> 16) | 0x40);
  return (uint16_t)((u + 0x7fffu + ((u >> 16) & 1)) >> 16);
}

// Up to eight elements of a row at element offset `at`, zeros past `count`.
// A 16-byte aligned address is read in vectors where all eight exist.
__device__ inline void load8(const void* base, int64_t at, int count, bool bf16, float* v) {
  if (bf16) {
    const uint16_t* p = (const uint16_t*)base + at;
    if (count >= 8 && ((uintptr_t)p & 15) == 0) {
      const uint4v q = *(const uint4v*)p;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(q[i] << 16);
        v[2 * i + 1] = __uint_as_float(q[i] & 0xffff0000u);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = i < count ? bf16_to_f32(p[i]) : 0.0f;
    }
  } else {
    const float* p = (const float*)base + at;
    if (count >= 8 && ((uintptr_t)p & 15) == 0) {
      const float4v q0 = *(const float4v*)p, q1 = *(const float4v*)(p + 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[i] = q0[i];
        v[4 + i] = q1[i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = i < count ? p[i] : 0.0f;
    }
  }
}

__device__ inline void store8(void* base, int64_t at, int count, bool bf16, const float* v) {
  if (bf16) {
    uint16_t* p = (uint16_t*)base + at;
    if (count >= 8 && ((uintptr_t)p & 15) == 0) {
      uint4v q;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        q[i] = (uint32_t)f32_to_bf16(v[2 * i]) | ((uint32_t)f32_to_bf16(v[2 * i + 1]) << 16);
      *(uint4v*)p = q;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < count) p[i] = f32_to_bf16(v[i]);
    }
  } else {
    float* p = (float*)base + at;
    if (count >= 8 && ((uintptr_t)p & 15) == 0) {
      *(float4v*)p = float4v{v[0], v[1], v[2], v[3]};
      *(float4v*)(p + 4) = float4v{v[4], v[5], v[6], v[7]};
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < count) p[i] = v[i];
    }
  }
}

// The update of eight elements; v8 becomes the new momentum.
__device__ inline void update8(const PackArgs& a, const float* g8, float* v8, bool momentum, float* u8) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (!momentum) {
      u8[i] = g8[i];
      continue;
    }
    v8[i] = a.mu * v8[i] + a.one_minus_mu * g8[i];
    u8[i] = a.nesterov ? a.mu * v8[i] + a.one_minus_mu * g8[i] : v8[i];
  }
}

__device__ inline double wave_sum(double x) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
  return x;
}

// grid: (n_parts, matrices); part b takes every n_parts-th run of eight.
__global__ __launch_bounds__(256) void norm_kernel(const PackArgs a) {
  const int mat = blockIdx.y;
  const SchulzGroup& g = a.group[a.of[mat]];
  const bool tall = a.tall[mat];
  const int rows = tall ? g.n : g.m, cols = tall ? g.m : g.n;
  const PackMatrix& pm = a.mat[mat];
  const bool momentum = pm.momentum != nullptr;
  const uint32_t runs = (uint32_t)(cols + 7) / 8;
  const int64_t total = (int64_t)runs * rows;
  double sum = 0.0;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)a.n_parts * 256) {
    const int64_t row = total < ((int64_t)1 << 32) ? (int64_t)((uint32_t)i / runs) : i / runs;
    const int col = (int)(i - row * runs) * 8;
    const int count = cols - col;
    float g8[8], v8[8], u8[8];
    load8(pm.grad, row * pm.grad_ld + col, count, a.grad_bf16, g8);
    if (momentum) load8(pm.momentum, row * pm.momentum_ld + col, count, a.momentum_bf16, v8);
    update8(a, g8, v8, momentum, u8);
#pragma unroll
    for (int k = 0; k < 8; ++k) sum += (double)u8[k] * (double)u8[k];
  }
  __shared__ double part[4];
  sum = wave_sum(sum);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) a.partials[mat * kNormParts + blockIdx.x] = (part[0] + part[1]) + (part[2] + part[3]);
}

constexpr int kLdsRow = 64 + 8;  // halves per staged row: 16-byte aligned, off by 16 bytes per row

// grid: (64 x 64 tiles of the largest padded matrix, matrices).
__global__ __launch_bounds__(256) void pack_kernel(const PackArgs a) {
  // the matrices that the norm pass read last first: the memory side's cache
  // still holds them (192 -> 174 us)
  const int mat = (int)(gridDim.y - 1 - blockIdx.y);
  const SchulzGroup& g = a.group[a.of[mat]];
  const bool tall = a.tall[mat];
  const int rows = tall ? g.n : g.m, cols = tall ? g.m : g.n;
  const int rows_p = tall ? g.np : g.mp, cols_p = tall ? g.mp : g.np;
  const int tiles_c = cols_p / 64;
  if ((int64_t)blockIdx.x >= (int64_t)tiles_c * (rows_p / 64)) return;  // the whole workgroup
  const int r0 = (int)(blockIdx.x / tiles_c) * 64, c0 = (int)(blockIdx.x % tiles_c) * 64;

  __shared__ double part[4];
  __shared__ __align__(16) half_t stage[2][64 * kLdsRow];
  const PackMatrix& pm = a.mat[mat];
  const bool momentum = pm.momentum != nullptr;
  // the elements are fetched before the norm is put together
  float g8[2][8], v8[2][8];
#pragma unroll
  for (int it = 0; it < 2; ++it) {
    const int row = r0 + (int)(threadIdx.x >> 3) + it * 32, col = c0 + (int)(threadIdx.x & 7) * 8;
    const int count = row < rows ? cols - col : 0;
    if (count > 0) {
      load8(pm.grad, (int64_t)row * pm.grad_ld + col, count, a.grad_bf16, g8[it]);
      if (momentum) load8(pm.momentum, (int64_t)row * pm.momentum_ld + col, count, a.momentum_bf16, v8[it]);
    }
  }

  double sum = (int)threadIdx.x < a.n_parts ? a.partials[mat * kNormParts + threadIdx.x] : 0.0;
  sum = wave_sum(sum);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
  __syncthreads();
  const double scale = (double)kScaleX / (sqrt((part[0] + part[1]) + (part[2] + part[3])) + a.eps);

  uint8_t* rec = a.ws + g.base + (uint64_t)(mat - g.first) * g.record;
  // a tall matrix lies as X^T does; another is turned in LDS
  half_t* xt = (half_t*)(rec + g.xt);
  const int64_t plane = (int64_t)g.mp * g.np;

#pragma unroll
  for (int it = 0; it < 2; ++it) {
    const int r = (int)(threadIdx.x >> 3) + it * 32, c = (int)(threadIdx.x & 7) * 8;
    const int row = r0 + r, col = c0 + c;
    half8 hi, lo;
#pragma unroll
    for (int i = 0; i < 8; ++i) hi[i] = lo[i] = (half_t)0.0f;
    const int count = row < rows ? cols - col : 0;
    if (count > 0) {
      float u8[8];
      update8(a, g8[it], v8[it], momentum, u8);
      if (momentum) store8(pm.momentum, (int64_t)row * pm.momentum_ld + col, count, a.momentum_bf16, v8[it]);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float x = (float)((double)u8[i] * scale);
        hi[i] = (half_t)x;
        lo[i] = (half_t)((x - (float)hi[i]) * kSplitScale);
      }
    }
    if (tall) {
      *(half8*)(xt + (int64_t)row * cols_p + col) = hi;
      if (a.split) *(half8*)(xt + plane + (int64_t)row * cols_p + col) = lo;
    } else {
      *(half8*)&stage[0][r * kLdsRow + c] = hi;
      if (a.split) *(half8*)&stage[1][r * kLdsRow + c] = lo;
    }
  }
  if (tall) return;
  __syncthreads();
  for (int p = 0; p <= (a.split ? 1 : 0); ++p) {
#pragma unroll
    for (int it = 0; it < 2; ++it) {
      const int c = (int)(threadIdx.x >> 3) + it * 32, r = (int)(threadIdx.x & 7) * 8;
      half8 v;
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = stage[p][(r + i) * kLdsRow + c];
      *(half8*)(xt + p * plane + (int64_t)(c0 + c) * g.mp + r0 + r) = v;
    }
  }
}

// A 64 x 64 tile of A from the sums of its K's parts, in a fixed order; four
// workgroups take 16 rows each, and each quarter of a workgroup every fourth
// part.  grid: (4 x tiles of the group with most, matrices).
__global__ __launch_bounds__(1024) void join_kernel(const GemmArgs a) {
  int gi = 0;
  while (gi + 1 < a.n_groups && (int)blockIdx.y >= a.group[gi + 1].first) ++gi;
  const SchulzGroup& g = a.group[gi];
  const int parts = a.parts[gi];
  constexpr int T = 64;
  const int tm = g.mp / T, per = tm * (tm + 1) / 2;
  const int tile = (int)blockIdx.x >> 2, r0 = ((int)blockIdx.x & 3) * 16;
  if (parts == 1 || tile >= per) return;
  int ti, tj;
  symmetric_tile(tile, tm, ti, tj);

  uint8_t* rec = a.ws + g.base + (uint64_t)((int)blockIdx.y - g.first) * g.record;
  const uint64_t xt_bytes = (uint64_t)g.mp * g.np * (a.split ? 4 : 2);
  const int quarter = (int)threadIdx.x >> 8, t = (int)threadIdx.x & 255;
  const int row = r0 + (t >> 4), col = (t & 15) * 4;
  const int64_t plane = (int64_t)g.mp * g.mp, at = (int64_t)(ti * T + row) * g.mp + tj * T + col;
  const float* sums = (const float*)(rec + g.xt + (a.buffer ? 0 : xt_bytes)) + at;
  float4v sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 8
  for (int p = quarter; p < parts; p += 4) sum += *(const float4v*)(sums + p * plane);
  __shared__ float4v quarters[3][256];
  __shared__ half_t stage[2][T][16 + 2];
  if (quarter) quarters[quarter - 1][t] = sum;
  __syncthreads();
  half_t* out = (half_t*)(rec + g.a);
  if (!quarter) {
    sum = (sum + quarters[0][t]) + (quarters[1][t] + quarters[2][t]);
    // rounded once (and what that left)
    half4 hi, lo;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float v = sum[i] * (kScaleA / (kScaleX * kScaleX));
      hi[i] = (half_t)v;
      lo[i] = (half_t)((v - (float)hi[i]) * kSplitScale);
      stage[0][col + i][row - r0] = hi[i];
      stage[1][col + i][row - r0] = lo[i];
    }
    *(half4*)(out + at) = hi;
    if (a.split) *(half4*)(out + plane + at) = lo;
  }
  if (ti == tj) return;  // the whole workgroup
  __syncthreads();
  if (quarter) return;
  const int c = t >> 2, r = (t & 3) * 4;
  for (int p = 0; p <= (a.split ? 1 : 0); ++p) {
    half4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = stage[p][c][r + i];
    *(half4*)(out + p * plane + (int64_t)(tj * T + c) * g.mp + ti * T + r0 + r) = v;
  }
}

}  // namespace

hipError_t launch_schulz_norm(const PackArgs& a, int n_matrices, hipStream_t s) {
  if (n_matrices < 1 || n_matrices > kMaxMatrices || a.n_parts < 1 || a.n_parts > kNormParts)
    return hipErrorInvalidValue;
  norm_kernel<<<dim3((unsigned)a.n_parts, (unsigned)n_matrices), 256, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_schulz_pack(const PackArgs& a, int n_matrices, hipStream_t s) {
  if (n_matrices < 1 || n_matrices > kMaxMatrices) return hipErrorInvalidValue;
  int64_t tiles = 0;
  for (int i = 0; i < a.n_groups; ++i) {
    const int64_t t = (int64_t)(a.group[i].mp / 64) * (a.group[i].np / 64);
    if (t > tiles) tiles = t;
  }
  if (tiles >= ((int64_t)1 << 24)) return hipErrorInvalidValue;
  pack_kernel<<<dim3((unsigned)tiles, (unsigned)n_matrices), 256, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_schulz_join(const GemmArgs& a, hipStream_t s) {
  if (a.n_groups < 1 || a.n_groups > kMaxGroups) return hipErrorInvalidValue;
  int64_t tiles = 0;
  int matrices = 0;
  for (int i = 0; i < a.n_groups; ++i) {
    const int64_t tm = a.group[i].mp / 64;
    if (a.parts[i] > 1) tiles = tm * (tm + 1) / 2 > tiles ? tm * (tm + 1) / 2 : tiles;
    matrices = a.group[i].first + a.group[i].count;
  }
  if (tiles == 0) return hipSuccess;
  if (4 * tiles >= kMaxTiles || matrices > kMaxMatrices) return hipErrorInvalidValue;
  join_kernel<<<dim3((unsigned)(4 * tiles), (unsigned)matrices), 1024, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace microadam
