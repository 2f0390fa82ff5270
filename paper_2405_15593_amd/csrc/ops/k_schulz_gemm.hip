// The products of a Newton-Schulz step on the matrix cores: D = P Q^T with
// binary16 operands whose rows are contiguous along the summed dimension, and
// binary32 accumulators.
//
// A workgroup computes a T x T tile of D in K steps of 64: the P and Q tiles
// of the next step go straight from memory to LDS while the matrix
// instructions (32x32x16) of the current one run.  A row of a step is 128
// bytes; its 16-byte chunk c is kept at position c ^ (row & 7), so that the
// eight rows of a read's 128-byte phase lie on different banks.
//
// In split precision an operand is hi + lo / 2048.  The product is taken as
// three runs over K into the same accumulators: lo hi, hi lo, then, after a
// factor 1/2048, hi hi.
//
// The symmetric products compute the tiles on and below the diagonal and
// store each twice.
#include "schulz_device.h"

namespace microadam {
namespace {

typedef _Float16 half_t;
typedef half_t half4 __attribute__((ext_vector_type(4)));
typedef half_t half8 __attribute__((ext_vector_type(8)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float16v __attribute__((ext_vector_type(16)));
typedef uint32_t uint2v __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) void* lds_ptr;

__device__ inline float bf16_to_f32(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }

__device__ inline uint16_t f32_to_bf16(float x) {
  const uint32_t u = __float_as_uint(x);
  if ((u & 0x7fffffffu) > 0x7f800000u) return (uint16_t)((u >> 16) | 0x40);
  return (uint16_t)((u + 0x7fffu + ((u >> 16) & 1)) >> 16);
}

constexpr int kStep = 64;            // K elements per step
constexpr int kRowBytes = kStep * 2;

template <int T>
struct Shape;
// waves along P's rows, along Q's rows
template <>
struct Shape<256> {
  static constexpr int wp = 2, wq = 4;
};
template <>
struct Shape<128> {
  static constexpr int wp = 2, wq = 2;
};
template <>
struct Shape<64> {
  static constexpr int wp = 2, wq = 2;
};

template <int T, int PHASE>
__global__ __launch_bounds__(64 * Shape<T>::wp * Shape<T>::wq, T == 256 ? 2 : 2) void gemm_kernel(const GemmArgs a) {
  constexpr int kWaves = Shape<T>::wp * Shape<T>::wq;
  constexpr int kTP = T / Shape<T>::wp, kTQ = T / Shape<T>::wq;  // a wave's tile
  constexpr int kI = kTP / 32, kJ = kTQ / 32;
  constexpr int kOperand = T * kRowBytes;                         // bytes of an operand's step
  constexpr int kStageRow = T + 8;                                // halves per row of the staged result
  constexpr int kLds = 4 * kOperand > T * kStageRow * 2 ? 4 * kOperand : T * kStageRow * 2;
  __shared__ __align__(1024) uint8_t lds[kLds];

  // Workgroups go to the eight XCDs in turn: give each XCD one run of
  // neighbouring tiles, which share operand rows in its L2.
  const int total = a.tile_begin[a.n_groups];
  int tile;
  {
    const int x = (int)blockIdx.x & 7, y = (int)blockIdx.x >> 3;
    const int each = total >> 3, more = total & 7;
    tile = x * each + (x < more ? x : more) + y;
  }
  int gi = 0;
  while (gi + 1 < a.n_groups && tile >= a.tile_begin[gi + 1]) ++gi;
  const SchulzGroup& g = a.group[gi];
  tile -= a.tile_begin[gi];

  const int tm = (g.mp + T - 1) / T, tn = (g.np + T - 1) / T;
  constexpr bool kSym = PHASE == kGram || PHASE == kPoly;
  const int per = kSym ? tm * (tm + 1) / 2 : tm * tn;
  const int which = tile / per;
  tile -= which * per;
  const int mat = g.first + which;
  const bool swap = PHASE == kFinal && a.tall[mat];

  // tile (ti, tj) of D
  int ti, tj;
  if (kSym) {
    ti = (int)((__builtin_amdgcn_sqrtf(8.0f * (float)tile + 1.0f) - 1.0f) * 0.5f);
    while (ti * (ti + 1) / 2 > tile) --ti;
    while ((ti + 1) * (ti + 2) / 2 <= tile) ++ti;
    tj = tile - ti * (ti + 1) / 2;
  } else {
    // columns of tiles along the longer dimension, so that a run of tiles
    // shares its rows of X^T and walks over B
    ti = tile % tm;
    tj = tile / tm;
  }

  uint8_t* rec = a.ws + g.base + (uint64_t)which * g.record;
  const uint64_t plane_x = (uint64_t)g.mp * g.np * 2, plane_a = (uint64_t)g.mp * g.mp * 2;
  const uint64_t xt_bytes = plane_x << a.split;
  const uint8_t* xt = rec + g.xt + (a.buffer ? xt_bytes : 0);
  const uint8_t *p, *q;
  uint64_t plane_p, plane_q;
  int ld, rows_p, rows_q;  // ld: halves per row, also the summed length
  if (PHASE == kGram) {
    p = q = rec + g.x;
    plane_p = plane_q = plane_x;
    ld = g.np;
    rows_p = rows_q = g.mp;
  } else if (PHASE == kPoly) {
    p = q = rec + g.a;
    plane_p = plane_q = plane_a;
    ld = g.mp;
    rows_p = rows_q = g.mp;
  } else {
    p = swap ? xt : rec + g.b;
    q = swap ? rec + g.b : xt;
    plane_p = swap ? plane_x : plane_a;
    plane_q = swap ? plane_a : plane_x;
    ld = g.mp;
    rows_p = swap ? g.np : g.mp;
    rows_q = swap ? g.mp : g.np;
  }
  if (swap) {
    const int t = ti;
    ti = tj;
    tj = t;
  }
  const int p0 = ti * T, q0 = tj * T;
  const int left_p = rows_p - p0 < T ? rows_p - p0 : T, left_q = rows_q - q0 < T ? rows_q - q0 : T;

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int wp0 = (wave % Shape<T>::wp) * kTP, wq0 = (wave / Shape<T>::wp) * kTQ;

  // rows past the operand read as zeros (the resource's size)
  const uint32_t row_bytes = (uint32_t)ld * 2;
  const uint8_t* tp = p + (uint64_t)p0 * row_bytes;
  const uint8_t* tq = q + (uint64_t)q0 * row_bytes;
  const int size_p = (int)((uint32_t)left_p * row_bytes), size_q = (int)((uint32_t)left_q * row_bytes);
  auto rp = __builtin_amdgcn_make_buffer_rsrc((void*)tp, 0, size_p, 0x00020000);
  auto rq = __builtin_amdgcn_make_buffer_rsrc((void*)tq, 0, size_q, 0x00020000);
  auto rp2 = __builtin_amdgcn_make_buffer_rsrc((void*)(tp + (a.split ? plane_p : 0)), 0, size_p, 0x00020000);
  auto rq2 = __builtin_amdgcn_make_buffer_rsrc((void*)(tq + (a.split ? plane_q : 0)), 0, size_q, 0x00020000);
  const int voff = (lane >> 3) * (int)row_bytes + ((lane & 7) ^ (lane >> 3)) * 16;
  const int ksteps = ld / kStep;
  const int steps = a.split ? 3 * ksteps : ksteps;

  auto load = [&](int s, int buf) {
    int k = s;
    int part = 2;
    if (a.split) {
      part = s >= 2 * ksteps ? 2 : s >= ksteps ? 1 : 0;
      k = s - part * ksteps;
    }
    uint8_t* dst = lds + buf * 2 * kOperand;
#pragma unroll
    for (int i = 0; i < T / 8 / kWaves; ++i) {
      const int c = i * kWaves + wave;
      const int soff = c * 8 * (int)row_bytes + k * kRowBytes;
      if (part == 0)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rp2, (lds_ptr)(dst + c * 1024), 16, voff, soff, 0, 0);
      else
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rp, (lds_ptr)(dst + c * 1024), 16, voff, soff, 0, 0);
      if (part == 1)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rq2, (lds_ptr)(dst + kOperand + c * 1024), 16, voff, soff, 0, 0);
      else
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rq, (lds_ptr)(dst + kOperand + c * 1024), 16, voff, soff, 0, 0);
    }
  };

  float16v acc[kI][kJ];
#pragma unroll
  for (int i = 0; i < kI; ++i)
#pragma unroll
    for (int j = 0; j < kJ; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;

  load(0, 0);
  for (int s = 0; s < steps; ++s) {
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): this wave's loads of step s
    __syncthreads();
    if (s + 1 < steps) load(s + 1, (s + 1) & 1);
    const uint8_t* b = lds + (s & 1) * 2 * kOperand;
    if (a.split && s == 2 * ksteps) {
#pragma unroll
      for (int i = 0; i < kI; ++i)
#pragma unroll
        for (int j = 0; j < kJ; ++j) acc[i][j] *= 1.0f / kSplitScale;
    }
#pragma unroll
    for (int kk = 0; kk < kStep / 16; ++kk) {
      half8 fp[kI], fq[kJ];
      const int off = (lane & 31) * kRowBytes + (((kk * 2 + (lane >> 5)) ^ (lane & 7)) * 16);
#pragma unroll
      for (int i = 0; i < kI; ++i) fp[i] = *(const half8*)(b + off + (wp0 + i * 32) * kRowBytes);
#pragma unroll
      for (int j = 0; j < kJ; ++j) fq[j] = *(const half8*)(b + kOperand + off + (wq0 + j * 32) * kRowBytes);
#pragma unroll
      for (int i = 0; i < kI; ++i)
#pragma unroll
        for (int j = 0; j < kJ; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(fq[j], fp[i], acc[i][j], 0, 0, 0);
    }
  }

  // Element 4 e + r of acc[i][j] is D at row (of the wave's tile) i * 32 +
  // lane % 32 and column j * 32 + 8 e + 4 (lane / 32) + r.
  const int lrow = lane & 31, lcol = (lane >> 5) * 4;

  if constexpr (PHASE == kFinal) {
    const OutMatrix& om = a.mat[mat];
    const int out_rows = swap ? g.n : g.m, out_cols = swap ? g.m : g.n;
    const float f = om.scale * (1.0f / (kScaleA * kScaleX));
#pragma unroll
    for (int i = 0; i < kI; ++i) {
      const int row = p0 + wp0 + i * 32 + lrow;
      if (row >= out_rows) continue;
#pragma unroll
      for (int j = 0; j < kJ; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int col = q0 + wq0 + j * 32 + e * 8 + lcol;
          const int64_t at = (int64_t)row * om.out_ld + col;
          float v[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) v[r] = acc[i][j][4 * e + r] * f;
          if (a.out_bf16) {
            uint16_t* o = (uint16_t*)om.out + at;
            if (col + 4 <= out_cols && ((uintptr_t)o & 7) == 0) {
              if (a.update) {
                const uint2v w = *(const uint2v*)o;
                v[0] = a.decay * __uint_as_float(w[0] << 16) - v[0];
                v[1] = a.decay * __uint_as_float(w[0] & 0xffff0000u) - v[1];
                v[2] = a.decay * __uint_as_float(w[1] << 16) - v[2];
                v[3] = a.decay * __uint_as_float(w[1] & 0xffff0000u) - v[3];
              }
              uint2v w;
              w[0] = (uint32_t)f32_to_bf16(v[0]) | ((uint32_t)f32_to_bf16(v[1]) << 16);
              w[1] = (uint32_t)f32_to_bf16(v[2]) | ((uint32_t)f32_to_bf16(v[3]) << 16);
              *(uint2v*)o = w;
            } else {
#pragma unroll
              for (int r = 0; r < 4; ++r)
                if (col + r < out_cols) o[r] = f32_to_bf16(a.update ? a.decay * bf16_to_f32(o[r]) - v[r] : v[r]);
            }
          } else {
            float* o = (float*)om.out + at;
            if (col + 4 <= out_cols && ((uintptr_t)o & 15) == 0) {
              if (a.update) {
                const float4v w = *(const float4v*)o;
#pragma unroll
                for (int r = 0; r < 4; ++r) v[r] = a.decay * w[r] - v[r];
              }
              *(float4v*)o = float4v{v[0], v[1], v[2], v[3]};
            } else {
#pragma unroll
              for (int r = 0; r < 4; ++r)
                if (col + r < out_cols) o[r] = a.update ? a.decay * o[r] - v[r] : v[r];
            }
          }
        }
    }
  } else {
    if constexpr (PHASE == kPoly) {
      // b A + c D + a I, at the stored scale
      const half_t* am = (const half_t*)(rec + g.a);
#pragma unroll
      for (int i = 0; i < kI; ++i) {
        const int row = p0 + wp0 + i * 32 + lrow;
#pragma unroll
        for (int j = 0; j < kJ; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int col = q0 + wq0 + j * 32 + e * 8 + lcol;
            if (row >= g.mp || col >= g.mp) continue;
            const half4 h = *(const half4*)(am + (int64_t)row * g.mp + col);
            half4 l = {};
            if (a.split) l = *(const half4*)(am + (int64_t)g.mp * g.mp + (int64_t)row * g.mp + col);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              float v = (float)h[r];
              if (a.split) v += (float)l[r] * (1.0f / kSplitScale);
              acc[i][j][4 * e + r] = a.cb * v + a.cc * acc[i][j][4 * e + r] + (row == col + r ? a.ca : 0.0f);
            }
          }
      }
    } else {
      const float f = PHASE == kGram ? kScaleA / (kScaleX * kScaleX) : 1.0f / kScaleA;
#pragma unroll
      for (int i = 0; i < kI; ++i)
#pragma unroll
        for (int j = 0; j < kJ; ++j) acc[i][j] *= f;
    }
    // D at (p0, q0) of an array with rows of `width`, or its transpose at
    // (q0, p0), staged in LDS so that rows are stored whole
    half_t* const stage = (half_t*)lds;
    auto store = [&](uint8_t* dst, int width, int height, bool flip, int plane) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kI; ++i)
#pragma unroll
        for (int j = 0; j < kJ; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            half4 h;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const float v = acc[i][j][4 * e + r];
              h[r] = (half_t)v;
              if (plane) h[r] = (half_t)((v - (float)h[r]) * kSplitScale);
            }
            const int row = wp0 + i * 32 + lrow, col = wq0 + j * 32 + e * 8 + lcol;
            if (flip) {
#pragma unroll
              for (int r = 0; r < 4; ++r) stage[(col + r) * kStageRow + row] = h[r];
            } else {
              *(half4*)(stage + row * kStageRow + col) = h;
            }
          }
      __syncthreads();
      const int r0 = flip ? q0 : p0, c0 = flip ? p0 : q0;
      half_t* d = (half_t*)dst + (int64_t)r0 * width + c0;
      for (int c = threadIdx.x; c < T * (T / 8); c += 64 * kWaves) {
        const int row = c / (T / 8), col = (c % (T / 8)) * 8;
        if (r0 + row < height && c0 + col < width)
          *(half8*)(d + (int64_t)row * width + col) = *(const half8*)(stage + row * kStageRow + col);
      }
    };
    for (int pl = 0; pl <= a.split; ++pl) {
      if constexpr (kSym) {
        uint8_t* dst = rec + (PHASE == kGram ? g.a : g.b) + (pl ? plane_a : 0);
        store(dst, g.mp, g.mp, false, pl);
        if (ti != tj) store(dst, g.mp, g.mp, true, pl);
      } else {
        store(rec + g.x + (pl ? plane_x : 0), g.np, g.mp, false, pl);
        store(rec + g.xt + (a.buffer ? 0 : xt_bytes) + (pl ? plane_x : 0), g.mp, g.np, true, pl);
      }
    }
  }
}

template <int T>
hipError_t launch(const GemmArgs& a, SchulzPhase phase, hipStream_t s) {
  const unsigned n = (unsigned)a.tile_begin[a.n_groups];
  constexpr int threads = 64 * Shape<T>::wp * Shape<T>::wq;
  switch (phase) {
    case kGram: gemm_kernel<T, kGram><<<n, threads, 0, s>>>(a); break;
    case kPoly: gemm_kernel<T, kPoly><<<n, threads, 0, s>>>(a); break;
    case kApply: gemm_kernel<T, kApply><<<n, threads, 0, s>>>(a); break;
    case kFinal: gemm_kernel<T, kFinal><<<n, threads, 0, s>>>(a); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace

int64_t schulz_tiles(const SchulzGroup& g, SchulzPhase phase, int tile) {
  const int64_t tm = (g.mp + tile - 1) / tile, tn = (g.np + tile - 1) / tile;
  return (phase == kGram || phase == kPoly ? tm * (tm + 1) / 2 : tm * tn) * g.count;
}

hipError_t launch_schulz_gemm(GemmArgs& a, SchulzPhase phase, int tile, hipStream_t s) {
  if (a.n_groups < 1 || a.n_groups > kMaxGroups) return hipErrorInvalidValue;
  int64_t total = 0;
  for (int i = 0; i < a.n_groups; ++i) {
    a.tile_begin[i] = (int32_t)total;
    total += schulz_tiles(a.group[i], phase, tile);
    if (total >= ((int64_t)1 << 24)) return hipErrorInvalidValue;
  }
  a.tile_begin[a.n_groups] = (int32_t)total;
  switch (tile) {
    case 64: return launch<64>(a, phase, s);
    case 128: return launch<128>(a, phase, s);
    case 256: return launch<256>(a, phase, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace microadam
