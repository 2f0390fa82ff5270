// Layer norm over the rows of a matrix, forward and backward.
//
//   m = mean x, r = 1 / sqrt(mean (x - m)^2 + eps), h = (x - m) r, y = h w + b
//   g = dy w:  dx = r (g - mean g - h mean(g h))
//   dw = sum over rows of dy h,  db = sum over rows of dy
//
// A row stays in the registers of a group of threads (a wave, up to a whole
// workgroup), so that x is read once forward, and x and dy once backward.  The
// variance is summed from differences to the mean, and corrected by what they
// sum to: forward a mean far from zero costs no bits.  Backward the mean comes
// from memory, rounded to binary32, which moves a row's h by up to 2^-24 |m| r, less
// than its other roundings while |m| r is below 64.  (Summing the differences again
// and taking their mean from h: 3 to 8% of the backward pass, and rows above 8192
// elements spill, 82 -> 264 us for 4096 x 16384.)  Backward a group keeps its columns'
// sums of dw and db in registers over all its rows; the groups of a workgroup are
// joined in LDS, the workgroups' sums by a second kernel, each in a fixed order.
// Rows too long for registers are read once more per pass, and their dw and db
// summed by columns.
//
// The bound is memory.  16384 x 4096 bfloat16, forward and backward in turn: 125 us
// (5.4 TB/s), 49 of them forward, 4 to 5 the join.  Small matrices take a row's own
// time: 4096 x 256 binary32 5, 6 and 3 us.
#include "elements.h"
#include "layer_norm_device.h"

namespace microadam {
namespace {

template <bool BF16>
__device__ inline uint4v load_some(const void* p, int64_t at, int left) {
  uint4v q = {0, 0, 0, 0};
  if (BF16) {
    const uint16_t* e = (const uint16_t*)p + at;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < left) q[i / 2] |= (uint32_t)e[i] << (16 * (i & 1));
  } else {
    const uint32_t* e = (const uint32_t*)p + at;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < left) q[i] = e[i];
  }
  return q;
}

// Up to sixteen bytes of a row from element `at` on, zeros from `left` elements on.
template <bool BF16, bool PAST = false>
__device__ inline uint4v load_piece(const void* p, int64_t at, int left) {
  typedef Elements<BF16> E;
  if (left >= E::kPer) return PAST ? E::load_past(p, at) : E::load(p, at);
  return load_some<BF16>(p, at, left);
}

template <bool BF16>
__device__ inline void store_piece(void* p, int64_t at, int left, const float* v) {
  typedef Elements<BF16> E;
  if (left >= E::kPer) {
    E::store(p, at, E::put(v));
    return;
  }
#pragma unroll
  for (int i = 0; i < E::kPer; ++i)
    if (i < left) E::store1(p, at + i, v[i]);
}

// N elements of the weight or bias from column `at` on; `other` where there is
// none, zeros from `left` on.
template <int N>
__device__ inline void load_side(const void* p, bool bf16, int at, int left, float other, float* v) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = p ? 0.0f : other;
  if (!p) return;
  if (bf16) {
#pragma unroll
    for (int j = 0; j < N; j += 8) {
      const uint4v q = load_piece<true>(p, at + j, left - j < N - j ? left - j : N - j);
#pragma unroll
      for (int i = 0; i < 8 && j + i < N; ++i) v[j + i] = Elements<true>::get(q, i);
    }
  } else {
#pragma unroll
    for (int j = 0; j < N; j += 4) {
      const uint4v q = load_piece<false>(p, at + j, left - j);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[j + i] = Elements<false>::get(q, i);
    }
  }
}

__device__ inline void store_side(void* p, bool bf16, int at, float v) {
  if (bf16)
    Elements<true>::store1(p, at, v);
  else
    Elements<false>::store1(p, at, v);
}

// Two sums over a group of G threads (the same for all of them).  `turn`
// alternates between the two places in LDS, so that one barrier is enough.
template <int G>
struct GroupSum {
  static constexpr int kWaves = G / 64;
  float2v part[2][kWaves];
  __device__ float2v sum(float a, float b, int turn) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
      a += __shfl_xor(a, d);
      b += __shfl_xor(b, d);
    }
    if (G == 64) return float2v{a, b};
    float2v* p = part[turn & 1];
    const int wave = (threadIdx.x % G) >> 6;
    if ((threadIdx.x & 63) == 0) p[wave] = float2v{a, b};
    __syncthreads();
    float2v s = p[0];
#pragma unroll
    for (int i = 1; i < kWaves; ++i) s += p[i];
    return s;
  }
};

// A row's pieces in the registers: G threads to a row, P pieces each.  SETTLED: a
// row's last piece, where it is not whole, is loaded with what lies before it, so
// that no load waits for another, and settled when it is used.  (Forward and
// backward, bfloat16, with a load per element there: 16384 x 4004 148 instead of
// 203 us, 100000 x 100 73 instead of 108.  binary32's pieces are four elements:
// forward up to 3% more.  Backward with two pieces a thread it spills: 132 instead
// of 111.)
template <bool BF16, int P, int G, bool SETTLED>
struct Row {
  typedef Elements<BF16> E;
  uint4v q[P];
  template <bool PAST>
  __device__ void load(const void* p, int64_t from, int t, int cols) {
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int at = (i * G + t) * E::kPer, last = cols - E::kPer;
      if constexpr (!SETTLED) {
        q[i] = load_piece<BF16, PAST>(p, from + at, cols - at);
      } else {
        q[i] = uint4v{0, 0, 0, 0};
        if (last < 0)
          q[i] = load_some<BF16>(p, from + at, cols - at);
        else if (at < cols)
          q[i] = PAST ? E::load_past(p, from + (at < last ? at : last)) : E::load(p, from + (at < last ? at : last));
      }
    }
  }
  __device__ void settle(int t, int cols) {
    if (!SETTLED || cols < E::kPer) return;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int left = cols - (i * G + t) * E::kPer;
      if (left <= 0 || left >= E::kPer) continue;
      const int off = (E::kPer - left) * E::kSize;  // bytes of the elements before
      if (off & 8) q[i] = uint4v{q[i][2], q[i][3], 0, 0};
      if (off & 4) q[i] = uint4v{q[i][1], q[i][2], q[i][3], 0};
      if (BF16 && (off & 2))
        q[i] = uint4v{q[i][0] >> 16 | q[i][1] << 16, q[i][1] >> 16 | q[i][2] << 16, q[i][2] >> 16 | q[i][3] << 16, q[i][3] >> 16};
    }
  }
  __device__ float get(int i, int j) const { return E::get(q[i], j); }
};

// ... R rows of a workgroup at a time.
template <bool BF16, int P, int G, int R>
struct Shape {
  static constexpr int kRows = R, kGroup = G, kPer = Elements<BF16>::kPer;
  static constexpr int kCols = P * G * kPer;  // at most
};

template <bool BF16, int P, int G, int R, bool PAST>
__global__ __launch_bounds__(G* R) void layer_norm_kernel(const LayerNormArgs a) {
  typedef Elements<BF16> E;
  constexpr int per = E::kPer;
  __shared__ GroupSum<G> sums[R];
  GroupSum<G>& group = sums[threadIdx.x / G];
  const int t = threadIdx.x % G, cols = a.cols;
  const float over = 1.0f / (float)cols;
  // every group takes as many turns as the others: they meet at barriers
  constexpr bool kAhead = G == 256 || G == 1024;  // the next row's pieces are loaded while a row is summed
  const int64_t step = (int64_t)gridDim.x * R;
  int64_t row = (int64_t)blockIdx.x * R + threadIdx.x / G;
  Row<BF16, P, G, BF16> next;
  auto load = [&](int64_t r) { next.template load<PAST>(a.x, r < a.rows ? r * a.x_ld : 0, t, r < a.rows ? cols : 0); };
  if (kAhead) load(row);
  float w[P][per], b[P][per];
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const int at = (i * G + t) * per, left = cols - at;
    load_side<per>(a.weight, a.weight_bf16, at, left, 1.0f, w[i]);
    load_side<per>(a.bias, a.weight_bf16, at, left, 0.0f, b[i]);
  }
  for (int64_t first = (int64_t)blockIdx.x * R; first < a.rows; first += step, row += step) {
    if (!kAhead) load(row);
    Row<BF16, P, G, BF16> x = next;
    const bool live = row < a.rows;
    if (kAhead && first + step < a.rows) load(row + step);
    x.settle(t, cols);
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < P; ++i)
#pragma unroll
      for (int j = 0; j < per; ++j) sum += x.get(i, j);
    const float about = group.sum(sum, 0.0f, 0)[0] * over;
    float d1 = 0.0f, d2 = 0.0f;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int left = cols - (i * G + t) * per;
#pragma unroll
      for (int j = 0; j < per; ++j) {
        const float d = j < left ? x.get(i, j) - about : 0.0f;
        d1 += d;
        d2 = __builtin_fmaf(d, d, d2);
      }
    }
    const float2v d = group.sum(d1, d2, 1);
    const float off = d[0] * over, var = fmaxf(__builtin_fmaf(-off, off, d[1] * over), 0.0f);
    const float mean = about + off, rstd = 1.0f / sqrtf((d[1] != d[1] ? d[1] : var) + a.eps);
    if (!live) continue;
    if (a.mean && t == 0) {
      a.mean[row] = mean;
      a.rstd[row] = rstd;
    }
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int at = (i * G + t) * per;
      if (at >= cols) break;
      float v[per];
#pragma unroll
      for (int j = 0; j < per; ++j) v[j] = __builtin_fmaf(((x.get(i, j) - about) - off) * rstd, w[i][j], b[i][j]);
      store_piece<BF16>(a.y, row * a.y_ld + at, cols - at, v);
    }
  }
}

// The partial sums of a workgroup lie as its threads hold them, dw then db: sum j
// of piece i of thread t at (i per + j) G + t, so that they are written and read
// in whole lines.
template <bool BF16, int P, int G, int R, bool PAST>
__global__ __launch_bounds__(G* R) void layer_norm_grad_kernel(const LayerNormArgs a) {
  typedef Elements<BF16> E;
  constexpr int per = E::kPer, kSums = P * G * per;
  // (half of the groups' sums of dw and db)
  __shared__ float joined[R > 1 ? R / 2 * 2 * kSums : 1];
  __shared__ GroupSum<G> sums[R];
  const int which = threadIdx.x / G, t = threadIdx.x % G, cols = a.cols;
  GroupSum<G>& group = sums[which];
  const float over = 1.0f / (float)cols;
  constexpr bool kAhead = P == 1;  // (two pieces': 129 instead of 89 us)
  const int64_t step = (int64_t)gridDim.x * R;
  int64_t row = (int64_t)blockIdx.x * R + which;
  Row<BF16, P, G, BF16 && kAhead> next_x, next_dy;
  float next_mean = 0.0f, next_rstd = 0.0f;
  auto load = [&](int64_t r) {
    const bool there = r < a.rows;
    next_x.template load<PAST>(a.x, there ? r * a.x_ld : 0, t, there ? cols : 0);
    next_dy.template load<PAST>(a.dy, there ? r * a.dy_ld : 0, t, there ? cols : 0);
    next_mean = there ? a.mean[r] : 0.0f;
    next_rstd = there ? a.rstd[r] : 0.0f;
  };
  if (kAhead) load(row);
  float w[P][per], dw[P][per], db[P][per];
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const int at = (i * G + t) * per;
    load_side<per>(a.weight, a.weight_bf16, at, cols - at, 1.0f, w[i]);
#pragma unroll
    for (int j = 0; j < per; ++j) dw[i][j] = db[i][j] = 0.0f;
  }
  int turn = 0;
  for (int64_t first = (int64_t)blockIdx.x * R; first < a.rows; first += step, row += step) {
    const bool live = row < a.rows;
    if (!kAhead) load(row);
    Row<BF16, P, G, BF16 && kAhead> x = next_x, dy = next_dy;
    const float mean = next_mean, rstd = next_rstd;
    if (kAhead && first + step < a.rows) load(row + step);
    x.settle(t, cols);
    dy.settle(t, cols);
    float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
    for (int i = 0; i < P; ++i)
#pragma unroll
      for (int j = 0; j < per; ++j) {
        const float d = dy.get(i, j), h = (x.get(i, j) - mean) * rstd, g = d * w[i][j];
        dw[i][j] = __builtin_fmaf(d, h, dw[i][j]);
        db[i][j] += d;
        s1 += g;
        s2 = __builtin_fmaf(g, h, s2);
      }
    const float2v s = group.sum(s1, s2, turn++);
    if (!live || !a.dx) continue;
    const float m1 = s[0] * over, m2 = s[1] * over;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int at = (i * G + t) * per;
      if (at >= cols) break;
      float v[per];
#pragma unroll
      for (int j = 0; j < per; ++j) {
        const float h = (x.get(i, j) - mean) * rstd, g = dy.get(i, j) * w[i][j];
        v[j] = (g - m1 - h * m2) * rstd;
      }
      store_piece<BF16>(a.dx, row * a.dx_ld + at, cols - at, v);
    }
  }
  if (!a.dweight && !a.dbias) return;
#pragma unroll
  for (int half = R / 2; half > 0; half /= 2) {
    __syncthreads();
    if (which >= half && which < 2 * half) {
      float* to = joined + (which - half) * 2 * kSums + t;
#pragma unroll
      for (int i = 0; i < P * per; ++i) {
        to[i * G] = dw[i / per][i % per];
        to[kSums + i * G] = db[i / per][i % per];
      }
    }
    __syncthreads();
    if (which < half) {
      const float* from = joined + which * 2 * kSums + t;
#pragma unroll
      for (int i = 0; i < P * per; ++i) {
        dw[i / per][i % per] += from[i * G];
        db[i / per][i % per] += from[kSums + i * G];
      }
    }
  }
  if (which != 0) return;
  if (a.parts == 1) {  // one workgroup: these are the sums
#pragma unroll
    for (int i = 0; i < P * per; ++i) {
      const int c = (i / per * G + t) * per + i % per;
      if (c >= cols) continue;
      if (a.dweight) store_side(a.dweight, a.weight_bf16, c, dw[i / per][i % per]);
      if (a.dbias) store_side(a.dbias, a.weight_bf16, c, db[i / per][i % per]);
    }
    return;
  }
  float* to = a.partial + (int64_t)blockIdx.x * 2 * kSums + t;
#pragma unroll
  for (int i = 0; i < P * per; ++i) {
    to[i * G] = dw[i / per][i % per];
    to[kSums + i * G] = db[i / per][i % per];
  }
}

// The partial sums of 64 places, sixteen runs of them side by side.
constexpr int kJoinPlaces = 64, kJoinRuns = 16;

__global__ __launch_bounds__(kJoinPlaces* kJoinRuns) void join_sides_kernel(const LayerNormArgs a) {
  __shared__ float part[kJoinRuns][kJoinPlaces];
  const int n = blockIdx.x * kJoinPlaces + (threadIdx.x & 63), run = threadIdx.x >> 6;
  void* out = blockIdx.y ? a.dbias : a.dweight;
  if (!out) return;
  const float* from = a.partial + (blockIdx.y ? a.sums : 0) + n;
  float sum = 0.0f;
  if (n < a.sums) {
#pragma unroll 8
    for (int p = run; p < a.parts; p += kJoinRuns) sum += from[(int64_t)p * 2 * a.sums];
  }
  part[run][threadIdx.x & 63] = sum;
  __syncthreads();
  if (run != 0 || n >= a.sums) return;
  sum = part[0][threadIdx.x];
#pragma unroll
  for (int i = 1; i < kJoinRuns; ++i) sum += part[i][threadIdx.x];
  const int t = n & ((1 << a.group_bits) - 1), k = n >> a.group_bits;
  const int j = k & ((1 << a.per_bits) - 1), i = k >> a.per_bits;
  const int c = (((i << a.group_bits) + t) << a.per_bits) + j;
  if (c < a.cols) store_side(out, a.weight_bf16, c, sum);
}

// ------------------------------------------------- rows beyond the registers
constexpr int kLongThreads = 1024;

// (binary64: a thread adds up to 2^14 terms in a chain)
__device__ inline double long_sum(double x) {
  __shared__ double part[kLongThreads / 64];
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
  __syncthreads();  // the last sum has been read
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
  __syncthreads();
  double s = part[0];
#pragma unroll
  for (int i = 1; i < kLongThreads / 64; ++i) s += part[i];
  return s;
}

template <bool BF16>
__global__ __launch_bounds__(kLongThreads) void long_norm_kernel(const LayerNormArgs a) {
  typedef Elements<BF16> E;
  constexpr int per = E::kPer;
  const int cols = a.cols;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const int64_t from = row * a.x_ld;
    double sum = 0.0, squares = 0.0;
    for (int at = threadIdx.x * per; at < cols; at += kLongThreads * per) {
      const uint4v q = load_piece<BF16>(a.x, from + at, cols - at);
#pragma unroll
      for (int j = 0; j < per; ++j) sum += (double)E::get(q, j);
    }
    const double mean = long_sum(sum) / cols;
    for (int at = threadIdx.x * per; at < cols; at += kLongThreads * per) {
      const uint4v q = load_piece<BF16>(a.x, from + at, cols - at);
#pragma unroll
      for (int j = 0; j < per; ++j) {
        const double d = j < cols - at ? (double)E::get(q, j) - mean : 0.0;
        squares = __builtin_fma(d, d, squares);
      }
    }
    const float rstd = (float)(1.0 / sqrt(long_sum(squares) / cols + (double)a.eps));
    const float m = (float)mean;
    if (a.mean && threadIdx.x == 0) {
      a.mean[row] = m;
      a.rstd[row] = rstd;
    }
    for (int at = threadIdx.x * per; at < cols; at += kLongThreads * per) {
      const uint4v q = load_piece<BF16>(a.x, from + at, cols - at);
      float w[per], b[per], v[per];
      load_side<per>(a.weight, a.weight_bf16, at, cols - at, 1.0f, w);
      load_side<per>(a.bias, a.weight_bf16, at, cols - at, 0.0f, b);
#pragma unroll
      for (int j = 0; j < per; ++j) v[j] = __builtin_fmaf((float)((double)E::get(q, j) - mean) * rstd, w[j], b[j]);
      store_piece<BF16>(a.y, row * a.y_ld + at, cols - at, v);
    }
  }
}

template <bool BF16>
__global__ __launch_bounds__(kLongThreads) void long_norm_grad_kernel(const LayerNormArgs a) {
  typedef Elements<BF16> E;
  constexpr int per = E::kPer;
  const int cols = a.cols;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const float mean = a.mean[row], rstd = a.rstd[row];
    double s1 = 0.0, s2 = 0.0;
    for (int at = threadIdx.x * per; at < cols; at += kLongThreads * per) {
      const uint4v x = load_piece<BF16>(a.x, row * a.x_ld + at, cols - at);
      const uint4v dy = load_piece<BF16>(a.dy, row * a.dy_ld + at, cols - at);
      float w[per];
      load_side<per>(a.weight, a.weight_bf16, at, cols - at, 1.0f, w);
#pragma unroll
      for (int j = 0; j < per; ++j) {
        const float g = E::get(dy, j) * w[j];
        s1 += (double)g;
        s2 += (double)(g * ((E::get(x, j) - mean) * rstd));
      }
    }
    const float m1 = (float)(long_sum(s1) / cols), m2 = (float)(long_sum(s2) / cols);
    for (int at = threadIdx.x * per; at < cols; at += kLongThreads * per) {
      const uint4v x = load_piece<BF16>(a.x, row * a.x_ld + at, cols - at);
      const uint4v dy = load_piece<BF16>(a.dy, row * a.dy_ld + at, cols - at);
      float w[per], v[per];
      load_side<per>(a.weight, a.weight_bf16, at, cols - at, 1.0f, w);
#pragma unroll
      for (int j = 0; j < per; ++j) {
        const float h = (E::get(x, j) - mean) * rstd;
        v[j] = (E::get(dy, j) * w[j] - m1 - h * m2) * rstd;
      }
      store_piece<BF16>(a.dx, row * a.dx_ld + at, cols - at, v);
    }
  }
}

constexpr int kSideThreads = 256;

template <bool BF16>
__global__ __launch_bounds__(kSideThreads) void long_sides_kernel(const LayerNormArgs a) {
  typedef Elements<BF16> E;
  constexpr int per = E::kPer;
  const int at = (blockIdx.x * kSideThreads + threadIdx.x) * per, cols = a.cols;
  if (at >= cols) return;
  float dw[per], db[per];
#pragma unroll
  for (int j = 0; j < per; ++j) dw[j] = db[j] = 0.0f;
  for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
    const uint4v x = load_piece<BF16>(a.x, row * a.x_ld + at, cols - at);
    const uint4v dy = load_piece<BF16>(a.dy, row * a.dy_ld + at, cols - at);
    const float mean = a.mean[row], rstd = a.rstd[row];
#pragma unroll
    for (int j = 0; j < per; ++j) {
      const float d = E::get(dy, j);
      dw[j] = __builtin_fmaf(d, (E::get(x, j) - mean) * rstd, dw[j]);
      db[j] += d;
    }
  }
  float* to = a.partial + (int64_t)blockIdx.y * 2 * cols;
#pragma unroll
  for (int j = 0; j < per; ++j)
    if (at + j < cols) {
      to[at + j] = dw[j];
      to[cols + at + j] = db[j];
    }
}

// Calls f with the shape of a row's group, the smallest that holds it; false where
// none does.  Of the sizes of group, pieces and workgroup that were tried, and
// with the next row's loads ahead or not, these took the least time or nearly.
//
// Forward, 2^26 bfloat16 elements (two pieces a thread, 16 waves to a CU; 32 of one
// piece: 65536 x 512 25 instead of 31 us):
//   cols      1024  2048  4096  8192  16384
//   us        45    44    46    47    53
//   others    45-53 46-58 47-69 49-84 54-63    (one piece; four; more workgroups)
template <bool BF16, class F>
bool with_forward_shape(int64_t cols, F f) {
  constexpr int e = Elements<BF16>::kPer;
  if (cols <= 64 * e) return f(Shape<BF16, 1, 64, 4>()), true;
  if (cols <= 128 * e) return f(Shape<BF16, 2, 64, 4>()), true;
  if (cols <= 256 * e) return f(Shape<BF16, 2, 128, 1>()), true;
  if (cols <= 512 * e) return f(Shape<BF16, 2, 256, 1>()), true;
  if (cols <= 1024 * e) return f(Shape<BF16, 2, 512, 1>()), true;
  if (cols <= 2048 * e) return f(Shape<BF16, 2, 1024, 1>()), true;
  if constexpr (!BF16) {  // (as many elements as bfloat16's two pieces)
    if (cols <= 4096 * e) return f(Shape<BF16, 4, 1024, 1>()), true;
  }
  return false;
}

// Backward, with the join (one piece a thread, one workgroup of 16 waves to a CU,
// whose sums of dw and db are the fewest; longer rows two pieces, none ahead):
//   us        75    75    76    79    89
//   others    75-86 76-95 77-92 79-90 93-129   (two pieces; smaller workgroups)
template <bool BF16, class F>
bool with_backward_shape(int64_t cols, F f) {
  constexpr int e = Elements<BF16>::kPer;
  if (cols <= 64 * e) return f(Shape<BF16, 1, 64, 16>()), true;
  if (cols <= 128 * e) return f(Shape<BF16, 1, 128, 8>()), true;
  if (cols <= 256 * e) return f(Shape<BF16, 1, 256, 4>()), true;
  if (cols <= 512 * e) return f(Shape<BF16, 1, 512, 2>()), true;
  if (cols <= 1024 * e) return f(Shape<BF16, 1, 1024, 1>()), true;
  if (cols <= 2048 * e) return f(Shape<BF16, 2, 1024, 1>()), true;
  if constexpr (!BF16) {  // (as many elements as bfloat16's two pieces)
    if (cols <= 4096 * e) return f(Shape<BF16, 4, 1024, 1>()), true;
  }
  return false;
}

// Whether what a pass reads and writes, so many matrices, fills the last-level
// cache's 256 MiB: it is read past the caches then.  Forward and backward in turn,
// and each with an operator that reads its result (a product; a sum), with / without, us:
//   32768 x 4096 bfloat16  244 / 254   307 + 286 / 309 + 288
//   16384 x 4096           125 / 132   152 + 138 / 155 + 146
//    8192 x 4096            69 /  66    92 +  72 /  92 +  74   (neither is)
//    2048 x 4096            27 /  26    45 +  26 /  45 +  26
// (Results that are written past the caches: 117 for the second, but 160 + 148.)
bool past_caches(const LayerNormArgs& a, int matrices) {
  return a.rows * a.cols * (a.bf16 ? 2 : 4) * matrices >= (int64_t)256 << 20;
}

template <bool BF16, int P, int G, int R>
void forward(const LayerNormArgs& a, hipStream_t s, Shape<BF16, P, G, R>) {
  const int64_t turns = (a.rows + R - 1) / R, most = 256 * (P == 1 ? 2048 : 1024) / (G * R);
  const dim3 grid((unsigned)(turns < most ? turns : most));
  if (past_caches(a, 2))
    layer_norm_kernel<BF16, P, G, R, true><<<grid, dim3(G * R), 0, s>>>(a);
  else
    layer_norm_kernel<BF16, P, G, R, false><<<grid, dim3(G * R), 0, s>>>(a);
}

template <bool BF16, int P, int G, int R>
void backward(const LayerNormArgs& a, hipStream_t s, Shape<BF16, P, G, R>) {
  if (past_caches(a, 3))
    layer_norm_grad_kernel<BF16, P, G, R, true><<<dim3(a.parts), dim3(G * R), 0, s>>>(a);
  else
    layer_norm_grad_kernel<BF16, P, G, R, false><<<dim3(a.parts), dim3(G * R), 0, s>>>(a);
}

template <bool BF16>
void launch_forward(const LayerNormArgs& a, hipStream_t s) {
  if (with_forward_shape<BF16>(a.cols, [&](auto shape) { forward(a, s, shape); })) return;
  long_norm_kernel<BF16><<<dim3((unsigned)(a.rows < 1024 ? a.rows : 1024)), dim3(kLongThreads), 0, s>>>(a);
}

template <bool BF16>
void launch_backward(const LayerNormArgs& a, hipStream_t s) {
  if (with_backward_shape<BF16>(a.cols, [&](auto shape) { backward(a, s, shape); })) return;
  constexpr int wide = kSideThreads * Elements<BF16>::kPer;
  if (a.dweight || a.dbias)
    long_sides_kernel<BF16><<<dim3((a.cols + wide - 1) / wide, a.parts), dim3(kSideThreads), 0, s>>>(a);
  if (a.dx && a.rows > 0)
    long_norm_grad_kernel<BF16><<<dim3((unsigned)(a.rows < 1024 ? a.rows : 1024)), dim3(kLongThreads), 0, s>>>(a);
}

int bits_of(int n) {
  int b = 0;
  while (1 << b < n) ++b;
  return b;
}

}  // namespace

LayerNormSums layer_norm_sums(int64_t rows, int64_t cols, bool bf16) {
  LayerNormSums n;
  auto of = [&](auto shape) {
    typedef decltype(shape) S;
    // two turns of a workgroup at least: what it leaves costs as much as a row
    const int64_t parts = (rows + 2 * S::kRows - 1) / (2 * S::kRows);
    n.parts = (int)(parts < 1 ? 1 : parts < kNormMostParts ? parts : kNormMostParts);
    n.sums = S::kCols;
    n.group_bits = bits_of(S::kGroup);
    n.per_bits = bits_of(S::kPer);
  };
  if (bf16 ? with_backward_shape<true>(cols, of) : with_backward_shape<false>(cols, of)) return n;
  n.parts = (int)(rows < 2 ? 2 : rows < 64 ? rows : 64);  // (two: the join kernel writes the result)
  n.sums = (int)cols;
  n.group_bits = 30;
  n.per_bits = 0;
  return n;
}

hipError_t launch_layer_norm(const LayerNormArgs& a, hipStream_t s) {
  if (a.bf16)
    launch_forward<true>(a, s);
  else
    launch_forward<false>(a, s);
  return hipGetLastError();
}

hipError_t launch_layer_norm_grad(const LayerNormArgs& a, hipStream_t s) {
  if (a.bf16)
    launch_backward<true>(a, s);
  else
    launch_backward<false>(a, s);
  if ((a.dweight || a.dbias) && a.parts > 1)
    join_sides_kernel<<<dim3((a.sums + kJoinPlaces - 1) / kJoinPlaces, 2), dim3(kJoinPlaces * kJoinRuns), 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace microadam
