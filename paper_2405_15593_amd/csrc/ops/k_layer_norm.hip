// Layer norm over the rows of a matrix, forward and backward.
//
//   m = mean x, r = 1 / sqrt(mean (x - m)^2 + eps), h = (x - m) r, y = h w + b
//   g = dy w:  dx = r (g - mean g - h mean(g h))
//   dw = sum over rows of dy h,  db = sum over rows of dy
//
// A row stays in the registers of a group of threads (a wave, up to a whole
// workgroup), so that x is read once forward, and x and dy once backward.  The
// variance is summed from differences to the mean, and corrected by what they
// sum to: a mean far from zero costs no bits.  Backward a group keeps its
// columns' sums of dw and db in registers over all its rows; the groups of a
// workgroup are joined in LDS, the workgroups' sums by a second kernel, each in
// a fixed order.  Rows too long for registers are read once more per pass, and
// their dw and db summed by columns.
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
template <bool BF16>
__device__ inline uint4v load_piece(const void* p, int64_t at, int left) {
  if (left >= Elements<BF16>::kPer) return Elements<BF16>::load(p, at);
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

// G threads to a row, P pieces of it each, R rows of a workgroup at a time.
template <bool BF16, int P, int G, int R>
struct Shape {
  typedef Elements<BF16> E;
  static constexpr int kPer = E::kPer;
  static constexpr int kRows = R;
};

template <bool BF16, int P, int G, int R>
__global__ __launch_bounds__(G* R) void layer_norm_kernel(const LayerNormArgs a) {
  typedef Elements<BF16> E;
  constexpr int per = E::kPer;
  __shared__ GroupSum<G> sums[R];
  GroupSum<G>& group = sums[threadIdx.x / G];
  const int t = threadIdx.x % G, cols = a.cols;
  const float over = 1.0f / (float)cols;
  float w[P][per], b[P][per];
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const int at = (i * G + t) * per, left = cols - at;
    load_side<per>(a.weight, a.weight_bf16, at, left, 1.0f, w[i]);
    load_side<per>(a.bias, a.weight_bf16, at, left, 0.0f, b[i]);
  }
  // every group takes as many turns as the others: they meet at barriers
  const int64_t step = (int64_t)gridDim.x * R;
  for (int64_t first = (int64_t)blockIdx.x * R; first < a.rows; first += step) {
    const int64_t row = first + threadIdx.x / G;
    const bool live = row < a.rows;
    const int64_t from = live ? row * a.x_ld : 0;
    uint4v q[P];
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int at = (i * G + t) * per;
      q[i] = load_piece<BF16>(a.x, from + at, live ? cols - at : 0);
    }
#pragma unroll
    for (int i = 0; i < P; ++i)
#pragma unroll
      for (int j = 0; j < per; ++j) sum += E::get(q[i], j);
    const float about = group.sum(sum, 0.0f, 0)[0] * over;
    float d1 = 0.0f, d2 = 0.0f;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int left = cols - (i * G + t) * per;
#pragma unroll
      for (int j = 0; j < per; ++j) {
        const float d = j < left ? E::get(q[i], j) - about : 0.0f;
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
      for (int j = 0; j < per; ++j)
        v[j] = __builtin_fmaf(((E::get(q[i], j) - about) - off) * rstd, w[i][j], b[i][j]);
      store_piece<BF16>(a.y, row * a.y_ld + at, cols - at, v);
    }
  }
}

template <bool BF16, int P, int G, int R>
__global__ __launch_bounds__(G* R) void layer_norm_grad_kernel(const LayerNormArgs a) {
  typedef Elements<BF16> E;
  constexpr int per = E::kPer;
  // (the groups' sums of dw and db, one group at a time)
  __shared__ float joined[R > 1 ? 2 * G * P * per : 1];
  __shared__ GroupSum<G> sums[R];
  const int which = threadIdx.x / G, t = threadIdx.x % G, cols = a.cols;
  GroupSum<G>& group = sums[which];
  const float over = 1.0f / (float)cols;
  float w[P][per], dw[P][per], db[P][per];
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const int at = (i * G + t) * per;
    load_side<per>(a.weight, a.weight_bf16, at, cols - at, 1.0f, w[i]);
#pragma unroll
    for (int j = 0; j < per; ++j) dw[i][j] = db[i][j] = 0.0f;
  }
  int turn = 0;
  for (int64_t first = (int64_t)blockIdx.x * R; first < a.rows; first += (int64_t)gridDim.x * R) {
    const int64_t row = first + which;
    const bool live = row < a.rows;
    const int64_t x0 = live ? row * a.x_ld : 0, dy0 = live ? row * a.dy_ld : 0;
    uint4v x[P], dy[P];
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int at = (i * G + t) * per, left = live ? cols - at : 0;
      x[i] = load_piece<BF16>(a.x, x0 + at, left);
      dy[i] = load_piece<BF16>(a.dy, dy0 + at, left);
    }
    const float mean = live ? a.mean[row] : 0.0f, rstd = live ? a.rstd[row] : 0.0f;
    float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
    for (int i = 0; i < P; ++i)
#pragma unroll
      for (int j = 0; j < per; ++j) {
        const float d = E::get(dy[i], j), h = (E::get(x[i], j) - mean) * rstd, g = d * w[i][j];
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
        const float h = (E::get(x[i], j) - mean) * rstd, g = E::get(dy[i], j) * w[i][j];
        v[j] = (g - m1 - h * m2) * rstd;
      }
      store_piece<BF16>(a.dx, row * a.dx_ld + at, cols - at, v);
    }
  }
  if (!a.dweight && !a.dbias) return;
  for (int r = 1; r < R; ++r) {
    __syncthreads();
    if (which == r) {
#pragma unroll
      for (int i = 0; i < P; ++i)
#pragma unroll
        for (int j = 0; j < per; ++j) {
          joined[(i * per + j) * G + t] = dw[i][j];
          joined[(P * per + i * per + j) * G + t] = db[i][j];
        }
    }
    __syncthreads();
    if (which == 0) {
#pragma unroll
      for (int i = 0; i < P; ++i)
#pragma unroll
        for (int j = 0; j < per; ++j) {
          dw[i][j] += joined[(i * per + j) * G + t];
          db[i][j] += joined[(P * per + i * per + j) * G + t];
        }
    }
  }
  if (which != 0) return;
  float* to = a.partial + (int64_t)blockIdx.x * 2 * cols;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const int at = (i * G + t) * per;
#pragma unroll
    for (int j = 0; j < per; ++j)
      if (at + j < cols) {
        if (a.parts == 1) {  // one workgroup: these are the sums
          if (a.dweight) store_side(a.dweight, a.weight_bf16, at + j, dw[i][j]);
          if (a.dbias) store_side(a.dbias, a.weight_bf16, at + j, db[i][j]);
        } else {
          to[at + j] = dw[i][j];
          to[cols + at + j] = db[i][j];
        }
      }
  }
}

// The partial sums of 64 columns, sixteen runs of them side by side.
constexpr int kJoinCols = 64, kJoinRuns = 16;

__global__ __launch_bounds__(kJoinCols* kJoinRuns) void join_sides_kernel(const LayerNormArgs a) {
  __shared__ float part[kJoinRuns][kJoinCols];
  const int c = blockIdx.x * kJoinCols + (threadIdx.x & 63), run = threadIdx.x >> 6;
  void* out = blockIdx.y ? a.dbias : a.dweight;
  if (!out) return;
  const float* from = a.partial + (blockIdx.y ? a.cols : 0);
  float sum = 0.0f;
  if (c < a.cols) {
#pragma unroll 8
    for (int p = run; p < a.parts; p += kJoinRuns) sum += from[(int64_t)p * 2 * a.cols + c];
  }
  part[run][threadIdx.x & 63] = sum;
  __syncthreads();
  if (run != 0 || c >= a.cols) return;
  sum = part[0][threadIdx.x];
#pragma unroll
  for (int i = 1; i < kJoinRuns; ++i) sum += part[i][threadIdx.x];
  store_side(out, a.weight_bf16, c, sum);
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

// Calls f with the shape of a row's group: the smallest that holds it.  False
// where none does.
template <bool BF16, class F>
bool with_shape(int64_t cols, F f) {
  constexpr int e = Elements<BF16>::kPer;
  if (cols <= 64 * 1 * e) return f(Shape<BF16, 1, 64, 4>()), true;
  if (cols <= 64 * 2 * e) return f(Shape<BF16, 2, 64, 4>()), true;
  if (cols <= 256 * 1 * e) return f(Shape<BF16, 1, 256, 1>()), true;
  if (cols <= 256 * 2 * e) return f(Shape<BF16, 2, 256, 1>()), true;
  if (cols <= 512 * 2 * e) return f(Shape<BF16, 2, 512, 1>()), true;
  if (cols <= 1024 * 2 * e) return f(Shape<BF16, 2, 1024, 1>()), true;
  return false;
}

template <bool BF16, int P, int G, int R>
void forward(const LayerNormArgs& a, hipStream_t s, Shape<BF16, P, G, R>) {
  const int64_t turns = (a.rows + R - 1) / R, most = 2048 * 256 / (G * R);
  layer_norm_kernel<BF16, P, G, R><<<dim3((unsigned)(turns < most ? turns : most)), dim3(G * R), 0, s>>>(a);
}

template <bool BF16, int P, int G, int R>
void backward(const LayerNormArgs& a, hipStream_t s, Shape<BF16, P, G, R>) {
  layer_norm_grad_kernel<BF16, P, G, R><<<dim3(a.parts), dim3(G * R), 0, s>>>(a);
}

template <bool BF16>
void launch_forward(const LayerNormArgs& a, hipStream_t s) {
  if (with_shape<BF16>(a.cols, [&](auto shape) { forward(a, s, shape); })) return;
  long_norm_kernel<BF16><<<dim3((unsigned)(a.rows < 1024 ? a.rows : 1024)), dim3(kLongThreads), 0, s>>>(a);
}

template <bool BF16>
void launch_backward(const LayerNormArgs& a, hipStream_t s) {
  if (with_shape<BF16>(a.cols, [&](auto shape) { backward(a, s, shape); })) return;
  constexpr int wide = kSideThreads * Elements<BF16>::kPer;
  if (a.dweight || a.dbias)
    long_sides_kernel<BF16><<<dim3((a.cols + wide - 1) / wide, a.parts), dim3(kSideThreads), 0, s>>>(a);
  if (a.dx && a.rows > 0)
    long_norm_grad_kernel<BF16><<<dim3((unsigned)(a.rows < 1024 ? a.rows : 1024)), dim3(kLongThreads), 0, s>>>(a);
}

}  // namespace

int layer_norm_parts(int64_t rows, int64_t cols, bool bf16) {
  int64_t parts = 0;
  auto of = [&](auto shape) {
    constexpr int r = decltype(shape)::kRows;
    parts = (rows + r - 1) / r;
  };
  const bool held = bf16 ? with_shape<true>(cols, of) : with_shape<false>(cols, of);
  if (!held) return (int)(rows < 2 ? 2 : rows < 64 ? rows : 64);  // (two: the join kernel writes the result)
  return (int)(parts < 1 ? 1 : parts < kNormMostParts ? parts : kNormMostParts);
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
    join_sides_kernel<<<dim3((a.cols + kJoinCols - 1) / kJoinCols, 2), dim3(kJoinCols * kJoinRuns), 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace microadam
