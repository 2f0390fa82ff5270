// The 2-norm over a list of gradients, and their scaling to a limit.
//
//   n = sqrt(sum g^2),  c = max_norm / (n + eps) where that is below 1, else 1
//   g <- c g
//
// The list is cut into chunks of 32 KiB that the workgroups take in turn; each
// keeps its sum of squares in binary64, which neither tiny nor huge gradients
// leave, and writes one partial sum.  Every workgroup of the scaling pass adds
// the partial sums itself, in one fixed order, so that no launch stands between
// and the same list gives the same bits; of a list past the caches, whose
// workgroups are many, a kernel before it does.  The scaling takes the chunks from the
// last to the first: what the norm read last is still in the cache.  Where the
// factor is 1 nothing is written.
//
// The bound is memory.  1.9e9 bfloat16 gradients (3.8 GB): the sum 540 us (6.9
// TB/s), the scaling 1325 (5.7 TB/s, read and written).  A list of 53 MB, which the
// last-level cache holds: 13 and 20 us; one of 15 MB: 6 us and 2 for the norm.
#include "clip_device.h"
#include "elements.h"

namespace microadam {
namespace {

constexpr int kThreads = 256;
// Workgroups of the scaling pass, at most, and the parts of a chunk that they take
// one each, of a list past the caches: 3.8 GB clipped / below the limit 1870 / 565 us.
// (More would cost what is not clipped: one workgroup a part 1813 / 599, 4096 that
// take chunk after chunk 1960 / 561.  Within the caches halves cost 105 MB 33
// instead of 31 us.)
constexpr int kScaleGroups = 1 << 16;
template <bool PAST>
constexpr int kScaleParts = PAST ? 2 : 1;
constexpr int kPieces = (int)(kClipChunk / 16 / kThreads);  // a thread's, of a chunk

__device__ inline double wave_sum(double x) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
  return x;
}

__device__ inline double block_sum(double x) {
  __shared__ double part[kThreads / 64];
  x = wave_sum(x);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
  __syncthreads();
  double sum = part[0];
#pragma unroll
  for (int i = 1; i < kThreads / 64; ++i) sum += part[i];
  return sum;
}

// The tensor that a chunk belongs to: the last whose first chunk is not behind it.
__device__ inline int tensor_of(const ClipArgs& a, int chunk) {
  int lo = 0, hi = a.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.first[mid] <= chunk)
      lo = mid;
    else
      hi = mid - 1;
  }
  return lo;
}

template <bool BF16>
__device__ inline double squares(const uint4v& q) {
  typedef Elements<BF16> E;
  double s = 0.0;
#pragma unroll
  for (int i = 0; i < E::kPer; ++i) {
    const double g = (double)E::get(q, i);
    s = __builtin_fma(g, g, s);
  }
  return s;
}

// Of the sixteen bytes at `p`, those elements that lie in [at, end); f takes
// each with its place.
template <bool BF16, class F>
__device__ inline void each_inside(uint64_t p, uint64_t at, uint64_t end, F f) {
  typedef Elements<BF16> E;
#pragma unroll
  for (int i = 0; i < E::kPer; ++i) {
    const uint64_t e = p + (uint64_t)(i * E::kSize);
    if (e >= at && e < end) f((void*)e);
  }
}

// A list that no cache holds is read and written past them.
template <bool PAST>
__device__ inline uint4v load_piece(const uint4v* p) {
  return PAST ? __builtin_nontemporal_load(p) : *p;
}
template <bool PAST>
__device__ inline void store_piece(uint4v* p, const uint4v& q) {
  if (PAST)
    __builtin_nontemporal_store(q, p);
  else
    *p = q;
}

template <bool BF16, bool PAST>
__device__ inline double chunk_squares(uint64_t from, uint64_t at, uint64_t end) {
  typedef Elements<BF16> E;
  double sum = 0.0;
  if (from >= at && from + kClipChunk <= end) {
    uint4v q[kPieces];
#pragma unroll
    for (int i = 0; i < kPieces; ++i) q[i] = load_piece<PAST>((const uint4v*)from + i * kThreads + threadIdx.x);
#pragma unroll
    for (int i = 0; i < kPieces; ++i) sum += squares<BF16>(q[i]);
    return sum;
  }
  for (int i = threadIdx.x; i < (int)(kClipChunk / 16); i += kThreads) {
    const uint64_t p = from + (uint64_t)i * 16;
    if (p >= end) break;
    if (p >= at && p + 16 <= end)
      sum += squares<BF16>(*(const uint4v*)p);
    else
      each_inside<BF16>(p, at, end, [&](void* e) {
        const double g = (double)E::load1(e, 0);
        sum = __builtin_fma(g, g, sum);
      });
  }
  return sum;
}

template <bool PAST>
__global__ __launch_bounds__(kThreads) void square_sums_kernel(const ClipArgs a) {
  double sum = 0.0;
  const int chunks = a.first[a.n];
  for (int c = blockIdx.x; c < chunks; c += gridDim.x) {
    const int t = tensor_of(a, c);
    const bool bf16 = a.at[t] & 1;
    const uint64_t at = a.at[t] & ~(uint64_t)1, end = a.end[t];
    const uint64_t from = (at & ~(uint64_t)15) + (uint64_t)(c - a.first[t]) * kClipChunk;
    sum += bf16 ? chunk_squares<true, PAST>(from, at, end) : chunk_squares<false, PAST>(from, at, end);
  }
  sum = block_sum(sum);
  if (threadIdx.x == 0) a.partial[blockIdx.x] = a.add ? a.partial[blockIdx.x] + sum : sum;
}

__device__ inline double norm_of(const ClipArgs& a) {
  double sum = 0.0;
  for (int i = threadIdx.x; i < a.slots; i += kThreads) sum += a.partial[i];
  return sqrt(block_sum(sum));
}

__global__ __launch_bounds__(kThreads) void grad_norm_kernel(const ClipArgs a) {
  const double norm = norm_of(a);
  if (threadIdx.x) return;
  *a.norm = (float)norm;
  a.partial[kClipSlots] = norm;
}

// (the product in binary64: a factor below binary32's normal range, of
// gradients near its end, would lose its bits)
__device__ inline float scaled(float g, double c) { return (float)((double)g * c); }

template <bool BF16>
__device__ inline uint4v scale_piece(const uint4v& q, double c) {
  typedef Elements<BF16> E;
  float v[E::kPer];
#pragma unroll
  for (int i = 0; i < E::kPer; ++i) v[i] = scaled(E::get(q, i), c);
  return E::put(v);
}

template <bool BF16, bool PAST>
__device__ inline void scale_part(uint64_t from, uint64_t at, uint64_t end, double c) {
  typedef Elements<BF16> E;
  constexpr int kBytes = (int)kClipChunk / kScaleParts<PAST>, kOwn = kBytes / 16 / kThreads;
  if (from >= at && from + kBytes <= end) {
    uint4v* p = (uint4v*)from;
    uint4v q[kOwn];
#pragma unroll
    for (int i = 0; i < kOwn; ++i) q[i] = load_piece<PAST>(p + i * kThreads + threadIdx.x);
#pragma unroll
    for (int i = 0; i < kOwn; ++i)
      store_piece<PAST>(p + i * kThreads + threadIdx.x, scale_piece<BF16>(q[i], c));
    return;
  }
  for (int i = threadIdx.x; i < kBytes / 16; i += kThreads) {
    const uint64_t p = from + (uint64_t)i * 16;
    if (p >= end) break;
    if (p >= at && p + 16 <= end)
      *(uint4v*)p = scale_piece<BF16>(*(const uint4v*)p, c);
    else
      each_inside<BF16>(p, at, end, [&](void* e) { E::store1(e, 0, scaled(E::load1(e, 0), c)); });
  }
}

template <bool PAST>
__global__ __launch_bounds__(kThreads) void scale_grads_kernel(const ClipArgs a) {
  const double norm = PAST ? a.partial[kClipSlots] : norm_of(a);
  if (!PAST && a.norm && blockIdx.x == 0 && threadIdx.x == 0) *a.norm = (float)norm;
  if (norm + a.eps <= a.max_norm) return;
  const double c = a.max_norm / (norm + a.eps);  // NaN of a NaN norm
  constexpr int parts = kScaleParts<PAST>;
  for (int k = a.first[a.n] * parts - 1 - (int)blockIdx.x; k >= 0; k -= (int)gridDim.x) {
    const int t = tensor_of(a, k / parts);
    const bool bf16 = a.at[t] & 1;
    const uint64_t at = a.at[t] & ~(uint64_t)1, end = a.end[t];
    const uint64_t from = (at & ~(uint64_t)15) + (uint64_t)(k - a.first[t] * parts) * (kClipChunk / parts);
    if (bf16)
      scale_part<true, PAST>(from, at, end, c);
    else
      scale_part<false, PAST>(from, at, end, c);
  }
}

}  // namespace

hipError_t launch_square_sums(const ClipArgs& a, hipStream_t s) {
  if (a.past)
    square_sums_kernel<true><<<dim3(a.slots), dim3(kThreads), 0, s>>>(a);
  else
    square_sums_kernel<false><<<dim3(a.slots), dim3(kThreads), 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_grad_norm(const ClipArgs& a, hipStream_t s) {
  grad_norm_kernel<<<dim3(1), dim3(kThreads), 0, s>>>(a);
  return hipGetLastError();
}

template <bool PAST>
static void scale_grads(const ClipArgs& a, hipStream_t s) {
  const int64_t parts = (int64_t)a.first[a.n] * kScaleParts<PAST>;
  const int grid = parts < 1 ? 1 : parts < kScaleGroups ? (int)parts : kScaleGroups;
  scale_grads_kernel<PAST><<<dim3(grid), dim3(kThreads), 0, s>>>(a);
}

hipError_t launch_scale_grads(const ClipArgs& a, hipStream_t s) {
  if (a.past)
    scale_grads<true>(a, s);
  else
    scale_grads<false>(a, s);
  return hipGetLastError();
}

}  // namespace microadam
