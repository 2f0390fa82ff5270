// Log probability of a given token per row of logits, with the entropy, the
// k most probable alternatives and the gradient with respect to the logits.
//
// With z = x / T, m = max z and d = z - m (in units of ln 2 here: d2 = (x -
// max x) c, c = log2(e) / T):
//   s = sum 2^d2, w = sum 2^d2 d2
//   log p_v = ln 2 (d2_v - log2 s),  H = ln 2 (log2 s - w / s)
//   dL/dx_v = (g_p ([v = t] - p_v) - g_H p_v (log p_v + H)) / T
//           = 2^d2 (A + B d2),  A = -(g_p + g_H (H - ln s)) / (s T),
//             B = -g_H ln 2 / (s T); at the target g_p counts with 1 - p
//
// One workgroup takes a row.  The row is read once, into registers; every
// thread sums against its own maximum, and one reduction joins (max, s, w) of
// the threads, so that no pass over the row waits for a maximum of all.  The
// alternatives and the gradient come from the registers.  A row too long for
// them is taken in segments, and read again for the alternatives or the
// gradient.  The bound is memory, a row's bytes once and once more for the
// gradient: 8192 x 32000 bf16 with the gradient takes 185 us (5.7 TB/s), 157 to
// 161 us with a fifth of the rows ignored, which are not read (5.9 to 6.0 TB/s).
// 4096 x 32000 with 8 alternatives and no gradient takes 69 us (3.8 TB/s): 13
// vector operations and an exponential per element, and two rows a CU to
// overlap them with the loads.
#include "logprobs_device.h"

namespace microadam {
namespace {

typedef uint32_t uint4v __attribute__((ext_vector_type(4)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr float kLn2 = 0.69314718055994531f;
constexpr float kLowest = -3.402823466e38f;
constexpr int kMaxThreads = 1024;
constexpr int kMaxWaves = kMaxThreads / 64;
constexpr int kCandidates = 1024;

__device__ inline float minus_inf() { return __uint_as_float(0xff800000u); }
__device__ inline float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// 16 bytes of a row: 8 bfloat16 or 4 binary32 elements.
template <bool BF16>
struct Chunk {
  static constexpr int kElems = BF16 ? 8 : 4;
  static constexpr int kSize = BF16 ? 2 : 4;
  uint4v q;
  __device__ static Chunk empty() {
    const uint32_t w = BF16 ? 0xff80ff80u : 0xff800000u;  // -inf
    return {uint4v{w, w, w, w}};
  }
  __device__ float get(int i) const {
    if (BF16) return __uint_as_float((i & 1) ? q[i / 2] & 0xffff0000u : q[i / 2] << 16);
    return __uint_as_float(q[i]);
  }
  __device__ static float load1(const void* p, int64_t i) {
    if (BF16) return __uint_as_float((uint32_t)((const uint16_t*)p)[i] << 16);
    return ((const float*)p)[i];
  }
  __device__ static uint32_t pack2(float a, float b) {
    const bf16x2 v = __builtin_convertvector(float2v{a, b}, bf16x2);
    return __builtin_bit_cast(uint32_t, v);
  }
  __device__ void set(const float* v) {
    if (BF16) {
#pragma unroll
      for (int i = 0; i < 4; ++i) q[i] = pack2(v[2 * i], v[2 * i + 1]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) q[i] = __float_as_uint(v[i]);
    }
  }
  __device__ static void store1(void* p, int64_t i, float v) {
    if (BF16)
      ((uint16_t*)p)[i] = (uint16_t)pack2(v, v);
    else
      ((float*)p)[i] = v;
  }
};

struct Sums {
  float m, s, w;  // maximum of x, sum of 2^d2, sum of 2^d2 d2
};

// What a thread adds up over the segments of a row, of which 2^24 logits have
// up to 2048: in binary32 the chain's rounding, one way where the terms are
// alike, reached 5e-4 of log s.
template <bool MULTI>
struct Running {
  typedef float type;
};
template <>
struct Running<true> {
  typedef double type;
};

// The sums of x's against `from` taken against the larger maximum `to`.
__device__ inline void rebase(Sums& a, float to, float c) {
  const float delta = (a.m - to) * c;
  const float f = exp2_fast(delta);
  // f = 0 where delta is far below: 0 * -inf must not arise
  a.w = f * (a.w + fmaxf(delta, -1000.0f) * a.s);
  a.s = f * a.s;
  a.m = to;
}

// The sums of a wave; `lane_s` becomes this lane's part of s.
__device__ inline Sums join_wave(Sums a, float c, float& lane_s) {
  float m = a.m;
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
  rebase(a, m, c);
  lane_s = a.s;
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    a.s += __shfl_xor(a.s, d);
    a.w += __shfl_xor(a.w, d);
  }
  return a;
}

// (value, index) order of the alternatives: larger first, ties to the lower index.
__device__ inline bool before(float va, int ia, float vb, int ib) { return va > vb || (va == vb && ia < ib); }

struct Shared {
  Sums sums[kMaxWaves];
  float best_v[kMaxWaves];
  int best_i[kMaxWaves];
  float thread_max[kMaxThreads];
  uint4v own[16];  // a thread's chunks
  float cand_v[kCandidates];
  int cand_i[kCandidates];
  int count;
  float rest;
};

// Whole numbers in the order of floats (no NaN).
__device__ inline uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);
  return (u >> 31) ? ~u : u | 0x80000000u;
}
__device__ inline float from_ordered(uint32_t u) { return __uint_as_float((u >> 31) ? u & 0x7fffffffu : ~u); }

// A value that at least k (at most 64) elements reach: with the threads'
// maxima taken together lane by lane over the waves, the k-th largest of the
// 64, down to the low 16 bits of its order.  Every wave finds it for itself.
__device__ inline float reached_by(const float* maxima, int waves, int k) {
  const int lane = threadIdx.x & 63;
  float m = maxima[lane];
  for (int w = 1; w < waves; ++w) m = fmaxf(m, maxima[w * 64 + lane]);
  const uint32_t key = ordered(m);
  uint32_t t = 0;
#pragma unroll
  for (int bit = 31; bit >= 16; --bit) {
    const uint32_t probe = t | (1u << bit);
    if (__popcll(__ballot(key >= probe)) >= k) t = probe;
  }
  return t <= ordered(minus_inf()) ? minus_inf() : from_ordered(t);
}

// MULTI: the row takes several segments of blockDim.x * NV chunks.
template <bool BF16, int NV, bool GRAD, bool ENTGRAD, bool MULTI>
__global__ __launch_bounds__(kMaxThreads) void row_kernel(const LogprobArgs a) {
  typedef Chunk<BF16> C;
  constexpr int E = C::kElems;
  __shared__ Shared sh;
  const int64_t row = blockIdx.x;
  const int tid = threadIdx.x, nt = blockDim.x, waves = nt >> 6;
  const int lane = tid & 63, wave = tid >> 6;
  const int64_t target = a.targets[row];
  const int k = GRAD ? 0 : a.top_k;
  int64_t start = row * a.ld;
  if (a.group_rows) {
    const uint32_t group = (uint32_t)row / (uint32_t)a.group_rows;
    start = group * a.group_stride + (int64_t)((uint32_t)row - group * (uint32_t)a.group_rows) * a.ld;
  }
  const uint8_t* const x = (const uint8_t*)a.logits + start * C::kSize;
  uint8_t* const dx = GRAD ? (uint8_t*)a.grad + row * a.grad_ld * C::kSize : nullptr;
  const int V = a.vocab;

  // [0, head) and [V - tail, V): one element each for the first threads;
  // between them whole chunks at 16-byte aligned addresses
  int head = (int)((0u - (uint32_t)(uintptr_t)x) & 15u) / C::kSize;
  if (head > V) head = V;
  const int chunks = (V - head) / E;
  const int tail = V - head - chunks * E;
  const int edge = tid < head ? tid : tid < head + tail ? V - tail + (tid - head) : -1;
  const uint4v* const body = (const uint4v*)(x + head * C::kSize);

  if (target == a.ignore_index) {
    if (tid == 0) {
      if (a.logp) a.logp[row] = 0.0f;
      if (a.entropy) a.entropy[row] = 0.0f;
    }
    for (int i = tid; i < k; i += nt) {
      a.top_logprobs[row * k + i] = 0.0f;
      a.top_indices[row * k + i] = -1;
    }
    if (GRAD) {
      const int dhead = (int)((0u - (uint32_t)(uintptr_t)dx) & 15u) / C::kSize;
      const int h = dhead > V ? V : dhead, n = (V - h) / E;
      for (int i = tid; i < n; i += nt) ((uint4v*)(dx + h * C::kSize))[i] = uint4v{0, 0, 0, 0};
      for (int i = tid; i < V - n * E; i += nt) C::store1(dx, i < h ? i : i + n * E, 0.0f);
    }
    return;
  }

  C r[NV];
  const int per_segment = nt * NV;
  const int segments = MULTI ? (chunks + per_segment - 1) / per_segment : 1;
  auto load = [&](int seg) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int j = seg * per_segment + i * nt + tid;
      r[i] = C::empty();
      if (j < chunks) r[i].q = __builtin_nontemporal_load(body + j);
    }
  };

  const float xe = edge >= 0 ? C::load1(x, edge) : minus_inf();
  Sums t;
  t.m = fmaxf(xe, kLowest);
  {
    const float d = (xe - t.m) * a.c;
    t.s = exp2_fast(d);
    t.w = t.s * fmaxf(d, -1000.0f);
  }
  typedef typename Running<MULTI>::type Wide;
  Wide all_s = t.s, all_w = t.w;  // of the segments before
  for (int seg = 0; seg < segments; ++seg) {
    load(seg);
    float m = t.m;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < E; ++e) m = fmaxf(m, r[i].get(e));
    if constexpr (MULTI) {
      if (m != t.m) {
        const float delta = (t.m - m) * a.c, f = exp2_fast(delta);
        all_w = f * (all_w + fmaxf(delta, -1000.0f) * all_s);
        all_s *= f;
      }
      t = {m, 0.0f, 0.0f};
    } else {
      rebase(t, m, a.c);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float d = (r[i].get(e) - m) * a.c;
        const float p = exp2_fast(d);
        t.s += p;
        t.w = __builtin_fmaf(p, fmaxf(d, -1000.0f), t.w);
      }
    if constexpr (MULTI) {
      all_s += t.s;
      all_w += t.w;
    }
  }
  if constexpr (MULTI) {
    t.s = (float)all_s;
    t.w = (float)all_w;
  }
  const float thread_max = t.m;
  const bool known = target >= 0 && target < V;
  // before the barrier: in place, the gradient's stores come after it
  const float x_target = tid == 0 && known ? C::load1(x, target) : 0.0f;

  float lane_s, unused;
  t = join_wave(t, a.c, lane_s);
  if (lane == 0) sh.sums[wave] = t;
  if (k) {
    sh.thread_max[tid] = thread_max;
    if (tid == 0) sh.count = 0;
  }
  __syncthreads();
  t = sh.sums[lane < waves ? lane : 0];
  if (lane >= waves) t.s = t.w = 0.0f;
  t = join_wave(t, a.c, unused);

  // t.s = 0: every logit is -inf (otherwise the largest adds 1); NaN: a NaN
  // or +inf logit.  Where one token has more than half the probability, s - 1
  // is summed apart from it, so that 1 - p and log s of that token are no
  // differences of rounded numbers.  Only the thread that holds it had it in
  // its sum: its wave takes that thread's elements again, one a lane.
  const bool empty = t.s == 0.0f;
  float rest = t.s - 1.0f;
  float log_s;
  if (!empty && t.s < 2.0f) {
    const uint64_t holds = __ballot(thread_max == t.m && lane_s >= 1.0f);  // its 2^0
    if (holds) {
      const int owner = __ffsll((unsigned long long)holds) - 1;
      auto other = [&](float v) { return v < t.m ? exp2_fast((v - t.m) * a.c) : 0.0f; };
      Wide wide = lane == owner ? other(xe) : lane_s;
      for (int seg = 0; seg < segments; ++seg) {
        if (MULTI) load(seg);
        if (lane == owner) {
#pragma unroll
          for (int i = 0; i < NV; ++i) sh.own[i] = r[i].q;
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        for (int i = lane; i < NV * E; i += 64) {
          C one;
          one.q = sh.own[i / E];
          float v = one.get(0);
#pragma unroll
          for (int e = 1; e < E; ++e) v = i % E == e ? one.get(e) : v;
          wide += other(v);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
      }
      float sum = (float)wide;
#pragma unroll
      for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
      if (lane == 0) sh.rest = sum;
    }
    __syncthreads();
    Sums u = sh.sums[lane < waves ? lane : 0];
    if (lane >= waves || u.m == t.m) u.s = 0.0f;
    rebase(u, t.m, a.c);
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) u.s += __shfl_xor(u.s, d);
    rest = u.s + sh.rest;
    t.s = 1.0f + rest;
  }
  if (rest < 1.0f / 128)  // log(1 + rest)
    log_s = rest * (1.0f - rest * (0.5f - rest * (1.0f / 3 - rest * 0.25f)));
  else
    log_s = kLn2 * __builtin_amdgcn_logf(t.s);
  const float below = empty ? 0.0f : -kLn2 * (t.w / t.s);  // H - log s
  auto logprob = [&](float v) { return (v - t.m) * a.inv_t - log_s; };
  if (tid == 0) {
    if (a.logp)
      a.logp[row] = !known ? __uint_as_float(0x7fc00000u) : empty ? minus_inf() : logprob(x_target);
    if (a.entropy) a.entropy[row] = empty ? 0.0f : below + log_s;
  }

  if constexpr (GRAD) {
    const float gp = known ? a.grad_logp[row] : __uint_as_float(0x7fc00000u);
    const float gh = ENTGRAD ? a.grad_entropy[row] : 0.0f;
    const float inv = a.inv_t / t.s;
    const float Ah = ENTGRAD ? -gh * below * inv : 0.0f;
    const float A = Ah - gp * inv;
    const float B = -gh * kLn2 * inv;
    const float none = known ? 0.0f : gp;  // of a row with no possible token
    auto part = [&](float v, float factor) {
      const float d = (v - t.m) * a.c;
      const float p = exp2_fast(d);
      const float g = ENTGRAD ? p * __builtin_fmaf(B, fmaxf(d, -1000.0f), factor) : p * factor;
      return empty ? none : g;
    };
    auto grad = [&](float v) { return part(v, A); };
    // g_p (1 - p) without the difference where p is nearly 1
    auto grad_target = [&](float v) {
      const float others = v == t.m ? rest : t.s - exp2_fast((v - t.m) * a.c);
      return empty ? none : part(v, Ah) + gp * others * inv;
    };
    const bool aligned = (((uintptr_t)x ^ (uintptr_t)dx) & 15) == 0;
    uint4v* const dbody = (uint4v*)(dx + head * C::kSize);
    const int tb = known ? (int)target - head : -1;  // the target's place in the body
    for (int seg = 0; seg < segments; ++seg) {
      if (MULTI) load(seg);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int j = seg * per_segment + i * nt + tid;
        if (j >= chunks) continue;
        float v[E];
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = grad(r[i].get(e));
        if (tb >= j * E && tb < j * E + E) {
#pragma unroll
          for (int e = 0; e < E; ++e)
            if (tb == j * E + e) v[e] = grad_target(r[i].get(e));
        }
        if (aligned) {
          C o;
          o.set(v);
          __builtin_nontemporal_store(o.q, dbody + j);
        } else {
#pragma unroll
          for (int e = 0; e < E; ++e) C::store1(dx, head + j * E + e, v[e]);
        }
      }
    }
    if (edge >= 0) C::store1(dx, edge, edge == target ? grad_target(xe) : grad(xe));
    return;
  }

  if (k == 0) return;
  float* const out_v = a.top_logprobs + row * k;
  int64_t* const out_i = a.top_indices + row * k;
  if (!(t.s > 0.0f)) {
    for (int i = tid; i < k; i += nt) {
      out_v[i] = empty ? minus_inf() : __uint_as_float(0x7fc00000u);
      out_i[i] = empty ? i : -1;
    }
    return;
  }
  // The first k are among the elements that reach the threshold: few more
  // than k, unless many are equal.
  const float threshold = reached_by(sh.thread_max, waves, k);
  auto collect = [&](float v, int i) {
    if (v >= threshold) {
      const int n = atomicAdd(&sh.count, 1);
      if (n < kCandidates) {
        sh.cand_v[n] = v;
        sh.cand_i[n] = i;
      }
    }
  };
  if (threshold > kLowest) {
    for (int seg = 0; seg < segments; ++seg) {
      if (MULTI) load(seg);
      if (!MULTI && thread_max < threshold) break;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int j = seg * per_segment + i * nt + tid;
        float m = r[i].get(0);
#pragma unroll
        for (int e = 1; e < E; ++e) m = fmaxf(m, r[i].get(e));
        if (m < threshold) continue;  // also past the last chunk
#pragma unroll
        for (int e = 0; e < E; ++e) collect(r[i].get(e), head + j * E + e);
      }
    }
    if (edge >= 0) collect(xe, edge);
  }
  __syncthreads();
  const int n = sh.count;
  auto emit = [&](int at, float v, int i) {
    out_v[at] = logprob(v);
    out_i[at] = i;
  };
  if (threshold > kLowest && n <= kCandidates) {
    for (int i = tid; i < n; i += nt) {
      const float v = sh.cand_v[i];
      const int at = sh.cand_i[i];
      int rank = 0;
      for (int j = 0; j < n; ++j) rank += before(sh.cand_v[j], sh.cand_i[j], v, at) ? 1 : 0;
      if (rank < k) emit(rank, v, at);
    }
    return;
  }
  // Many equal values (or fewer than k threads with one): k rounds, each the
  // first element after the last round's.
  float last_v = __uint_as_float(0x7f800000u);
  int last_i = -1;
  for (int round = 0; round < k; ++round) {
    float bv = minus_inf();
    int bi = 0x7fffffff;
    auto look = [&](float v, int i) {
      if (before(last_v, last_i, v, i) && before(v, i, bv, bi)) {
        bv = v;
        bi = i;
      }
    };
    for (int seg = 0; seg < segments; ++seg) {
      if (MULTI) load(seg);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int j = seg * per_segment + i * nt + tid;
        if (j >= chunks) continue;
#pragma unroll
        for (int e = 0; e < E; ++e) look(r[i].get(e), head + j * E + e);
      }
    }
    if (edge >= 0) look(xe, edge);
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
      const float ov = __shfl_xor(bv, d);
      const int oi = __shfl_xor(bi, d);
      if (before(ov, oi, bv, bi)) {
        bv = ov;
        bi = oi;
      }
    }
    if (lane == 0) {
      sh.best_v[wave] = bv;
      sh.best_i[wave] = bi;
    }
    __syncthreads();
    bv = sh.best_v[0];
    bi = sh.best_i[0];
    for (int i = 1; i < waves; ++i)
      if (before(sh.best_v[i], sh.best_i[i], bv, bi)) {
        bv = sh.best_v[i];
        bi = sh.best_i[i];
      }
    __syncthreads();
    if (tid == 0) emit(round, bv, bi);
    last_v = bv;
    last_i = bi;
  }
}

template <bool BF16, bool GRAD, bool ENTGRAD>
hipError_t launch_rows(const LogprobArgs& a, hipStream_t s) {
  const int chunks = a.vocab / Chunk<BF16>::kElems;  // at most
  const dim3 grid((unsigned)a.rows);
  auto threads = [&](int nv) {
    const int n = ((chunks + nv - 1) / nv + 63) / 64 * 64;
    return n < 64 ? 64 : n;
  };
  // With few rows a row's own time counts: few chunks in up to 1024 threads
  // (1 x 32000 bf16: 8.7 us, with 8 chunks in 512 threads 9.3).  With many, up
  // to 8 chunks in small workgroups, of which a CU holds more (2048 x 16384
  // bf16 with 8 alternatives: 18.9 us in 256 threads, 27.5 in 512 with 4).
  //
  // Values alone read a row once in segments too, in a third of the registers:
  // long rows without alternatives take 256 threads (2048 x 50257 bf16: 42 us,
  // held whole 61), and so do longer ones with them, which are then read twice
  // (67 us, held whole 81; binary32, twice the bytes, gains only beyond its
  // registers).
  const bool few = a.rows <= 128;
  const int most = few ? kMaxThreads : 64;
  if (!GRAD && !few && threads(8) > (a.top_k == 0 ? 256 : BF16 ? 512 : 2 * kMaxThreads))
    row_kernel<BF16, 8, GRAD, ENTGRAD, true><<<grid, 256, 0, s>>>(a);
  else if (threads(1) <= most)
    row_kernel<BF16, 1, GRAD, ENTGRAD, false><<<grid, threads(1), 0, s>>>(a);
  else if (threads(2) <= most)
    row_kernel<BF16, 2, GRAD, ENTGRAD, false><<<grid, threads(2), 0, s>>>(a);
  else if (threads(4) <= (few ? kMaxThreads : 256))
    row_kernel<BF16, 4, GRAD, ENTGRAD, false><<<grid, threads(4), 0, s>>>(a);
  else if (threads(8) <= kMaxThreads)
    row_kernel<BF16, 8, GRAD, ENTGRAD, false><<<grid, threads(8), 0, s>>>(a);
  // 16 binary32 chunks a thread still fit its registers (2000 x 50257 with the
  // gradient: 166 us, in segments 232 us); as many bfloat16 ones, twice the
  // elements, spill
  else if (!BF16 && threads(16) <= kMaxThreads)
    row_kernel<BF16, BF16 ? 8 : 16, GRAD, ENTGRAD, false><<<grid, threads(16), 0, s>>>(a);
  else
    row_kernel<BF16, 8, GRAD, ENTGRAD, true><<<grid, kMaxThreads, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_token_logprobs(const LogprobArgs& a, bool bf16, hipStream_t s) {
  if (a.rows < 1 || a.rows >= ((int64_t)1 << 31) / kMaxThreads || a.vocab < 1 || a.top_k > kMaxTopK)
    return hipErrorInvalidValue;
  if (!a.grad) return bf16 ? launch_rows<true, false, false>(a, s) : launch_rows<false, false, false>(a, s);
  if (!a.grad_entropy) return bf16 ? launch_rows<true, true, false>(a, s) : launch_rows<false, true, false>(a, s);
  return bf16 ? launch_rows<true, true, true>(a, s) : launch_rows<false, true, true>(a, s);
}

}  // namespace microadam
