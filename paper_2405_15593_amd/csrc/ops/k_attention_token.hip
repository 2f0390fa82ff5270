// Softmax attention of a few binary32 rows of a key head, a generated token's, as a
// stream over keys and values.
//
// The matrix cores would multiply 32 rows for a few, which costs binary32 more
// time than the reading (one query of 32 heads on 8, 32768 keys of 128: 73 us, here
// 51; bfloat16, whose products are sixteen times as fast, 33 and 34).  Here G lanes
// hold a key, eight elements each, and R rows of q: a score is a sum over G lanes
// (in-row permutes), and out's part of the key is added where v lies.  Nothing
// passes through LDS before the end.  Every group of G lanes keeps its own maximum,
// sum and output over every so many keys; a workgroup's groups are joined in LDS,
// parts of the keys by attention_join_kernel.  The bound is memory: those 268 MB
// take 43 to 47 us (5.7 to 6.3 TB/s) and 4 to 5 for the join.
#include "attention_tile.h"

namespace microadam {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr float kAhead = 8.0f;

template <int CTRL>
__device__ inline float add_permuted(float x) {
  return x + __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), CTRL, 0xf, 0xf, true));
}

// The sum over G lanes, in each of them.
template <int G>
__device__ inline float sum_lanes(float x) {
  x = add_permuted<0xb1>(x);               // neighbours
  x = add_permuted<0x4e>(x);               // pairs
  if (G >= 8) x = add_permuted<0x141>(x);  // halves of eight, mirrored
  if (G >= 16) x = add_permuted<0x140>(x); // halves of sixteen
  return x;
}

template <int G, int R, bool PAST>
__global__ __launch_bounds__(kThreads, 2) void attention_token_kernel(const AttentionArgs a) {
  constexpr int kPolicy = PAST ? kNonTemporal : 0;
  constexpr int kKeys = 64 / G;            // keys of a wave at once
  constexpr int kDeep = R == 8 ? 2 : 4;    // one behind the other (as registers allow)
  constexpr int kStep = kKeys * kDeep;
  constexpr int kLoads = 2;                // sixteen bytes each
  constexpr int kGroups = kWaves * kKeys;  // of lanes, in the workgroup
  __shared__ float sums[R][kGroups][G * 8];
  __shared__ float stats[R][kGroups][2];
  const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6);
  const int in = lane % G, group = lane / G;
  int head_of = blockIdx.x, part = 0;
  if (a.parts) {
    part = head_of % a.parts;
    head_of /= a.parts;
  }
  const int kv_head = head_of % a.kv_heads, batch = head_of / a.kv_heads;
  const int length = keys_of(a, batch);
  int limits[R], end = 0, least = length;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    limits[r] = r < a.rows ? limit_of(a, row_at(a, kv_head, r).query, length) : 0;
    if (r >= a.rows) continue;
    end = limits[r] > end ? limits[r] : end;
    least = limits[r] < least ? limits[r] : least;
  }
  const int steps = (end + kStep - 1) / kStep;
  const int first = a.parts ? (int)((int64_t)part * steps / a.parts) : 0;
  const int last = a.parts ? (int)((int64_t)(part + 1) * steps / a.parts) : steps;

  constexpr int size = 4;
  const int64_t k_pos = a.k.pos * size, v_pos = a.v.pos * size;
  const uint8_t* k_at = (const uint8_t*)a.k.at + (batch * a.k.batch + kv_head * a.k.head) * size;
  const uint8_t* v_at = (const uint8_t*)a.v.at + (batch * a.v.batch + kv_head * a.v.head) * size;
  // (element 4 (i G + in) + j of a row is a lane's 4 i + j: each load takes whole lines)
  auto element = [&](int i) { return 4 * (i * G + in); };
  uint32_t k_from[kDeep][kLoads], v_from[kDeep][kLoads];
#pragma unroll
  for (int u = 0; u < kDeep; ++u)
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int key = u * kKeys + group, e = element(i);
      k_from[u][i] = e < a.dim ? (uint32_t)(key * (int)k_pos + e * size) : 0x80000000u;
      v_from[u][i] = e < a.dim ? (uint32_t)(key * (int)v_pos + e * size) : 0x80000000u;
    }
  struct Loaded {
    uint4v k[kDeep][kLoads], v[kDeep][kLoads];
  };
  auto load = [&](Loaded& to, int step) {
    const int at = step * kStep, there = end - at < kStep ? end - at : kStep;
    const int k_bytes = there > 0 ? (there - 1) * (int)k_pos + a.dim * size : 0;
    const int v_bytes = there > 0 ? (there - 1) * (int)v_pos + a.dim * size : 0;
    const auto k_buffer = __builtin_amdgcn_make_buffer_rsrc((void*)(k_at + at * k_pos), 0, k_bytes, 0x00020000);
    const auto v_buffer = __builtin_amdgcn_make_buffer_rsrc((void*)(v_at + at * v_pos), 0, v_bytes, 0x00020000);
#pragma unroll
    for (int u = 0; u < kDeep; ++u)
#pragma unroll
      for (int i = 0; i < kLoads; ++i) to.k[u][i] = __builtin_amdgcn_raw_buffer_load_b128(k_buffer, (int)k_from[u][i], 0, kPolicy);
#pragma unroll
    for (int u = 0; u < kDeep; ++u)
#pragma unroll
      for (int i = 0; i < kLoads; ++i) to.v[u][i] = __builtin_amdgcn_raw_buffer_load_b128(v_buffer, (int)v_from[u][i], 0, kPolicy);
  };
  Loaded next;
  int step = first + wave;
  if (step < last) load(next, step);

  float q[R][8], out[R][8], m[R], l[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const RowAt at = row_at(a, kv_head, r < a.rows ? r : 0);
    const int64_t q_at = batch * a.q.batch + at.head * a.q.head + at.query * a.q.pos;
    m[r] = -infinity();
    l[r] = 0.0f;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const uint4v f = r < a.rows && element(i) < a.dim ? Elements<false>::load(a.q.at, q_at + element(i)) : uint4v{0, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        q[r][4 * i + j] = __uint_as_float(f[j]);
        out[r][4 * i + j] = 0.0f;
      }
    }
  }
  for (; step < last; step += kWaves) {
    const Loaded now = next;
    if (step + kWaves < last) load(next, step + kWaves);
    float s[kDeep][R];
#pragma unroll
    for (int u = 0; u < kDeep; ++u) {
#pragma unroll
      for (int r = 0; r < R; ++r) s[u][r] = 0.0f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float x = __uint_as_float(now.k[u][j / 4][j % 4]);
#pragma unroll
        for (int r = 0; r < R; ++r) s[u][r] = __builtin_fmaf(x, q[r][j], s[u][r]);
      }
#pragma unroll
      for (int r = 0; r < R; ++r) s[u][r] = sum_lanes<G>(s[u][r]);
    }
    const int at = step * kStep + group;
    if (step * kStep + kStep > least) {
#pragma unroll
      for (int u = 0; u < kDeep; ++u)
#pragma unroll
        for (int r = 0; r < R; ++r) s[u][r] = at + u * kKeys < limits[r] ? s[u][r] : -infinity();
    }
    bool moved = false;
    float top[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      top[r] = s[0][r];
#pragma unroll
      for (int u = 1; u < kDeep; ++u) top[r] = fmaxf(top[r], s[u][r]);
      top[r] *= a.c;
      moved = moved || top[r] > m[r] + kAhead;
    }
    if (__any(moved)) {  // (as k_attention.hip's add_tile: most steps pass without a factor)
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const bool ahead = top[r] > m[r] + kAhead;
        const float to = ahead ? top[r] : m[r], factor = ahead ? exp2_fast(m[r] - to) : 1.0f;
        m[r] = to;
        l[r] *= factor;
#pragma unroll
        for (int j = 0; j < 8; ++j) out[r][j] *= factor;
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const float from = m[r] == -infinity() ? 0.0f : -m[r];
#pragma unroll
      for (int u = 0; u < kDeep; ++u) {
        s[u][r] = exp2_fast(__builtin_fmaf(s[u][r], a.c, from));
        l[r] += s[u][r];
      }
    }
#pragma unroll
    for (int u = 0; u < kDeep; ++u)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float x = __uint_as_float(now.v[u][j / 4][j % 4]);
#pragma unroll
        for (int r = 0; r < R; ++r) out[r][j] = __builtin_fmaf(x, s[u][r], out[r][j]);
      }
  }

  const int slot = wave * kKeys + group;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if (in == 0) {
      stats[r][slot][0] = m[r];
      stats[r][slot][1] = l[r];
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) sums[r][slot][element(j / 4) + j % 4] = out[r][j];
  }
  __syncthreads();
  // a thread an element of a row
  for (int n = threadIdx.x; n < R * G * 8; n += kThreads) {
    const int r = n / (G * 8), e = n % (G * 8);
    if (r >= a.rows || e >= a.dim) continue;
    float top = stats[r][0][0];
#pragma unroll
    for (int i = 1; i < kGroups; ++i) top = fmaxf(top, stats[r][i][0]);
    const float from = top == -infinity() ? 0.0f : top;
    float sum = 0.0f, o = 0.0f;
#pragma unroll
    for (int i = 0; i < kGroups; ++i) {
      const float factor = exp2_fast(stats[r][i][0] - from);
      sum = __builtin_fmaf(stats[r][i][1], factor, sum);
      o = __builtin_fmaf(sums[r][i][e], factor, o);
    }
    if (a.parts) {
      const int64_t row = ((int64_t)head_of * a.parts + part) * a.rows + r;
      a.part_out[row * a.dim + e] = o;
      if (e < 2) a.part_stats[2 * row + e] = e ? sum : top;
      continue;
    }
    const RowAt at = row_at(a, kv_head, r);
    o = sum == 0.0f ? 0.0f : o / sum;
    ((float*)a.out.at)[batch * a.out.batch + at.head * a.out.head + at.query * a.out.pos + e] = o;
    if (a.lse && e == 0)
      a.lse[((int64_t)batch * a.heads + at.head) * a.queries + at.query] =
          sum == 0.0f ? infinity() : top + __builtin_amdgcn_logf(sum);
  }
}

template <int G, int R>
void launch_rows(const AttentionArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)(a.kv_heads * a.batch * (a.parts ? a.parts : 1)));
  if (past_caches(a))
    attention_token_kernel<G, R, true><<<grid, dim3(kThreads), 0, s>>>(a);
  else
    attention_token_kernel<G, R, false><<<grid, dim3(kThreads), 0, s>>>(a);
}

template <int G>
void launch_group(const AttentionArgs& a, hipStream_t s) {
  if (a.rows <= 1)
    launch_rows<G, 1>(a, s);
  else if (a.rows <= 2)
    launch_rows<G, 2>(a, s);
  else if (a.rows <= 4)
    launch_rows<G, 4>(a, s);
  else
    launch_rows<G, 8>(a, s);
}

}  // namespace

void launch_attention_token(const AttentionArgs& a, hipStream_t s) {
  if (a.dim <= 32)
    launch_group<4>(a, s);
  else if (a.dim <= 64)
    launch_group<8>(a, s);
  else
    launch_group<16>(a, s);
}

}  // namespace microadam
