// Softmax attention, forward.
//
//   z = scale q k, masked: a query sees the first min(length, query + 1 + keys -
//   queries if causal) keys;  p = softmax z;  out = p v;  lse = log2 sum 2^(c q k)
//
// One pass over the keys with the running maximum and sum.  The query heads that
// share a key head are the rows of one matrix.  A wave takes 32 rows: it keeps
// their q as B fragments and out^T in the accumulators, and computes z^T = k q^T
// and out^T += v^T p^T, so that a row's maximum, sum and factor are its lane's
// own.  Four waves share the tiles of keys and values in LDS, which the next
// tile's loads pass in registers.
//
// The bound of many rows is the matrix cores beside the exponentials: 2 sequences
// of 4096 tokens, 32 heads of 128, causal, bfloat16 take 306 to 349 us (790 to 900
// TFLOP/s; a large library product 1390), the matrix cores 44% busy at 2.0 GHz
// (alone they run at 1.6), vector instructions 42% of the time, no bank conflicts.
// Two waves a SIMD interleave them; eight waves in two groups that take turns at
// the two kinds of work gave 1%.  The bound of few rows is memory: one query of 32
// heads on 8 over 8 x 4096 keys 25 us and 4 for the join (134 MB, 5.4 TB/s).
#include <algorithm>

#include "attention_tile.h"

namespace microadam {
namespace {

constexpr int kThreads = 256;
constexpr int kRows = 128;  // of a workgroup

template <bool BF16>
constexpr int kKeys = BF16 ? 64 : 32;  // of a tile

// z^T of a tile.
template <bool BF16, int D, int KEYS>
__device__ inline void scores(float16v (&s)[KEYS / 32], const uint8_t* tile, const typename Tile<BF16, D, KEYS>::Lane& at,
                              const Frag<BF16> (&q)[D / 16]) {
  constexpr int n = KEYS / 32;
  schedule_here();
  __builtin_amdgcn_s_setprio(1);
#pragma unroll
  for (int i = 0; i < n; ++i) s[i] = zeros();
#pragma unroll
  for (int step = 0; step < D / 16; ++step)
#pragma unroll
    for (int i = 0; i < n; ++i) multiply(s[i], Tile<BF16, D, KEYS>::along(tile, at, 32 * i, step), q[step]);
  if (BF16) interleave<4, D / 16 * n, D / 16 * n>();
  schedule_here();
  __builtin_amdgcn_s_setprio(0);
}

template <int N>
__device__ inline void mask(float16v (&s)[N], int first, int limit, int lane, float with) {
  const int h = lane >> 5;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) s[i][r] = first + 32 * i + 8 * (r / 4) + 4 * h + r % 4 < limit ? s[i][r] : with;
}

// out^T += v^T p^T of a tile, with the running maximum m (in units of ln 2) and
// the lane's part l of the sum.  m follows a row's maximum only where that is
// more than kAhead above it: the probabilities' common factor cancels, and most
// tiles pass without a factor for sum and output.  Each row decides for itself
// (its factor is 1 where another row's is not), so that no row's bits go by its
// neighbours.
//
// The matrix instruction takes p in bfloat16 where v is that.  WHOLE: what p's
// rounding leaves over is multiplied too, so that p has 16 bits and out's own
// rounding is the error that is left, 1.6e-3 of the result's norm instead of 2.1e-3
// to 2.4e-3.  It is taken where a workgroup's waves share rows: one token's time
// goes by memory (8 x 4096 keys 28.2 -> 28.7 us, 64 x 2048 83 -> 84), some hundred
// rows' by the way of a tile (3 x 515 rows, 1031 keys of 80, 17.7 -> 20.3).  Full
// workgroups of 128 rows, which the matrix cores bound, would take 360 -> 450 us for
// 2 x 4096 tokens, 32 heads of 128, causal: there p is rounded, half a step, 2^-8 of
// each, with random signs.
constexpr float kAhead = 8.0f;

template <bool BF16, int D, int KEYS, bool WHOLE>
__device__ inline void add_tile(float16v (&s)[KEYS / 32], const uint8_t* values,
                                const typename Tile<BF16, D, KEYS>::Lane& at, float c, float& m, float& l,
                                float16v (&out)[D / 32]) {
  float top = s[0][0];
#pragma unroll
  for (int i = 0; i < KEYS / 32; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) top = fmaxf(top, s[i][r]);
  top = max_halves(top) * c;
  const bool ahead = top > m + kAhead;  // (of -infinity: any score)
  if (__any(ahead)) {
    const float next = ahead ? top : m;
    const float factor = ahead ? exp2_fast(m - next) : 1.0f;
    m = next;
    l *= factor;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) out[i] *= factor;
  }
  const float from = m == -infinity() ? 0.0f : -m;
  typedef Tile<BF16, D, KEYS> T;
  constexpr int n = KEYS / 32, parts = D / 32;
  auto weights = [&](float16v& x) {
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      x[r] = exp2_fast(__builtin_fmaf(x[r], c, from));
      l += x[r];
    }
  };
  Frag<BF16> v[2 * parts];
  auto read = [&](int i) {
#pragma unroll
    for (int k = 0; k < 2 * parts; ++k) v[k] = T::across(values, at, 32 * i + 16 * (k % 2), k / 2);
  };
  schedule_here();
  read(0);
  weights(s[0]);
  schedule_here();
#pragma unroll
  for (int i = 0; i < n; ++i) {
    const Frag<BF16> p0 = as_frag<BF16, 0>(s[i]), p1 = as_frag<BF16, 1>(s[i]);
#pragma unroll
    for (int part = 0; part < parts; ++part) {
      multiply(out[part], v[2 * part], p0);
      multiply(out[part], v[2 * part + 1], p1);
    }
    if constexpr (BF16 && WHOLE) {
      const Frag<true> r0 = rest_of<0>(s[i], p0), r1 = rest_of<1>(s[i], p1);
#pragma unroll
      for (int part = 0; part < parts; ++part) {
        multiply(out[part], v[2 * part], r0);
        multiply(out[part], v[2 * part + 1], r1);
      }
    }
    if (i + 1 < n) {
      read(i + 1);
      weights(s[i + 1]);
      schedule_here();
    }
  }
}

// What a wave has of its rows when its keys are through (l the lanes' sum):
// the result, or where the keys are split a part of it.
template <bool BF16, int D>
__device__ inline void finish(const AttentionArgs& a, int head_of, int batch, int row, const RowAt& at, int part, float m,
                              float l, const float16v (&out)[D / 32], int lane) {
  if (a.parts) {
    const int64_t n = ((int64_t)head_of * a.parts + part) * a.rows + row;
    if (lane < 32) *(float2v*)(a.part_stats + 2 * n) = float2v{m, l};
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
      store_column<false>(a.part_out, n * a.dim + 32 * i, a.dim - 32 * i, out[i], 1.0f, lane);
    return;
  }
  const float over = l == 0.0f ? 0.0f : 1.0f / l;
  const int64_t o_at = batch * a.out.batch + at.head * a.out.head + at.query * a.out.pos;
#pragma unroll
  for (int i = 0; i < D / 32; ++i) store_column<BF16>(a.out.at, o_at + 32 * i, a.dim - 32 * i, out[i], over, lane);
  if (!a.lse) return;
  const int64_t stat = ((int64_t)batch * a.heads + at.head) * a.queries + at.query;
  if (lane < 32) a.lse[stat] = l == 0.0f ? infinity() : m + __builtin_amdgcn_logf(l);
  if (BF16) {
#pragma unroll
    for (int i = 0; i < D / 32; ++i) store_rest(a.rest, stat * a.dim + 32 * i, a.dim - 32 * i, out[i], over, lane);
  }
}

// The tiles [first, last) of a part of `tiles`.
struct Part {
  int first, last;
};
__device__ inline Part part_of(const AttentionArgs& a, int part, int tiles) {
  if (!a.parts) return {0, tiles};
  return {(int)((int64_t)part * tiles / a.parts), (int)((int64_t)(part + 1) * tiles / a.parts)};
}

template <bool BF16, int D>
__global__ __launch_bounds__(kThreads, BF16 || D <= 64 ? 2 : 1) void attention_kernel(const AttentionArgs a) {
  constexpr int keys = kKeys<BF16>;
  typedef Tile<BF16, D, keys> T;
  __shared__ __align__(16) uint8_t lds[2][2][T::kBytes];  // [turn][keys, values]
  const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6);
  const int tiles = (a.rows + kRows - 1) / kRows;
  const Work work = work_of(blockIdx.x, gridDim.x, a.kv_heads * a.batch);
  const int tile = tiles - 1 - work.order, head_of = work.head;  // (the last rows see the most keys)
  const typename T::Lane places(lane);
  const int kv_head = head_of % a.kv_heads, batch = head_of / a.kv_heads;
  const int length = keys_of(a, batch);

  const int row = tile * kRows + wave * 32 + (lane & 31);
  const bool live = row < a.rows;
  const RowAt at = row_at(a, kv_head, live ? row : 0);
  const int limit = live ? limit_of(a, at.query, length) : 0;
  const int most = wave_max(limit), least = wave_min(live ? limit : a.keys);
  Frag<BF16> q[D / 16];
  const int64_t q_at = batch * a.q.batch + at.head * a.q.head + at.query * a.q.pos;
#pragma unroll
  for (int s = 0; s < D / 16; ++s) {
    const int d = 16 * s + 8 * (lane >> 5);
    q[s] = load_frag<BF16>(a.q.at, q_at + d, live && d < a.dim);
  }

  const int turns = (last_key(a, tile * kRows, kRows, length) + keys - 1) / keys;

  Staged<BF16, D, keys, kThreads> next_k, next_v;
  constexpr int size = T::kSize;
  const int64_t k_pos = a.k.pos * size, v_pos = a.v.pos * size;
  const uint8_t* k_at = (const uint8_t*)a.k.at + (batch * a.k.batch + kv_head * a.k.head) * size;
  const uint8_t* v_at = (const uint8_t*)a.v.at + (batch * a.v.batch + kv_head * a.v.head) * size;
  next_k.start(a.dim, (int)k_pos, threadIdx.x);
  next_v.start(a.dim, (int)v_pos, threadIdx.x);
  auto load = [&](int turn) {
    next_k.load(k_at, k_pos, a.dim, turn * keys, length);
    next_v.load(v_at, v_pos, a.dim, turn * keys, length);
  };
  auto store = [&](int turn) {
    next_k.store(lds[turn & 1][0], threadIdx.x);
    next_v.store(lds[turn & 1][1], threadIdx.x);
  };

  float m = -infinity(), l = 0.0f;
  float16v out[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) out[i] = zeros();
  if (turns > 0) {
    load(0);
    store(0);
  }
  wait_all();
  __syncthreads();
  for (int turn = 0; turn < turns; ++turn) {
    if (turn + 1 < turns) load(turn + 1);
    const int first = turn * keys;
    if (first < most) {
      float16v s[keys / 32];
      scores<BF16, D, keys>(s, lds[turn & 1][0], places, q);
      if (first + keys > least) mask(s, first, limit, lane, -infinity());
      add_tile<BF16, D, keys, false>(s, lds[turn & 1][1], places, a.c, m, l, out);
    }
    if (turn + 1 < turns) store(turn + 1);
    __syncthreads();
  }

  l = add_halves(l);
  if (live) finish<BF16, D>(a, head_of, batch, row, at, 0, m, l, out, lane);
}

// Where there are few rows for the CUs, a token's or some hundred: the four waves
// of a workgroup take the same 32 rows and every fourth tile of the part's keys,
// each on its own way through its own place in LDS, and are joined at the end.
constexpr int kFewRows = 32, kFewKeys = 32;

template <bool BF16, int D, bool PAST>
__global__ __launch_bounds__(kThreads, BF16 || D <= 64 ? 2 : 1) void attention_few_kernel(const AttentionArgs a) {
  typedef Tile<BF16, D, kFewKeys> T;
  constexpr int kWaves = kThreads / 64;
  constexpr int kSums = D / 32 * 16 + 2;  // floats that a lane hands over
  __shared__ __align__(16) uint8_t lds[kWaves][2][T::kBytes];
  static_assert((kWaves - 1) * kSums * 64 * sizeof(float) <= sizeof(lds), "the waves' sums");
  const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6);
  int block = blockIdx.x, part = 0;
  if (a.parts) {
    part = block % a.parts;
    block /= a.parts;
  }
  const int tiles = (a.rows + kFewRows - 1) / kFewRows;
  const Work work = work_of(block, gridDim.x / (a.parts ? a.parts : 1), a.kv_heads * a.batch);
  const int tile = tiles - 1 - work.order, head_of = work.head;  // (the last rows see the most keys)
  const int kv_head = head_of % a.kv_heads, batch = head_of / a.kv_heads;
  const int length = keys_of(a, batch);
  const Part own = part_of(a, part, (last_key(a, tile * kFewRows, kFewRows, length) + kFewKeys - 1) / kFewKeys);

  Staged<BF16, D, kFewKeys, 64> next_k, next_v;
  constexpr int size = T::kSize;
  const int64_t k_pos = a.k.pos * size, v_pos = a.v.pos * size;
  const uint8_t* k_at = (const uint8_t*)a.k.at + (batch * a.k.batch + kv_head * a.k.head) * size;
  const uint8_t* v_at = (const uint8_t*)a.v.at + (batch * a.v.batch + kv_head * a.v.head) * size;
  next_k.start(a.dim, (int)k_pos, lane);
  next_v.start(a.dim, (int)v_pos, lane);
  int turn = own.first + wave;
  auto load = [&](int t) {
    next_k.template load<PAST>(k_at, k_pos, a.dim, t * kFewKeys, length);
    next_v.template load<PAST>(v_at, v_pos, a.dim, t * kFewKeys, length);
  };
  if (turn < own.last) load(turn);

  const int row = tile * kFewRows + (lane & 31);
  const bool live = row < a.rows;
  const RowAt at = row_at(a, kv_head, live ? row : 0);
  const int limit = live ? limit_of(a, at.query, length) : 0;
  const int least = wave_min(live ? limit : a.keys);
  Frag<BF16> q[D / 16];
  const int64_t q_at = batch * a.q.batch + at.head * a.q.head + at.query * a.q.pos;
#pragma unroll
  for (int s = 0; s < D / 16; ++s) {
    const int d = 16 * s + 8 * (lane >> 5);
    q[s] = load_frag<BF16>(a.q.at, q_at + d, live && d < a.dim);
  }
  float m = -infinity(), l = 0.0f;
  float16v out[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) out[i] = zeros();
  wait_all();
  uint8_t *keys = lds[wave][0], *values = lds[wave][1];
  const typename T::Lane places(lane);
  for (; turn < own.last; turn += kWaves) {
    next_k.store(keys, lane);
    next_v.store(values, lane);
    if (turn + kWaves < own.last) load(turn + kWaves);
    wave_order();
    const int first = turn * kFewKeys;
    float16v s[1];
    scores<BF16, D, kFewKeys>(s, keys, places, q);
    if (first + kFewKeys > least) mask(s, first, limit, lane, -infinity());
    add_tile<BF16, D, kFewKeys, true>(s, values, places, a.c, m, l, out);
    wave_order();
  }
  l = add_halves(l);

  __syncthreads();
  float* sums = (float*)&lds[0][0][0];
  if (wave > 0) {
    float* to = sums + (wave - 1) * kSums * 64 + lane;
    to[0] = m;
    to[64] = l;
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) to[(2 + 16 * i + r) * 64] = out[i][r];
  }
  __syncthreads();
  if (wave > 0 || !live) return;
  float top = m;
#pragma unroll
  for (int w = 0; w < kWaves - 1; ++w) top = fmaxf(top, sums[w * kSums * 64 + lane]);
  const float from = top == -infinity() ? 0.0f : top;
  const float own_factor = exp2_fast(m - from);
  l *= own_factor;
#pragma unroll
  for (int i = 0; i < D / 32; ++i) out[i] *= own_factor;
#pragma unroll
  for (int w = 0; w < kWaves - 1; ++w) {
    const float* other = sums + w * kSums * 64 + lane;
    const float factor = exp2_fast(other[0] - from);
    l = __builtin_fmaf(other[64], factor, l);
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) out[i][r] = __builtin_fmaf(other[(2 + 16 * i + r) * 64], factor, out[i][r]);
  }
  finish<BF16, D>(a, head_of, batch, row, at, part, top, l, out, lane);
}

// The parts of a row's keys joined by WAVES waves: lane i has the sums of parts i,
// i + 64, .., then two elements of the row; the waves share the parts.
template <bool BF16, int WAVES>
__global__ __launch_bounds__(WAVES == 1 ? kThreads : 64 * WAVES) void attention_join_kernel(const AttentionArgs a) {
  constexpr int kEach = kMostParts / 64, kRowsHere = WAVES == 1 ? kThreads / 64 : 1;
  __shared__ float2v others[WAVES * kRowsHere][64];
  const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6), which = wave % WAVES;
  const int64_t rows = (int64_t)a.batch * a.kv_heads * a.rows, n = (int64_t)blockIdx.x * kRowsHere + wave / WAVES;
  const bool live = n < rows;
  const int64_t head_of = live ? n / a.rows : 0;
  const int row = live ? (int)(n - head_of * a.rows) : 0;
  const int batch = (int)(head_of / a.kv_heads);
  const RowAt at = row_at(a, (int)(head_of % a.kv_heads), row);
  const int64_t first = head_of * a.parts * a.rows + row;
  float m[kEach], l[kEach], top = -infinity();
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int part = 64 * i + lane;
    const bool there = live && part < a.parts;
    const float2v s = there ? *(const float2v*)(a.part_stats + 2 * (first + (int64_t)part * a.rows)) : float2v{0.0f, 0.0f};
    m[i] = there ? s[0] : -infinity();
    l[i] = s[1];
    top = fmaxf(top, m[i]);
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  const float from = top == -infinity() ? 0.0f : top;
  float sum = 0.0f;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    m[i] = exp2_fast(m[i] - from);
    sum = __builtin_fmaf(m[i], l[i], sum);
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
  const int d = 2 * lane;
  float2v o = {0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int parts = a.parts - 64 * i < 64 ? a.parts - 64 * i : 64;
    const float* from_part = a.part_out + (first + (int64_t)64 * i * a.rows) * a.dim + d;
    for (int p = 8 * which; p < parts; p += 8 * WAVES) {
      float2v x[8];
#pragma unroll
      for (int u = 0; u < 8; ++u)
        x[u] = live && p + u < parts && d < a.dim ? *(const float2v*)(from_part + (int64_t)(p + u) * a.rows * a.dim)
                                                  : float2v{0.0f, 0.0f};
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const float factor = __shfl(m[i], (p + u) & 63);
        o[0] = __builtin_fmaf(factor, x[u][0], o[0]);
        o[1] = __builtin_fmaf(factor, x[u][1], o[1]);
      }
    }
  }
  if (WAVES > 1) {
    others[wave][lane] = o;
    __syncthreads();
    if (which != 0) return;
#pragma unroll
    for (int w = 1; w < WAVES; ++w) o += others[wave + w][lane];
  }
  if (!live) return;
  const float over = sum == 0.0f ? 0.0f : 1.0f / sum;
  const int64_t stat = ((int64_t)batch * a.heads + at.head) * a.queries + at.query;
  if (d < a.dim) {
    const int64_t to = batch * a.out.batch + at.head * a.out.head + at.query * a.out.pos + d;
    o *= over;
    Elements<BF16>::store1(a.out.at, to, o[0]);
    Elements<BF16>::store1(a.out.at, to + 1, o[1]);
    if (BF16 && a.lse) {
      const uint32_t q = pack_bf16(o[0], o[1]);
      *(uint32_t*)(a.rest + stat * a.dim + d) =
          pack_bf16(o[0] - __uint_as_float(q << 16), o[1] - __uint_as_float(q & 0xffff0000u));
    }
  }
  if (a.lse && lane == 0) a.lse[stat] = sum == 0.0f ? infinity() : top + __builtin_amdgcn_logf(sum);
}

// Whether the rows go to attention_few_kernel: besides few_groups' rule causal ones
// of many keys whatever the head's size (bfloat16, shared or not, us: 16 heads of 96,
// 2048 keys, 256 workgroups 38 / 45; 4 of 128, 8192 keys, 256 148 / 164; 10 of 128,
// 4096 keys, 320 98 / 90; 12 of 128, 4096 keys, 384 110 / 91).
bool few_rows(const AttentionArgs& a) {
  const int64_t groups = (int64_t)((a.rows + kRows - 1) / kRows) * a.kv_heads * a.batch;
  const bool uneven = a.bf16 && a.causal && a.keys >= 2048 && a.queries >= a.keys / 2;
  return a.rows <= kFewRows || few_groups(a, a.rows) || (uneven && groups <= 256);
}

template <bool BF16, int D>
void launch_rows(const AttentionArgs& a, hipStream_t s) {
  const int heads = a.kv_heads * a.batch, parts = a.parts ? a.parts : 1;
  const bool few = few_rows(a);
  const int tiles = few ? (a.rows + kFewRows - 1) / kFewRows : (a.rows + kRows - 1) / kRows;
  if (!BF16 && token_rows(a))
    launch_attention_token(a, s);
  else if (few && tiles == 1 && past_caches(a))
    attention_few_kernel<BF16, D, true><<<dim3((unsigned)(heads * parts)), dim3(kThreads), 0, s>>>(a);
  else if (few)
    attention_few_kernel<BF16, D, false><<<dim3((unsigned)(tiles * heads * parts)), dim3(kThreads), 0, s>>>(a);
  else
    attention_kernel<BF16, D><<<dim3((unsigned)(tiles * heads)), dim3(kThreads), 0, s>>>(a);
  if (a.parts) {
    // (waves to a row; of 32, 128 and 256 parts sixteen instead of four: 13.5 -> 12.7,
    // 14.0 -> 12.9 and 19.9 -> 16.9 us for both launches)
    const int64_t rows = (int64_t)heads * a.rows, waves = kThreads / 64;
    if (a.parts > 16)
      attention_join_kernel<BF16, 16><<<dim3((unsigned)rows), dim3(1024), 0, s>>>(a);
    else if (a.parts > 8)
      attention_join_kernel<BF16, 4><<<dim3((unsigned)rows), dim3(256), 0, s>>>(a);
    else
      attention_join_kernel<BF16, 1><<<dim3((unsigned)((rows + waves - 1) / waves)), dim3(kThreads), 0, s>>>(a);
  }
}

template <bool BF16>
void launch_dim(const AttentionArgs& a, hipStream_t s) {
  if (a.dim <= 32)
    launch_rows<BF16, 32>(a, s);
  else if (a.dim <= 64)
    launch_rows<BF16, 64>(a, s);
  else if (a.dim <= 96)
    launch_rows<BF16, 96>(a, s);
  else
    launch_rows<BF16, 128>(a, s);
}

}  // namespace

// Keys are split where the rows alone are too few workgroups for 256 CUs: into
// as many parts as give two to a CU, of at least so many keys that a part's work
// is worth the join (4 to 5 us with its launch).
int32_t attention_parts(const AttentionArgs& a) {
  if (!token_rows(a) && !few_rows(a)) return 0;
  const int64_t tiles = token_rows(a) ? 1 : (a.rows + kFewRows - 1) / kFewRows, groups = tiles * a.kv_heads * a.batch;
  if (groups < 1 || groups >= 256) return 0;
  const int64_t parts = std::min((512 + groups - 1) / groups, (int64_t)a.keys / (token_rows(a) ? 128 : 256));
  return parts > 1 ? (int32_t)std::min<int64_t>(parts, kMostParts) : 0;
}

hipError_t launch_attention(const AttentionArgs& a, hipStream_t s) {
  if (a.bf16)
    launch_dim<true>(a, s);
  else
    launch_dim<false>(a, s);
  return hipGetLastError();
}

}  // namespace microadam
