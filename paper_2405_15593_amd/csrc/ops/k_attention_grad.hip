// Softmax attention, backward: the probabilities are computed again from q, k
// and each row's log sum.
//
//   p = 2^(c q k - lse),  ds = p (dout v - delta),  delta = sum dout out
//   dq = scale ds k,  dk = scale ds^T q,  dv = p^T dout
//
// Two kernels, each with its sums in registers, so that nothing is added in an
// order that changes: dq by rows, as forward, in z^T = k q^T, dp^T = v dout^T and
// dq^T += k^T ds^T; then dk and dv by keys, in z = q k^T, dp = dout v^T, dv^T +=
// dout^T p and dk^T += q^T ds, over all rows of the query heads that share the
// keys (split into parts that a third kernel joins where the keys' workgroups are
// few).  Seven products where one kernel with shared sums would take five.
//
// The matrix instruction takes p and ds in bfloat16 where the operands are that;
// their sums are binary32.  Where a workgroup's waves share rows or keys (SPLIT),
// what the rounding leaves over is multiplied too: p and ds have 16 bits, and the
// results' own rounding is the error that is left, 1.65e-3 of their norm instead of
// 2.35e-3 (both kernels, 3 x 515 rows, 1031 keys of 80: 56 -> 62 us).  Full workgroups,
// which the matrix cores bound, would take 1010 -> 1590 us for 2 x 4096 tokens, 32
// heads of 128, causal (dk and dv of 128 elements spill 120 bytes a lane): there p and
// ds are rounded, half a step, 2^-8 of each, with random signs.
//
// The bound is the matrix cores beside the vector work: 2 sequences of 4096 tokens,
// 32 heads of 128, causal, bfloat16 take 423 to 472 and 542 to 619 us (890 to 1010
// TFLOP/s of the products that are computed; a large library product 1390), the
// matrix cores 49 and 50% busy at 2.0 GHz, no bank conflicts.
#include <algorithm>

#include "attention_tile.h"

namespace microadam {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kRows = 128;      // of a workgroup, rows or keys
constexpr int kTile = 32;       // keys or rows of a tile

// SPLIT: where there are few rows (keys) for the CUs, a workgroup has 32 of them
// for all four waves, which take every fourth tile, each on its own way through
// its own place in LDS, and are joined at the end.

// The sums of the waves' same results, in wave 0: `sums` is free and has room for
// three waves' results.
template <int N>
__device__ inline void join_waves(float16v (&x)[N], float* sums, int wave, int lane) {
  __syncthreads();
  if (wave > 0) {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) sums[(((wave - 1) * N + i) * 16 + r) * 64 + lane] = x[i][r];
  }
  __syncthreads();
  if (wave > 0) return;
#pragma unroll
  for (int w = 0; w < kWaves - 1; ++w)
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) x[i][r] += sums[((w * N + i) * 16 + r) * 64 + lane];
}

template <bool BF16, int D, bool SPLIT>
__global__ __launch_bounds__(kThreads, (BF16 && !SPLIT) || D <= 64 ? 2 : 1) void attention_dq_kernel(const AttentionArgs a) {
  typedef Tile<BF16, D, kTile> T;
  constexpr int own_rows = SPLIT ? 32 : kRows;
  __shared__ __align__(16) uint8_t lds[SPLIT ? kWaves : 2][2][T::kBytes];  // [wave or turn][keys, values]
  static_assert(!SPLIT || sizeof(lds) >= (kWaves - 1) * D / 32 * 16 * 64 * sizeof(float), "the waves' sums");
  const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6);
  const int stager = SPLIT ? lane : (int)threadIdx.x;
  const int tiles = (a.rows + own_rows - 1) / own_rows;
  const Work work = work_of(blockIdx.x, gridDim.x, a.kv_heads * a.batch);
  const int tile = tiles - 1 - work.order, head_of = work.head;  // (the last rows see the most keys)
  const typename T::Lane places(lane);
  const int kv_head = head_of % a.kv_heads, batch = head_of / a.kv_heads;
  const int length = keys_of(a, batch);

  const int row = tile * own_rows + (SPLIT ? 0 : wave * 32) + (lane & 31);
  const bool live = row < a.rows;
  const RowAt at = row_at(a, kv_head, live ? row : 0);
  const int limit = live ? limit_of(a, at.query, length) : 0;
  const int most = wave_max(limit), least = wave_min(live ? limit : a.keys);
  Frag<BF16> q[D / 16], dout[D / 16];
  const int64_t q_at = batch * a.q.batch + at.head * a.q.head + at.query * a.q.pos;
  const int64_t do_at = batch * a.dout.batch + at.head * a.dout.head + at.query * a.dout.pos;
  const int64_t o_at = batch * a.out.batch + at.head * a.out.head + at.query * a.out.pos;
  const int64_t stat = ((int64_t)batch * a.heads + at.head) * a.queries + at.query;
  // (delta from out as it was before its rounding: of few keys ds is a small
  // difference to it; with out alone dk of three keys was off by 3.8e-3)
  float delta = 0.0f;
#pragma unroll
  for (int s = 0; s < D / 16; ++s) {
    const int d = 16 * s + 8 * (lane >> 5);
    const bool there = live && d < a.dim;
    q[s] = load_frag<BF16>(a.q.at, q_at + d, there);
    dout[s] = load_frag<BF16>(a.dout.at, do_at + d, there);
    const Frag<BF16> o = load_frag<BF16>(a.out.at, o_at + d, there);
#pragma unroll
    for (int j = 0; j < 8; ++j) delta = __builtin_fmaf((float)dout[s].v[j], (float)o.v[j], delta);
    if (BF16) {
      const Frag<BF16> rest = load_frag<BF16>(a.rest, stat * a.dim + d, there);
#pragma unroll
      for (int j = 0; j < 8; ++j) delta = __builtin_fmaf((float)dout[s].v[j], (float)rest.v[j], delta);
    }
  }
  delta = add_halves(delta);
  const float lse = live ? a.lse[stat] : infinity();
  if (live && lane < 32 && (!SPLIT || wave == 0)) a.delta[stat] = delta;

  const int turns = (last_key(a, tile * own_rows, own_rows, length) + kTile - 1) / kTile;

  Staged<BF16, D, kTile, SPLIT ? 64 : kThreads> next_k, next_v;
  constexpr int size = T::kSize;
  const int64_t k_pos = a.k.pos * size, v_pos = a.v.pos * size;
  const uint8_t* k_at = (const uint8_t*)a.k.at + (batch * a.k.batch + kv_head * a.k.head) * size;
  const uint8_t* v_at = (const uint8_t*)a.v.at + (batch * a.v.batch + kv_head * a.v.head) * size;
  next_k.start(a.dim, (int)k_pos, stager);
  next_v.start(a.dim, (int)v_pos, stager);
  auto load = [&](int turn) {
    next_k.load(k_at, k_pos, a.dim, turn * kTile, length);
    next_v.load(v_at, v_pos, a.dim, turn * kTile, length);
  };
  auto store = [&](int place) {
    next_k.store(lds[place][0], stager);
    next_v.store(lds[place][1], stager);
  };

  float16v dq[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) dq[i] = zeros();
  // (`more` loads the next tile: after the scores where what the loads pass through
  // is free only then)
  constexpr bool kLate = SPLIT && !BF16;
  auto add = [&](int turn, int place, auto more) {
    if (!kLate) more();
    const int first = turn * kTile;
    const uint8_t *keys = lds[place][0], *values = lds[place][1];
    if (first < most) {
      schedule_here();
      __builtin_amdgcn_s_setprio(1);
      float16v s = zeros(), dp = zeros();
#pragma unroll
      for (int step = 0; step < D / 16; ++step) {
        multiply(s, T::along(keys, places, 0, step), q[step]);
        multiply(dp, T::along(values, places, 0, step), dout[step]);
      }
      if (BF16) interleave<4, D / 8, D / 8>();
      schedule_here();
      __builtin_amdgcn_s_setprio(0);
      if (kLate) more();
      constexpr int ahead = D < 128 ? D / 16 : D / 32;  // (fragments that there are registers for)
      Frag<BF16> across[D / 16];
#pragma unroll
      for (int i = 0; i < ahead; ++i) across[i] = T::across(keys, places, 16 * (i % 2), i / 2);
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float p = exp2_fast(__builtin_fmaf(s[r], a.c, -lse));
        s[r] = p * (dp[r] - delta);
      }
      if (first + kTile > least) {
        // (a key that is a query's only one: p is 1 whatever the score, where dp -
        // delta would leave the rounding of two sums)
        const int end = limit > 1 ? limit : 0;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = first + 8 * (r / 4) + 4 * (lane >> 5) + r % 4 < end ? s[r] : 0.0f;
      }
      schedule_here();
      const Frag<BF16> d0 = as_frag<BF16, 0>(s), d1 = as_frag<BF16, 1>(s);
#pragma unroll
      for (int i = ahead; i < D / 16; ++i) across[i] = T::across(keys, places, 16 * (i % 2), i / 2);
#pragma unroll
      for (int part = 0; part < D / 32; ++part) {
        multiply(dq[part], across[2 * part], d0);
        multiply(dq[part], across[2 * part + 1], d1);
      }
      if constexpr (BF16 && SPLIT) {
        const Frag<true> r0 = rest_of<0>(s, d0), r1 = rest_of<1>(s, d1);
#pragma unroll
        for (int part = 0; part < D / 32; ++part) {
          multiply(dq[part], across[2 * part], r0);
          multiply(dq[part], across[2 * part + 1], r1);
        }
      }
    } else if (kLate) {
      more();
    }
  };
  if constexpr (SPLIT) {
    if (wave < turns) load(wave);
    wait_all();
    for (int turn = wave; turn < turns; turn += kWaves) {
      store(wave);
      wave_order();
      add(turn, wave, [&]() {
        if (turn + kWaves < turns) load(turn + kWaves);
      });
      wave_order();
    }
    join_waves(dq, (float*)&lds[0][0][0], wave, lane);
    if (wave > 0) return;
  } else {
    if (turns > 0) {
      load(0);
      store(0);
    }
    wait_all();
    __syncthreads();
    for (int turn = 0; turn < turns; ++turn) {
      add(turn, turn & 1, [&]() {
        if (turn + 1 < turns) load(turn + 1);
      });
      if (turn + 1 < turns) store((turn + 1) & 1);
      __syncthreads();
    }
  }
  if (!live) return;
  const int64_t dq_at = batch * a.dq.batch + at.head * a.dq.head + at.query * a.dq.pos;
#pragma unroll
  for (int i = 0; i < D / 32; ++i) store_column<BF16>(a.dq.at, dq_at + 32 * i, a.dim - 32 * i, dq[i], a.scale, lane);
}

template <bool BF16, int D, bool SPLIT>
__global__ __launch_bounds__(kThreads, (BF16 && !SPLIT) || D <= 64 ? 2 : 1) void attention_dkv_kernel(const AttentionArgs a) {
  typedef Tile<BF16, D, kTile> T;
  constexpr int own_keys = SPLIT ? 32 : kRows;
  constexpr int kPlaces = SPLIT ? kWaves : 2;
  // Two sums of 128 x 32, k and v are 192 registers with bfloat16's 128 elements:
  // two waves to a SIMD only with v in LDS.  Two workgroups then fill a CU's 160
  // KiB to the byte, so the rows' log sums and deltas lie in the tiles' padding.
  constexpr bool kKeep = SPLIT || !(BF16 && D == 128);
  typedef Tile<BF16, D, kRows> Own;
  constexpr bool kPadded = T::kPad == 4;
  constexpr int kTiles = kPlaces * 2 * T::kBytes;
  __shared__ __align__(16) uint8_t lds[kTiles + (kPadded ? 0 : kPlaces * 2 * kTile * 4) + (kKeep ? 0 : Own::kBytes)];
  uint8_t* const values = lds + kTiles;  // (128 elements a row are padded)
  static_assert(kKeep || kPadded, "values");
  static_assert(!SPLIT || sizeof(lds) >= (kWaves - 1) * D / 32 * 16 * 64 * sizeof(float), "the waves' sums");
  auto tile_at = [&](int place, int which) { return lds + (place * 2 + which) * T::kBytes; };  // queries, dout
  // log sums, deltas; four from a multiple of four on
  auto stats_at = [&](int place, int which, int i) {
    const int n = which * kTile + i;
    return (float*)(kPadded ? tile_at(place, 0) + (n >> 4) * T::kStride + T::kChunks * 16 + (n & 15) * 4
                            : lds + kTiles + (place * 2 * kTile + n) * 4);
  };
  const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6), h = lane >> 5;
  const int parts = !SPLIT && a.grad_parts ? a.grad_parts : 1;
  const Work work = work_of(blockIdx.x, gridDim.x, a.kv_heads * a.batch * parts);
  const int tile = work.order, head_of = work.head / parts;  // (the first keys are seen by the most rows)
  const int part = work.head - head_of * parts;
  const typename T::Lane places(lane);
  const int kv_head = head_of % a.kv_heads, batch = head_of / a.kv_heads;
  const int length = keys_of(a, batch);

  const int stager = SPLIT ? lane : (int)threadIdx.x;
  const int key0 = tile * own_keys, wave_key = key0 + (SPLIT ? 0 : wave * 32), key = wave_key + (lane & 31);
  const bool live = key < length;
  Frag<BF16> k[D / 16], v[kKeep ? D / 16 : 1];
  const int64_t k_at = batch * a.k.batch + kv_head * a.k.head + key * a.k.pos;
  const int64_t v_at = batch * a.v.batch + kv_head * a.v.head + key * a.v.pos;
#pragma unroll
  for (int s = 0; s < D / 16; ++s) {
    const int d = 16 * s + 8 * h;
    k[s] = load_frag<BF16>(a.k.at, k_at + d, live && d < a.dim);
    if (kKeep) v[kKeep ? s : 0] = load_frag<BF16>(a.v.at, v_at + d, live && d < a.dim);
  }
  if (!kKeep) {
    Staged<BF16, D, kRows, kThreads> all;
    const int64_t pos = a.v.pos * T::kSize;
    all.start(a.dim, (int)pos, threadIdx.x);
    all.load((const uint8_t*)a.v.at + (batch * a.v.batch + kv_head * a.v.head) * T::kSize, pos, a.dim, key0, length);
    all.store(values, threadIdx.x);
  }

  // The query heads one after the other, each from the first tile of queries that
  // see one of the workgroup's keys on.  The first tile of all begins with the first
  // query that sees a key: the others are not read, whose p of zero would not take
  // away a NaN.
  int from = 0, origin = 0;
  if (a.causal) {
    origin = a.queries > a.keys ? (a.queries - a.keys) % kTile : 0;
    from = key0 - (a.keys - a.queries) - origin;
    from = (from < 0 ? 0 : from) / kTile;
  }
  const int of_head = (a.queries - origin + kTile - 1) / kTile - from;
  const int all = key0 < length && of_head > 0 ? of_head * a.group : 0;
  const int start = (int)((int64_t)part * all / parts), turns = (int)((int64_t)(part + 1) * all / parts);

  Staged<BF16, D, kTile, SPLIT ? 64 : kThreads> next_q, next_do;
  float next_lse = 0.0f, next_delta = 0.0f;
  constexpr int size = T::kSize;
  const int64_t q_pos = a.q.pos * size, do_pos = a.dout.pos * size;
  next_q.start(a.dim, (int)q_pos, stager);
  next_do.start(a.dim, (int)do_pos, stager);
  auto load = [&](int turn) {
    const int of = uniform(turn / of_head), head = kv_head * a.group + of;
    const int first = (from + turn - of * of_head) * kTile + origin;
    next_q.load((const uint8_t*)a.q.at + (batch * a.q.batch + head * a.q.head) * size, q_pos, a.dim, first, a.queries);
    next_do.load((const uint8_t*)a.dout.at + (batch * a.dout.batch + head * a.dout.head) * size, do_pos, a.dim, first,
                 a.queries);
    if (stager < kTile) {
      const int64_t stat = ((int64_t)batch * a.heads + head) * a.queries;
      const int query = first + stager;
      next_lse = query < a.queries ? a.lse[stat + query] : infinity();
      next_delta = query < a.queries ? a.delta[stat + query] : 0.0f;
    }
  };
  auto store = [&](int place) {
    next_q.store(tile_at(place, 0), stager);
    next_do.store(tile_at(place, 1), stager);
    if (stager < kTile) {
      *stats_at(place, 0, stager) = next_lse;
      *stats_at(place, 1, stager) = next_delta;
    }
  };

  const typename Own::Lane own_places(lane);
  constexpr int kAhead = kKeep ? D / 32 : 2;  // of dout's fragments, read before the probabilities are done
  float16v dk[D / 32], dv[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) dk[i] = dv[i] = zeros();
  constexpr bool kLate = !kKeep || (SPLIT && !BF16);
  auto add = [&](int turn, int place, auto more) {
    if (!kLate) more();
    const uint8_t *queries = tile_at(place, 0), *douts = tile_at(place, 1);
    schedule_here();
    __builtin_amdgcn_s_setprio(1);
    float16v s = zeros(), dp = zeros();
#pragma unroll
    for (int step = 0; step < D / 16; ++step) {
      multiply(s, T::along(queries, places, 0, step), k[step]);
      const Frag<BF16> vs = kKeep ? v[kKeep ? step : 0] : Own::along(values, own_places, wave * 32, step);
      multiply(dp, T::along(douts, places, 0, step), vs);
    }
    if (BF16) interleave<4, D / 16 * (kKeep ? 2 : 3), D / 8, kKeep ? 1 : 2>();
    schedule_here();
    __builtin_amdgcn_s_setprio(0);
    if (kLate) more();
    Frag<BF16> across[D / 16];
    if (BF16) {
#pragma unroll
      for (int i = 0; i < kAhead; ++i) across[i] = T::across(douts, places, 16 * (i % 2), i / 2);
    }
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const float4v lse = *(const float4v*)stats_at(place, 0, 8 * g + 4 * h);
#pragma unroll
      for (int i = 0; i < 4; ++i) s[4 * g + i] = exp2_fast(__builtin_fmaf(s[4 * g + i], a.c, -lse[i]));
    }
    // the tile's first query does not see the wave's last key
    const int first = (from + turn - uniform(turn / of_head) * of_head) * kTile + origin;
    const int hidden = wave_key + 31 - (first + a.keys - a.queries);
    if (a.causal && hidden > 0) {
      const int at = (lane & 31) - 31 + hidden - 4 * h;  // rows below it do not see the lane's key
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = 8 * (r / 4) + r % 4 < at ? 0.0f : s[r];
    }
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const float4v delta = *(const float4v*)stats_at(place, 1, 8 * g + 4 * h);
#pragma unroll
      for (int i = 0; i < 4; ++i) dp[4 * g + i] = s[4 * g + i] * (dp[4 * g + i] - delta[i]);
    }
    // queries that see one key (as in dq): with one in all, or the first that sees any
    const int alone = a.queries - a.keys - first;
    if (length == 1 || (a.causal && wave_key == 0 && alone >= 0 && alone < kTile)) {
#pragma unroll
      for (int r = 0; r < 16; ++r) dp[r] = length == 1 || 8 * (r / 4) + 4 * h + r % 4 == alone ? 0.0f : dp[r];
    }
    const Frag<BF16> p0 = as_frag<BF16, 0>(s), p1 = as_frag<BF16, 1>(s);
    const Frag<BF16> d0 = as_frag<BF16, 0>(dp), d1 = as_frag<BF16, 1>(dp);
    if constexpr (BF16 && SPLIT) {
      schedule_here();
#pragma unroll
      for (int i = kAhead; i < D / 16; ++i) across[i] = T::across(douts, places, 16 * (i % 2), i / 2);
#pragma unroll
      for (int i = 0; i < D / 16; ++i) multiply(dv[i / 2], across[i], i % 2 ? p1 : p0);
      schedule_here();
      const Frag<BF16> pr0 = rest_of<0>(s, p0), pr1 = rest_of<1>(s, p1);
      const Frag<BF16> dr0 = rest_of<0>(dp, d0), dr1 = rest_of<1>(dp, d1);
#pragma unroll
      for (int i = 0; i < D / 16; ++i) multiply(dv[i / 2], across[i], i % 2 ? pr1 : pr0);
#pragma unroll
      for (int i = 0; i < D / 16; ++i) across[i] = T::across(queries, places, 16 * (i % 2), i / 2);
#pragma unroll
      for (int i = 0; i < D / 16; ++i) multiply(dk[i / 2], across[i], i % 2 ? d1 : d0);
#pragma unroll
      for (int i = 0; i < D / 16; ++i) multiply(dk[i / 2], across[i], i % 2 ? dr1 : dr0);
      schedule_here();
    } else if (BF16) {
      schedule_here();
#pragma unroll
      for (int i = kAhead; i < D / 16; ++i) across[i] = T::across(douts, places, 16 * (i % 2), i / 2);
#pragma unroll
      for (int i = 0; i < D / 16; ++i) multiply(dv[i / 2], across[i], i % 2 ? p1 : p0);
#pragma unroll
      for (int i = 0; i < D / 16; ++i) multiply(dk[i / 2], T::across(queries, places, 16 * (i % 2), i / 2), i % 2 ? d1 : d0);
      interleave<2 * (D / 16 - kAhead), 2 * (2 * (D / 16) - kAhead), D / 8, 2>();
      schedule_here();
    } else {
#pragma unroll
      for (int i = 0; i < D / 16; ++i) {
        multiply(dv[i / 2], T::across(douts, places, 16 * (i % 2), i / 2), i % 2 ? p1 : p0);
        multiply(dk[i / 2], T::across(queries, places, 16 * (i % 2), i / 2), i % 2 ? d1 : d0);
      }
    }
  };
  if constexpr (SPLIT) {
    if (wave < turns) load(wave);
    wait_all();
    for (int turn = wave; turn < turns; turn += kWaves) {
      store(wave);
      wave_order();
      add(turn, wave, [&]() {
        if (turn + kWaves < turns) load(turn + kWaves);
      });
      wave_order();
    }
    join_waves(dk, (float*)lds, wave, lane);
    join_waves(dv, (float*)lds, wave, lane);
    if (wave > 0) return;
  } else {
    if (turns > start) {
      load(start);
      store(start & 1);
    }
    wait_all();
    __syncthreads();
    for (int turn = start; turn < turns; ++turn) {
      add(turn, turn & 1, [&]() {
        if (turn + 1 < turns) load(turn + 1);
      });
      if (turn + 1 < turns) store((turn + 1) & 1);
      __syncthreads();
    }
  }
  if (key >= a.keys) return;
  // (a key behind the length has scores of its zeros: no gradient)
  if (parts > 1) {
    const int64_t rows = (int64_t)a.batch * a.kv_heads * a.keys, at = (int64_t)head_of * a.keys + key;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      store_column<false>(a.grad_part, (2 * part * rows + at) * a.dim + 32 * i, a.dim - 32 * i, live ? dk[i] : zeros(), 1.0f, lane);
      store_column<false>(a.grad_part, ((2 * part + 1) * rows + at) * a.dim + 32 * i, a.dim - 32 * i, live ? dv[i] : zeros(), 1.0f,
                          lane);
    }
    return;
  }
  const float one = live ? 1.0f : 0.0f;
  const int64_t dk_at = batch * a.dk.batch + kv_head * a.dk.head + key * a.dk.pos;
  const int64_t dv_at = batch * a.dv.batch + kv_head * a.dv.head + key * a.dv.pos;
#pragma unroll
  for (int i = 0; i < D / 32; ++i) {
    store_column<BF16>(a.dk.at, dk_at + 32 * i, a.dim - 32 * i, live ? dk[i] : zeros(), a.scale, lane);
    store_column<BF16>(a.dv.at, dv_at + 32 * i, a.dim - 32 * i, live ? dv[i] : zeros(), one, lane);
  }
}

// The parts of dk (blockIdx.y 0) and dv (1) joined, four elements a thread.
template <bool BF16>
__global__ __launch_bounds__(kThreads) void attention_dkv_join_kernel(const AttentionArgs a) {
  const int quads = a.dim / 4;
  const int64_t rows = (int64_t)a.batch * a.kv_heads * a.keys, n = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int64_t row = n / quads;
  if (row >= rows) return;
  const int d = (int)(n - row * quads) * 4, which = blockIdx.y;
  const float* from = a.grad_part + (which * rows + row) * a.dim + d;
  float4v sum = *(const float4v*)from;
  for (int p = 1; p < a.grad_parts; ++p) sum += *(const float4v*)(from + 2 * p * rows * a.dim);
  if (which == 0) sum *= a.scale;
  const int64_t head_of = row / a.keys, key = row - head_of * a.keys;
  const HeadTensor& to = which ? a.dv : a.dk;
  const int64_t at = head_of / a.kv_heads * to.batch + head_of % a.kv_heads * to.head + key * to.pos + d;
  if (BF16)
    ((Four2*)((uint16_t*)to.at + at))->q = uint2v{pack_bf16(sum[0], sum[1]), pack_bf16(sum[2], sum[3])};
  else
    ((Four4*)((float*)to.at + at))->q = sum;
}

template <bool BF16, int D>
void launch_both(const AttentionArgs& a, hipStream_t s) {
  const int heads = a.kv_heads * a.batch;
  const auto groups = [&](int n, int of) { return (unsigned)((int64_t)((n + of - 1) / of) * heads); };
  if (a.rows) {
    if (few_groups(a, a.rows))
      attention_dq_kernel<BF16, D, true><<<dim3(groups(a.rows, 32)), dim3(kThreads), 0, s>>>(a);
    else
      attention_dq_kernel<BF16, D, false><<<dim3(groups(a.rows, kRows)), dim3(kThreads), 0, s>>>(a);
  }
  if (a.keys) {
    if (a.grad_parts) {
      attention_dkv_kernel<BF16, D, false><<<dim3(groups(a.keys, kRows) * a.grad_parts), dim3(kThreads), 0, s>>>(a);
      const int64_t quads = (int64_t)heads * a.keys * (a.dim / 4);
      attention_dkv_join_kernel<BF16><<<dim3((unsigned)((quads + kThreads - 1) / kThreads), 2), dim3(kThreads), 0, s>>>(a);
    } else if (few_groups(a, a.keys))
      attention_dkv_kernel<BF16, D, true><<<dim3(groups(a.keys, 32)), dim3(kThreads), 0, s>>>(a);
    else
      attention_dkv_kernel<BF16, D, false><<<dim3(groups(a.keys, kRows)), dim3(kThreads), 0, s>>>(a);
  }
}

template <bool BF16>
void launch_dim(const AttentionArgs& a, hipStream_t s) {
  if (a.dim <= 32)
    launch_both<BF16, 32>(a, s);
  else if (a.dim <= 64)
    launch_both<BF16, 64>(a, s);
  else if (a.dim <= 96)
    launch_both<BF16, 96>(a, s);
  else
    launch_both<BF16, 128>(a, s);
}

}  // namespace

// Where the query heads that share a key head are many, its workgroups are few and
// long, causal ones of all lengths: the rows are then split into parts of 64 tiles
// and more, up to four (causal; else two) workgroups of them to a CU.  Where there
// are not even workgroups of 128 keys for the CUs, into parts of 16 tiles and more,
// instead of the shared ones, if there are eight.  dq, dk and dv, not split / split, us:
//   bfloat16  32 heads of 128 on 8   2 x 2048 causal 508 / 330   full 592 / 505
//                                    1 x 4096        973 / 572       1119 / 925
//             32 of 128 on 1         1 x 4096       1818 / 619
//             4 of 64 on 1           1 x 4096        151 / 82         166 / 106
//             (parts of 32 tiles: 32 on 32, 1 x 2048  191 / 200       247 / 289)
//   binary32  16 of 128 on 2         1 x 2048       1484 / 698       1692 / 1065
int32_t attention_grad_parts(const AttentionArgs& a) {
  const int64_t groups = (int64_t)((a.keys + kRows - 1) / kRows) * a.kv_heads * a.batch;
  if (groups < 1 || a.rows < 1) return 0;
  const int64_t turns = (int64_t)((a.queries + kTile - 1) / kTile) * a.group;  // of a workgroup, at most
  const bool few = few_groups(a, a.keys);
  const int64_t want = few || a.causal ? 1024 : 512;
  const int64_t parts = std::min((want + groups - 1) / groups, turns / (few ? 16 : 64));
  return parts >= (few ? 8 : 2) ? (int32_t)parts : 0;
}

hipError_t launch_attention_grad(const AttentionArgs& a, hipStream_t s) {
  if (a.bf16)
    launch_dim<true>(a, s);
  else
    launch_dim<false>(a, s);
  return hipGetLastError();
}

}  // namespace microadam
