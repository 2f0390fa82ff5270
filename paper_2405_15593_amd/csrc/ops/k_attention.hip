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
#include "attention_tile.h"

namespace microadam {
namespace {

constexpr int kThreads = 256;
constexpr int kRows = 128;  // of a workgroup

template <bool BF16>
constexpr int kKeys = BF16 ? 64 : 32;  // of a tile

// z^T of a tile, masked by the lane's limit where asked.
template <bool BF16, int D, int KEYS>
__device__ inline void scores(float16v (&s)[KEYS / 32], const uint8_t* tile, const Frag<BF16> (&q)[D / 16], int lane) {
#pragma unroll
  for (int i = 0; i < KEYS / 32; ++i) s[i] = zeros();
#pragma unroll
  for (int step = 0; step < D / 16; ++step)
#pragma unroll
    for (int i = 0; i < KEYS / 32; ++i) multiply(s[i], Tile<BF16, D, KEYS>::along(tile, 32 * i, step, lane), q[step]);
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
constexpr float kAhead = 8.0f;

template <bool BF16, int D, int KEYS>
__device__ inline void add_tile(float16v (&s)[KEYS / 32], const uint8_t* values, float c, float& m, float& l,
                                float16v (&out)[D / 32], int lane) {
  float top = s[0][0];
#pragma unroll
  for (int i = 0; i < KEYS / 32; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) top = fmaxf(top, s[i][r]);
  top = fmaxf(top, __shfl_xor(top, 32)) * c;
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
#pragma unroll
  for (int i = 0; i < KEYS / 32; ++i) {
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[i][r] = exp2_fast(__builtin_fmaf(s[i][r], c, from));
      l += s[i][r];
    }
    const Frag<BF16> p0 = as_frag<BF16, 0>(s[i]), p1 = as_frag<BF16, 1>(s[i]);
#pragma unroll
    for (int part = 0; part < D / 32; ++part) {
      multiply(out[part], Tile<BF16, D, KEYS>::across(values, 32 * i, part, lane), p0);
      multiply(out[part], Tile<BF16, D, KEYS>::across(values, 32 * i + 16, part, lane), p1);
    }
  }
}

template <bool BF16, int D>
__global__ __launch_bounds__(kThreads, BF16 ? 2 : 1) void attention_kernel(const AttentionArgs a) {
  constexpr int keys = kKeys<BF16>;
  typedef Tile<BF16, D, keys> T;
  __shared__ __align__(16) uint8_t lds[2][2][T::kBytes];  // [turn][keys, values]
  const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6);
  const int tiles = (a.rows + kRows - 1) / kRows;
  const int work = run_of_xcd(blockIdx.x, gridDim.x);
  // (the last rows see the most keys: first)
  const int tile = tiles - 1 - work % tiles, head_of = work / tiles;
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

  // the workgroup's last key
  int end;
  {
    const int first = tile * kRows, last = first + kRows < a.rows ? first + kRows - 1 : a.rows - 1;
    const int whole = first / a.queries != last / a.queries;  // rows of two heads: the last query is among them
    end = limit_of(a, whole ? a.queries - 1 : last % a.queries, length);
  }
  const int turns = (end + keys - 1) / keys;

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
      scores<BF16, D, keys>(s, lds[turn & 1][0], q, lane);
      if (first + keys > least) mask(s, first, limit, lane, -infinity());
      add_tile<BF16, D, keys>(s, lds[turn & 1][1], a.c, m, l, out, lane);
    }
    if (turn + 1 < turns) store(turn + 1);
    __syncthreads();
  }

  l += __shfl_xor(l, 32);
  if (!live) return;
  const float over = l == 0.0f ? 0.0f : 1.0f / l;
  const int64_t o_at = batch * a.out.batch + at.head * a.out.head + at.query * a.out.pos;
#pragma unroll
  for (int i = 0; i < D / 32; ++i) store_column<BF16>(a.out.at, o_at + 32 * i, a.dim - 32 * i, out[i], over, lane);
  if (a.lse && lane < 32)
    a.lse[((int64_t)batch * a.heads + at.head) * a.queries + at.query] =
        l == 0.0f ? infinity() : m + __builtin_amdgcn_logf(l);
}

template <bool BF16, int D>
void launch_rows(const AttentionArgs& a, hipStream_t s) {
  const int tiles = (a.rows + kRows - 1) / kRows;
  attention_kernel<BF16, D><<<dim3((unsigned)(tiles * a.kv_heads * a.batch)), dim3(kThreads), 0, s>>>(a);
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

void attention_parts(const AttentionArgs&, int32_t& parts, int32_t& part_keys) { parts = part_keys = 0; }

hipError_t launch_attention(const AttentionArgs& a, hipStream_t s) {
  if (a.bf16)
    launch_dim<true>(a, s);
  else
    launch_dim<false>(a, s);
  return hipGetLastError();
}

}  // namespace microadam
