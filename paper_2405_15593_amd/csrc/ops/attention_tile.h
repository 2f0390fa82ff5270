// What the attention kernels share: fragments of the matrix instruction, tiles
// in LDS, rows and their limits.
//
// All products run on the 32x32 matrix instructions in one form, D = A B with D's
// column in lane % 32: its rows 8 (i / 4) + 4 (lane / 32) + i % 4 are the lane's
// sixteen results i.  A product's results are then the next one's B as they lie,
// eight of them a step of sixteen, when its A is read with the rows of the sum in
// that order: scores never leave the registers.  A fragment is eight elements a
// lane for both types: one 32x32x16 instruction of bfloat16, eight 32x32x2 of
// binary32.
//
// Tiles keep the rows of q, k, v or dout.  A row's 16-byte chunks c lie at
// c ^ (row / 4 % 4), and rows are padded to 4 or 12 chunks modulo 16, so that
// neither sixteen rows' same chunk (a fragment along the row) nor four rows' four
// chunks (the transposing read) meet on a bank.
#pragma once
#include "attention_device.h"
#include "elements.h"

namespace microadam {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float16v __attribute__((ext_vector_type(16)));
typedef uint32_t uint2v __attribute__((ext_vector_type(2)));
typedef short short4v __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) short4v* lds_short4;

__device__ inline float infinity() { return __uint_as_float(0x7f800000u); }
__device__ inline float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
// All loads are back: the loop after it waits for its own alone.
__device__ inline void wait_all() { __builtin_amdgcn_s_waitcnt(0); }
// What a wave's lanes wrote to LDS before is there for its other lanes after (a
// wave's accesses to LDS are done in order; this keeps the compiler to it).
__device__ inline void wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}
__device__ inline int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// The order of the instructions since the last scheduling barrier: AHEAD reads
// from LDS, then with each of the matrix instructions EACH more of what is left
// of READS, and WORK vector operations.  A read is then on its way for some
// instructions before its data is used; left to itself the compiler reads a
// fragment, waits and multiplies.
template <int AHEAD, int READS, int MFMAS, int EACH = 1, int WORK = 0>
__device__ inline void interleave() {
  int left = READS - AHEAD;
  if (AHEAD > 0) __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 0);
#pragma unroll
  for (int i = 0; i < MFMAS; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    if (WORK > 0) __builtin_amdgcn_sched_group_barrier(0x002, WORK, 0);
    if (left > 0) __builtin_amdgcn_sched_group_barrier(0x100, EACH, 0);
    left -= EACH;
  }
}
__device__ inline void schedule_here() { __builtin_amdgcn_sched_barrier(0); }

template <bool BF16>
struct Frag;
template <>
struct Frag<true> {
  bf16x8 v;
};
template <>
struct Frag<false> {
  float v[8];
};

__device__ inline void multiply(float16v& d, const Frag<true>& a, const Frag<true>& b) {
  d = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.v, b.v, d, 0, 0, 0);
}

__device__ inline void multiply(float16v& d, const Frag<false>& a, const Frag<false>& b) {
#pragma unroll
  for (int j = 0; j < 8; ++j) d = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[j], b.v[j], d, 0, 0, 0);
}

__device__ inline float16v zeros() {
  float16v z;
#pragma unroll
  for (int i = 0; i < 16; ++i) z[i] = 0.0f;
  return z;
}

// Results 8 HALF to 8 HALF + 7 as a fragment.
template <bool BF16, int HALF>
__device__ inline Frag<BF16> as_frag(const float16v& d) {
  Frag<BF16> f;
  if constexpr (BF16) {
    uint4v q;
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = pack_bf16(d[8 * HALF + 2 * i], d[8 * HALF + 2 * i + 1]);
    f.v = __builtin_bit_cast(bf16x8, q);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f.v[i] = d[8 * HALF + i];
  }
  return f;
}

// What bfloat16's rounding of the same results left over, 2^-8 of each rounded in
// turn: the two fragments together are 16 bits of a result.
template <int HALF>
__device__ inline Frag<true> rest_of(const float16v& d, const Frag<true>& rounded) {
  const uint4v r = __builtin_bit_cast(uint4v, rounded.v);
  uint4v q;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    q[i] = pack_bf16(d[8 * HALF + 2 * i] - __uint_as_float(r[i] << 16), d[8 * HALF + 2 * i + 1] - __uint_as_float(r[i] & 0xffff0000u));
  Frag<true> f;
  f.v = __builtin_bit_cast(bf16x8, q);
  return f;
}

// Eight elements of memory, zeros where there are none.
template <bool BF16>
__device__ inline Frag<BF16> load_frag(const void* p, int64_t at, bool there) {
  Frag<BF16> f;
  if constexpr (BF16) {
    f.v = __builtin_bit_cast(bf16x8, there ? Elements<true>::load(p, at) : uint4v{0, 0, 0, 0});
  } else {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const uint4v q = there ? Elements<false>::load(p, at + 4 * u) : uint4v{0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < 4; ++i) f.v[4 * u + i] = __uint_as_float(q[i]);
    }
  }
  return f;
}

// ROWS rows of D elements in LDS.
template <bool BF16, int D, int ROWS>
struct Tile {
  static constexpr int kSize = BF16 ? 2 : 4;
  static constexpr int kChunks = D * kSize / 16;
  static constexpr int kMod = kChunks % 16;
  static constexpr int kPad = kMod == 0 ? 4 : kMod == 8 ? 4 : 0;
  static_assert((kChunks + kPad) % 16 == 4 || (kChunks + kPad) % 16 == 12, "rows' places");
  static constexpr int kStride = (kChunks + kPad) * 16;
  static constexpr int kBytes = ROWS * kStride;

  __device__ static int place(int row, int chunk) { return row * kStride + ((chunk ^ ((row >> 2) & 3)) << 4); }

  // What a lane adds to a tile's address for the reads below; the rest of their
  // places is the same for all lanes.
  struct Lane {
    int along[2], across[2];
    __device__ explicit Lane(int lane) {
      const int r = lane & 31, h = lane >> 5;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        along[u] = place(r, BF16 ? 2 * u + h : 2 * h + u);
        // (sixteen lanes address four rows' four times four elements, and
        // receive one element of four rows each)
        across[u] = BF16 ? place(8 * u + 4 * h + ((lane & 15) >> 2), 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) + (lane & 1) * 8
                         : place(8 * u + 4 * h, r >> 2) + (r & 3) * 4;
      }
    }
  };

  // Row lane % 32 of the rows from `row` on (a multiple of 16), elements 16 step
  // + 8 (lane / 32) + j.
  __device__ static Frag<BF16> along(const uint8_t* tile, const Lane& at, int row, int step) {
    Frag<BF16> f;
    if constexpr (BF16) {
      f.v = __builtin_bit_cast(bf16x8, *(const uint4v*)(tile + at.along[step & 1] + (row * kStride + (step >> 1) * 64)));
    } else {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const float4v q = *(const float4v*)(tile + at.along[u] + (row * kStride + step * 64));
#pragma unroll
        for (int i = 0; i < 4; ++i) f.v[4 * u + i] = q[i];
      }
    }
    return f;
  }

  // Element 32 part + lane % 32 of rows row + 8 (j / 4) + 4 (lane / 32) + j % 4.
  __device__ static Frag<BF16> across(const uint8_t* tile, const Lane& at, int row, int part) {
    Frag<BF16> f;
    if constexpr (BF16) {
      const uint8_t* p = tile + (row * kStride + part * 64);
      const short4v a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4)(p + at.across[0]));
      const short4v b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4)(p + at.across[1]));
      f.v = __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        f.v[j] = *(const float*)(tile + at.across[j / 4] + ((row + j % 4) * kStride + part * 128));
    }
    return f;
  }
};

constexpr int kNonTemporal = 2;  // a buffer load's cache policy

// A tile on its way from memory to LDS through THREADS threads' registers: rows
// of one head, `pos` bytes apart.  The buffer's size ends with the last row that
// there is, so that rows past it read as zeros without a branch.
template <bool BF16, int D, int ROWS, int THREADS>
struct Staged {
  typedef Tile<BF16, D, ROWS> T;
  static constexpr int kCount = (ROWS * T::kChunks + THREADS - 1) / THREADS;
  static constexpr bool kEven = ROWS * T::kChunks % THREADS == 0;
  uint4v q[kCount];
  uint32_t from[kCount];

  __device__ void start(int dim, int pos, int thread) {
#pragma unroll
    for (int i = 0; i < kCount; ++i) {
      const int n = thread + i * THREADS, row = n / T::kChunks, chunk = n % T::kChunks;
      // (2^31: past the end of any tile)
      from[i] = row < ROWS && chunk * (16 / T::kSize) < dim ? (uint32_t)(row * pos + chunk * 16) : 0x80000000u;
    }
  }
  // The rows [first, first + ROWS) of which those below `end` are there.
  template <bool PAST = false>
  __device__ void load(const void* base, int64_t pos, int dim, int first, int end) {
    const int rows = end - first < ROWS ? end - first : ROWS;
    const int bytes = rows > 0 ? (rows - 1) * (int)pos + dim * T::kSize : 0;
    const auto buffer =
        __builtin_amdgcn_make_buffer_rsrc((void*)((const uint8_t*)base + first * pos), 0, bytes, 0x00020000);
#pragma unroll
    for (int i = 0; i < kCount; ++i) q[i] = __builtin_amdgcn_raw_buffer_load_b128(buffer, (int)from[i], 0, PAST ? kNonTemporal : 0);
  }
  __device__ void store(uint8_t* tile, int thread) const {
#pragma unroll
    for (int i = 0; i < kCount; ++i) {
      const int n = thread + i * THREADS, row = n / T::kChunks, chunk = n % T::kChunks;
      if (!kEven && row >= ROWS) continue;
      *(uint4v*)(tile + T::place(row, chunk)) = q[i];
    }
  }
};

struct __attribute__((packed, aligned(2))) Four2 {
  uint2v q;
};
struct __attribute__((packed, aligned(4))) Four4 {
  float4v q;
};

// A lane's sixteen results of 32 elements from `at` on, its column's row in
// memory: four runs of four.
template <bool BF16>
__device__ inline void store_column(void* p, int64_t at, int left, const float16v& d, float factor, int lane) {
  const int h = lane >> 5;
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    const int e = 8 * g + 4 * h;
    if (e >= left) continue;
    const float a = d[4 * g] * factor, b = d[4 * g + 1] * factor, c = d[4 * g + 2] * factor, f = d[4 * g + 3] * factor;
    if (BF16)
      ((Four2*)((uint16_t*)p + at + e))->q = uint2v{pack_bf16(a, b), pack_bf16(c, f)};
    else
      ((Four4*)((float*)p + at + e))->q = float4v{a, b, c, f};
  }
}

// What bfloat16's rounding of the same elements left over, to `at` on.
__device__ inline void store_rest(uint16_t* p, int64_t at, int left, const float16v& d, float factor, int lane) {
  const int h = lane >> 5;
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    const int e = 8 * g + 4 * h;
    if (e >= left) continue;
    float r[4];
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
      const float a = d[4 * g + i] * factor, b = d[4 * g + i + 1] * factor;
      const uint32_t q = pack_bf16(a, b);
      r[i] = a - __uint_as_float(q << 16);
      r[i + 1] = b - __uint_as_float(q & 0xffff0000u);
    }
    *(uint2v*)(p + at + e) = uint2v{pack_bf16(r[0], r[1]), pack_bf16(r[2], r[3])};
  }
}

// The value of the lane 32 away joined with one's own (a lane and that one hold
// the halves of a column).
__device__ inline float max_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float add_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Which tile (by its work, the largest first) of which head (of all sequences') a
// workgroup takes.  Workgroups go to the eight XCDs in turn: where the heads are
// a multiple of eight a head's tiles stay on one, in whose L2 they find its keys
// (or queries).  The longest go first, of all heads: a long one that starts last
// would be waited for (causal, 64 heads of 32 tiles, head by head: 20% of the
// time the average CU had nothing to do).  Of at most 512, which all run at once,
// those from 256 on go the other way, so that a CU's two are a long and a short one
// (causal, forward / backward: 32 heads of 64, 2048 keys, binary32 208 / 688 -> 161 /
// 526 us; 32 of 128, bfloat16 57 / 191 -> 55 / 183).
struct Work {
  int order, head;
};
__device__ inline Work work_of(int block, int blocks, int heads) {
  const bool back = blocks > 256 && blocks <= 512;
  if (heads % 8) {
    if (back && block >= 256) block = blocks - 1 - (block - 256);
    return {block / heads, block % heads};
  }
  const int per = heads / 8;
  int n = block >> 3;
  if (back && n >= 32) n = (blocks >> 3) - 1 - (n - 32);
  return {n / per, (block & 7) * per + n % per};
}

// A row of the rows that share a key head: its query head and query.
struct RowAt {
  int head, query;
};
__device__ inline RowAt row_at(const AttentionArgs& a, int kv_head, int row) {
  const int h = row / a.queries;
  return {kv_head * a.group + h, row - h * a.queries};
}

// (without queries nothing is read)
__device__ inline int keys_of(const AttentionArgs& a, int batch) {
  if (!a.queries) return 0;
  if (!a.lengths) return a.keys;
  const int n = a.lengths[batch];
  return n < 0 ? 0 : n < a.keys ? n : a.keys;
}

// How many of the first keys a query sees.
__device__ inline int limit_of(const AttentionArgs& a, int query, int length) {
  if (!a.causal) return length;
  const int n = query + 1 + a.keys - a.queries;
  return n < 0 ? 0 : n < length ? n : length;
}

// How many of the first keys the rows [first, first + count) see together.
__device__ inline int last_key(const AttentionArgs& a, int first, int count, int length) {
  const int last = first + count < a.rows ? first + count - 1 : a.rows - 1;
  // rows of two heads: the last query is among them
  const bool two = first / a.queries != last / a.queries;
  return limit_of(a, two ? a.queries - 1 : last % a.queries, length);
}

__device__ inline int wave_min(int x) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    const int y = __shfl_xor(x, d);
    x = x < y ? x : y;
  }
  return uniform(x);
}
__device__ inline int wave_max(int x) { return -wave_min(-x); }

}  // namespace
}  // namespace microadam
