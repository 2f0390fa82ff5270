// The products of a Newton-Schulz step on the matrix cores, with binary16
// operands and binary32 accumulators: D = P Q^T with the operands' rows
// contiguous along the summed dimension, and X X^T = P^T Q from X^T, whose rows
// run along it.  So only X^T is kept, and one product writes it once.
//
// A workgroup computes a T x T tile of D.  K is taken in stages of 64 elements
// that go straight from memory to LDS, one to three stages ahead of the matrix
// instructions (16x16x32).  Rows are kept with their 16-byte chunks permuted, so
// that sixteen rows' chunks, which a 16-byte read takes in one cycle, lie on
// different banks (64 of 4 bytes).  Stages of X^T are kept as they lie, 64 rows
// of T elements, with their 32-byte segments permuted likewise, and read with
// the transposing LDS read (four rows of 16 elements to sixteen lanes of four).
//
// In split precision an operand is hi + lo / 2048.  The product is taken as
// three runs over K into the same accumulators: lo hi, hi lo, then, after a
// factor 1/2048, hi hi; tiles of 64 take all three at once.
//
// The symmetric products compute the tiles on and below the diagonal and
// store each twice.
//
// X X^T of few rows is a few tiles with a long K: the K of tiles up to 128
// can be split over workgroups, whose sums join_kernel (k_schulz_pack.hip)
// adds up (what it gives stands in schulz_launch.cpp).
//
// Large products are bound by the power limit: X^T B of 4096 x 11008 takes 285
// to 305 us in 256-tiles (1.2 to 1.3 PFLOP/s; the library's 8192^3 in binary16:
// 1.33), the matrix cores busy for 65% of 1.6 to 1.8 GHz.  With K = 768 the
// stores of all CUs at once are 40% of a 256-tile's time (0.85 PFLOP/s); a few
// 64-tiles take 4 to 5 us however little they compute.
#pragma once
#include "schulz_device.h"

namespace microadam {
namespace {

typedef _Float16 half_t;
typedef half_t half4 __attribute__((ext_vector_type(4)));
typedef half_t half8 __attribute__((ext_vector_type(8)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef uint32_t uint2v __attribute__((ext_vector_type(2)));
typedef short short4v __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void* lds_ptr;
typedef __attribute__((address_space(3))) short4v* lds_short4;

__device__ inline float bf16_to_f32(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }

__device__ inline uint16_t f32_to_bf16(float x) {
  const uint32_t u = __float_as_uint(x);
  if ((u & 0x7fffffffu) > 0x7f800000u) return (uint16_t)((u >> 16) | 0x40);
  return (uint16_t)((u + 0x7fffu + ((u >> 16) & 1)) >> 16);
}

// Forms of the kernel by tile: the places in LDS for an operand's stage (T
// rows of kStep elements) and the waves along Q's rows (two along P's).
// Stage s of P is load 2 s and stage s of Q load 2 s + 1; load u goes to place
// u % places.  Five places hold two stages and half of a third.
constexpr int kStep = 64;  // whole 128-byte lines: half lines cost the L2 twice the requests
template <int T>
struct Form;
template <>
struct Form<256> {
  static constexpr int places = 5, wq = 4;
};
template <>
struct Form<192> {
  static constexpr int places = 5, wq = 4;
};
template <>
struct Form<128> {
  static constexpr int places = 5, wq = 2;
};
// (eight waves: few of these tiles are on a CU, and a wave alone on its SIMD
// waits for its LDS reads; 1024^2 split 14.7 us with four, 13.0 with eight)
template <>
struct Form<64> {
  static constexpr int places = 8, wq = 4;
};

// A value that is the same in every lane, as a scalar.
__device__ inline int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// The transposing LDS read: of sixteen lanes, lanes 4 r to 4 r + 3 address row
// r's four times four elements, and lane i receives element i of four rows.
// (`restrict`: without alias information the compiler waits for all loads to
// LDS before it; the loop below waits for those of its stage.)
__device__ inline short4v read_tr16(const uint8_t* __restrict__ p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4)p);
}

template <int N>
__device__ inline void wait_vmcnt() {
  // vmcnt is split in two fields; the other counters are left at their most
  __builtin_amdgcn_s_waitcnt(0x0f70 | (N & 15) | ((N >> 4) << 14));
}

// The order of the instructions since the last scheduling barrier: two reads
// from LDS before each of the first matrix instructions, so that the reads are
// done when the next set of them starts, then a load after each.
template <int READS, int LOADS, int MFMAS>
__device__ inline void interleave() {
  int reads = READS, loads = LOADS;
#pragma unroll
  for (int i = 0; i < MFMAS; ++i) {
    const int left = MFMAS - i;
    if (reads > 0) {
      const int n = reads < 2 ? reads : reads > 2 * left ? reads / left : 2;
      if (n == 1) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      if (n == 2) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
      reads -= n;
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    } else {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      if (loads > 0) {
        if (loads > left)
          __builtin_amdgcn_sched_group_barrier(0x010, 2, 0);
        else
          __builtin_amdgcn_sched_group_barrier(0x010, 1, 0);
        loads -= loads > left ? 2 : 1;
      }
    }
  }
}

template <int T, int PHASE, bool SPLIT>
__global__ __launch_bounds__(128 * Form<T>::wq, 2) void gemm_kernel(const GemmArgs a) {
  constexpr int kWQ = Form<T>::wq, kWaves = 2 * kWQ;
  // A split stage of the small tile holds both planes of both operands and is
  // multiplied at once, the cross terms into accumulators of their own: a
  // third of the stages and two thirds of the loads, which such a tile's time
  // goes by.  Larger tiles have no registers for that.
  constexpr bool kFused = SPLIT && T == 64;
  constexpr int kOps = kFused ? 4 : 2;             // loads per stage: P, Q (, what was left of P, of Q)
  constexpr int kPlaces = kFused ? 10 : Form<T>::places, kAhead = (kPlaces + kOps - 1) / kOps;
  constexpr int kRowBytes = kStep * 2;             // of an operand's row in a stage
  constexpr int kLoads = T / 8 / kWaves;           // of an operand's stage, eight rows each, per wave
  constexpr int kI = T / 32, kJ = T / (16 * kWQ);  // a wave's 16 x 16 results
  constexpr int kK = kStep / 32;                   // matrix instructions along a stage
  constexpr int kOperand = T * kRowBytes;          // bytes of an operand's stage
  constexpr int kStageRow = T + 8;                 // halves per row of the staged result
  constexpr int kLds = kPlaces * kOperand > T * kStageRow * 2 ? kPlaces * kOperand : T * kStageRow * 2;
  __shared__ __align__(1024) uint8_t lds[kLds];

  // Workgroups go to the eight XCDs in turn: give each XCD one run of every
  // group's tiles, which share operand rows in its L2.
  const int xcd = (int)blockIdx.x & 7;
  // (the first group's fields are fetched along with the number of groups)
  int turn = (int)blockIdx.x >> 3;
  SchulzGroup g = a.group[0];
  int tiles = a.tiles[0];
  constexpr bool kRuns = PHASE == kGram && T <= kPartTile;
  int parts = kRuns ? a.parts[0] : 1, part_stages = kRuns ? a.part_stages[0] : 0;
  if (a.n_groups > 1 && turn >= a.turns[0]) {
    int gi = 0;
    while (gi + 1 < a.n_groups && turn >= a.turns[gi]) turn -= a.turns[gi++];
    g = a.group[gi];
    tiles = a.tiles[gi];
    if (kRuns) {
      parts = a.parts[gi];
      part_stages = a.part_stages[gi];
    }
  }
  const int each = tiles >> 3, more = tiles & 7;
  if (turn >= each + (xcd < more ? 1 : 0)) return;
  int tile = xcd * each + (xcd < more ? xcd : more) + turn;

  const int tm = (g.mp + T - 1) / T, tn = (g.np + T - 1) / T;
  constexpr bool kSym = PHASE == kGram || PHASE == kPoly;
  const int per = kSym ? tm * (tm + 1) / 2 : tm * tn;
  int which = uniform(tile / per), part = 0;
  tile -= which * per;
  if (kRuns && parts > 1) {
    part = uniform(which % parts);
    which = uniform(which / parts);
  }
  const int mat = g.first + which;
  // X^T's rows are D's rows: always to keep X^T, at the end for a tall matrix
  const bool swap = PHASE == kApply || (PHASE == kFinal && uniform(a.tall[mat]));

  // Tile (ti, tj) of D: strips of kStrip tile rows, column by column, so that
  // the 32 tiles an XCD's CUs take at a time need about 8 + 4 operand tiles.
  int ti, tj;
  if (kSym) {
    symmetric_tile(tile, tm, ti, tj);
  } else {
    const int strip = uniform(tile / (kStrip * tn)), first = strip * kStrip;
    const int high = tm - first < kStrip ? tm - first : kStrip;
    const int in = tile - strip * kStrip * tn;
    tj = uniform(in / high);
    ti = first + in - tj * high;
  }

  uint8_t* rec = a.ws + g.base + (uint64_t)which * g.record;
  const uint64_t plane_x = (uint64_t)g.mp * g.np * 2, plane_a = (uint64_t)g.mp * g.mp * 2;
  const uint64_t xt_bytes = plane_x << (SPLIT ? 1 : 0);
  const uint8_t* xt = rec + g.xt + (a.buffer ? xt_bytes : 0);
  const uint8_t *p, *q;
  uint64_t plane_p, plane_q;
  int rows_p, rows_q;
  if (PHASE == kGram) {
    p = q = xt;
    plane_p = plane_q = plane_x;
    rows_p = rows_q = g.mp;
  } else if (PHASE == kPoly) {
    p = q = rec + g.a;
    plane_p = plane_q = plane_a;
    rows_p = rows_q = g.mp;
  } else {
    p = swap ? xt : rec + g.b;
    q = swap ? rec + g.b : xt;
    plane_p = swap ? plane_x : plane_a;
    plane_q = swap ? plane_a : plane_x;
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
  const int wave = uniform((int)threadIdx.x >> 6);
  const int wp0 = (wave & 1) * (T / 2), wq0 = (wave >> 1) * (T / kWQ);

  // What lies past the operand reads as zeros (the resource's size).  kGram: a
  // stage's 64 rows of X^T from column p0 (q0) on; columns past the matrix read
  // the next row's, whose results are not stored.
  const uint32_t row_bytes = (uint32_t)g.mp * 2;
  const int first_stage = kRuns ? part * part_stages : 0;
  const uint8_t* tp = p + (PHASE == kGram ? (uint64_t)p0 * 2 + (uint64_t)((uint32_t)first_stage * kStep) * row_bytes : (uint64_t)p0 * row_bytes);
  const uint8_t* tq = q + (PHASE == kGram ? (uint64_t)q0 * 2 + (uint64_t)((uint32_t)first_stage * kStep) * row_bytes : (uint64_t)q0 * row_bytes);
  const int size_p = (int)(PHASE == kGram ? kStep * row_bytes - (uint32_t)p0 * 2 : (uint32_t)left_p * row_bytes);
  const int size_q = (int)(PHASE == kGram ? kStep * row_bytes - (uint32_t)q0 * 2 : (uint32_t)left_q * row_bytes);
  // the 16-byte chunk c of row r is kept at position c ^ spread(r)
  auto spread = [](int r) { return (r >> 1) & 7; };
  const int load_row = lane >> 3;
  const int voff = load_row * (int)row_bytes + ((lane & 7) ^ spread(load_row)) * 16;
  int ksteps = (PHASE == kGram ? g.np : g.mp) / kStep;
  if (kRuns && parts > 1) ksteps = ksteps - first_stage < part_stages ? ksteps - first_stage : part_stages;
  // kGram: the 32-byte segment s of row r is kept at position s ^ turn, by the
  // bits of r that the rows of one read differ in
  constexpr bool kWide = T % 128 == 0;  // whole 256-byte rows: all of a read's eight rows on the same banks
  auto turn_of = [](int r) { return kWide ? (r & 3) | ((r >> 3 & 1) << 2) : (r >> 1 & 1) | ((r >> 3 & 1) << 1); };
  int voff_gram[PHASE == kGram ? kLoads : 1];
  if constexpr (PHASE == kGram) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int at = (wave * kLoads + i) * 1024 + lane * 16;
      const int r = at / (2 * T), in = at % (2 * T);
      voff_gram[i] = r * (int)row_bytes + (((in >> 5) ^ turn_of(r)) << 5) + (in & 31);
    }
  }
  const int steps = SPLIT && !kFused ? 3 * ksteps : ksteps;

  // load op of stage t
  auto load = [&](int op, int t, int place) {
    const bool is_q = op & 1;
    const uint8_t* base = is_q ? tq : tp;
    if (kFused) {
      if (op >= 2) base += is_q ? plane_q : plane_p;
    } else if (SPLIT) {
      const int part = t >= 2 * ksteps ? 2 : t >= ksteps ? 1 : 0;
      t -= part * ksteps;
      if (part == (is_q ? 1 : 0)) base += is_q ? plane_q : plane_p;
    }
    if (PHASE == kGram) base += (uint64_t)((uint32_t)t * kStep) * row_bytes;
    auto rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, is_q ? size_q : size_p, 0x00020000);
    uint8_t* dst = lds + place * kOperand;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int c = wave * kLoads + i;
      // the second eight of sixteen rows have bit 2 of their chunks' places flipped
      const int v = PHASE == kGram ? voff_gram[PHASE == kGram ? i : 0] : c & 1 ? voff ^ 64 : voff;
      const int soff = PHASE == kGram ? 0 : c * 8 * (int)row_bytes + t * kRowBytes;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_ptr)(dst + c * 1024), 16, v, soff, 0, 0);
    }
  };

  // Element r of acc[i][j] is D at row (of the wave's tile) i * 16 + lane % 16
  // and column j * 16 + 4 (lane / 16) + r.
  const int lrow = lane & 15, lcol = (lane >> 4) * 4;

  // kPoly adds A, which the smaller tiles have registers to fetch before the
  // product (a memory round trip less at the end)
  auto load_a = [&](int i, int j, int plane) {
    const int row = p0 + wp0 + i * 16 + lrow, col = q0 + wq0 + j * 16 + lcol;
    half4 h = {};
    if (row < g.mp && col < g.mp)
      h = *(const half4*)((const half_t*)(rec + g.a) + (plane ? (int64_t)g.mp * g.mp : 0) + (int64_t)row * g.mp + col);
    return h;
  };
  constexpr bool kEarly = PHASE == kPoly && T <= 128;
  constexpr int kEarlyPlanes = SPLIT ? 2 : 1;
  half4 early[kEarly ? kEarlyPlanes : 1][kEarly ? kI : 1][kEarly ? kJ : 1];
  if constexpr (kEarly) {
#pragma unroll
    for (int pl = 0; pl < kEarlyPlanes; ++pl)
#pragma unroll
      for (int i = 0; i < kI; ++i)
#pragma unroll
        for (int j = 0; j < kJ; ++j) early[pl][i][j] = load_a(i, j, pl);
  }

  float4v acc[kI][kJ];
#pragma unroll
  for (int i = 0; i < kI; ++i)
#pragma unroll
    for (int j = 0; j < kJ; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) acc[i][j][r] = 0.0f;

  constexpr int kParts = kFused ? 2 : 1;
  float4v cross[kFused ? kI : 1][kFused ? kJ : 1] = {};
  half8 fp[2][kParts][kI], fq[2][kParts][kJ];
  // place: of the stage's P; its other loads follow
  auto at = [&](int place, int op) { return place + op >= kPlaces ? place + op - kPlaces : place + op; };
  // kGram: fragment i of an operand is its segment i of 16 columns; lane l
  // takes part in rows 8 (l / 16) + (l % 16) / 4 and four on
  auto read_turned = [&](const uint8_t* operand, int segment, int kk) {
    const int r = (lane >> 4) * 8 + ((lane & 15) >> 2);
    const uint8_t* b = operand + r * (2 * T) + ((segment ^ turn_of(r)) << 5) + (lane & 3) * 8 + kk * 32 * (2 * T);
    const short4v lo = read_tr16(b), hi = read_tr16(b + 4 * (2 * T));
    return __builtin_bit_cast(half8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  };
  auto read = [&](int place, int kk, int set) {
    const uint8_t* b = lds + (lane & 15) * kRowBytes + (((kk * 4 + (lane >> 4)) ^ spread(lane & 15)) * 16);
#pragma unroll
    for (int part = 0; part < kParts; ++part) {
      const int op = at(place, 2 * part) * kOperand, oq = at(place, 2 * part + 1) * kOperand;
#pragma unroll
      for (int j = 0; j < kJ; ++j)
        fq[set][part][j] = PHASE == kGram ? read_turned(lds + oq, wq0 / 16 + j, kk)
                                          : *(const half8*)(b + oq + (wq0 + j * 16) * kRowBytes);
#pragma unroll
      for (int i = 0; i < kI; ++i)
        fp[set][part][i] = PHASE == kGram ? read_turned(lds + op, wp0 / 16 + i, kk)
                                          : *(const half8*)(b + op + (wp0 + i * 16) * kRowBytes);
    }
  };
  auto multiply = [&](int set) {
#pragma unroll
    for (int i = 0; i < kI; ++i)
#pragma unroll
      for (int j = 0; j < kJ; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fq[set][0][j], fp[set][0][i], acc[i][j], 0, 0, 0);
    if constexpr (kFused) {
#pragma unroll
      for (int i = 0; i < kI; ++i)
#pragma unroll
        for (int j = 0; j < kJ; ++j)
          cross[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fq[set][1][j], fp[set][0][i], cross[i][j], 0, 0, 0);
#pragma unroll
      for (int i = 0; i < kI; ++i)
#pragma unroll
        for (int j = 0; j < kJ; ++j)
          cross[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fq[set][0][j], fp[set][1][i], cross[i][j], 0, 0, 0);
    }
  };
  constexpr int kReads = kParts * (kI + kJ) * (PHASE == kGram ? 2 : 1), kMfmas = (kFused ? 3 : 1) * kI * kJ;

  // The places of stage s are loaded again as soon as every wave has read the
  // last of s into registers; the fragments of each half stage are read half a
  // stage ahead.
#pragma unroll
  for (int u = 0; u < kPlaces; ++u)
    if (u / kOps < steps) load(u % kOps, u / kOps, u);
  if (steps >= kAhead)
    wait_vmcnt<(kPlaces - kOps) * kLoads>();
  else
    wait_vmcnt<0>();
  __builtin_amdgcn_s_barrier();
  read(0, 0, 0);
  int place = 0;  // of stage s of P
  auto stage = [&](int s, bool more, bool next) {
    if (SPLIT && !kFused && s == 2 * ksteps) {
#pragma unroll
      for (int i = 0; i < kI; ++i)
#pragma unroll
        for (int j = 0; j < kJ; ++j) acc[i][j] *= 1.0f / kSplitScale;
    }
#pragma unroll
    for (int kk = 0; kk < kK - 1; ++kk) {
      read(place, kk + 1, (kk + 1) & 1);
      multiply(kk & 1);
      interleave<kReads, 0, kMfmas>();
      __builtin_amdgcn_sched_barrier(0);
    }
    if (next) {
      __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): stage s is in registers
      if (more)
        wait_vmcnt<(kPlaces - 2 * kOps) * kLoads>();
      else
        wait_vmcnt<0>();
      __builtin_amdgcn_s_barrier();
      __builtin_amdgcn_sched_barrier(0);
      const int after = at(place, kOps);
      read(after, 0, 0);
      // loads kOps * s + kPlaces and on
#pragma unroll
      for (int i = 0; i < kOps; ++i) {
        const int later = (kPlaces + i) / kOps;  // stages after s
        if (more || s + later < steps) load((kPlaces + i) % kOps, s + later, at(place, i));
      }
      place = after;
    }
    multiply((kK - 1) & 1);
    if (next) {
      if (more)
        interleave<kReads, kOps * kLoads, kMfmas>();
      else
        interleave<kReads, 0, kMfmas>();
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  int s = 0;
  for (; s < steps - kAhead; ++s) stage(s, true, true);
  for (; s < steps - 1; ++s) stage(s, false, true);
  stage(s, false, false);
  if constexpr (kFused) {
#pragma unroll
    for (int i = 0; i < kI; ++i)
#pragma unroll
      for (int j = 0; j < kJ; ++j) acc[i][j] += cross[i][j] * (1.0f / kSplitScale);
  }

  if constexpr (kRuns) {
    if (parts > 1) {
      float* sums = (float*)(rec + g.xt + (a.buffer ? 0 : xt_bytes)) + (int64_t)part * g.mp * g.mp;
#pragma unroll
      for (int i = 0; i < kI; ++i)
#pragma unroll
        for (int j = 0; j < kJ; ++j) {
          const int row = p0 + wp0 + i * 16 + lrow, col = q0 + wq0 + j * 16 + lcol;
          if (row < g.mp && col < g.mp) *(float4v*)(sums + (int64_t)row * g.mp + col) = acc[i][j];
        }
      return;
    }
  }
  if constexpr (PHASE == kFinal) {
    const OutMatrix& om = a.mat[mat];
    const int out_rows = swap ? g.n : g.m, out_cols = swap ? g.m : g.n;
    const float f = om.scale * (1.0f / (kScaleA * kScaleX));
#pragma unroll
    for (int i = 0; i < kI; ++i) {
      const int row = p0 + wp0 + i * 16 + lrow;
      if (row >= out_rows) continue;
#pragma unroll
      for (int j = 0; j < kJ; ++j)
        {
          const int col = q0 + wq0 + j * 16 + lcol;
          const int64_t at = (int64_t)row * om.out_ld + col;
          float v[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) v[r] = acc[i][j][r] * f;
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
    // the result at its stored scale, rounded once (and what that left)
    constexpr int kPlanes = SPLIT ? 2 : 1;
    half4 out[kPlanes][kI][kJ];
#pragma unroll
    for (int i = 0; i < kI; ++i) {
      const int row = p0 + wp0 + i * 16 + lrow;
#pragma unroll
      for (int j = 0; j < kJ; ++j)
        {
          const int col = q0 + wq0 + j * 16 + lcol;
          float v[4];
          if constexpr (PHASE == kPoly) {  // b A + c D + a I
            half4 h, l;
            if constexpr (kEarly) {
              h = early[0][i][j];
              l = early[kEarlyPlanes - 1][i][j];
            } else {
              h = load_a(i, j, 0);
              if (SPLIT) l = load_a(i, j, 1);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              float x = (float)h[r];
              if (SPLIT) x += (float)l[r] * (1.0f / kSplitScale);
              v[r] = a.cb * x + a.cc * acc[i][j][r] + (row == col + r ? a.ca : 0.0f);
            }
          } else {
            constexpr float f = PHASE == kGram ? kScaleA / (kScaleX * kScaleX) : 1.0f / kScaleA;
#pragma unroll
            for (int r = 0; r < 4; ++r) v[r] = acc[i][j][r] * f;
          }
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            out[0][i][j][r] = (half_t)v[r];
            if (SPLIT) out[kPlanes - 1][i][j][r] = (half_t)((v[r] - (float)out[0][i][j][r]) * kSplitScale);
          }
        }
    }
    // D at (p0, q0) of an array of `height` rows, or its transpose at
    // (q0, p0), staged in LDS so that rows are stored whole
    half_t* const stage = (half_t*)lds;
    auto store = [&](uint8_t* dst, int height, bool flip, int plane) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kI; ++i)
#pragma unroll
        for (int j = 0; j < kJ; ++j)
          {
            const half4 h = out[plane][i][j];
            const int row = wp0 + i * 16 + lrow, col = wq0 + j * 16 + lcol;
            if (flip) {
#pragma unroll
              for (int r = 0; r < 4; ++r) stage[(col + r) * kStageRow + row] = h[r];
            } else {
              *(half4*)(stage + row * kStageRow + col) = h;
            }
          }
      __syncthreads();
      const int r0 = flip ? q0 : p0, c0 = flip ? p0 : q0;
      half_t* d = (half_t*)dst + (int64_t)r0 * g.mp + c0;
      for (int c = threadIdx.x; c < T * (T / 8); c += 64 * kWaves) {
        const int row = c / (T / 8), col = (c % (T / 8)) * 8;
        if (r0 + row < height && c0 + col < g.mp)
          *(half8*)(d + (int64_t)row * g.mp + col) = *(const half8*)(stage + row * kStageRow + col);
      }
    };
#pragma unroll
    for (int pl = 0; pl < kPlanes; ++pl) {
      if constexpr (kSym) {
        uint8_t* dst = rec + (PHASE == kGram ? g.a : g.b) + (pl ? plane_a : 0);
        store(dst, g.mp, false, pl);
        if (ti != tj) store(dst, g.mp, true, pl);
      } else {
        store(rec + g.xt + (a.buffer ? 0 : xt_bytes) + (pl ? plane_x : 0), g.np, false, pl);
      }
    }
  }
}

template <int T, bool SPLIT>
hipError_t launch_products(const GemmArgs& a, SchulzPhase phase, hipStream_t s) {
  unsigned n = 0;
  for (int i = 0; i < a.n_groups; ++i) n += 8 * (unsigned)a.turns[i];
  constexpr int threads = 128 * Form<T>::wq;
  switch (phase) {
    case kGram: gemm_kernel<T, kGram, SPLIT><<<n, threads, 0, s>>>(a); break;
    case kPoly: gemm_kernel<T, kPoly, SPLIT><<<n, threads, 0, s>>>(a); break;
    case kApply: gemm_kernel<T, kApply, SPLIT><<<n, threads, 0, s>>>(a); break;
    case kFinal: gemm_kernel<T, kFinal, SPLIT><<<n, threads, 0, s>>>(a); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace
}  // namespace microadam
