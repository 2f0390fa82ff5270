// Launch interface of the Newton-Schulz kernels (orthogonalize, Muon).
//
// A launch works on up to kMaxGroups groups of matrices.  The matrices of a
// group have one working shape m x n with m <= n (a matrix with more rows
// than columns is worked on as its transpose), padded with zeros to multiples
// of kPad, and one record each in the workspace:
//   XT  [np][mp]   the iterate X transposed, in two buffers that the steps alternate
//   A   [mp][mp]   S_A X X^T
//   B   [mp][mp]   S_A (a I + b A + c A^2)
// All are binary16, X scaled by S_X; in split precision each is followed by a
// second plane with 2048 times what the rounding of the first left.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace microadam {

constexpr int kMaxGroups = 8;     // working shapes per launch
constexpr int kMaxMatrices = 96;  // matrices per launch (their addresses are kernel arguments)
constexpr int kPad = 64;          // working dimensions are padded to this
constexpr int64_t kMaxTiles = (int64_t)1 << 24;  // of a product's launch
constexpr int kNormParts = 256;   // partial sums of a matrix's norm
constexpr int kPartTile = 128;    // the largest tile whose products may be split over K

// Powers of two, so that scaling rounds nothing.  Elements of X are at most
// about 1 and around 1/sqrt(mn) at the start (1.5e-4 for 4096 x 11008), those
// of A around 1/(m sqrt(n)) off the diagonal (2e-6): scaled, both are normal
// binary16 numbers (6e-5 to 65504).
constexpr float kScaleX = 256.0f;
constexpr float kScaleA = 1024.0f;
constexpr float kSplitScale = 2048.0f;

struct SchulzGroup {
  uint64_t base;        // of the group's first record, bytes from the workspace
  uint64_t record;      // bytes of a record
  uint64_t xt, a, b;    // offsets in a record (xt: of the first of its two buffers)
  int32_t m, n;         // working shape, m <= n
  int32_t mp, np;       // padded
  int32_t first, count; // matrices of the launch
};

// What the norm and pack kernels read of a matrix, and what the last product
// writes.
struct PackMatrix {
  const void* grad;
  void* momentum;
  int32_t grad_ld, momentum_ld;
};
struct OutMatrix {
  void* out;
  int32_t out_ld;
  float scale;
};

struct PackArgs {
  uint8_t* ws;
  double* partials;  // [matrix][kNormParts]
  float mu, one_minus_mu;
  double eps;
  int32_t n_groups, n_parts, split, nesterov;
  int32_t grad_bf16, momentum_bf16;
  SchulzGroup group[kMaxGroups];
  PackMatrix mat[kMaxMatrices];
  uint8_t tall[kMaxMatrices];
  uint8_t of[kMaxMatrices];  // matrix -> group
};

// Products of a step.
enum SchulzPhase {
  kGram = 0,   // A = X X^T (symmetric)
  kPoly = 1,   // B = a I + b A + c A A^T (symmetric)
  kApply = 2,  // X^T <- X^T B, into the other buffer
  kFinal = 3   // the caller's matrix from B X
};

struct GemmArgs {
  uint8_t* ws;
  int32_t n_groups, split;
  int32_t buffer;            // which XT buffer holds the transpose of X
  float ca, cb, cc;          // kPoly: factors of I, the stored A and the product
  float decay;               // kFinal: 1 - lr * weight_decay
  int32_t out_bf16, update;  // kFinal: update out in place (out = decay * out - scale * D) or store scale * D
  int32_t tiles[kMaxGroups];           // of each group, and an eighth of them, rounded up
  int32_t turns[kMaxGroups];
  // kGram in tiles of up to kPartTile: a tile's K is taken in `parts` runs of
  // `part_stages` stages of 64 by as many workgroups.  Where they are more than
  // one, their binary32 sums lie in the XT buffer that the step has yet to
  // write, [part][mp][mp] with the tiles on and below the diagonal, until they
  // are joined.
  int32_t parts[kMaxGroups], part_stages[kMaxGroups];
  SchulzGroup group[kMaxGroups];
  OutMatrix mat[kMaxMatrices];         // kFinal
  uint8_t tall[kMaxMatrices];
};

constexpr int kStrip = 8;  // tile rows

#ifdef __HIPCC__
// The row r of a triangle of rows 0, 1, 2, .. of 1, 2, 3, .. that entry t
// falls in.
__device__ inline int triangle_row(int t) {
  int r = (int)((__builtin_amdgcn_sqrtf(8.0f * (float)t + 1.0f) - 1.0f) * 0.5f);
  while (r * (r + 1) / 2 > t) --r;
  while ((r + 1) * (r + 2) / 2 <= t) ++r;
  return r;
}

// Tile `tile` of the tiles on and below the diagonal of tm x tm, in strips of
// kStrip tile rows, column by column.  The same in every lane.
__device__ inline void symmetric_tile(int tile, int tm, int& ti, int& tj) {
  auto uniform = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
  // rows before a strip of a triangle hold first * (first + 1) / 2 tiles
  const int first = uniform(triangle_row(tile)) / kStrip * kStrip;
  const int high = tm - first < kStrip ? tm - first : kStrip;
  const int in = tile - first * (first + 1) / 2;
  if (in < high * first) {
    tj = uniform(in / high);
    ti = first + in - tj * high;
  } else {
    const int corner = in - high * first;
    const int r = uniform(triangle_row(corner));
    ti = first + r;
    tj = first + corner - r * (r + 1) / 2;
  }
}
#endif

hipError_t launch_schulz_norm(const PackArgs& a, int n_matrices, hipStream_t s);
hipError_t launch_schulz_pack(const PackArgs& a, int n_matrices, hipStream_t s);

int64_t schulz_tiles(const SchulzGroup& g, SchulzPhase phase, int tile);
// The tile (64, 128, 192 or 256) that takes a launch's products least time;
// sets parts and part_stages for kGram.
int choose_schulz_tile(GemmArgs& a, SchulzPhase phase);
hipError_t launch_schulz_gemm(GemmArgs& a, SchulzPhase phase, int tile, hipStream_t s);
hipError_t launch_schulz_join(const GemmArgs& a, hipStream_t s);
hipError_t launch_schulz_gemm_64(const GemmArgs& a, SchulzPhase phase, hipStream_t s);
hipError_t launch_schulz_gemm_128(const GemmArgs& a, SchulzPhase phase, hipStream_t s);
hipError_t launch_schulz_gemm_192(const GemmArgs& a, SchulzPhase phase, hipStream_t s);
hipError_t launch_schulz_gemm_256(const GemmArgs& a, SchulzPhase phase, hipStream_t s);  // not split

}  // namespace microadam
