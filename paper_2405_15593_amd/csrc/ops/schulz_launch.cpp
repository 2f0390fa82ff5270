// Host side of a Newton-Schulz product's launch: the tile that suits its sizes.
#include "schulz_device.h"

namespace microadam {

int64_t schulz_tiles(const SchulzGroup& g, SchulzPhase phase, int tile) {
  const int64_t tm = (g.mp + tile - 1) / tile, tn = (g.np + tile - 1) / tile;
  return (phase == kGram || phase == kPoly ? tm * (tm + 1) / 2 : tm * tn) * g.count;
}

namespace {

// What a workgroup of each tile takes for a stage of 64 elements of K and for
// the rest of its work (microseconds), with few others on the device and with
// every CU holding per_cu of them; the rest of a symmetric product, which
// stores off-diagonal tiles twice, apart.  Measured on products of 1024^2,
// 4096^2, 4096 x 11008 and on 72 matrices of 768 x 768 and 768 x 3072, where
// the rest, mostly the stores of all CUs at once, is 40% of a 256-tile's time;
// "few" also on 1 to 250 tiles of 1 to 64 stages, with a kernel's own start.
struct TileForm {
  int tile, per_cu;
  float few_stage, few_rest, full_stage, full_rest, full_rest_symmetric;
};
constexpr TileForm kTileForms[] = {
    {256, 1, 1.40f, 4.0f, 1.60f, 10.0f, 15.0f},
    {192, 1, 0.95f, 3.5f, 1.08f, 7.0f, 11.0f},
    {128, 2, 0.70f, 3.0f, 1.04f, 4.0f, 8.0f},
    {64, 2, 0.24f, 3.0f, 0.45f, 1.2f, 2.1f},
};
// the 64-tile in split precision, whose stage holds all three products (the
// others take three stages)
constexpr TileForm kSplit64 = {64, 2, 0.65f, 3.2f, 0.95f, 2.0f, 3.0f};
constexpr int kCus = 256;
// Joining the sums of a K in parts: a launch, a workgroup's time per part, and
// the bytes of the sums, written and read.  X X^T of 64 x 8192 in split
// precision, one tile, is 10 us in 32 parts, 77 us whole (128 stages); of 256 x
// 11008 12 us in 18, 41 whole; of 768 x 30522 42 us in 11 parts of 128-tiles,
// 115 in whole 64-tiles.  64-tiles of 1024 x 4096, 136 of 64 stages, are taken
// whole: 18 us, in two parts 24.
constexpr float kJoin = 5.0f, kJoinPart = 0.035f, kJoinByte = 0.25e-6f;

int stages_of(const SchulzGroup& g, SchulzPhase phase) { return (phase == kGram ? g.np : g.mp) / 64; }

// Runs of about `stages` stages for the K of every group's X X^T (0: all of
// it), as far as the sums have room.
struct Parts {
  int32_t parts[kMaxGroups], stages[kMaxGroups];
};
int64_t sum_bytes(const SchulzGroup& g) {  // of one part
  return (int64_t)g.mp * g.mp * (int64_t)sizeof(float);
}
int64_t sum_room(const GemmArgs& a, const SchulzGroup& g) { return (int64_t)g.mp * g.np * (a.split ? 4 : 2); }
Parts parts_of(const GemmArgs& a, SchulzPhase phase, int stages) {
  Parts p;
  for (int i = 0; i < a.n_groups; ++i) {
    const int all = stages_of(a.group[i], phase);
    int64_t n = stages ? (all + stages - 1) / stages : 1;
    if (n > 1) {
      const int64_t room = sum_room(a, a.group[i]) / sum_bytes(a.group[i]);
      n = room < 1 ? 1 : n < room ? n : room;
    }
    p.stages[i] = (int32_t)((all + n - 1) / n);
    p.parts[i] = (all + p.stages[i] - 1) / p.stages[i];
  }
  return p;
}

// Time until the last workgroup is done when the groups' tiles are handed out
// in order to the next free place, and the parts' sums are joined.
float makespan(const GemmArgs& a, SchulzPhase phase, const TileForm& f, const Parts& p) {
  int64_t all = 0, joined = 0;
  int most = 0;
  for (int i = 0; i < a.n_groups; ++i) {
    all += schulz_tiles(a.group[i], phase, f.tile) * p.parts[i];
    if (p.parts[i] > most) most = p.parts[i];
    if (p.parts[i] > 1) joined += sum_bytes(a.group[i]) * p.parts[i] * a.group[i].count;
  }
  // (up to one workgroup a CU, those of two a CU run alone)
  const bool full = all > (f.per_cu > 1 ? kCus : 3 * kCus / 4);
  const int64_t places = (int64_t)kCus * (full ? f.per_cu : 1);
  // two planes to store in split precision (the 64-tile's figures have them)
  const float planes = a.split && f.tile != 64 ? 3.0f : 0.0f;
  const float rest = (phase == kGram || phase == kPoly ? f.full_rest_symmetric : f.full_rest) + planes;
  // places that become free at the same time, earliest first
  struct Level {
    float at;
    int64_t places;
  };
  constexpr int kLevels = 2 * kMaxGroups + 2;
  Level level[kLevels + 1] = {{0.0f, places}};
  int levels = 1;
  for (int i = 0; i < a.n_groups; ++i) {
    const SchulzGroup& g = a.group[i];
    const float stages = (float)(p.stages[i] * (a.split && f.tile != 64 ? 3 : 1));
    const float each = full ? stages * f.full_stage + rest : stages * f.few_stage + f.few_rest + planes;
    int64_t left = schulz_tiles(g, phase, f.tile) * p.parts[i];
    // whole rounds leave the differences between the places as they are
    const int64_t rounds = left / places;
    for (int l = 0; l < levels; ++l) level[l].at += (float)rounds * each;
    left -= rounds * places;
    while (left > 0) {
      Level first = level[0];
      const int64_t n = left < first.places ? left : first.places;
      left -= n;
      level[0].places -= n;
      if (level[0].places == 0) {
        for (int l = 1; l < levels; ++l) level[l - 1] = level[l];
        --levels;
      }
      const float at = first.at + each;
      int l = levels;
      while (l > 0 && level[l - 1].at > at) --l;
      for (int m = levels; m > l; --m) level[m] = level[m - 1];
      level[l] = {at, n};
      ++levels;
      if (levels > kLevels) {  // join the two earliest
        level[1].places += level[0].places;
        for (int m = 1; m < levels; ++m) level[m - 1] = level[m];
        --levels;
      }
    }
  }
  return level[levels - 1].at + (joined ? kJoin + (float)most * kJoinPart + (float)joined * kJoinByte : 0.0f);
}

}  // namespace

int choose_schulz_tile(GemmArgs& a, SchulzPhase phase) {
  int best = 0;
  float least = 0.0f;
  Parts runs = parts_of(a, phase, 0);
  const Parts whole = runs;
  for (const TileForm& f : kTileForms) {
    if (a.split && f.tile == 256) continue;
    int64_t tiles = 0;
    for (int i = 0; i < a.n_groups; ++i) tiles += schulz_tiles(a.group[i], phase, f.tile);
    if (tiles >= kMaxTiles) continue;
    const TileForm& form = a.split && f.tile == 64 ? kSplit64 : f;
    const float time = makespan(a, phase, form, whole);
    if (!best || time < least) {
      least = time;
      best = f.tile;
      runs = whole;
    }
    if (phase != kGram || f.tile > kPartTile) continue;
    // K in runs, from four stages (which a workgroup has in flight) on
    for (int stages = 4; stages <= 256; stages += stages < 16 ? 2 : stages / 4) {
      const Parts p = parts_of(a, phase, stages);
      int64_t n = 0;
      for (int i = 0; i < a.n_groups; ++i) n += schulz_tiles(a.group[i], phase, f.tile) * p.parts[i];
      if (n >= kMaxTiles) continue;
      const float t = makespan(a, phase, form, p);
      if (t < least) {
        least = t;
        best = f.tile;
        runs = p;
      }
    }
  }
  if (phase == kGram) {
    for (int i = 0; i < a.n_groups; ++i) {
      a.parts[i] = runs.parts[i];
      a.part_stages[i] = runs.stages[i];
    }
  }
  return best;
}

hipError_t launch_schulz_gemm(GemmArgs& a, SchulzPhase phase, int tile, hipStream_t s) {
  if (a.n_groups < 1 || a.n_groups > kMaxGroups) return hipErrorInvalidValue;
  int64_t total = 0;
  bool joined = false;
  for (int i = 0; i < a.n_groups; ++i) {
    int64_t n = schulz_tiles(a.group[i], phase, tile);
    if (phase == kGram && tile <= kPartTile) {
      const SchulzGroup& g = a.group[i];
      const int64_t parts = a.parts[i], stages = a.part_stages[i], all = stages_of(g, phase);
      // every part has a stage, and its sums room
      if (parts < 1 || (parts - 1) * stages >= all || parts * stages < all ||
          (parts > 1 && parts * sum_bytes(g) > sum_room(a, g)))
        return hipErrorInvalidValue;
      n *= parts;
      joined = joined || parts > 1;
    }
    total += n;
    if (total >= kMaxTiles) return hipErrorInvalidValue;
    a.tiles[i] = (int32_t)n;
    a.turns[i] = (int32_t)((n + 7) / 8);
  }
  hipError_t e = hipSuccess;
  switch (tile) {
    case 64: e = launch_schulz_gemm_64(a, phase, s); break;
    case 128: e = launch_schulz_gemm_128(a, phase, s); break;
    case 192: e = launch_schulz_gemm_192(a, phase, s); break;
    case 256: e = launch_schulz_gemm_256(a, phase, s); break;
    default: return hipErrorInvalidValue;
  }
  return e == hipSuccess && joined ? launch_schulz_join(a, s) : e;
}

}  // namespace microadam
