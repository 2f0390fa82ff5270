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
// the rest, mostly the stores of all CUs at once, is 40% of a 256-tile's time.
struct TileForm {
  int tile, per_cu;
  float few_stage, few_rest, full_stage, full_rest, full_rest_symmetric;
};
constexpr TileForm kTileForms[] = {
    {256, 1, 1.40f, 4.0f, 1.60f, 10.0f, 15.0f},
    {192, 1, 0.95f, 3.0f, 1.08f, 7.0f, 11.0f},
    {128, 2, 0.70f, 2.0f, 1.04f, 4.0f, 8.0f},
    {64, 2, 0.38f, 1.5f, 0.45f, 1.2f, 2.1f},
};
// the 64-tile in split precision, whose stage holds all three products (the
// others take three stages)
constexpr TileForm kSplit64 = {64, 2, 0.62f, 2.0f, 0.90f, 2.0f, 3.0f};
constexpr int kCus = 256;

// Time until the last workgroup is done when the groups' tiles are handed out
// in order to the next free place.
float makespan(const GemmArgs& a, SchulzPhase phase, const TileForm& f) {
  int64_t all = 0;
  for (int i = 0; i < a.n_groups; ++i) all += schulz_tiles(a.group[i], phase, f.tile);
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
    const int k = phase == kGram ? g.np : g.mp;
    const float stages = (float)(k / 64 * (a.split && f.tile != 64 ? 3 : 1));
    const float each = full ? stages * f.full_stage + rest : stages * f.few_stage + f.few_rest + planes;
    int64_t left = schulz_tiles(g, phase, f.tile);
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
  return level[levels - 1].at;
}

}  // namespace

int choose_schulz_tile(const GemmArgs& a, SchulzPhase phase) {
  int best = 0;
  float least = 0.0f;
  for (const TileForm& f : kTileForms) {
    if (a.split && f.tile == 256) continue;
    int64_t tiles = 0;
    for (int i = 0; i < a.n_groups; ++i) tiles += schulz_tiles(a.group[i], phase, f.tile);
    if (tiles >= kMaxTiles) continue;
    const float time = makespan(a, phase, a.split && f.tile == 64 ? kSplit64 : f);
    if (!best || time < least) {
      least = time;
      best = f.tile;
    }
  }
  return best;
}

hipError_t launch_schulz_gemm(GemmArgs& a, SchulzPhase phase, int tile, hipStream_t s) {
  if (a.n_groups < 1 || a.n_groups > kMaxGroups) return hipErrorInvalidValue;
  int64_t total = 0;
  for (int i = 0; i < a.n_groups; ++i) {
    const int64_t n = schulz_tiles(a.group[i], phase, tile);
    total += n;
    if (total >= kMaxTiles) return hipErrorInvalidValue;
    a.tiles[i] = (int32_t)n;
    a.turns[i] = (int32_t)((n + 7) / 8);
  }
  switch (tile) {
    case 64: return launch_schulz_gemm_64(a, phase, s);
    case 128: return launch_schulz_gemm_128(a, phase, s);
    case 192: return launch_schulz_gemm_192(a, phase, s);
    case 256: return launch_schulz_gemm_256(a, phase, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace microadam
