// Which kernel and form a dense product takes, by estimated time. Internal.
#pragma once
#include <cuda_bf16.h>

#include <algorithm>
#include <cstdint>

#include "launch.h"

namespace ecmoe {

// Forms of linear_tile.cuh: one-CTA tiles of 128 x 64 and 128 x 128, pair tiles of 256 x 128; for long sums
// pair tiles of 256 x 256. (Those were the fastest at none of 65 other products: where they are many, the
// persistent kernel is.)
struct TileForm {
  int rows, cols, ctas;   // of a tile; CTAs that work on one block of K
  double planes_us;       // the least a k-slice of fp32 planes, 24 MMAs, takes; 256 x 256: six times four
};
constexpr TileForm kTileForms[4] = {{128, 64, 1, 0.8}, {128, 128, 1, 1.1}, {256, 128, 2, 0.92},
                                    {256, 256, 2, 1.7}};

// Rows of A that a CTA loads: of a product of fewer than 128 rows only those there are, in eights (the
// swizzle's unit), where they are rows in memory. The MMA still reads 128: what stands in the others' place
// ends up in rows of the accumulator that nobody reads.
inline int tile_a_rows(int form, bool a_rows, int64_t M) {
  return a_rows && kTileForms[form].ctas == 1 && M < 128 ? (int)(M + 7) / 8 * 8 : 128;
}
// Operand bytes of a k-slice of 64 in one CTA's shared memory, and the slices its ring holds. One CTA to an
// SM takes a deep ring (a load's round trip is 1.2 us and more: 96 KB in flight are 80 GB/s, 43 bytes a
// clock), two share the shared memory. Clusters of eight always share it: they must find eight SMs of one
// GPC, and 128 CTAs of them one to an SM did not all run at once.
inline int tile_stage(int form, int planes, int a_rows) {
  return planes * (a_rows * 128 + kTileForms[form].cols * 128 / kTileForms[form].ctas);
}
constexpr int kTileMaxStages = 16;
constexpr int kTileExtra = 2048;                        // alignment, barriers
constexpr int kTileDeep = 232448 - kTileExtra, kTileShared = 98304;
inline int tile_ring(int stage, bool deep) {
  return std::min(kTileMaxStages, (deep ? kTileDeep : kTileShared) / stage);
}
inline bool tile_deep(int64_t ctas, int cluster) { return ctas <= kSms && cluster <= 4; }

struct TileChoice {
  int form, splits;
  double us;
};

// Which products: bf16 operands, fp32 ones as three planes, or bf16 ones with a sum too long for one
// accumulator. The last two keep the tile's sums in registers (SUMS in linear_tile.cuh).
enum TileKind { TILE_BF16, TILE_F32, TILE_LONG };
// k-slices that an accumulator of bf16 operands takes at most, 32768 of K: what the tensor cores cut off of a
// sum of one sign is 1.7e-4 of it then, a twentieth of half a bf16 step.
constexpr int64_t kLongSlices = 512;
// k-slices whose fp32 results are added in one chain; a power of two. (1000 x 500 x 364: 12.7 us, with the
// second level's registers 13.6.)
constexpr int kBlockSlices = 256;
inline int64_t tile_chain(int64_t slices, int splits) { return (slices + splits - 1) / splits; }

// The form and the number of blocks of K with the least estimated time. A CTA's k-slice takes a share of a
// load's round trip (1.42 us over the slices of the ring) or its bytes at 139 GB/s an SM from L2, whichever
// is longer, and its epilogue 0.09 us per 1000 outputs; a tile's joined blocks 0.093 us per 1000 of all of
// it, and 1.1 us. Constants fitted to 65 products in all their forms (9 to 8000 rows, K and N 200 to
// 8192), of which it takes the fastest form or one 2% slower on average, a quarter at worst. fp32 results
// (f32): one CTA to an SM, whose registers hold the tile's sums, clusters of four at most, and three planes
// an operand (19 products: the fastest form or one 2% slower at worst).
// Long sums: one CTA to an SM likewise, and split only where all their CTAs run at once (100000 rows of
// 2048 x 8192, 512 CTAs: dW 2.05 ms, split in two 2.20), into eight where there are no more than eight tiles
// (2097152 rows of 64 x 64: 710 us, in four 1400; 16 tiles and more: half as long again in eight as in four).
inline TileChoice tile_choice(TileKind kind, bool a_rows, int64_t M, int64_t N, int64_t slices) {
  TileChoice best{0, 1, 1e30};
  const bool sums = kind != TILE_BF16;
  for (int f = 0; f < (kind == TILE_LONG ? 4 : 3); ++f) {
    const TileForm& t = kTileForms[f];
    const int64_t tiles = ((M + t.rows - 1) / t.rows) * ((N + t.cols - 1) / t.cols);
    const int stage = tile_stage(f, kind == TILE_F32 ? 3 : 1, tile_a_rows(f, a_rows, M));
    const int most = kind == TILE_BF16 || (kind == TILE_LONG && tiles <= 8) ? 8 : 4;
    for (int s = 1; s * t.ctas <= most && s <= slices; s *= 2) {
      const int64_t ctas = tiles * t.ctas * s;
      if (kind == TILE_BF16 && tile_chain(slices, s) > kLongSlices) continue;
      if (kind == TILE_LONG && s > 1 && ctas > kSms) continue;
      const bool deep = sums || tile_deep(ctas, t.ctas * s);
      const int on = deep ? 1 : 2;   // CTAs an SM runs at once
      const int64_t turns = (ctas + kSms * on - 1) / (kSms * on);
      const double at_once = (double)std::min<int64_t>(on, (ctas + kSms - 1) / kSms);
      const double slice = std::max({1.42 / tile_ring(stage, deep), at_once * stage / 139e3,
                                     !sums ? 0.0 : kind == TILE_F32 ? t.planes_us : t.planes_us / 6});
      const double outputs = std::min<double>((double)M, 128.0) * t.cols / 1000;
      const double finish = s == 1 ? 0.09 * outputs : 1.1 + 0.093 * outputs;
      const double us =
          3.4 + (double)turns * ((double)((slices + s - 1) / s) * slice + at_once * finish);
      if (us < best.us) best = {f, s, us};
    }
  }
  return best;
}

// The tile kernel for sums too long for one accumulator (bf16) or one chain of fp32 sums, in a chosen form.
template <typename T>
struct TileProblem;
cudaError_t tc_linear_long(const TileProblem<__nv_bfloat16>& t, const TileChoice& c, LaunchStream st);
cudaError_t tc_linear_long(const TileProblem<float>& t, const TileChoice& c, LaunchStream st);

// The persistent kernel's 256 x 256 pair tiles, for sums that one accumulator takes: 0.275 us a k-slice and
// wave of tiles (64 tiles of 32 slices: 15.7 us, of 128: 42.0 us; pair tiles of 256 x 128: 16.3 and 44.5 us).
inline double pairs_us(int64_t M, int64_t N, int64_t slices) {
  const int64_t tiles = ((M + 255) / 256) * ((N + 255) / 256), walkers = kSms / 2;
  return 6.8 + 0.275 * (double)((tiles + walkers - 1) / walkers) * (double)slices;
}

}  // namespace ecmoe
