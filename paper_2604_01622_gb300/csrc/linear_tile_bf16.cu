// The tile kernel of dense products on bf16 operands, and the choice between it, the persistent kernel and the
// tile kernel for long sums.
#include "linear_tile.cuh"
#include "linear_tile.h"

namespace ecmoe {

template <>
cudaError_t tc_linear<bf16>(const TileProblem<bf16>& t, LaunchStream st) {
  const int64_t slices = (t.K + BK - 1) / BK;
  const bool a_rows = t.form != LIN_DW;
  const TileChoice c = tile_choice(TILE_BF16, a_rows, t.M, t.N, slices);
  if (slices > kLongSlices) {
    const TileChoice l = tile_choice(TILE_LONG, a_rows, t.M, t.N, slices);
    return l.us < c.us ? tc_linear_long(t, l, st) : tile_launch<0>(t, c, st);
  }
  return pairs_us(t.M, t.N, slices) < c.us ? tc_linear_pairs(t, st) : tile_launch<0>(t, c, st);
}

}  // namespace ecmoe
