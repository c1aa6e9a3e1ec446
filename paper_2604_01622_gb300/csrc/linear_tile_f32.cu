// The tile kernel of dense products on fp32 operands, as planes.
#include "linear_tile.cuh"
#include "linear_tile.h"

namespace ecmoe {

template <>
cudaError_t tc_linear<float>(const TileProblem<float>& t, LaunchStream st) {
  const int64_t slices = (t.K + BK - 1) / BK;
  const TileChoice c = tile_choice(TILE_F32, t.form != LIN_DW, t.M, t.N, slices);
  if (tile_chain(slices, c.splits) > kBlockSlices) return tc_linear_long(t, c, st);
  return tile_launch<1>(t, c, st);
}

}  // namespace ecmoe
