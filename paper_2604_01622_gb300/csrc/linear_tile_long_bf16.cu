// The tile kernel of dense products on bf16 operands whose sums are too long for one accumulator.
#include "linear_tile.cuh"
#include "linear_tile.h"

namespace ecmoe {

cudaError_t tc_linear_long(const TileProblem<bf16>& t, const TileChoice& c, LaunchStream st) {
  return tile_launch<1>(t, c, st);
}

}  // namespace ecmoe
