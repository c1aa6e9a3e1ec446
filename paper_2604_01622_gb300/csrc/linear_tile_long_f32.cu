// The tile kernel of dense products on fp32 operands whose sums are too long for one chain of fp32 sums.
#include "linear_tile.cuh"
#include "linear_tile.h"

namespace ecmoe {

cudaError_t tc_linear_long(const TileProblem<float>& t, const TileChoice& c, LaunchStream st) {
  return tile_launch<2>(t, c, st);
}

}  // namespace ecmoe
