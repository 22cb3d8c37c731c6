// The tiled products of linear_tile.h for f32 operands.
#include "linear_tile.h"

namespace bo {

hipError_t launch_product_f32(TileProduct what, const TileArgs& p, TileShape shape, hipStream_t st) {
  return launch_product<BO_TYPE_F32>(what, p, shape, st);
}

}  // namespace bo
