// The tiled products of linear_tile.h for bf16 operands.
#include "linear_tile.h"

namespace bo {

hipError_t launch_product_bf16(TileProduct what, const TileArgs& p, TileShape shape, hipStream_t st) {
  return launch_product<BO_TYPE_BF16>(what, p, shape, st);
}

}  // namespace bo
