// Tiles of moe_grouped_product (see product_tiles.hpp): instances of their own object.
#include "product_tiles.hpp"

namespace exf {

int launch_forward_tiles(const RowsTiles& p, hipStream_t stream) { return launch_rows_tiles<256, kForward>(p, stream, "moe_grouped_product"); }

}  // namespace exf
