// Tiles of moe_grouped_product_dx (see product_tiles.hpp): instances of their own object.
#include "product_tiles.hpp"

namespace exf {

int launch_rows_gradient_tiles(const RowsTiles& p, hipStream_t stream) { return launch_rows_tiles<256, kRowsGradient>(p, stream, "moe_grouped_product_dx"); }

}  // namespace exf
