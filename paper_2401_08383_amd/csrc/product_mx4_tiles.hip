// Tiles of moe_grouped_product_mx4 (see product_tiles.hpp): instances of their own object.
#include "product_tiles.hpp"

namespace exf {

int launch_mx4_tiles(const RowsTiles& p, hipStream_t stream) { return launch_rows_tiles<256, kMx4>(p, stream, "moe_grouped_product_mx4"); }

}  // namespace exf
