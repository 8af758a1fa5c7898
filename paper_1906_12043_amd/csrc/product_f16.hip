// Grouped products in f16 (see product_tiles.hpp).
#include "product_tiles.hpp"

namespace cocod {

hipError_t launch_store_f16(hipStream_t stream, Layout layout, Tile tile, const ProductParams &p) { return launch_store<F16>(stream, layout, tile, p); }

}  // namespace cocod
