// Grouped products in bf16 (see product_tiles.hpp).
#include "product_tiles.hpp"

namespace cocod {

hipError_t launch_store_bf16(hipStream_t stream, Layout layout, Tile tile, const ProductParams &p) { return launch_store<Bf16>(stream, layout, tile, p); }

}  // namespace cocod
