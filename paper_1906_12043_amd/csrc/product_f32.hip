// Grouped products in f32 (see product_tiles.hpp).
#include "product_tiles.hpp"

namespace cocod {

hipError_t launch_store_f32(hipStream_t stream, Layout layout, Tile tile, const ProductParams &p) { return launch_store<F32>(stream, layout, tile, p); }

}  // namespace cocod
