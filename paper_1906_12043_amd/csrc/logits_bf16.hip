// Logits in bf16: statistics of their rows, slopes of the loss (see product_tiles.hpp).
#include "product_tiles.hpp"

namespace cocod {

hipError_t launch_logits_bf16(hipStream_t stream, Finish finish, Tile tile, const ProductParams &p) { return launch_logits<Bf16>(stream, finish, tile, p); }

}  // namespace cocod
