#include "product_tile.h"

namespace craft {

hipError_t launch_product_tiles_bf16(const ProductArgs &a, int32_t width, int32_t height, hipStream_t s) {
    return launch_tiles<CRAFT_BF16>(a, width, height, s);
}

}  // namespace craft
