// The int8 product with scales for each token and channel.
#include "nmspmm_products.h"

namespace nmspmm {

int launch_scaled(int kind, int tile, const BlockArgs &a, int grid, void *stream) {
    return launch_kinds<ScaledOut>(kind, tile, a, grid, stream);
}

}  // namespace nmspmm
