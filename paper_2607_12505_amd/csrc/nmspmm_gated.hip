// The gated feed-forward block: both products, the activation and their
// product in one kernel.
#include "nmspmm_products.h"

namespace nmspmm {

int launch_gated(int kind, int tile, const BlockArgs &a, int grid, void *stream) {
    return launch_kinds<GatedOut, kScaledTiles>(kind, tile, a, grid, stream);
}

}  // namespace nmspmm
