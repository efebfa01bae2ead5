// The gated feed-forward block: both products, the activation and their
// product in one kernel.
#include "nmspmm_products.h"
#include "nmspmm_rows.h"

namespace nmspmm {
namespace {

__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(4))) void k_gated_rows(BlockArgs a) {
    constexpr RowTile t = kRowTileShape;
    using G = RowGeometry<t.wn, t.wm, t.fn, t.fm>;
    __shared__ __attribute__((aligned(1024))) int8_t lds[G::LDSB];
    gemm_rows<t.wn, t.wm, t.fn, t.fm, GatedOut>(a, lds);
}

}  // namespace

int launch_gated(int kind, int tile, const BlockArgs &a, int grid, void *stream) {
    if (tile != kRowTile) return launch_kinds<GatedOut>(kind, tile, a, grid, stream);
    if (kind != NM_KIND_DENSE) return (int)hipErrorInvalidValue;
    hipLaunchKernelGGL(k_gated_rows, dim3(grid), dim3(512), 0, (hipStream_t)stream, a);
    return (int)hipGetLastError();
}

}  // namespace nmspmm
