// The tiled kernel on f16 operands: forward (A in k rows, B not), gradient of A (both), gradient of B (neither).
#include "ops_tile.h"

namespace {
template <bool AKC, bool BKC>
int launch_tile(const OpsGemm& g, OpsTile tile)
{
    using namespace ops_tile;
    if (tile == TILE_256) return launch_tiles<ELEM_F16, AKC, BKC, 256, 256, 2>(g);
    if constexpr (AKC && !BKC) { if (tile == TILE_128x256) return launch_tiles<ELEM_F16, true, false, 128, 256, 3>(g); }
    if (tile == TILE_128_ANY) return launch_tiles<ELEM_F16, AKC, BKC, 128, 128, 2, ANY_ALIGNMENT>(g);
    return launch_tiles<ELEM_F16, AKC, BKC, 128, 128, 2>(g);
}
}  // namespace

int ops_launch_tiles_f16(const OpsGemm& g, OpsTile tile)
{
    if (g.a_kc) return g.b_kc ? launch_tile<true, true>(g, tile) : launch_tile<true, false>(g, tile);
    return launch_tile<false, false>(g, tile);
}
