// The tiled kernel on operands of a 16-bit type: forward (A in k rows, B not), gradient of A (both), gradient of B (neither).
#pragma once
#include "ops_tile.h"

namespace ops_tile {

template <int ELEM, bool AKC, bool BKC>
int launch_16bit_layout(const OpsGemm& g, OpsTile tile)
{
    if (tile == TILE_256) return launch_tiles<ELEM, AKC, BKC, 256, 256, 2>(g);
    if constexpr (AKC && !BKC) { if (tile == TILE_128x256) return launch_tiles<ELEM, true, false, 128, 256, 3>(g); }
    if (tile == TILE_128_ANY) return launch_tiles<ELEM, AKC, BKC, 128, 128, 2, ANY_ALIGNMENT>(g);
    return launch_tiles<ELEM, AKC, BKC, 128, 128, 2>(g);
}

template <int ELEM>
int launch_16bit(const OpsGemm& g, OpsTile tile)
{
    if (g.a_kc) return g.b_kc ? launch_16bit_layout<ELEM, true, true>(g, tile) : launch_16bit_layout<ELEM, true, false>(g, tile);
    return launch_16bit_layout<ELEM, false, false>(g, tile);
}

}  // namespace ops_tile
