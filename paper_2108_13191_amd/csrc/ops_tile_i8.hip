// The tiled kernel on 8-bit integers with scales for each row and column.
#include "ops_tile.h"

int ops_launch_tiles_i8(const OpsGemm& g, OpsTile tile)
{
    using namespace ops_tile;
    if (tile == TILE_256_LONG) return ops_launch_long_i8(g);
    if (tile == TILE_256) return launch_tiles<ELEM_I8, true, true, 256, 256, 2>(g);
    return launch_tiles<ELEM_I8, true, true, 128, 128, 2>(g);
}
