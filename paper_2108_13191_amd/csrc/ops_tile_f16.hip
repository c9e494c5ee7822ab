#include "ops_tile_16bit.h"

int ops_launch_tiles_f16(const OpsGemm& g, OpsTile tile) { return ops_tile::launch_16bit<ELEM_F16>(g, tile); }
