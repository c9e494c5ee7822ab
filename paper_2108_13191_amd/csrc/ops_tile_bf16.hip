#include "ops_tile_16bit.h"

int ops_launch_tiles_bf16(const OpsGemm& g, OpsTile tile) { return ops_tile::launch_16bit<ELEM_BF16>(g, tile); }
