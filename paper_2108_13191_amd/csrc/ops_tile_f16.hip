// The tiled kernel on f16 operands: forward (A in k rows, B not), gradient of A (both), gradient of B (neither).
#include "ops_tile.h"

int ops_launch_tiles_f16(const OpsGemm& g, int block)
{
    using namespace ops_tile;
    if (g.a_kc) {
        if (g.b_kc) return block == 256 ? launch_tiles<ELEM_F16, true, true, 256, 256>(g) : launch_tiles<ELEM_F16, true, true, 128, 128>(g);
        return block == 256 ? launch_tiles<ELEM_F16, true, false, 256, 256>(g) : launch_tiles<ELEM_F16, true, false, 128, 128>(g);
    }
    return block == 256 ? launch_tiles<ELEM_F16, false, false, 256, 256>(g) : launch_tiles<ELEM_F16, false, false, 128, 128>(g);
}
