// The tiled kernel on e4m3 operands with block scales.
//
// The e4m3 matrix instructions (all four shapes) add the products of neighbouring k with the bits below 2^-13 of the largest one's
// exponent cut off: a sum of 128 of normally distributed values is off by 1.4e-5 of itself and by up to 2e-5 of its magnitudes, at the most by 2^-10 of them.
// A caller has them for large 16-bit results, whose own rounding is coarser, unless it asks for exact products.  Products of
// values widened to f16 are exact and their sums f32, at half the matrix rate: 4000^3 127 us, 1.0 PFLOP/s.  Those are bound by the conversions, 8 cycles each
// (two values), beside the MFMAs: a SIMD has 320 of them (10 fragments of 16 for each of two wavefronts), 2560 cycles, and 174 other vector instructions, for 128 MFMAs of 16
// cycles in a k step of 256 x 128, 4400 cycles in all: the two seldom run side by side.  (Each value is converted by every wavefront that reads it; converting once, on the way into
// LDS, has not been built.)  (In one phase, conversions between the MFMAs, and wavefronts of 64 x 64 in place of 128 x 32: 129; in two phases 135.)  Two workgroups of 128 x 128 a compute unit,
// with a few registers spilled around the loop, fill each other's gaps: (3000,3000,2048) 66 -> 53 us, (4096,8192,1024) 90 -> 79.
#include "ops_tile.h"

int ops_launch_tiles_e4m3(const OpsGemm& g, OpsTile tile)
{
    using namespace ops_tile;
    if (tile == TILE_256) return launch_tiles<ELEM_E4M3, true, true, 256, 256, 2>(g);
    if (tile == TILE_128_FAST) return launch_tiles<ELEM_E4M3, true, true, 128, 128, 2>(g);
    if (tile == TILE_128_SHORT) return launch_tiles<ELEM_E4M3, true, true, 128, 128, 2, WIDENED_SHORT>(g);
    if (tile == TILE_128_PAIR) return launch_tiles<ELEM_E4M3, true, true, 128, 128, 2, WIDENED_PAIR>(g);
    return tile == TILE_256x128 ? launch_tiles<ELEM_E4M3, true, true, 256, 128, 2, WIDENED>(g) : launch_tiles<ELEM_E4M3, true, true, 128, 128, 2, WIDENED>(g);
}
