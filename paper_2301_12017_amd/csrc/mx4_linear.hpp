// Products of two operands in microscaled 4-bit floating point: arguments of their kernels (gfx950).
#pragma once
#include "common.hpp"

namespace w4a4 {

struct MX4LinearArgs {
    const uint8_t *a, *w;
    const uint32_t *sa, *sw;
    const uint16_t *bias;
    uint16_t *out;
    int M, N, planes, act, tiles_m, tiles_n;
    int whole;                                                     // tiles that are not taken in parts
};

// Tiles in LDS (mx4_tiles.hip); N < 2^22.
enum MX4Tile { kMX4Tile64x64, kMX4Tile64x128, kMX4Tile128x128, kMX4Tile128x256, kMX4Tile256x256 };
int mx4_tiles(const MX4LinearArgs &g, int dtype, MX4Tile tile, hipStream_t st);

}  // namespace w4a4
