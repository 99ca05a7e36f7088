// Tiles of the 8-bit integer product, gated, to fp32 (see q8_tile.h)
#define Q8_TILE_INSTANTIATE
#include "q8_tile.h"

template void launch_q8_tile<true, float>(const Q8View& w, const Q8GemmArgs& a, const Q8TilePlan& p, hipStream_t st);
