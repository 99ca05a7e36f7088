// The tiles of the 8-bit integer product of 128 rows and more (see q8_tile.h)
#include "q8_tile.h"

template void launch_q8_tiles<true>(const Q8View& w, const Q8GemmArgs& a, const Q8TilePlan& p, hipStream_t st);
