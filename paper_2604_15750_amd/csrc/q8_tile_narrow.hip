// The tiles of the 8-bit integer product of fewer than 128 rows (see q8_tile.h)
#include "q8_tile.h"

template void launch_q8_tiles<false>(const Q8View& w, const Q8GemmArgs& a, const Q8TilePlan& p, hipStream_t st);
