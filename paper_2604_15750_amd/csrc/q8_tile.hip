// The tiles of the 8-bit integer product (see q8_tile.h)
#include "q8_tile.h"

void launch_q8_tiles(const Q8View& w, const Q8GemmArgs& a, const Q8TilePlan& p, hipStream_t st) {
  int i = 0;
#define GO(WM, WN, KB, NS, MORE) \
  if (p.tile == i++) return launch_tile<WM, WN, KB>(w, a, p, st);
  Q8_TILES(GO)
#undef GO
}
