// The bands of the 8-bit integer product (see q8_band.h)
#include "q8_band.h"

void launch_q8_bands(const Q8View& w, const Q8GemmArgs& a, const Q8TilePlan& p, hipStream_t st) {
  int i = Q8_TILE_COUNT;
#define GO(WM, CW, S, NS, MORE) \
  if (p.tile == i++) return p.mblocks == 1 ? launch_band<WM, CW, S, true>(w, a, p, st) : launch_band<WM, CW, S, false>(w, a, p, st);
  Q8_BANDS(GO)
#undef GO
}
