// The launches of the few rows' product (q8_stream.h).
#include "q8_plan.h"
#include "q8_stream.h"

void launch_q8_stream(const Q8View& w, const Q8GemmArgs& a, const Q8StreamPlan& p, hipStream_t st) {
  if (a.M <= 16) {
    if (p.subs == 1) launch_stream<1, 1, 4, 6>(w, a, st);
    else if (p.subs == 3) launch_stream<1, 3, 4, 3>(w, a, st);
    else launch_stream<1, 2, 4, 6>(w, a, st);
  } else if (p.subs == 1) {
    launch_stream<2, 1, 4, 4>(w, a, st);
  } else {
    launch_stream<2, 2, 4, 4>(w, a, st);
  }
}
