// Which launch serves a product in 8-bit integers.
#pragma once
#include "q8.h"

// The shape of a tile {WM, WN, RW, CW, KB, MF, NT, ns}: see q8_tile.h.  NT: a W that one row block reads is read non-temporally, past the memory-side cache, in
// which the weights of a model do not stay from pass to pass (5 % of launches of up to 64 rows; nothing beyond).  ns: nanoseconds per k-tile of 64 that a workgroup alone on the
// chip takes.  16 of 60 shapes that were timed (29 row counts from 8 to 2822, 15 weights from 640 x 640 to 3584 x 18944, random codes), chosen by leaving out, one by
// one, the shape whose absence costs least: what the planner takes is 2 % behind the best of these in the mean.
#define Q8_TILES(X) \
  X(4, 2, 2, 4, 2, 16, false, 586) X(3, 3, 2, 4, 1, 16, false, 675) X(3, 2, 2, 4, 2, 16, false, 506) X(2, 3, 2, 4, 1, 16, false, 499) \
  X(2, 2, 2, 4, 2, 16, false, 325) X(5, 1, 1, 6, 2, 32, false, 348) X(5, 1, 1, 8, 2, 32, false, 351) X(3, 1, 2, 4, 2, 32, false, 231) \
  X(1, 2, 4, 2, 2, 16, false, 202) X(3, 1, 1, 4, 2, 32, false, 190) X(1, 1, 2, 5, 2, 16, true, 173) X(1, 1, 2, 4, 2, 16, true, 149) \
  X(1, 1, 2, 2, 2, 16, true, 121) X(1, 1, 1, 5, 1, 16, true, 151) X(1, 1, 1, 4, 2, 16, true, 128) X(1, 1, 1, 2, 2, 16, true, 114)
// rows x packed rows: 256 x 256, 192 x 384, 192 x 256, 128 x 384, 128 x 256, 160 x 192, 160 x 256, 192 x 128, 128 x 128, 96 x 128, 64 x 160, 64 x 128, 64 x 64, 32 x 160,
// 32 x 128, 32 x 64

struct Q8TilePlan {
  int tile;  // index into Q8_TILES
  int rows, cols;  // of a tile
  int nblocks, mblocks;
  int splits, stages;  // workgroups that share a tile's K, and how many stages each has
  size_t workspace;    // bytes: the sums of every split of a launch that splits K, 4 KiB a unit and 32 rows
  float us;            // estimated
};
constexpr int Q8_SPLIT_WGS = 256, Q8_MAX_SPLITS = 16;  // (a launch that splits K is one round)
Q8TilePlan q8_tile_plan(int M, int units, int K);
template <bool WIDE>
void launch_q8_tiles(const Q8View& w, const Q8GemmArgs& a, const Q8TilePlan& p, hipStream_t st);

void launch_q8_join(const Q8View& w, const Q8GemmArgs& a, const Q8TilePlan& p, hipStream_t st);  // behind one that splits K

constexpr int Q8_STREAM_ROWS = 32;  // up to as many rows may be the streamed product's (q8_stream.h)
struct Q8StreamPlan {
  int subs;  // of a workgroup: 1, 2 or 3
  float us;  // estimated
};
Q8StreamPlan q8_stream_plan(int M, int units, int K, bool gated);
void launch_q8_stream(const Q8View& w, const Q8GemmArgs& a, const Q8StreamPlan& p, hipStream_t st);

struct Q8Plan {
  bool streamed;
  Q8StreamPlan stream;
  Q8TilePlan tile;
  size_t workspace;  // bytes that the launch needs
};
Q8Plan q8_plan(int M, int units, int K, bool gated, int64_t x_stride);
void launch_q8_gemm(const Q8View& w, const Q8GemmArgs& a, const Q8Plan& p, hipStream_t st);
