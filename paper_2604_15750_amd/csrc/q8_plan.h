// Which launch serves a product in 8-bit integers.
#pragma once
#include "q8.h"

// The shapes of a tile {WM, WN, KB, ns, more} (see q8_tile.h) and of a band {WM, CW, S, ns, more} (q8_band.h).  ns: nanoseconds per k-tile of 64 that a workgroup
// alone on the chip takes; more: what one adds that shares its compute unit.  15 of 36 shapes that were timed (29 row counts from 8 to 2822, 15 weights from 640 x 640
// to 3584 x 18944, random codes), chosen by leaving out, one by one, the shape whose absence costs least (0.8 % in the mean); what the planner takes is 1 to 2 % behind the best of
// these in the mean, 21 % at most (768 x 1024 x 8192).  (W through LDS in tiles of 32, 64 and 96 rows is among those left out: bands are faster by 8 to 16 % from 24 to 340 rows.)
#define Q8_TILES(X) X(4, 2, 2, 531, 531) X(3, 3, 1, 717, 717) X(2, 3, 1, 472, 472) X(2, 2, 2, 314, 314) X(3, 1, 2, 277, 277)
#define Q8_BANDS(X) \
  X(1, 2, 6, 64, 36) X(1, 3, 6, 90, 62) X(1, 4, 6, 87, 51) X(2, 3, 6, 133, 95) X(2, 4, 5, 133, 108) X(3, 4, 5, 175, 121) X(3, 6, 5, 230, 230) X(4, 4, 4, 208, 122) \
  X(5, 4, 4, 269, 128) X(5, 6, 4, 374, 374)
// rows x packed rows: 256 x 256, 192 x 384, 128 x 384, 128 x 256, 192 x 128; 32 x 64, 32 x 96, 32 x 128, 64 x 96, 64 x 128, 96 x 128, 96 x 192, 128 x 128,
// 160 x 128, 160 x 192
#define ONE(...) +1
constexpr int Q8_TILE_COUNT = 0 Q8_TILES(ONE);
#undef ONE

struct Q8TilePlan {
  int tile;  // index into Q8_TILES, or behind those into Q8_BANDS
  int rows, cols;  // of a tile
  int nblocks, mblocks;
  int splits, stages;  // workgroups that share a tile's K, and how many stages each has
  size_t workspace;    // bytes: the sums of every split of a launch that splits K, 4 KiB a unit and 32 rows
  float us;            // estimated
};
// threads of its launch: 8 wavefronts a tile, one a unit of a band; workgroups in eights (see tile_of)
inline int64_t q8_tile_threads(const Q8TilePlan& p) {
  return ((int64_t)p.nblocks * p.mblocks * p.splits + 7) / 8 * 8 * (p.tile < Q8_TILE_COUNT ? 512 : p.cols / 32 * 64);
}
constexpr int Q8_SPLIT_WGS = 256, Q8_MAX_SPLITS = 16;  // (a launch that splits K is one round)
Q8TilePlan q8_tile_plan(int M, int units, int K);
void launch_q8_tiles(const Q8View& w, const Q8GemmArgs& a, const Q8TilePlan& p, hipStream_t st);
void launch_q8_bands(const Q8View& w, const Q8GemmArgs& a, const Q8TilePlan& p, hipStream_t st);

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
