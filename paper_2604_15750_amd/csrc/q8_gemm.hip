// Products in 8-bit integers: the packing of a weight, and the choice of the kernel.
#include <cmath>

#include "q8_gemm.h"
#include "q8_plan.h"

namespace {

// a thread: the 16 bytes of one (unit, k-tile, sub, chunk, row)
__global__ __launch_bounds__(256) void q8_pack_kernel(const int8_t* __restrict__ codes, int64_t stride, int n, int k, int gated, int kt, i32x4* __restrict__ out, int64_t chunks) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= chunks) return;
  const int row = i & 15, chunk = (i >> 4) & 3, sub = (i >> 6) & 1;
  const int64_t tile = i >> 7;
  const int unit = (int)(tile / kt), k0 = (int)(tile % kt) * 64 + chunk * 16, channel = q8_channel(unit, 16 * sub + row, n, gated);
  union { i32x4 v; int8_t b[16]; } o;
  o.v = i32x4{0, 0, 0, 0};
  if (channel < n && k0 < k) {
    o.v = *(const i32x4*)(codes + channel * stride + k0);
    if (k0 + 16 > k)
#pragma unroll
      for (int j = 0; j < 16; ++j)
        if (k0 + j >= k) o.b[j] = 0;
  }
  out[i] = o.v;
}
__global__ __launch_bounds__(256) void q8_pack_scale_kernel(const float* __restrict__ scale, int n, int gated, int units, float* __restrict__ out) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= units * 32) return;
  const int channel = q8_channel(i >> 5, i & 31, n, gated);
  out[i] = channel < n ? scale[channel] : 0.f;
}

// The sums of a launch that splits K, added up and finished: a wavefront, a workgroup of its own, has a unit's 32 packed rows of 32 tokens (four of them in a workgroup leave
// compute units without work where there are few: 24 x 3584 x 18944 15.7 us with both launches, 15.3 so)
__global__ __launch_bounds__(64) void q8_join_kernel(const i32x4* __restrict__ parts, int splits, int M, int units, const float* __restrict__ wscale, const float* __restrict__ x_scale,
                                                      void* __restrict__ out, int64_t out_stride, int outputs, int form) {
  const int lane = threadIdx.x, blocks = (M + 31) >> 5, frag = blockIdx.x;
  const int u = frag / blocks, m = (frag - u * blocks) * 32 + (lane & 15);
  const i32x4* from = parts + (int64_t)frag * 256 + lane;
  i32x4 t[4];
#pragma unroll
  for (int a = 0; a < 4; ++a) t[a] = from[a * 64];
#pragma unroll 4
  for (int sp = 1; sp < splits; ++sp) {
    from += (int64_t)units * blocks * 256;
#pragma unroll
    for (int a = 0; a < 4; ++a) t[a] += from[a * 64];
  }
  const float xs[2] = {x_scale[min(m, M - 1)], x_scale[min(m + 16, M - 1)]};
  with_form(form, out, [&](auto gated, auto* to) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      finish8<decltype(gated)::value>(t[2 * i], t[2 * i + 1], xs[i], wscale, to + (int64_t)(m + 16 * i) * out_stride, u, lane >> 4, outputs, m + 16 * i < M);
  });
}

}  // namespace

void launch_q8_pack(const int8_t* codes, int64_t stride, const float* scale, const Q8View& w, void* data, hipStream_t st) {
  const int64_t chunks = (int64_t)w.units * w.kt * 128;
  q8_pack_kernel<<<(unsigned)((chunks + 255) / 256), 256, 0, st>>>(codes, stride, w.n, w.k, w.gated, w.kt, (i32x4*)data, chunks);
  q8_pack_scale_kernel<<<(w.units * 32 + 255) / 256, 256, 0, st>>>(scale, w.n, w.gated, w.units, (float*)w.scale);
}

void launch_q8_join(const Q8View& w, const Q8GemmArgs& a, const Q8TilePlan& p, hipStream_t st) {
  q8_join_kernel<<<w.units * ((a.M + 31) / 32), 64, 0, st>>>((const i32x4*)a.workspace, p.splits, a.M, w.units, w.scale, a.x_scale, a.out, a.out_stride, w.outputs(),
                                                                        out_form(w, a));
}

// The shape and K split with the least estimated time.  A k-tile takes what a workgroup alone on the chip takes (ns), or what the matrix cores give when all are busy (4.04
// POP/s, at the 1.93 GHz that power leaves), what the L2s (25.6 TB/s) or, for W, HBM (7.07 TB/s) give to all of the workgroups that run at a time, whichever is most, joined by a 4-norm; row blocks
// share W, up to 8 of them and not perfectly: their number to the power 0.633.  256 further workgroups add `more` to that, and their epilogues; a K split adds a launch, and the
// sums' way to memory and back.  Constants fitted to the launches named at Q8_TILES: 10 % off in the root mean square.
Q8TilePlan q8_tile_plan(int M, int units, int K) {
  struct Shape {
    int bm, un, kb;
    float ns_4, more_4, chip_4, hbm;  // 4th powers of ns, of `more`, and of what the matrix cores and the L2s allow on a full chip; ns that HBM allows where one row block reads W
  };
  constexpr float CUS = 256.f;
  static const auto shape = [](int bm, int un, int kb, float ns, float more) {
    auto p4 = [](float x) { return x * x * x * x; };
    return Shape{bm, un, kb, p4(ns), p4(more), p4(bm * un * 32 * 128 * CUS / 4.04e6f) + p4((bm + un * 32) * 64 * CUS / 25.6e3f), un * 2048 * CUS / 7.07e3f};
  };
#define TILE(WM, WN, KB, NS, MORE) shape(64 * WM, 4 * WN, KB, NS, MORE),
#define BAND(WM, CW, S, NS, MORE) shape(32 * WM, CW, 2, NS, MORE),
  static const Shape shapes[] = {Q8_TILES(TILE) Q8_BANDS(BAND)};
#undef TILE
#undef BAND
  static constexpr float shared[9] = {1, 1, 0.645f, 0.499f, 0.416f, 0.361f, 0.322f, 0.292f, 0.268f};  // n^-0.633
  const int KT = (K + 63) / 64;
  Q8TilePlan best{};
  best.us = 1e30f;
  int i = -1;
  for (const Shape& t : shapes) {
    ++i;
    const int mb = (M + t.bm - 1) / t.bm, nb = (units + t.un - 1) / t.un, stages = (KT + t.kb - 1) / t.kb;
    const float out = t.bm * t.un * 32.f, edge = t.bm + t.un * 32.f, hbm = t.hbm * shared[mb < 8 ? mb : 8], full_4 = t.chip_4 + hbm * hbm * hbm * hbm;
    auto ns = [&](float own_4, float share) { return sqrtf(sqrtf(own_4 + full_4 * (share * share) * (share * share))); };
    const int64_t wgs = (int64_t)mb * nb;
    for (int sp = 1; sp <= Q8_MAX_SPLITS; ++sp) {
      if (sp > 1 && (wgs * sp > Q8_SPLIT_WGS || stages < 4 * sp)) break;
      const int per = (stages + sp - 1) / sp;
      if ((stages + per - 1) / per != sp) continue;  // (a split without stages)
      const int64_t all = wgs * sp, full = (all - 1) / 256;
      const float last = (all - 256 * full) / CUS;
      float us = per * t.kb * 1e-3f * ((full ? full * ns(t.more_4, 1.f) : 0.f) + ns(t.ns_4, last)) + 1.67f + (full + last) * 1.336e-4f * out + (0.44f * full + 1) * 9.76e-3f * edge;
      if (sp > 1) us += 1.8f + sp * (0.194f + 5e-4f * units * ((M + 31) / 32));
      if (us < best.us) best = Q8TilePlan{i, t.bm, t.un * 32, nb, mb, sp, per, sp > 1 ? (size_t)sp * units * ((M + 31) / 32) * 4096 : 0, us};
    }
  }
  return best;
}

// Subs of a workgroup, for the least that the busiest compute unit has to read (its subs of W, and X once a workgroup) at 34 bytes a nanosecond, up to 50 on a
// chip that is partly full: within 10 % of what was measured from 512 x 16000 to 37888 x 3584 at 8 and 16 rows
Q8StreamPlan q8_stream_plan(int M, int units, int K, bool gated) {
  const int subs = 2 * units, rows = M < Q8_STREAM_ROWS ? M : Q8_STREAM_ROWS;
  Q8StreamPlan best{2, 1e30f};
  for (int n = gated ? 2 : 1; n <= (gated || rows > 16 ? 2 : 3); ++n) {
    const int wgs = (subs + n - 1) / n;
    const float rate = (n == 3 ? 31e3f : 34e3f) + (wgs < 256 ? 16e3f * (256 - wgs) / 256 : 0.f);
    const float us = 2.2f + (wgs + 255) / 256 * (16.f * n + rows) * K / rate;
    if (us < best.us) best = Q8StreamPlan{n, us};
  }
  return best;
}

// Few rows are either's, whichever is estimated to take less; rows so far apart that a tile's would be past 32 bits are streamed, however many
Q8Plan q8_plan(int M, int units, int K, bool gated, int64_t x_stride) {
  Q8Plan c{};
  const bool far = x_stride > 1 << 22;
  if (M <= Q8_STREAM_ROWS || far) c.stream = q8_stream_plan(M, units, K, gated);
  if (!far) c.tile = q8_tile_plan(M, units, K);
  c.streamed = far || (M <= Q8_STREAM_ROWS && c.stream.us <= c.tile.us);
  c.workspace = c.streamed ? 0 : c.tile.workspace;
  return c;
}

size_t q8_gemm_workspace(int rows, int n, int k, int gated) {
  // (a tile's plan depends on the rows through their blocks of 32, and one that splits K has at most Q8_SPLIT_WGS / 2 tiles, of at most 256 rows or 12 units)
  const int units = q8_units(n, gated), most = 256 * (Q8_SPLIT_WGS / 2 / ((units + 11) / 12));
  size_t bytes = 0;
  for (int m = 1; m <= rows && m <= most; m += 32) {
    const size_t need = q8_tile_plan(m, units, k).workspace;
    if (need > bytes) bytes = need;
  }
  return bytes;
}

void launch_q8_gemm(const Q8View& w, const Q8GemmArgs& a, const Q8Plan& c, hipStream_t st) {
  if (c.streamed) return launch_q8_stream(w, a, c.stream, st);
  c.tile.tile < Q8_TILE_COUNT ? launch_q8_tiles(w, a, c.tile, st) : launch_q8_bands(w, a, c.tile, st);
  if (c.tile.splits > 1) launch_q8_join(w, a, c.tile, st);
}
