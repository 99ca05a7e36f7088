// Products in 8-bit integers: the packing of a weight, and the choice of the kernel.
#include "q8_gemm.h"
#include "q8_tile.h"

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

}  // namespace

void launch_q8_pack(const int8_t* codes, int64_t stride, const float* scale, const Q8View& w, void* data, hipStream_t st) {
  const int64_t chunks = (int64_t)w.units * w.kt * 128;
  q8_pack_kernel<<<(unsigned)((chunks + 255) / 256), 256, 0, st>>>(codes, stride, w.n, w.k, w.gated, w.kt, (i32x4*)data, chunks);
  q8_pack_scale_kernel<<<(w.units * 32 + 255) / 256, 256, 0, st>>>(scale, w.n, w.gated, w.units, (float*)w.scale);
}

size_t q8_gemm_workspace(int, int, int, int) { return 0; }

// The tile with the least estimated time.  A round is what 256 compute units take together; a chip that is partly full runs its workgroups up to 40 %
// faster, and every round pays for its pipeline's start and its epilogue.
Q8TilePlan q8_tile_plan(int M, int units, int K) {
  const struct { int wm, wn, rw, cw, kb; float ns4, ns2, ns1; } tiles[] = {
#define ROW(WM, WN, RW, CW, KB, NS4, NS2, NS1) {WM, WN, RW, CW, KB, NS4, NS2, NS1},
      Q8_TILES(ROW)
#undef ROW
  };
  constexpr int CUS = 256;
  const int KT = (K + 63) / 64;
  Q8TilePlan best{0, 1, 1, 1e30f};
  int i = -1;
  for (auto& t : tiles) {
    ++i;
    const int bm = 32 * t.rw * t.wm, un = t.cw * t.wn, mb = (M + bm - 1) / bm, nb = (units + un - 1) / un, kt = (KT + t.kb - 1) / t.kb * t.kb;
    const int64_t wgs = (int64_t)mb * nb, full = (wgs - 1) / CUS, last = wgs - CUS * full;
    const float ns = mb == 1 ? t.ns1 : mb < 4 ? t.ns2 : t.ns4, fixed = 3.f + bm * un * 32 * 1e-4f;
    const float us = kt * ns * 1e-3f * (full + 0.6f + 0.4f * last / CUS) + (full + 1) * fixed;
    if (us < best.us) best = Q8TilePlan{i, nb, mb, us};
  }
  return best;
}

void launch_q8_stream(const Q8View& w, const Q8GemmArgs& a, hipStream_t st);
void launch_q8_gemm(const Q8View& w, const Q8GemmArgs& a, hipStream_t st) {
  // few rows; or rows so far apart that a tile's would be past 32 bits
  if (a.M <= 64 || a.x_stride > 1 << 22) return launch_q8_stream(w, a, st);
  const Q8TilePlan p = q8_tile_plan(a.M, w.units, w.k);
  if (a.out_dtype == DLM_BF16) w.gated ? launch_q8_tile<true, bf16_t>(w, a, p, st) : launch_q8_tile<false, bf16_t>(w, a, p, st);
  else w.gated ? launch_q8_tile<true, float>(w, a, p, st) : launch_q8_tile<false, float>(w, a, p, st);
}
