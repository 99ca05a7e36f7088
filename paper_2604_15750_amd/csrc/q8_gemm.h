// What the kernels of the 8-bit integer product share: loads of their operands, and the epilogue.
#pragma once
#include <type_traits>

#include "q8.h"

namespace {

template <typename TO> struct Out4;
template <> struct Out4<bf16_t> { typedef bf16x4 vec; };
template <> struct Out4<float> { typedef f32x4 vec; };

// y = q-sum x scale of the token x scales of the channels, in this order (each rounded once: 2^-24 of the value, besides the conversion's)
__device__ inline f32x4 scaled(i32x4 sum, float token, f32x4 channel) {
  f32x4 y;
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = (float)sum[i] * token * channel[i];
  return y;
}
// silu(g) u, (13 + 6 |g|) 2^-24 of itself off: the exponential's argument is rounded (2 |g| 2^-24 of the result, and 3 |g| from g's own error), the exponential
// and the reciprocal are within a few units of fp32's last place; below g = -87.3 the reciprocal is below 2^-126 and may be taken as zero.  A division instead (2 of the
// 13 units) takes 41.5 us for 2048 x 24576 x 256 in fp32, and 47.9 with an exponential to the last place; 37.7 so
__device__ inline f32x4 gated_unit(f32x4 g, f32x4 u) {
  f32x4 y;
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = g[i] * __builtin_amdgcn_rcpf(1.f + __expf(-g[i])) * u[i];
  return y;
}
// outputs n .. n + 3 of a row of `outputs`: what is past its end is left as it is
template <typename TO>
__device__ inline void store4(TO* row, int n, int outputs, f32x4 y) {
  if (n + 4 <= outputs) {
    typename Out4<TO>::vec v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (TO)y[i];
    *(typename Out4<TO>::vec*)(row + n) = v;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (n + i < outputs) row[n + i] = (TO)y[i];
  }
}

// outputs n .. n + 7
template <typename TO>
__device__ inline void store8(TO* row, int n, int outputs, f32x4 lo, f32x4 hi) {
  if constexpr (sizeof(TO) == 2) {
    if (n + 8 <= outputs) {
      bf16x8 v;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[i] = (bf16_t)lo[i];
        v[4 + i] = (bf16_t)hi[i];
      }
      *(bf16x8*)(row + n) = v;
      return;
    }
  }
  store4(row, n, outputs, lo);
  store4(row, n + 4, outputs, hi);
}

// What a product writes: bit 0: fp32, not bf16; bit 1: gated.  f(gated, out) with both in its arguments' types (the branch is uniform, behind the product's loop)
inline int out_form(const Q8View& w, const Q8GemmArgs& a) { return (a.out_dtype == DLM_F32) | (int)w.gated << 1; }
template <typename F>
__device__ inline void with_form(int form, void* out, F f) {
  if (form == 0) f(std::false_type{}, (bf16_t*)out);
  else if (form == 1) f(std::false_type{}, (float*)out);
  else if (form == 2) f(std::true_type{}, (bf16_t*)out);
  else f(std::true_type{}, (float*)out);
}

// The outputs of 4 packed rows of each sub of a unit and of a token, as 16x16 products leave them to a lane (g: lane / 16): neighbours
template <bool GATED, typename TO>
__device__ inline void finish8(i32x4 first, i32x4 second, float token, const float* wscale, TO* row, int u, int g, int outputs, bool there) {
  const f32x4 y0 = scaled(first, token, *(const f32x4*)(wscale + u * 32 + 4 * g)), y1 = scaled(second, token, *(const f32x4*)(wscale + u * 32 + 16 + 4 * g));
  if (!there) return;
  if constexpr (GATED) store4(row, 16 * u + 4 * g, outputs, gated_unit(y0, y1));
  else store8(row, 32 * u + 8 * g, outputs, y0, y1);
}

// 1 KiB, 16 bytes a lane, from a buffer to LDS (dst: the wavefront's)
__device__ inline void copy_to_lds(__amdgpu_buffer_rsrc_t from, unsigned char* dst, int lane_at, int at) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)dst, 16, lane_at, at, 0, 0);
}

// Workgroup id -> tile and share of K: ids congruent mod 8 share an XCD, which gets one contiguous eighth of the tiles; in groups of 8 row blocks, row blocks
// fastest, so that the tiles an XCD works on at a time share both operands in its L2
struct Q8At {
  int split, rb, cb;  // split < 0: none
};
__device__ inline Q8At tile_of(int id, int nblocks, int mblocks, int splits) {
  const int tiles = nblocks * mblocks, lin = (id & 7) * ((tiles * splits + 7) >> 3) + (id >> 3);
  if (lin >= tiles * splits) return Q8At{-1, 0, 0};
  const int split = lin / tiles, tile = lin - split * tiles;
  const int group = tile / (8 * nblocks), rows_in = min(8, mblocks - 8 * group), at = tile - group * 8 * nblocks;
  const int cb = at / rows_in;
  return Q8At{split, 8 * group + at - cb * rows_in, cb};
}

// The end of a tile: WN units from u0 on by WM x 32 rows from m0 on of a wavefront, acc[2 unit + sub][2 (rows / 32) + half] as 16x16 products leave them.
// A launch that splits K leaves its sums in the workspace, [split][unit][32 rows][sub + 2 (row / 16)][group][row % 16], where a second launch adds them up
// and finishes; any other finishes straight from the accumulators.
template <int WN, int WM>
__device__ inline __attribute__((always_inline)) void finish_tile(const i32x4 (&acc)[2 * WN][2 * WM], int u0, int m0, int lane, int split, int splits, int M, int units, const float* wscale,
                                                                  const float* x_scale, void* out, int64_t out_stride, int outputs, int form, i32x4* parts) {
  const int g = lane >> 4;
  if (splits > 1) {
    const int blocks = (M + 31) >> 5;
#pragma unroll
    for (int j = 0; j < WN; ++j)
#pragma unroll
      for (int i = 0; i < WM; ++i) {
        const int u = u0 + j, block = (m0 >> 5) + i;
        if (u >= units || block >= blocks) continue;
        i32x4* to = parts + ((int64_t)split * units + u) * blocks * 256 + block * 256 + lane;
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
          for (int s = 0; s < 2; ++s) to[(s + 2 * p) * 64] = acc[2 * j + s][2 * i + p];
      }
    return;
  }
  with_form(form, out, [&](auto gated, auto* to) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 2 * WM; ++i) {
      const int m = m0 + 16 * i + (lane & 15);
      const float xs = x_scale[min(m, M - 1)];
#pragma unroll
      for (int j = 0; j < WN; ++j)
        if (u0 + j < units) finish8<decltype(gated)::value>(acc[2 * j][i], acc[2 * j + 1][i], xs, wscale, to + (int64_t)m * out_stride, u0 + j, g, outputs, m < M);
    }
  });
}

}  // namespace
