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
// silu(g) u: the exponential and the reciprocal within a few units of fp32's last place
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

}  // namespace
