// Rows in 8-bit integers, alone or behind the residual's addition and a root-mean-square norm: one pass over the row.
//
//   t = x                                    s = max|t| / 127                             (dlm_q8_rows)
//   h = residual + x, t = h gain             s = max|t| rsqrt(mean(h^2) + eps) / 127      (dlm_add_norm_q8)
//   q = 127 t / max|t| rounded to the nearest integer, ties to even
//
// The norm multiplies every t of a row by the same number, which cancels in q: codes depend on no sum and on no square root, and t is a product of two
// numbers as they are stored, rounded to fp32 once (exact for bf16).  So q can be what the formula says to the last bit: an fp32 quotient
// (off by at most 127 x 2^-23) decides all but those next to a border k + 1/2, and for these the sign of 127 t - (k + 1/2) max|t| does, which 64
// bits hold (31 and 32 bits of product before one rounding).  A border is hit exactly whenever t = +-max|t| / 2.
// Bound by memory where there are many rows: each value is read once and kept in registers until the row's maximum and sum are known.  2048 x 3584 in bf16 with the residual takes 9.7 us
// (5.3 TB/s read and written, what a copy reaches), 1500 x 12288 bf16 rows alone 11.3 (4.9), 333 x 5003 in fp32 6.6 (3.3: 333 workgroups are not two for every compute unit).
// 8 rows take the launch and two trips to memory: 3.5 us.
#include "q8.h"

namespace {

template <typename T> struct V8;  // eight values of a row
template <> struct V8<bf16_t> {
  bf16x8 v;
  __device__ inline void load(const bf16_t* p) { v = *(const bf16x8*)p; }
  __device__ inline float get(int i) const { return (float)v[i]; }
  __device__ inline void set(int i, float x) { v[i] = (bf16_t)x; }
  __device__ inline void store(bf16_t* p) const { *(bf16x8*)p = v; }
};
template <> struct V8<float> {
  f32x4 v[2];
  __device__ inline void load(const float* p) { v[0] = *(const f32x4*)p; v[1] = *(const f32x4*)(p + 4); }
  __device__ inline float get(int i) const { return v[i >> 2][i & 3]; }
  __device__ inline void set(int i, float x) { v[i >> 2][i & 3] = x; }
  __device__ inline void store(float* p) const { *(f32x4*)p = v[0]; *(f32x4*)(p + 4) = v[1]; }
};
// The code of t where the row's largest magnitude is top, in the low byte: inv is 127 / top rounded up to fp32.  Added to 1.5 2^23 a product is rounded to an
// integer; what that leaves of t inv (at most 127 x 2^-23 of which is inv's rounding) says whether the quotient may be on the other side of a border
constexpr float SHIFT = 12582912.f, NEAR = 0.49998f;
__device__ inline unsigned rounded(float t, float inv, float* left) {
  const float f = fmaf(t, inv, SHIFT);
  *left = fmaf(t, inv, SHIFT - f);
  return __float_as_uint(f);
}
__device__ inline unsigned exact_code(unsigned f, float left, float t, float top) {
  const float k = __uint_as_float(f) - SHIFT;
  const double border = (double)k + (left > 0.f ? 0.5 : -0.5), e = fma(-border, (double)top, 127.0 * (double)t);
  const int below = (int)k - (left > 0.f ? 0 : 1);
  return (unsigned)(e > 0.0 ? below + 1 : e < 0.0 ? below : below + (below & 1));
}
// ... of eight, with one check for all.  t = +-top / 2, which one in 600 bf16 values is, is the border 63.5 itself: it belongs to 64, where a product that is
// no smaller than the quotient takes it.  One in 25000 others is looked at in 64 bits.
__device__ inline uint64_t codes8(const float (&t)[8], float top, float inv) {
  unsigned y[8];
  float left[8], most = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    y[i] = rounded(t[i], inv, &left[i]);
    most = fmaxf(most, fabsf(left[i]));
  }
  if (most > NEAR) {
    most = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) most = fmaxf(most, fabsf(t[i]) == 0.5f * top ? 0.f : fabsf(left[i]));
    if (most > NEAR)
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (fabsf(left[i]) > NEAR) y[i] = exact_code(y[i], left[i], t[i], top);
  }
  unsigned w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
    w[i] = __builtin_amdgcn_perm(y[4 * i + 1], y[4 * i], 0x0c0c0400u) | __builtin_amdgcn_perm(y[4 * i + 3], y[4 * i + 2], 0x04000c0cu);
  return (uint64_t)w[1] << 32 | w[0];
}

// T threads a row; a thread keeps ITERS times eight values, T x 8 of the row apart.  LOOP: rows of any length, read (or, of a sum, read back from h)
// a second time.
template <typename TX, typename TH, bool NORM, bool RES, int T, int ITERS, bool LOOP>
__global__ __launch_bounds__(T < 256 ? 256 : T) void q8_rows_kernel(const TX* x, int64_t x_stride, const TH* residual, int64_t r_stride, TH* h_out, int64_t h_stride,
                                                                    const TX* __restrict__ gain, float eps, int8_t* __restrict__ codes, int64_t codes_stride,
                                                                    float* __restrict__ scale, int rows, int width) {
  constexpr int TPB = T < 256 ? 256 : T, STEP = T * 8;
  const int row = blockIdx.x * (TPB / T) + threadIdx.x / T, d0 = threadIdx.x % T * 8;
  if (T == 64 && row >= rows) return;  // (a wavefront has one row, and meets no other)
  const TX* px = x + row * x_stride;
  const TH* pr = RES ? residual + row * r_stride : nullptr;
  TH* ph = RES ? h_out + row * h_stride : nullptr;
  int8_t* pc = codes + row * codes_stride;

  // The last width % 8 values of a row are a thread's own, one each, so that eights have no bounds; their loads go out first
  const int whole = width & ~7, e = whole + (int)(threadIdx.x % T);
  const bool odd = e < width;  // (T > 7)
  TX ox, og;
  TH orr;
  if (odd) {
    ox = px[e];
    if (RES) orr = pr[e];
    if (NORM) og = gain[e];
  }
  float t[ITERS][8], ot = 0.f;
  unsigned top = 0;
  float ss = 0.f;
  auto take = [&](int d, float (&v)[8], bool first) __attribute__((always_inline)) {  // the t's of d .. d + 7
    if (RES && !first) {
      V8<TH> h;
      h.load(ph + d);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = h.get(i);
    } else {
      V8<TX> a;
      a.load(px + d);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = a.get(i);
      if (RES) {
        V8<TH> h;
        h.load(pr + d);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          h.set(i, h.get(i) + v[i]);
          v[i] = h.get(i);
        }
        h.store(ph + d);
      }
    }
    if (NORM) {
      V8<TX> g;
      g.load(gain + d);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (first) ss += v[i] * v[i];
        v[i] *= g.get(i);
      }
    }
    if (first)
#pragma unroll
      for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[i]) & 0x7FFFFFFFu);  // (a NaN is above infinity here)
  };
  if (LOOP) {
    for (int d = d0; d < whole; d += STEP) take(d, t[0], true);
  } else {
#pragma unroll
    for (int j = 0; j < ITERS; ++j)
      if (d0 + j * STEP < whole) take(d0 + j * STEP, t[j], true);
  }
  if (odd) {
    ot = (float)ox;
    if (RES) {
      const TH h = (TH)((float)orr + ot);
      ph[e] = h;
      ot = (float)h;
    }
    if (NORM) {
      ss += ot * ot;
      ot *= (float)og;
    }
    top = max(top, __float_as_uint(ot) & 0x7FFFFFFFu);
  }
  struct BitsUMax { __device__ unsigned operator()(unsigned a, unsigned b) const { return max(a, b); } };
  top = butterfly(top, BitsUMax());
  if (NORM) ss = wave_sum(ss);
  if (T > 64) {
    __shared__ unsigned s_top[T / 64];
    __shared__ float s_ss[T / 64];
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) {
      s_top[wave] = top;
      s_ss[wave] = ss;
    }
    __syncthreads();
    top = 0;
    ss = 0.f;
#pragma unroll
    for (int i = 0; i < T / 64; ++i) {
      top = max(top, s_top[i]);
      if (NORM) ss += s_ss[i];
    }
  }
  const float a = __uint_as_float(top);
  const bool bad = top >= 0x7F800000u || (NORM && !(ss < __builtin_inff()));
  if (threadIdx.x % T == 0) {
    float y = a, up = 1.f;
    if (NORM && a > 0.f) {
      const float r = rsqrtf(ss / (float)width + eps);
      y = a * r;
      if (y == __builtin_inff()) {  // (the row's largest value may be past fp32's range where its 127th is not)
        y = a * 0x1p-16f * r;
        up = 0x1p16f;
      }
    }
    const float s = y / 127.f * up;
    scale[row] = bad ? __builtin_nanf("") : s;
  }
  // a row of zeros: every quotient 0 x 0; a tiny maximum: 127 / max would be past fp32's range, so the row is scaled by a power of two first
  const bool tiny = a < 0x1p-100f;
  const float big = tiny ? a * 0x1p64f : a;
  float inv = 0.f;
  if (!bad && big != 0.f) {
    inv = 127.f / big;
    if (fmaf(inv, big, -127.f) < 0.f) inv = __uint_as_float(__float_as_uint(inv) + 1);
  }
  auto put = [&](int d, float (&v)[8]) __attribute__((always_inline)) {
    if (tiny)  // (the whole row)
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] *= 0x1p64f;
    const uint64_t w = codes8(v, big, inv);
    *(uint64_t*)(pc + d) = bad || big == 0.f ? 0 : w;
  };
  if (LOOP) {
    for (int d = d0; d < whole; d += STEP) {
      take(d, t[0], false);
      put(d, t[0]);
    }
  } else {
#pragma unroll
    for (int j = 0; j < ITERS; ++j)
      if (d0 + j * STEP < whole) put(d0 + j * STEP, t[j]);
  }
  if (odd) {
    const float v = tiny ? ot * 0x1p64f : ot;
    float left;
    unsigned f = rounded(v, inv, &left);
    if (fabsf(left) > NEAR) f = exact_code(f, left, v, big);
    pc[e] = (int8_t)(bad || big == 0.f ? 0 : f);
  }
}

template <typename TX, typename TH, bool NORM, bool RES>
void launch(const Q8RowsArgs& a, hipStream_t st) {
  auto go = [&](auto kernel, int threads) {
    const int per = threads < 256 ? 256 / threads : 1;
    kernel<<<(a.rows + per - 1) / per, threads * per, 0, st>>>((const TX*)a.x, a.x_stride, (const TH*)a.residual, a.r_stride, (TH*)a.h, a.h_stride,
                                                               (const TX*)a.gain, a.eps, a.codes, a.codes_stride, a.scale, a.rows, a.width);
  };
#define GO(T, ITERS, LOOP) go(q8_rows_kernel<TX, TH, NORM, RES, T, ITERS, LOOP>, T)
  if (a.width <= 512) GO(64, 1, false);
  else if (a.width <= 1024) GO(64, 2, false);
  else if (a.width <= 2048) GO(256, 1, false);
  else if (a.width <= 4096) GO(256, 2, false);
  else if (a.width <= 8192) GO(512, 2, false);
  else if (a.width <= 16384) GO(1024, 2, false);
  else if (a.width <= 32768) GO(1024, 4, false);
  else GO(1024, 1, true);
#undef GO
}

}  // namespace

void launch_q8_rows(const Q8RowsArgs& a, hipStream_t st) {
  if (a.dtype == DLM_BF16) {
    if (!a.gain) launch<bf16_t, bf16_t, false, false>(a, st);
    else if (!a.residual) launch<bf16_t, bf16_t, true, false>(a, st);
    else if (a.h_dtype == DLM_BF16) launch<bf16_t, bf16_t, true, true>(a, st);
    else launch<bf16_t, float, true, true>(a, st);
  } else {
    if (!a.gain) launch<float, float, false, false>(a, st);
    else if (!a.residual) launch<float, float, true, false>(a, st);
    else launch<float, float, true, true>(a, st);
  }
}
