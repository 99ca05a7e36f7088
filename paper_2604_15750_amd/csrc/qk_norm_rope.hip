// Queries and keys as an attention reads them: RMSNorm of every head and the rotation by the row's position, in one pass.
//
// y = x rsqrt(mean(x^2) + eps) gain;  (y1, y2) -> (y1 cos a - y2 sin a, y2 cos a + y1 sin a), a = position theta^(-2i/hd), pairs
// (i, i + hd/2).  Bound by memory (each value read and written once).  A lane holds 16 bytes of a head's first half and the 16 bytes
// of the second half that they are paired with, so the rotation exchanges nothing and the norm's sum goes over 2 to 16 lanes; a
// wavefront has one row's angles and up to ITERS x 64 / LANES of its heads: the angles (a sine and a cosine in 64-bit turns, by far the
// most instructions) are computed while its loads are on their way.  2048 rows x 32 heads of 128 bf16 8.6 us (6.8 at the rate of a large
// copy), fp32 600 rows x 64 heads 8.9 (8.0); 8 rows 3.8: a launch.
#include "kv8.h"

namespace {

constexpr int ITERS = 4;  // heads a lane works on, all their loads in flight together

template <typename T> struct Half16;
template <> struct Half16<bf16_t> {
  typedef bf16x8 vec;
  static constexpr int N = 8;
};
template <> struct Half16<float> {
  typedef f32x4 vec;
  static constexpr int N = 4;
};

template <int N>
__device__ inline float group_sum(float v) {  // over N neighbouring lanes (N = 2 .. 16, a power of two)
  auto add = [](float a, unsigned b) { return a + __uint_as_float(b); };
  v = add(v, rotate<0xB1>(__float_as_uint(v)));                // quad_perm [1,0,3,2]
  if (N > 2) v = add(v, rotate<0x4E>(__float_as_uint(v)));     // quad_perm [2,3,0,1]
  if (N > 4) v = add(v, rotate<0x141>(__float_as_uint(v)));    // mirrored within 8 lanes: the other quad
  if (N > 8) v = add(v, rotate<0x140>(__float_as_uint(v)));    // mirrored within 16: the other 8
  return v;
}

// log2_theta_hd = 2 log2(theta) / hd
template <typename T, int HD>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(const T* x, int64_t x_stride, const int32_t* __restrict__ positions, T* out, int64_t out_stride, int rows,
                                                           int n_q, int heads, float eps, double log2_theta_hd, const T* __restrict__ q_gain,
                                                           const T* __restrict__ k_gain) {
  typedef typename Half16<T>::vec vec;
  constexpr int N = Half16<T>::N, HALF = HD / 2, LANES = HALF / N, HEADS = 64 / LANES;
  __shared__ __align__(16) float cs[4][2][HALF];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, d = lane % LANES * N;
  const int row = blockIdx.x * 4 + wave, h0 = blockIdx.y * (ITERS * HEADS) + lane / LANES;
  const bool there = row < rows;
  const T* from = x + (int64_t)(there ? row : 0) * x_stride + d;
  vec a[ITERS], b[ITERS];
#pragma unroll
  for (int t = 0; t < ITERS; ++t) {
    const int h = h0 + t * HEADS;
    if (there && h < heads) {
      a[t] = *(const vec*)(from + (int64_t)h * HD);
      b[t] = *(const vec*)(from + (int64_t)h * HD + HALF);
    }
  }
  if (there && lane < HALF) {
    // the angle in turns, in 64 bits; what a float leaves of its fraction is put back by the derivative
    constexpr double INV_2PI = 0.15915494309189533577, PI = 3.14159265358979323846;
    const double t = (double)positions[row] * (exp2(-log2_theta_hd * lane) * INV_2PI), u = 2.0 * (t - rint(t));
    const float r = (float)u, rest = (float)((u - (double)r) * PI);
    float s, c;
    sincospif(r, &s, &c);
    cs[wave][0][lane] = c - s * rest;
    cs[wave][1][lane] = s + c * rest;
  }
  __syncthreads();
  if (!there) return;
  float co[N], si[N];
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    const f32x4 c4 = *(const f32x4*)&cs[wave][0][d + i], s4 = *(const f32x4*)&cs[wave][1][d + i];
#pragma unroll
    for (int j = 0; j < 4; ++j) { co[i + j] = c4[j]; si[i + j] = s4[j]; }
  }
  T* to = out + (int64_t)row * out_stride + d;
#pragma unroll
  for (int t = 0; t < ITERS; ++t) {
    const int h = h0 + t * HEADS;
    float y1[N], y2[N], ss = 0.f;
    if (h < heads) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        y1[i] = to_f32(a[t][i]);
        y2[i] = to_f32(b[t][i]);
        ss += y1[i] * y1[i] + y2[i] * y2[i];
      }
    }
    ss = group_sum<LANES>(ss);
    if (h >= heads) continue;
    const T* gain = h < n_q ? q_gain : k_gain;
    if (gain) {
      const float rs = rsqrtf(ss * (1.f / HD) + eps);
      const vec g1 = *(const vec*)(gain + d), g2 = *(const vec*)(gain + d + HALF);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        y1[i] *= rs * to_f32(g1[i]);
        y2[i] *= rs * to_f32(g2[i]);
      }
    }
    vec o1, o2;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      o1[i] = (T)(y1[i] * co[i] - y2[i] * si[i]);
      o2[i] = (T)(y2[i] * co[i] + y1[i] * si[i]);
    }
    *(vec*)(to + (int64_t)h * HD) = o1;
    *(vec*)(to + (int64_t)h * HD + HALF) = o2;
  }
}

template <typename T, int HD>
void launch(const void* x, int64_t x_stride, int rows, int n_q, int n_kv, const void* q_gain, const void* k_gain, float eps, float theta,
            const int32_t* positions, void* out, int64_t out_stride, hipStream_t st) {
  constexpr int HEADS = 64 / (HD / 2 / Half16<T>::N);
  const int heads = n_q + n_kv;
  qk_norm_rope_kernel<T, HD><<<dim3((rows + 3) / 4, (heads + ITERS * HEADS - 1) / (ITERS * HEADS)), 256, 0, st>>>(
      (const T*)x, x_stride, positions, (T*)out, out_stride, rows, n_q, heads, eps, 2.0 * log2((double)theta) / HD, (const T*)q_gain, (const T*)k_gain);
}

}  // namespace

void launch_qk_norm_rope(const void* x, int64_t x_stride, int rows, int n_q, int n_kv, int hd, int dtype, const void* q_gain, const void* k_gain, float eps,
                         float theta, const int32_t* positions, void* out, int64_t out_stride, hipStream_t st) {
  auto go = [&](auto f) { f(x, x_stride, rows, n_q, n_kv, q_gain, k_gain, eps, theta, positions, out, out_stride, st); };
  if (dtype == DLM_BF16) hd == 128 ? go(launch<bf16_t, 128>) : hd == 64 ? go(launch<bf16_t, 64>) : go(launch<bf16_t, 32>);
  else hd == 128 ? go(launch<float, 128>) : hd == 64 ? go(launch<float, 64>) : go(launch<float, 32>);
}
