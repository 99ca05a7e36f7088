// Writing K and V rows into the 8-bit cache and reading them back (layout, formats and scales: kv8.h).
//
// Write, per vector x: E = the smallest integer in [-60, 60] with max|x| <= M 2^E (M = 448 e4m3, 127 i8), code = x 2^-E rounded to the
// format (to even), saturated.  E follows from the bits of max|x|, so nothing is rounded but the code.  Read: code 2^E, exact in
// bf16 and fp32.  Both are bound by memory: every value is moved once, one workgroup a block of 32 positions of one head, whose
// image is put together (taken apart) in LDS, because V's codes lie transposed in it.
#include <type_traits>

#include "kv8.h"

namespace {

// 16 bytes of a row: 8 bf16 or 4 fp32
template <typename T> struct Piece;
template <> struct Piece<bf16_t> {
  static constexpr int N = 8;
  static __device__ inline void load(const bf16_t* p, float (&x)[N]) {
    const bf16x8 v = *(const bf16x8*)p;
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = (float)v[i];
  }
  static __device__ inline void store(bf16_t* p, const float (&x)[N]) {
    bf16x8 v;
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = (bf16_t)x[i];  // (exact: at most 8 significant bits)
    *(bf16x8*)p = v;
  }
};
template <> struct Piece<float> {
  static constexpr int N = 4;
  static __device__ inline void load(const float* p, float (&x)[N]) {
    const f32x4 v = *(const f32x4*)p;
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = v[i];
  }
  static __device__ inline void store(float* p, const float (&x)[N]) { *(f32x4*)p = f32x4{x[0], x[1], x[2], x[3]}; }
};

template <int N>
__device__ inline unsigned group_max(unsigned v) {  // over N neighbouring lanes (N = 4 .. 32, a power of two)
  auto mx = [](unsigned a, unsigned b) { return a > b ? a : b; };
  v = mx(v, rotate<0xB1>(v));                  // quad_perm [1,0,3,2]
  v = mx(v, rotate<0x4E>(v));                  // quad_perm [2,3,0,1]
  if (N > 4) v = mx(v, rotate<0x141>(v));      // mirrored within 8 lanes: the other quad
  if (N > 8) v = mx(v, rotate<0x140>(v));      // mirrored within 16: the other 8
  if (N > 16) {
    const auto x = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = mx(x[0], x[1]);
  }
  return v;
}

// scale byte of a vector whose largest magnitude has the bits `top`
template <int FMT>
__device__ inline unsigned scale_byte(unsigned top) {
  if (top >= 0x7F800000u) return KV8_NAN;
  // M = 1.75 2^8 (e4m3), 1.984375 2^6 (i8)
  const int E = (int)(top >> 23) - 127, e = E - (FMT == DLM_KV8_E4M3 ? 8 : 6) + ((top & 0x7FFFFFu) > (FMT == DLM_KV8_E4M3 ? 0x600000u : 0x7E0000u));
  return (unsigned)(min(max(e, -KV8_E_MAX), KV8_E_MAX) + 127);
}

// four codes in a word.  i8 is stored as code + 128
template <int FMT>
__device__ inline unsigned codes4(const float* x, float inv, bool bad) {
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = bad ? 0.f : __builtin_amdgcn_fmed3f(x[i] * inv, FMT == DLM_KV8_E4M3 ? -448.f : -127.f, FMT == DLM_KV8_E4M3 ? 448.f : 127.f);
  if (FMT == DLM_KV8_E4M3) {
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], lo, true);
  }
  // 2^23 + 2^22 + 128 added: one unit in the last place is 1, so the sum rounds y to an integer, halves to even, and its low byte is the code
  unsigned b[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) b[i] = __float_as_uint(y[i] + 12583040.f) & 0xFFu;
  return b[0] | b[1] << 8 | b[2] << 16 | b[3] << 24;
}

template <int FMT>
__device__ inline float value_of(unsigned code, unsigned scale) {
  if (scale == KV8_NAN) return __uint_as_float(0x7FC00000u);
  const float s = __uint_as_float(scale << 23);  // (0 for a position that was never written)
  if (FMT == DLM_KV8_E4M3) return __builtin_amdgcn_cvt_f32_fp8((int)code, 0) * s;
  return (float)((int)code - 128) * s;
}

struct Place {  // of a workgroup: its block of 32 positions, and which of them the span has
  int head, slot, block, lo, hi, row0;  // positions [lo, hi) of the block; row0: row of position 0 (may lie before the rows)
};
__device__ inline Place place_of(const Kv8Meta& m, int n_kv) {
  Place p;
  p.head = blockIdx.x % n_kv;
  const int i = blockIdx.x / n_kv, b = seq_of(m.block_off, m.n_seqs, i);
  const int start = m.start[b], end = start + m.row_off[b + 1] - m.row_off[b];
  p.block = (start >> 5) + i - m.block_off[b];
  p.slot = m.slot[b];
  p.lo = max(start - 32 * p.block, 0);
  p.hi = min(end - 32 * p.block, 32);
  p.row0 = m.row_off[b] - start + 32 * p.block;
  return p;
}

template <typename T, int HD, int FMT>
__global__ __launch_bounds__(256) void kv8_write_kernel(const T* __restrict__ k, const T* __restrict__ v, int64_t stride, Kv8View c, Kv8Meta m) {
  constexpr int N = Piece<T>::N, LANES = HD / N, ROWS = 256 / LANES < 32 ? 256 / LANES : 32, PASSES = 32 / ROWS;
  __shared__ __align__(16) unsigned char img[kv8_block_bytes(HD)];
  const Place w = place_of(m, c.n_kv);
  const int r = threadIdx.x / LANES, d = threadIdx.x % LANES * N;
  float x[2][PASSES][N];
#pragma unroll
  for (int t = 0; t < PASSES; ++t) {
    const int p = t * ROWS + r;
#pragma unroll
    for (int i = 0; i < N; ++i) x[0][t][i] = x[1][t][i] = 0.f;
    if (r < ROWS && p >= w.lo && p < w.hi) {
      const int64_t at = (int64_t)(w.row0 + p) * stride + w.head * HD + d;
      Piece<T>::load(k + at, x[0][t]);
      Piece<T>::load(v + at, x[1][t]);
    }
  }
#pragma unroll
  for (int t = 0; t < PASSES; ++t) {
    const int p = t * ROWS + r;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      unsigned top = 0;
#pragma unroll
      for (int i = 0; i < N; ++i) top = max(top, __float_as_uint(x[s][t][i]) & 0x7FFFFFFFu);
      const unsigned sb = scale_byte<FMT>(group_max<LANES>(top));
      if (r >= ROWS) continue;
      const float inv = __uint_as_float((254u - sb) << 23);
#pragma unroll
      for (int q = 0; q < N; q += 4) {
        const unsigned word = codes4<FMT>(&x[s][t][q], inv, sb == KV8_NAN);
        if (s == 0) *(unsigned*)&img[kv8_k_index(p, d + q, HD)] = word;
        else
#pragma unroll
          for (int i = 0; i < 4; ++i) img[kv8_v_index(p, d + q + i, HD)] = (unsigned char)(word >> 8 * i);
      }
      if (d == 0) img[kv8_scale_index(p, s, HD)] = (unsigned char)sb;
    }
  }
  __syncthreads();
  unsigned char* out = c.data + ((int64_t)w.slot * c.n_kv + w.head) * c.head_bytes + (int64_t)w.block * kv8_block_bytes(HD);
  if (w.lo == 0 && w.hi == 32) {
    for (int i = threadIdx.x; i < kv8_block_bytes(HD) / 16; i += 256) ((u32x4*)out)[i] = ((const u32x4*)img)[i];
    return;
  }
  // part of a block: the other positions' bytes stay as they are
  const unsigned here = (unsigned)((1ull << w.hi) - (1ull << w.lo));
  for (int i = threadIdx.x; i < kv8_block_bytes(HD) / 4; i += 256) {
    unsigned bits;  // which of the word's bytes
    if (i < 8 * HD) bits = here >> (i >> 2 & 31) & 1 ? 15u : 0u;                      // K: one position's
    else if (i < 16 * HD) bits = here >> ((i & 3) * 8 + (i >> 2 & 32) / 8) & 15u;     // V: four positions'
    else bits = here >> (i & 7) * 4 & 15u;
    const unsigned word = ((const unsigned*)img)[i];
    if (bits == 15u) ((unsigned*)out)[i] = word;
    else
      for (int j = 0; j < 4; ++j)
        if (bits >> j & 1) out[4 * i + j] = (unsigned char)(word >> 8 * j);
  }
}

template <typename T, int HD, int FMT>
__global__ __launch_bounds__(256) void kv8_read_kernel(T* __restrict__ k, T* __restrict__ v, int64_t stride, Kv8View c, Kv8Meta m) {
  constexpr int N = Piece<T>::N, LANES = HD / N, ROWS = 256 / LANES < 32 ? 256 / LANES : 32, PASSES = 32 / ROWS;
  __shared__ __align__(16) unsigned char img[kv8_block_bytes(HD)];
  const Place w = place_of(m, c.n_kv);
  const unsigned char* in = c.data + ((int64_t)w.slot * c.n_kv + w.head) * c.head_bytes + (int64_t)w.block * kv8_block_bytes(HD);
  for (int i = threadIdx.x; i < kv8_block_bytes(HD) / 16; i += 256) ((u32x4*)img)[i] = ((const u32x4*)in)[i];
  __syncthreads();
  const int r = threadIdx.x / LANES, d = threadIdx.x % LANES * N;
#pragma unroll
  for (int t = 0; t < PASSES; ++t) {
    const int p = t * ROWS + r;
    if (r >= ROWS || p < w.lo || p >= w.hi) continue;
    const int64_t at = (int64_t)(w.row0 + p) * stride + w.head * HD + d;
    float x[N];
    unsigned sb = img[kv8_scale_index(p, 0, HD)];
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = value_of<FMT>(img[kv8_k_index(p, d + i, HD)], sb);
    Piece<T>::store(k + at, x);
    sb = img[kv8_scale_index(p, 1, HD)];
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = value_of<FMT>(img[kv8_v_index(p, d + i, HD)], sb);
    Piece<T>::store(v + at, x);
  }
}

template <typename F>
void for_shape(int format, int hd, int dtype, F f) {
  auto with_hd = [&](auto hd_c) {
    auto with_fmt = [&](auto fmt_c) { dtype == DLM_BF16 ? f(bf16_t(), hd_c, fmt_c) : f(float(), hd_c, fmt_c); };
    format == DLM_KV8_E4M3 ? with_fmt(std::integral_constant<int, DLM_KV8_E4M3>()) : with_fmt(std::integral_constant<int, DLM_KV8_I8>());
  };
  hd == 128 ? with_hd(std::integral_constant<int, 128>()) : hd == 64 ? with_hd(std::integral_constant<int, 64>()) : with_hd(std::integral_constant<int, 32>());
}

}  // namespace

void launch_kv8_write(const Kv8View& c, int format, int hd, const void* k, const void* v, int64_t stride, int dtype, const Kv8Meta& m, hipStream_t st) {
  for_shape(format, hd, dtype, [&](auto t, auto hd_c, auto fmt_c) {
    typedef decltype(t) T;
    kv8_write_kernel<T, hd_c(), fmt_c()><<<m.block_off[m.n_seqs] * c.n_kv, 256, 0, st>>>((const T*)k, (const T*)v, stride, c, m);
  });
}
void launch_kv8_read(const Kv8View& c, int format, int hd, void* k, void* v, int64_t stride, int dtype, const Kv8Meta& m, hipStream_t st) {
  for_shape(format, hd, dtype, [&](auto t, auto hd_c, auto fmt_c) {
    typedef decltype(t) T;
    kv8_read_kernel<T, hd_c(), fmt_c()><<<m.block_off[m.n_seqs] * c.n_kv, 256, 0, st>>>((T*)k, (T*)v, stride, c, m);
  });
}
