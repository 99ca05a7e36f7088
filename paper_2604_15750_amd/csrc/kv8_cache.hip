// Writing K and V rows into the 8-bit cache and reading them back (layout, formats and scales: kv8.h).
//
// Write, per vector x: E = the smallest integer in [-60, 60] with max|x| <= M 2^E (M = 448 e4m3, 127 i8), code = x 2^-E rounded to the
// format (to even), saturated.  E follows from the bits of max|x|, so nothing is rounded but the code.  Read: code 2^E, exact in
// bf16 and fp32.  Both are bound by memory: every value is moved once, one workgroup a block of 32 positions of one head, whose
// image is put together (taken apart) in LDS, because V's codes lie transposed in it.  The heads of a block's rows are neighbours in the
// grid, so what the chip touches at a time is whole rows.  16384 rows (TB/s moved, written / read; a large copy reaches 4.9): 32 heads of
// 128 bf16 5.4 / 5.2, fp32 5.8 / 4.8; 16 of 64 4.4 / 4.2; 32 of 32 3.5 / 3.3 (a head's 64 bytes of a row are half a line).  1280 rows x 32
// heads of 128 9.0 / 8.5 us (floor 6.4), 8 rows 4.6 / 2.8 us: a launch and its trips to memory.
#include <type_traits>

#include "kv8.h"

namespace {

__device__ inline void store8(bf16_t* p, const float (&x)[8]) {
  bf16x8 v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (bf16_t)x[i];  // (exact: at most 8 significant bits)
  *(bf16x8*)p = v;
}
__device__ inline void store8(float* p, const float (&x)[8]) {
  *(f32x4*)p = f32x4{x[0], x[1], x[2], x[3]};
  *(f32x4*)(p + 4) = f32x4{x[4], x[5], x[6], x[7]};
}

template <int N>
__device__ inline unsigned group_max(unsigned v) {  // over N neighbouring lanes (4, 8 or 16)
  auto mx = [](unsigned a, unsigned b) { return a > b ? a : b; };
  v = mx(v, rotate<0xB1>(v));              // quad_perm [1,0,3,2]
  v = mx(v, rotate<0x4E>(v));              // quad_perm [2,3,0,1]
  if (N > 4) v = mx(v, rotate<0x141>(v));  // mirrored within 8 lanes: the other quad
  if (N > 8) v = mx(v, rotate<0x140>(v));  // mirrored within 16: the other 8
  return v;
}

// V lies transposed in a block: four neighbouring positions share a word.  A wavefront has four positions 16 lanes apart; a lane's two words
// (its position's codes of 8 dims) become dims 2i and 2i + 1 of all four positions, i its row of 16 lanes, and back.  (Byte by byte
// through LDS: 3904 blocks of 32 x 128 bf16 written in 26.4 us, 22.8 to
// 25 now; read in 23.6, 19 now.)
struct Two { unsigned a, b; };
__device__ inline Two swap16(Two v) { const auto r = __builtin_amdgcn_permlane16_swap(v.a, v.b, false, false); return Two{r[0], r[1]}; }
__device__ inline Two swap32(Two v) { const auto r = __builtin_amdgcn_permlane32_swap(v.a, v.b, false, false); return Two{r[0], r[1]}; }
__device__ inline Two by_dims(Two v) {
  v = swap16(swap32(v));
  v = swap16(Two{__builtin_amdgcn_perm(v.b, v.a, 0x05010400u), __builtin_amdgcn_perm(v.b, v.a, 0x07030602u)});
  return Two{__builtin_amdgcn_perm(v.b, v.a, 0x05040100u), __builtin_amdgcn_perm(v.b, v.a, 0x07060302u)};
}
__device__ inline Two by_positions(Two v) {
  v = swap16(Two{__builtin_amdgcn_perm(v.b, v.a, 0x05040100u), __builtin_amdgcn_perm(v.b, v.a, 0x07060302u)});
  return swap32(swap16(Two{__builtin_amdgcn_perm(v.b, v.a, 0x06040200u), __builtin_amdgcn_perm(v.b, v.a, 0x07050301u)}));
}

// a block's image in LDS: its 16-byte units in an order that spreads what a wavefront accesses together over the banks
__device__ inline int unit_at(int u) { return u ^ ((u >> 3 ^ u >> 5) & 7); }
__device__ inline int byte_at(int i) { return unit_at(i >> 4) * 16 + (i & 15); }

// scale byte of a vector whose largest magnitude has the bits `top`
template <int FMT>
__device__ inline unsigned scale_byte(unsigned top) {
  if (top >= 0x7F800000u) return KV8_NAN;
  // M = 1.75 2^8 (e4m3), 1.984375 2^6 (i8)
  const int E = (int)(top >> 23) - 127, e = E - (FMT == DLM_KV8_E4M3 ? 8 : 6) + ((top & 0x7FFFFFu) > (FMT == DLM_KV8_E4M3 ? 0x600000u : 0x7E0000u));
  return (unsigned)(min(max(e, -KV8_E_MAX), KV8_E_MAX) + 127);
}

// the codes of eight values, four in a word; i8 is stored as code + 128
template <int FMT, typename E>
__device__ inline Two codes8(const E& x, unsigned scale) {
  constexpr float M = FMT == DLM_KV8_E4M3 ? 448.f : 127.f;
  const float inv = __uint_as_float((254u - scale) << 23);
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = x[i] * inv;
  if (__builtin_amdgcn_ballot_w64(scale == 127u + KV8_E_MAX)) {  // (only there a value can be beyond the largest code)
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = __builtin_amdgcn_fmed3f(y[i], -M, M);
  }
  unsigned w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (FMT == DLM_KV8_E4M3) {
      w[i] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i], y[4 * i + 1], 0, false);
      w[i] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i + 2], y[4 * i + 3], (int)w[i], true);
    } else {
      // 2^23 + 2^22 + 128 added: one unit in the last place is 1, so the sum rounds y to an integer, halves to even, and its low byte is the code
      unsigned b[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) b[j] = __float_as_uint(y[4 * i + j] + 12583040.f);
      w[i] = __builtin_amdgcn_perm(b[1], b[0], 0x0C0C0400u) | __builtin_amdgcn_perm(b[3], b[2], 0x04000C0Cu);
    }
    if (scale == KV8_NAN) w[i] = FMT == DLM_KV8_E4M3 ? 0u : 0x80808080u;
  }
  return Two{w[0], w[1]};
}

template <int FMT>
__device__ inline void values8(Two w, unsigned scale, float (&x)[8]) {
  const float s = scale == KV8_NAN ? __uint_as_float(0x7FC00000u) : __uint_as_float(scale << 23);  // (0 for a position that was never written)
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const unsigned v = i ? w.b : w.a;
    if (FMT == DLM_KV8_E4M3) {
      const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)v, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)v, true);
      x[4 * i] = lo[0] * s; x[4 * i + 1] = lo[1] * s; x[4 * i + 2] = hi[0] * s; x[4 * i + 3] = hi[1] * s;
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) x[4 * i + j] = ((float)(v >> 8 * j & 0xFFu) - 128.f) * s;
    }
  }
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

// (heads of 32 with 256 threads, half of them idle: 16384 rows x 32 heads fp32 read in 49.6 us, 41.8 now, bf16 written in 30.5, 29.3 now)
// A thread has 8 dims of a position, 16 lanes the dims of one to four positions 4 apart, whose neighbours are in the other rows of 16 lanes
template <int HD>
struct Lanes {
  static constexpr int N = HD / 8, THREADS = 32 * N < 256 ? 32 * N : 256, ROWS = THREADS / N, PASSES = 32 / ROWS;  // ROWS: positions of a pass
  int p, d;
  __device__ inline Lanes() {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    p = (wave * (16 / N) + (lane & 15) / N) * 4 + (lane >> 4);
    d = lane % N * 8;
  }
};

template <typename T, int HD, int FMT>
__global__ __launch_bounds__(Lanes<HD>::THREADS) void kv8_write_kernel(const T* __restrict__ k, const T* __restrict__ v, int64_t stride, Kv8View c, Kv8Meta m) {
  typedef Lanes<HD> L;
  __shared__ __align__(16) unsigned char img[kv8_block_bytes(HD)];
  const Place w = place_of(m, c.n_kv);
  const L t;
  Eight<T> x[2][L::PASSES];
#pragma unroll
  for (int n = 0; n < L::PASSES; ++n) {
    const int p = n * L::ROWS + t.p;
    if (p >= w.lo && p < w.hi) {
      const int64_t at = (int64_t)(w.row0 + p) * stride + w.head * HD + t.d;
      x[0][n].load(k + at);
      x[1][n].load(v + at);
    }
  }
#pragma unroll
  for (int n = 0; n < L::PASSES; ++n) {
    const int p = n * L::ROWS + t.p;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const unsigned sb = scale_byte<FMT>(group_max<L::N>(x[s][n].top()));
      const Two codes = codes8<FMT>(x[s][n], sb);
      if (s == 0) {
        *(u32x2*)&img[byte_at(kv8_k_index(p, t.d, HD))] = u32x2{codes.a, codes.b};
      } else {
        const Two dims = by_dims(codes);
        const int d = t.d + 2 * (p & 3);
        *(unsigned*)&img[byte_at(kv8_v_index(p & ~3, d, HD))] = dims.a;
        *(unsigned*)&img[byte_at(kv8_v_index(p & ~3, d + 1, HD))] = dims.b;
      }
      if (t.d == 0) img[kv8_scale_index(p, s, HD)] = (unsigned char)sb;
    }
  }
  __syncthreads();
  unsigned char* out = c.data + ((int64_t)w.slot * c.n_kv + w.head) * c.head_bytes + (int64_t)w.block * kv8_block_bytes(HD);
  if (w.lo == 0 && w.hi == 32) {
#pragma unroll
    for (int i = threadIdx.x; i < 4 * HD; i += L::THREADS) ((u32x4*)out)[i] = ((const u32x4*)img)[unit_at(i)];
    if (threadIdx.x < 4) ((u32x4*)out)[4 * HD + threadIdx.x] = ((const u32x4*)img)[4 * HD + threadIdx.x];
    return;
  }
  // part of a block: the other positions' bytes stay as they are
  const unsigned here = (unsigned)((1ull << w.hi) - (1ull << w.lo));
  auto put = [&](int i, unsigned word, unsigned bits) {  // bits: which of word i's bytes
    if (bits == 15u) ((unsigned*)out)[i] = word;
    else
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (bits >> j & 1) out[4 * i + j] = (unsigned char)(word >> 8 * j);
  };
#pragma unroll
  for (int i = threadIdx.x; i < 8 * HD; i += L::THREADS)  // K: a word is one position's
    if (here >> (i >> 2 & 31) & 1) ((unsigned*)out)[i] = *(const unsigned*)&img[byte_at(4 * i)];
#pragma unroll
  for (int i = 8 * HD + threadIdx.x; i < 16 * HD; i += L::THREADS)  // V: four positions'
    put(i, *(const unsigned*)&img[byte_at(4 * i)], here >> ((i & 3) * 8 + (i >> 2 & 32) / 8) & 15u);
  if (threadIdx.x < 16) put(16 * HD + threadIdx.x, ((const unsigned*)img)[16 * HD + threadIdx.x], here >> (threadIdx.x & 7) * 4 & 15u);
}

template <typename T, int HD, int FMT>
__global__ __launch_bounds__(Lanes<HD>::THREADS) void kv8_read_kernel(T* __restrict__ k, T* __restrict__ v, int64_t stride, Kv8View c, Kv8Meta m) {
  typedef Lanes<HD> L;
  __shared__ __align__(16) unsigned char img[kv8_block_bytes(HD)];
  const Place w = place_of(m, c.n_kv);
  const unsigned char* in = c.data + ((int64_t)w.slot * c.n_kv + w.head) * c.head_bytes + (int64_t)w.block * kv8_block_bytes(HD);
#pragma unroll
  for (int i = threadIdx.x; i < 4 * HD; i += L::THREADS) ((u32x4*)img)[unit_at(i)] = ((const u32x4*)in)[i];
  if (threadIdx.x < 4) ((u32x4*)img)[4 * HD + threadIdx.x] = ((const u32x4*)in)[4 * HD + threadIdx.x];
  __syncthreads();
  const L t;
#pragma unroll
  for (int n = 0; n < L::PASSES; ++n) {
    const int p = n * L::ROWS + t.p, d = t.d + 2 * (p & 3);
    const u32x2 kw = *(const u32x2*)&img[byte_at(kv8_k_index(p, t.d, HD))];
    const Two vw = by_positions(Two{*(const unsigned*)&img[byte_at(kv8_v_index(p & ~3, d, HD))], *(const unsigned*)&img[byte_at(kv8_v_index(p & ~3, d + 1, HD))]});
    if (p < w.lo || p >= w.hi) continue;
    const int64_t at = (int64_t)(w.row0 + p) * stride + w.head * HD + t.d;
    float x[8];
    values8<FMT>(Two{kw[0], kw[1]}, img[kv8_scale_index(p, 0, HD)], x);
    store8(k + at, x);
    values8<FMT>(vw, img[kv8_scale_index(p, 1, HD)], x);
    store8(v + at, x);
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
    kv8_write_kernel<T, hd_c(), fmt_c()><<<m.block_off[m.n_seqs] * c.n_kv, Lanes<hd_c()>::THREADS, 0, st>>>((const T*)k, (const T*)v, stride, c, m);
  });
}
void launch_kv8_read(const Kv8View& c, int format, int hd, void* k, void* v, int64_t stride, int dtype, const Kv8Meta& m, hipStream_t st) {
  for_shape(format, hd, dtype, [&](auto t, auto hd_c, auto fmt_c) {
    typedef decltype(t) T;
    kv8_read_kernel<T, hd_c(), fmt_c()><<<m.block_off[m.n_seqs] * c.n_kv, Lanes<hd_c()>::THREADS, 0, st>>>((T*)k, (T*)v, stride, c, m);
  });
}
