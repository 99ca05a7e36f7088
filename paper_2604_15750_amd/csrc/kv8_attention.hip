// Attention of packed rows over the 8-bit cache on the matrix cores: one pass over the keys with the running maximum and sum of a softmax.
//
// The queries of a kv head are the rows of a sequence times the query heads that share it (a group's heads read K and V together); a
// workgroup has up to 16 TILES of them, its wavefronts take every NWV-th block of 32 positions and are merged through LDS.  S^T = K Q^T
// leaves 8 keys of one query in a lane, in the order in which the cache holds V, so the probabilities feed O^T = V^T P^T from registers.
//
// 8-bit codes are exact in IEEE half, so what the matrix cores lose is what the other operand loses:
//   q  a power of two brings a query's largest magnitude to [2^14, 2^15); then one half term (bf16 queries: exact down to 2^-29 of the
//      largest) or two, high and low (fp32 queries: 22 bits)
//   p  one half term (bf16 outputs: 11 bits against the output's 8) or two (fp32: 22 bits)
// The scales: with K_j = 2^a_j code_j and V_j = 2^b_j code_j,
//   s'_j = (q . code_j) 2^a_j log2(e) / sqrt(hd) + b_j,   p'_j = 2^(s'_j - m'),   l = sum_j p'_j 2^-b_j,   o = sum_j p'_j code_j / l
// so V's scale costs no instruction: it is the addend of the multiply-add that applies K's, and the sum's addition becomes a
// multiply-add.  p' is at most 1 whatever the scales; b in [-60, 60] keeps every p' that weighs in l within 32 bits.  p' is kept times
// 2^15, the top of half's range, where it keeps 11 bits down to 2^-29 of the largest.
// A vector marked NaN: a key's scale byte 255 makes its score infinity times zero, a value's makes l minus infinity or NaN.
#include <type_traits>

#include "kv8.h"

namespace {

constexpr float NEG_BIG = -3.0e38f;
constexpr int P_BITS = 15;

struct Pair { float a, b; };
__device__ inline Pair across16(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return Pair{__uint_as_float(r[0]), __uint_as_float(r[1])};
}
__device__ inline Pair across32(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return Pair{__uint_as_float(r[0]), __uint_as_float(r[1])};
}
__device__ inline float query_max(float v) {  // over the four lanes of a query
  Pair t = across16(v);
  t = across32(fmaxf(t.a, t.b));
  return fmaxf(t.a, t.b);
}
__device__ inline float query_sum(float v) {
  Pair t = across16(v);
  t = across32(t.a + t.b);
  return t.a + t.b;
}

// 8 codes (8 bytes) as half
template <int FMT>
__device__ inline f16x8 halves(unsigned lo, unsigned hi) {
  f16x2 h[4];
  if (FMT == DLM_KV8_E4M3) {
    h[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)lo, 1.f, false);
    h[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)lo, 1.f, true);
    h[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)hi, 1.f, false);
    h[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)hi, 1.f, true);
  } else {  // a stored byte c + 128 behind 0x64 is 1024 + c + 128 as half
    const f16x2 bias = {(f16_t)1152.f, (f16_t)1152.f};
    h[0] = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, lo, 0x04010400u)) - bias;
    h[1] = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, lo, 0x04030402u)) - bias;
    h[2] = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, hi, 0x04010400u)) - bias;
    h[3] = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, hi, 0x04030402u)) - bias;
  }
  return f16x8{h[0][0], h[0][1], h[1][0], h[1][1], h[2][0], h[2][1], h[3][0], h[3][1]};
}

__device__ inline void load8(const bf16_t* p, float (&x)[8]) {
  const bf16x8 v = *(const bf16x8*)p;
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = (float)v[i];
}
__device__ inline void load8(const float* p, float (&x)[8]) {
  const f32x4 a = *(const f32x4*)p, b = *(const f32x4*)(p + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[i] = a[i]; x[4 + i] = b[i]; }
}

template <int HD, int NWV>
struct MergeLds {
  float m[NWV][16], l[NWV][16];
  float o[NWV][16][HD + 4];  // (rows 16 bytes apart from a multiple of the banks)
};

__device__ inline float finish(float o, float l) { return l > 0.f ? o / l : l == 0.f ? 0.f : __uint_as_float(0x7FC00000u); }

template <typename T, int HD, int FMT, int TILES, int NWV>
__global__ __launch_bounds__(NWV * 64) void kv8_attention_kernel(Kv8AttnArgs a, Kv8View cache, Kv8AttnMeta meta, int split_out) {
  constexpr bool F32 = std::is_same<T, float>::value;
  constexpr int KS = HD / 32, DT = HD / 16, TERMS = F32 ? 2 : 1;
  __shared__ MergeLds<HD, NWV> L;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g = lane >> 4, c = lane & 15;
  // (the heads of an item are neighbours: where their number is a multiple of 8 all items of a head are on one XCD, and its L2 has the head's K and V)
  const int head = blockIdx.x % cache.n_kv, item = blockIdx.x / cache.n_kv;
  const int b = seq_of(meta.item_off, meta.n_seqs, item);
  const int row0 = meta.row_off[b], nr = meta.row_off[b + 1] - row0, n_keys = meta.n_keys[b], group = a.n_q / cache.n_kv;
  const int nq = nr * group, qtiles = (nq + 16 * TILES - 1) / (16 * TILES);
  const int rel = item - meta.item_off[b], split = rel / qtiles, q0 = (rel - split * qtiles) * (16 * TILES);
  const int nblk = (n_keys + 31) >> 5, blk0 = split * meta.chunk, blk1 = min(nblk, blk0 + meta.chunk);
  const unsigned char* region = cache.data + ((int64_t)meta.slot[b] * cache.n_kv + head) * cache.head_bytes;

  // ---- queries: normalised by a power of two, in one or two half terms
  f16x8 qf[TILES][TERMS][KS];
  float qs[TILES];
  const uint32_t* words[TILES];
#pragma unroll
  for (int u = 0; u < TILES; ++u) {
    const int x = q0 + 16 * u + c, r = x / group;
    const bool there = x < nq;
    const T* from = (const T*)a.q + (int64_t)(row0 + (there ? r : 0)) * a.q_stride + (head * group + (there ? x - r * group : 0)) * HD + 8 * g;
    words[u] = a.mask + (int64_t)(row0 + (there ? r : 0)) * a.mask_words;
    float v[KS][8];
    unsigned top = 0;
#pragma unroll
    for (int t = 0; t < KS; ++t) {
      load8(from + 32 * t, v[t]);
#pragma unroll
      for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[t][i]) & 0x7FFFFFFFu);
    }
    const int e = min(max((int)(__float_as_uint(query_max(__uint_as_float(top & 0x7F800000u))) >> 23) - 127, -100), 127);
    const float up = __uint_as_float((unsigned)(127 + 14 - e) << 23);
    qs[u] = __uint_as_float((unsigned)(127 - 14 + e) << 23) * (1.44269504088896340736f / sqrtf((float)HD));
#pragma unroll
    for (int t = 0; t < KS; ++t)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float y = v[t][i] * up;
        const f16_t hi = (f16_t)y;
        qf[u][0][t][i] = hi;
        if (F32) qf[u][TERMS - 1][t][i] = (f16_t)(y - (float)hi);
      }
  }

  float m[TILES], l[TILES];
  f32x4 o[TILES][DT];
#pragma unroll
  for (int u = 0; u < TILES; ++u) {
    m[u] = NEG_BIG;
    l[u] = 0.f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[u][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // ---- blocks of 32 positions; the next one is in flight while this one is worked on
  constexpr int KP = HD / 32, VP = HD / 32;  // 1 KiB pieces of K and of V
  u32x4 raw[KP + VP + 1];
  auto load = [&](u32x4 (&w)[KP + VP + 1], int blk) __attribute__((always_inline)) {
    const u32x4* p = (const u32x4*)(region + (int64_t)blk * kv8_block_bytes(HD));
#pragma unroll
    for (int i = 0; i < KP + VP; ++i) w[i] = p[i * 64 + lane];
    w[KP + VP] = p[(KP + VP) * 64 + g];
  };
  const int first = a.mask ? n_keys - nr : n_keys;  // positions from here on are visible to whom the mask says
  if (blk0 + wave < blk1) load(raw, blk0 + wave);
  for (int blk = blk0 + wave; blk < blk1; blk += NWV) {
    f16x8 kf[2 * KS], vf[DT];
#pragma unroll
    for (int f = 0; f < 2 * KS; ++f) kf[f] = halves<FMT>(raw[f / 2][f % 2 * 2], raw[f / 2][f % 2 * 2 + 1]);
#pragma unroll
    for (int f = 0; f < DT; ++f) vf[f] = halves<FMT>(raw[KP + f / 2][f % 2 * 2], raw[KP + f / 2][f % 2 * 2 + 1]);
    float ks[8], vb[8], vi[8];  // 2^a, b, 2^-b of the lane's keys 4g + i (i < 4) and 16 + 4g + i - 4
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const unsigned kb = raw[KP + VP][i / 4] >> 8 * (i % 4) & 255u, vbyte = raw[KP + VP][2 + i / 4] >> 8 * (i % 4) & 255u;
      ks[i] = __uint_as_float(kb << 23);
      vb[i] = (float)vbyte - 127.f;
      vi[i] = __uint_as_float((254u - vbyte) << 23);
    }
    if (blk + NWV < blk1) load(raw, blk + NWV);
    const bool masked = 32 * blk + 32 > first;  // (uniform)
#pragma unroll
    for (int u = 0; u < TILES; ++u) {
      f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int x = 0; x < TERMS; ++x)
#pragma unroll
        for (int t = 0; t < KS; ++t) {
          s0 = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf[t], qf[u][x][t], s0, 0, 0, 0);
          s1 = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf[KS + t], qf[u][x][t], s1, 0, 0, 0);
        }
      float sv[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) sv[i] = __builtin_fmaf((i < 4 ? s0[i] : s1[i - 4]) * qs[u], ks[i], vb[i]);
      unsigned see = 0xFFFFFFFFu;
      if (masked) {
        const int left = n_keys - 32 * blk, ofs = 32 * blk - first;  // ofs: of the block in the masked positions
        if (left < 32) see = (1u << left) - 1u;
        if (a.mask) {
          const int w = ofs >> 5, sh = ofs & 31;  // (floors: a block that starts in front of them takes its upper bits from word 0)
          const unsigned lo = w >= 0 ? words[u][w] : 0xFFFFFFFFu, hi = sh && w + 1 < a.mask_words ? words[u][w + 1] : 0u;
          see &= sh ? lo >> sh | hi << (32 - sh) : lo;
        }
        see = see >> 4 * g;
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (!(see >> (i < 4 ? i : 12 + i) & 1u)) sv[i] = -__builtin_inff();
      }
      float mx = fmaxf(fmaxf(fmaxf(sv[0], sv[1]), fmaxf(sv[2], sv[3])), fmaxf(fmaxf(sv[4], sv[5]), fmaxf(sv[6], sv[7])));
      const float mn = fmaxf(m[u], query_max(mx) - (float)P_BITS);
      if (__builtin_amdgcn_ballot_w64(mn != m[u])) {
        const float corr = __builtin_amdgcn_exp2f(m[u] - mn);
        l[u] *= corr;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[u][dt] *= corr;
        m[u] = mn;
      }
      float p[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) p[i] = __builtin_amdgcn_exp2f(sv[i] - mn);
      if (masked) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (see >> (i < 4 ? i : 12 + i) & 1u) l[u] = __builtin_fmaf(p[i], vi[i], l[u]);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) l[u] = __builtin_fmaf(p[i], vi[i], l[u]);
      }
      f16x8 ph, pl;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        ph[i] = (f16_t)p[i];
        if (F32) pl[i] = (f16_t)(p[i] - (float)ph[i]);
      }
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        o[u][dt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf[dt], ph, o[u][dt], 0, 0, 0);
        if (F32) o[u][dt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf[dt], pl, o[u][dt], 0, 0, 0);
      }
    }
  }

  // ---- merge the wavefronts, a tile at a time
#pragma unroll
  for (int u = 0; u < TILES; ++u) {
    if (q0 + 16 * u >= nq) break;  // (uniform)
    if (u) __syncthreads();
    const float ls = query_sum(l[u]);
    if (g == 0) { L.m[wave][c] = m[u]; L.l[wave][c] = ls; }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) *(f32x4*)&L.o[wave][c][16 * dt + 4 * g] = o[u][dt];
    __syncthreads();
    for (int i = tid; i < 16 * HD / 4; i += NWV * 64) {
      const int x = i / (HD / 4), d = i % (HD / 4) * 4, qi = q0 + 16 * u + x, r = qi / group;
      if (qi >= nq) continue;
      float M = L.m[0][x], ls = 0.f;
#pragma unroll
      for (int w = 1; w < NWV; ++w) M = fmaxf(M, L.m[w][x]);
      f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < NWV; ++w) {
        const float f = __builtin_amdgcn_exp2f(L.m[w][x] - M);
        ls += f * L.l[w][x];
        acc += *(const f32x4*)&L.o[w][x][d] * f;
      }
      const int64_t at = (int64_t)(row0 + r) * a.n_q + head * group + (qi - r * group);
      if (split_out) {
        const int64_t part = (int64_t)split * a.rows * a.n_q + at;
        *(f32x4*)(a.part + part * HD + d) = acc;
        if (d == 0) { a.part_ml[2 * part] = M; a.part_ml[2 * part + 1] = ls; }
      } else {
        T* to = (T*)a.out + at * HD + d;
#pragma unroll
        for (int j = 0; j < 4; ++j) to[j] = (T)finish(acc[j], ls);
      }
    }
  }
}

// the shares of a sequence's keys joined: a wavefront a (row, head)
template <typename T, int HD>
__global__ __launch_bounds__(256) void kv8_attention_join_kernel(Kv8AttnArgs a, Kv8AttnMeta meta) {
  constexpr int N = HD / 64 ? HD / 64 : 1;
  const int lane = threadIdx.x & 63;
  const int64_t at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), all = (int64_t)a.rows * a.n_q;
  if (at >= all) return;
  const int row = (int)(at / a.n_q), b = seq_of(meta.row_off, meta.n_seqs, row);
  const int splits = max(1, ((meta.n_keys[b] + 31) / 32 + meta.chunk - 1) / meta.chunk);
  float M = NEG_BIG;
  for (int s = 0; s < splits; ++s) M = fmaxf(M, a.part_ml[2 * (s * all + at)]);
  float ls = 0.f, acc[N] = {};
  for (int s = 0; s < splits; ++s) {
    const int64_t i = s * all + at;
    const float f = __builtin_amdgcn_exp2f(a.part_ml[2 * i] - M);
    ls += f * a.part_ml[2 * i + 1];
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (lane * N < HD) acc[j] += f * a.part[i * HD + lane * N + j];
  }
#pragma unroll
  for (int j = 0; j < N; ++j)
    if (lane * N < HD) ((T*)a.out)[at * HD + lane * N + j] = (T)finish(acc[j], ls);
}

constexpr int64_t MAX_PARTIALS = 1 << 16;
constexpr int MAX_SPLITS = 32;

}  // namespace

size_t kv8_attention_partials(int64_t rows, int n_q) {
  const int64_t all = rows * n_q;
  return 2 * all > MAX_PARTIALS ? 0 : (size_t)(all * MAX_SPLITS < MAX_PARTIALS ? all * MAX_SPLITS : MAX_PARTIALS);
}

Kv8AttnPlan kv8_attention_plan(const int32_t* row_off, const int32_t* n_keys, int n_seqs, int n_q, int n_kv, int hd, int dtype) {
  Kv8AttnPlan p;
  int longest = 0, rows_max = 0;
  for (int b = 0; b < n_seqs; ++b) {
    const int nr = row_off[b + 1] - row_off[b];
    if (nr > rows_max) rows_max = nr;
    if (nr && n_keys[b] > longest) longest = n_keys[b];
  }
  const int64_t queries = (int64_t)rows_max * (n_q / n_kv);
  p.tiles = queries <= 16 ? 1 : queries <= 32 || dtype == DLM_F32 ? 2 : 4;
  p.waves = 4;
  int64_t wgs = 0;
  for (int b = 0; b < n_seqs; ++b) wgs += ((int64_t)(row_off[b + 1] - row_off[b]) * (n_q / n_kv) + 16 * p.tiles - 1) / (16 * p.tiles) * n_kv;
  const int blocks = (longest + 31) / 32;
  p.splits = 1;
  p.chunk = blocks ? blocks : 1;
  const int64_t all = (int64_t)row_off[n_seqs] * n_q;
  if (wgs > 0 && wgs < 256) {
    int64_t s = 512 / wgs, most = MAX_PARTIALS / all;
    if (s > most) s = most;
    if (s > MAX_SPLITS) s = MAX_SPLITS;
    if (s > 1) {
      int chunk = (int)((blocks + s - 1) / s);
      if (chunk < 8) chunk = 8;
      if (chunk < blocks) { p.chunk = chunk; p.splits = (blocks + chunk - 1) / chunk; }
    }
  }
  p.items = 0;
  return p;
}

namespace {
template <typename T, int HD, int FMT>
void launch_shape(const Kv8View& c, const Kv8AttnArgs& a, const Kv8AttnMeta& m, const Kv8AttnPlan& p, hipStream_t st) {
  const int grid = (int)(p.items * c.n_kv), sp = p.splits > 1;
  constexpr int MOST = std::is_same<T, float>::value ? 2 : 4;
  if (p.tiles == 1) kv8_attention_kernel<T, HD, FMT, 1, 4><<<grid, 256, 0, st>>>(a, c, m, sp);
  else if (p.tiles == 2) kv8_attention_kernel<T, HD, FMT, 2, 4><<<grid, 256, 0, st>>>(a, c, m, sp);
  else kv8_attention_kernel<T, HD, FMT, MOST, 4><<<grid, 256, 0, st>>>(a, c, m, sp);
  if (sp) kv8_attention_join_kernel<T, HD><<<(int)(((int64_t)a.rows * a.n_q + 3) / 4), 256, 0, st>>>(a, m);
}
template <typename T, int HD>
void launch_format(const Kv8View& c, int format, const Kv8AttnArgs& a, const Kv8AttnMeta& m, const Kv8AttnPlan& p, hipStream_t st) {
  format == DLM_KV8_E4M3 ? launch_shape<T, HD, DLM_KV8_E4M3>(c, a, m, p, st) : launch_shape<T, HD, DLM_KV8_I8>(c, a, m, p, st);
}
}  // namespace

void launch_kv8_attention(const Kv8View& c, int format, int hd, int dtype, const Kv8AttnArgs& a, const Kv8AttnMeta& m, const Kv8AttnPlan& p, hipStream_t st) {
  auto go = [&](auto f) { f(c, format, a, m, p, st); };
  if (dtype == DLM_BF16) hd == 128 ? go(launch_format<bf16_t, 128>) : hd == 64 ? go(launch_format<bf16_t, 64>) : go(launch_format<bf16_t, 32>);
  else hd == 128 ? go(launch_format<float, 128>) : hd == 64 ? go(launch_format<float, 64>) : go(launch_format<float, 32>);
}
