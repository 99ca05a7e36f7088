// Attention of packed rows over the 8-bit cache on the matrix cores: one pass over the keys with the running maximum and sum of a softmax.
//
// The queries of a kv head are the rows of a sequence times the query heads that share it (a group's heads read K and V together); a
// wavefront has 32 of them and takes blocks of 32 positions.  S^T = K Q^T leaves 16 keys of one query in a lane, in the order in which
// the cache holds V, so the probabilities feed O^T = V^T P^T from registers.
//
// 8-bit codes are exact in IEEE half, so what the matrix cores lose is what the other operand loses:
//   q  a power of two brings a query's largest magnitude to [2^14, 2^15); then one half term (bf16 queries: exact down to 2^-29 of the
//      largest) or two, high and low (fp32 queries: 22 bits)
//   p  one half term (bf16 outputs: 11 bits against the output's 8) or two (fp32: 22 bits)
// The scales: with K_j = 2^a_j code_j and V_j = 2^b_j code_j,
//   s'_j = (q . K_j) log2(e) / sqrt(hd) + b_j,   p'_j = 2^(s'_j - m),   l = sum_j p'_j 2^-b_j,   o = sum_j p'_j code_j / l
//   a  goes in where codes become half (the conversion scales; i8 takes it in the multiply-add that takes its offset off), relative to a
//      wavefront's `ref`, which moves where a block has a key 2^6 above it or 2^-16 below it: half holds every code in between exactly, so
//      a score does not depend on ref, nor on any other key.  The products of a block whose keys lie further apart are made once
//      for each range of scales in it, from codes that are loaded again (rare, and out of the way of other blocks)
//   b  is the addend of the multiply-add that applies the softmax's scale, and the sum's addition becomes a multiply-add.  p' stays
//      bounded whatever the scales.  b in [-60, 60] keeps l within 32 bits, and a value whose scale is 2^-B of the largest one's that its
//      wavefront has met has its part in l down to a probability of 2^(B-134) of that one's (fp32 2^(B-139)): 2^-34 (2^-39) for values
//      2^100 apart, 2^-14 (2^-19) for the 2^120 that is the most.  Where sums are rescaled and joined nothing more is lost.
// The softmax's instructions weigh as much as the products (16 scores a lane against 512 cycles of them for 32 x 32 scores), so each
// score costs a multiply-add, half a maximum, an exponential, a multiply-add and half a conversion: the products start from -m (bf16), and m
// moves only where a score would leave half's range: the largest p' is brought to about 2^8 (fp32: 2^13) and may grow to 2^15 before that.
// What bounds it: 1280 rows x 32 heads of 128 over themselves 40 to 45 us, 0.6 to 0.67 PFLOP/s (fp32 68 to 70), 4096 rows 320 to 330 us, 0.85 (a large half
// product reaches 1.12 to 1.22): vector instructions and products in turn.  155 instructions a block of 32 keys on the straight path beside 16 products,
// 187 at 4096 rows and 249 at 1280 with what is done once a wavefront: at 4096 the products have 41 % of the cycles and they 60 %, at 1280 29 and 56, and the
// rest is the chip's last round.  Single tokens of 24 sequences of up to 8192 keys, 28 of 4 heads: 30.6 us, 5 TB/s of cache.  Few rows: latency,
// 8 rows x 32 heads of 392 keys 6.6 us.
// The rare paths (scales too far apart, a maximum from far below) cost the others 0 to 3 %: 1280 rows 44.1 us without them, 45.6 with; 24 single tokens 35.0,
// 35.3; fp32 1280 rows 68.1, 70.0.  Written as a loop around the softmax they cost 10 %, with registers that spill up to 13.
// Why 32 queries, one wavefront's work: a group's heads of a few rows fill 32, not 128.  Four wavefronts share the keys because a decode
// has few tiles and many keys.  Tried and slower: K and V through LDS for 4 x 32 queries (1280 rows 55.6 us, 42 at that time; only 1024 rows
// of 4096 keys gained, 110 to 91), two tiles a wavefront (73), 8 wavefronts a workgroup (392 keys 7.9, 7.4 then), V loaded two blocks ahead
// (46.6, 44), queries in LDS so that three wavefronts fit a SIMD (392 keys 7.9, 6.7; 4096 rows 351, 343), the next block's scores under this
// block's exponentials (392 keys 6.85, 6.7; 4096 rows 370, 356).
#include <type_traits>

#include "kv8.h"

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float NEG_BIG = -3.0e38f;
constexpr float P_LIMIT = 15.f;  // log2 of where the largest p' may go
constexpr float P_FAR = 32.f;    // ... and from where on scores are made again: fp32's step at m is at most that of the score and 32
constexpr unsigned REF_ABOVE = 5, REF_BELOW = 15;  // of ref: 1152 2^5 and 448 2^5 are below half's largest, 2^-9 2^-15 (e4m3's smallest code) is its smallest

__device__ inline float halves_max(float v) {  // over the two lanes of a query
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float halves_sum(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// 8 codes (8 bytes) as half, times 2^e (e4m3: `scale`; i8: `mul`, and `add` = -1152 mul)
template <int FMT>
__device__ inline f16x8 halves(unsigned lo, unsigned hi, float scale, f16x2 mul, f16x2 add) {
  f16x2 h[4];
  if (FMT == DLM_KV8_E4M3) {
    h[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)lo, scale, false);
    h[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)lo, scale, true);
    h[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)hi, scale, false);
    h[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)hi, scale, true);
  } else {  // a stored byte c + 128 behind 0x64 is 1024 + c + 128 as half
    h[0] = __builtin_elementwise_fma(__builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, lo, 0x04010400u)), mul, add);
    h[1] = __builtin_elementwise_fma(__builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, lo, 0x04030402u)), mul, add);
    h[2] = __builtin_elementwise_fma(__builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, hi, 0x04010400u)), mul, add);
    h[3] = __builtin_elementwise_fma(__builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, hi, 0x04030402u)), mul, add);
  }
  return f16x8{h[0][0], h[0][1], h[1][0], h[1][1], h[2][0], h[2][1], h[3][0], h[3][1]};
}

__device__ inline void store4(bf16_t* p, f32x4 v) { *(bf16x4*)p = bf16x4{(bf16_t)v[0], (bf16_t)v[1], (bf16_t)v[2], (bf16_t)v[3]}; }
__device__ inline void store4(float* p, f32x4 v) { *(f32x4*)p = v; }

// what an output is multiplied with: a row that sees nothing gives 0, one whose sum is not a positive number NaN
__device__ inline float reciprocal(float l) { return l > 0.f ? 1.f / l : l == 0.f ? 0.f : __uint_as_float(0x7FC00000u); }

// sum 2^x of a whole number x <= 0.  (A sum with V's scales undone can be far above 1, 2^68 where they are 2^-60, and count where 2^x by itself is below 32
// bits' range; an output that small beside another does not.)
__device__ inline float rescaled(float sum, float x) { return __builtin_amdgcn_ldexpf(sum, (int)fmaxf(x, -1000.f)); }

// whether a scale byte of K is one: a position that was never written (zero beside any other) or is marked NaN is right with any ref
__device__ inline bool has_scale(unsigned kb) { return kb - 1u < KV8_NAN - 1u; }

// What a workgroup works on
struct Work {
  int head, row0, nq, group, q0, split, blk0, blk1, n_keys, first;  // first: positions from here on are visible to whom the mask says
  const unsigned char* region;
  __device__ inline int row_of(int x) const { return group == 1 ? x : (int)((unsigned)x / (unsigned)group); }  // of query x
};

// 32 queries of a wavefront and their running softmax
template <typename T, int HD, int FMT>
struct Tile {
  static constexpr bool F32 = std::is_same<T, float>::value;
  static constexpr float P_TOP = F32 ? 13.f : 8.f;  // log2 of where the largest p' is put: half ends 25 bits below 1
  static constexpr int PIECES = HD / 32, KF = HD / 16, TERMS = F32 ? 2 : 1;
  f16x8 qf[KF];
  f16x8* low;                      // fp32: LDS, the low terms (the same in all wavefronts of a workgroup, and each reads what it wrote)
  f32x16 o[PIECES], from_m;        // from_m: -m / cq in every element, what the products start from
  float qs, cq, rest, m, l, limit; // rest: what cq leaves of the scale (fp32); m: a whole number; limit: minus infinity until the query has seen a key
  int ref;                         // biased exponent that K's scales are relative to
  const uint32_t* words;           // of the query's row in the mask

  __device__ inline void start(const T* q, int64_t q_stride, const Kv8AttnArgs& a, const Work& w, int lane) {
    const int h = lane >> 5, x = w.q0 + (lane & 31), r = x < w.nq ? w.row_of(x) : 0, hq = x < w.nq ? x - r * w.group : 0;
    const T* from = q + (int64_t)(w.row0 + r) * q_stride + (w.head * w.group + hq) * HD + 16 * h;
    words = a.mask + (int64_t)(w.row0 + r) * a.mask_words;
    Eight<T> v[KF];
    unsigned top = 0;
#pragma unroll
    for (int f = 0; f < KF; ++f) v[f].load(from + 32 * (f >> 1) + 8 * (f & 1));
#pragma unroll
    for (int f = 0; f < KF; ++f) top = max(top, v[f].top());
    const int e = min(max((int)(__float_as_uint(halves_max(__uint_as_float(top & 0x7F800000u))) >> 23) - 127, -100), 127);
    const float up = __uint_as_float((unsigned)(127 + 14 - e) << 23);
    qs = __uint_as_float((unsigned)(127 - 14 + e) << 23);
#pragma unroll
    for (int f = 0; f < KF; ++f) {
      f16x8 rest_of;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float y = v[f][i] * up;
        qf[f][i] = (f16_t)y;
        rest_of[i] = (f16_t)(y - (float)qf[f][i]);
      }
      if (F32) low[f * 64 + lane] = rest_of;
    }
    m = l = 0.f;
    limit = -__builtin_inff();
    set_ref(127);  // (a largest magnitude of 2^-6 to 2^13: what normalised heads hold)
#pragma unroll
    for (int d = 0; d < PIECES; ++d) o[d] = from_m;
  }

  // which of a block's positions the lane's query sees, from bit 4h on
  __device__ inline unsigned visible(const Kv8AttnArgs& a, const Work& w, int blk, int h) const {
    unsigned see = 0xFFFFFFFFu;
    const int left = w.n_keys - 32 * blk, ofs = 32 * blk - w.first;  // ofs: of the block in the masked positions
    if (left < 32) see = left > 0 ? (1u << left) - 1u : 0u;
    if (a.mask) {
      const int i = ofs >> 5, sh = ofs & 31;  // (floors: a block that starts in front of them takes its upper bits from word 0)
      const unsigned lo = i >= 0 ? words[i] : 0xFFFFFFFFu, hi = sh && i + 1 < a.mask_words ? words[i + 1] : 0u;
      see &= sh ? lo >> sh | hi << (32 - sh) : lo;
    }
    return see >> 4 * h;
  }

  __device__ inline void start_from_m() {
    const float t = -m * __builtin_amdgcn_rcpf(cq);  // (a step of fp32 off: what the products start from is the same for all keys)
#pragma unroll
    for (int i = 0; i < 16; ++i) from_m[i] = t;
  }

  // K's scales from here on relative to `to`
  __device__ inline void set_ref(int to) {
    constexpr double SCALE = 1.44269504088896340736 / (HD == 128 ? 11.3137084989847603904 : HD == 64 ? 8.0 : 5.65685424949238019521);
    // 2^-64: scores are below 2^-28 then, as good as zero; 2^125: beyond it only where no key that the query sees has a score in range, and finite, so that
    // a position that was never written scores zero
    const float unit = __builtin_amdgcn_fmed3f(qs * __uint_as_float((unsigned)to << 23), 0x1p-64f, 0x1p125f);
    ref = to;
    cq = unit * (float)SCALE;
    rest = unit * (float)(SCALE - (double)(float)SCALE);
    start_from_m();
  }
  // ref at the largest scale of the positions whose bits are set (if any); returns those of them that it suits
  __device__ inline unsigned move_ref(unsigned kb, unsigned of, int lane) {
    unsigned t = of >> (lane & 31) & 1u ? kb : 0u;
    t = row_butterfly(t, [](unsigned p, unsigned q) { return p > q ? p : q; });
    const auto r = __builtin_amdgcn_permlane16_swap(t, t, false, false);
    const unsigned top = __builtin_amdgcn_readfirstlane(r[0] > r[1] ? r[0] : r[1]);
    if (top) set_ref((int)top);
    return of & (unsigned)__builtin_amdgcn_ballot_w64((int)kb + (int)REF_BELOW >= ref);
  }
  // s = K Q^T of a block, relative to ref (bf16: from -m on)
  template <typename K>
  __device__ __attribute__((always_inline)) inline f32x16 products(unsigned kb, K k, int lane) const {
    const float k_scale = __uint_as_float((unsigned)max((int)kb - ref + 127, 0) << 23);
    const f16x2 k_mul = {(f16_t)k_scale, (f16_t)k_scale}, k_add = k_mul * f16x2{(f16_t)-1152.f, (f16_t)-1152.f};
    f32x16 s;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = F32 ? 0.f : from_m[i];
#pragma unroll
    for (int f = 0; f < KF; ++f) {
      const u32x4 raw = k(f >> 1);
      const f16x8 kf = halves<FMT>(raw[f % 2 * 2], raw[f % 2 * 2 + 1], k_scale, k_mul, k_add);
#pragma unroll
      for (int x = 0; x < TERMS; ++x) s = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf, x ? low[f * 64 + lane] : qf[f], s, 0, 0, 0);
    }
    return s;
  }
  // log2 p' of the lane's keys 8j + 4h + i
  __device__ __attribute__((always_inline)) inline void logits(const f32x16& s, const float* vb, int h, float (&p)[16]) const {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const f32x4 t = *(const f32x4*)&vb[8 * j + 4 * h];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        // fp32: products that start from zero, and no rounding but at the size of the difference (b and m are whole numbers)
        p[4 * j + i] = __builtin_fmaf(s[4 * j + i], cq, F32 ? t[i] - m : t[i]);
        if (F32) p[4 * j + i] = __builtin_fmaf(s[4 * j + i], rest, p[4 * j + i]);
      }
    }
  }

  // NaN for positions so marked, minus infinity for those that the query does not see
  __device__ __attribute__((always_inline)) inline void hide(float (&p)[16], const Kv8AttnArgs& a, const Work& w, int blk, int h, unsigned nan_keys) const {
    if (__builtin_expect(nan_keys != 0, 0)) {
      asm volatile("; keys marked NaN");  // (keeps the branch: the compiler would make 48 instructions of every block out of it)
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (nan_keys >> (8 * (i >> 2) + 4 * h + (i & 3)) & 1u) p[i] = __uint_as_float(0x7FC00000u);
    }
    if (__builtin_expect(32 * blk + 32 > w.first, 0)) {  // (uniform)
      const unsigned see = visible(a, w, blk, h);
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (!(see >> (8 * (i >> 2) + (i & 3)) & 1u)) p[i] = -__builtin_inff();
    }
  }
  static __device__ inline float largest(const float (&p)[16]) {
    float mx = p[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = fmaxf(mx, p[i]);
    return mx;
  }

  // One block of 32 positions.  kb: K's scale byte of position lane % 32; nan_keys: bits of positions marked NaN in K or V (the same
  // in all lanes); vb, inv: LDS, V's exponents and what undoes them; k(i), v(i): the lane's 16 bytes of piece i; after_k, after_v: run
  // when they are used up; again_k: brings k back; kept: LDS, a place for the outputs.
  template <typename K, typename V, typename AK, typename AV, typename RK>
  __device__ __attribute__((always_inline)) inline void block(const Kv8AttnArgs& a, const Work& w, int blk, int h, unsigned kb, unsigned nan_keys, const float* vb,
                                                              const float* inv, K k, V v, AK after_k, AV after_v, RK again_k, float* kept) {
    const int lane = threadIdx.x & 63;
    const f16x2 v_mul = {(f16_t)1.f, (f16_t)1.f}, v_add = {(f16_t)-1152.f, (f16_t)-1152.f};
    bool again = false;  // (uniform) whether the block's keys are too far apart for one ref
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(kb - (unsigned)ref + REF_BELOW > REF_BELOW + REF_ABOVE && has_scale(kb)) != 0, 0)) {
      const unsigned all = (unsigned)__builtin_amdgcn_ballot_w64(has_scale(kb));
      again = move_ref(kb, all, lane) != all;
    }
    float p[16];
    {
      const f32x16 s = products(kb, k, lane);
      after_k();
      logits(s, vb, h, p);
    }
    hide(p, a, w, blk, h, nan_keys);
    float mx = largest(p);
    if (__builtin_expect(again || __builtin_amdgcn_ballot_w64(mx > limit) != 0, 0)) {  // some query's maximum moves
      const float was = m;
      const bool had = limit > 0.f;
      mx = halves_max(mx);
      // Scores come out relative to m, with the rounding of its size: those of a maximum far above that of the blocks before are made again, from zero
      if (__builtin_expect(again || __builtin_amdgcn_ballot_w64(had && mx > P_FAR) != 0, 0)) {
        // (the outputs so far wait in LDS: their registers would be needed, and those that the compiler would spill are used on every block)
#pragma unroll
        for (int i = 0; i < 16 * PIECES; ++i) kept[64 * i + lane] = o[i >> 4][i & 15];
        asm volatile("" ::: "memory");
        for (bool from_zero = !again;; from_zero = true) {
          if (from_zero) {
            const bool far = had && mx > P_FAR;
            if (__builtin_amdgcn_ballot_w64(far) == 0) break;
            if (far) {
              m = 0.f;
              limit = -__builtin_inff();
              start_from_m();
            }
          }
          const unsigned all = (unsigned)__builtin_amdgcn_ballot_w64(has_scale(kb));
          unsigned due = all;
          do {
            asm volatile("" ::: "memory");  // (nothing is loaded, or converted, in front of the loop)
            again_k();
            const unsigned now = move_ref(kb, due, lane), mine = (now | ~all) >> 4 * h;
            float x[16];
            logits(products(kb, k, lane), vb, h, x);
#pragma unroll
            for (int i = 0; i < 16; ++i)
              if (mine >> (8 * (i >> 2) + (i & 3)) & 1u) p[i] = x[i];
            due &= ~now;
          } while (due);
          after_k();
          hide(p, a, w, blk, h, nan_keys);
          mx = halves_max(largest(p));
          if (from_zero) break;
        }
        asm volatile("" ::: "memory");
#pragma unroll
        for (int i = 0; i < 16 * PIECES; ++i) o[i >> 4][i & 15] = kept[64 * i + lane];
      }
      const bool up = mx > limit;
      // (a maximum of 2^24 or more is put to 1: its steps are too coarse for P_TOP, and a step more than that passes half's range)
      float by = up ? floorf(mx) - (fabsf(mx) < 0x1p24f ? P_TOP : 0.f) : 0.f;
      if (had) by = fmaxf(by, was - m);  // (m never falls: made again, a score of many digits can turn out below the old maximum)
      m += by;
      if (up) limit = P_LIMIT;
      const float down = had ? was - m : NEG_BIG, corr = __builtin_amdgcn_exp2f(down);
      l = rescaled(l, down);
#pragma unroll
      for (int d = 0; d < PIECES; ++d) o[d] *= corr;
#pragma unroll
      for (int i = 0; i < 16; ++i) p[i] -= by;
      start_from_m();
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const f32x4 t = *(const f32x4*)&inv[8 * j + 4 * h];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        p[4 * j + i] = __builtin_amdgcn_exp2f(p[4 * j + i]);
        l = __builtin_fmaf(p[4 * j + i], t[i], l);
      }
    }
    f16x8 ph[TERMS][2];
#pragma unroll
    for (int x = 0; x < TERMS; ++x)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        ph[x][i >> 3][i & 7] = (f16_t)p[i];
        if (F32) p[i] -= (float)ph[x][i >> 3][i & 7];
      }
#pragma unroll
    for (int f = 0; f < KF; ++f) {
      const u32x4 raw = v(f >> 1);
      const f16x8 vf = halves<FMT>(raw[f % 2 * 2], raw[f % 2 * 2 + 1], 1.f, v_mul, v_add);
#pragma unroll
      for (int x = 0; x < TERMS; ++x) o[f >> 1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf, ph[x][f & 1], o[f >> 1], 0, 0, 0);
    }
    after_v();
  }

  __device__ inline float top() const { return limit > 0.f ? m : NEG_BIG; }
};

// V's scale byte as its exponent and what undoes it.  A position that was never written (0) counts at the least scale, as a vector of zeros that was
// (its codes: 0 in e4m3, -128 in i8, 2^-53 there): at 2^-127 the sum's terms would pass 32 bits.
__device__ inline unsigned v_scale(unsigned vb) { return max(vb, 127u - KV8_E_MAX); }
__device__ inline float exponent_of(unsigned vb) { return (float)v_scale(vb) - 127.f; }
__device__ inline float undo_of(unsigned vb) { return vb == KV8_NAN ? 0.f : __uint_as_float((254u - v_scale(vb)) << 23); }

// where a query's four dims from d on go: the output, or the workspace if the keys are split
template <typename T, int HD>
__device__ inline void put(const Kv8AttnArgs& a, const Work& w, int split_out, int x, int d, f32x4 v, float top, float sum_or_inv) {
  const int r = w.row_of(x);
  const int64_t at = (int64_t)(w.row0 + r) * a.n_q + w.head * w.group + (x - r * w.group);
  if (!split_out) {
    store4((T*)a.out + at * HD + d, v * sum_or_inv);
    return;
  }
  const int64_t part = (int64_t)w.split * a.rows * a.n_q + at;
  *(f32x4*)(a.part + part * HD + d) = v;
  if (d == 0) { a.part_ml[2 * part] = top; a.part_ml[2 * part + 1] = sum_or_inv; }
}

constexpr int NWV = 4;  // wavefronts of a workgroup, which share its keys

template <int HD, bool F32>
struct alignas(16) AttnLds {
  f16x8 low[F32 ? HD / 16 * 64 : 1];  // (in registers: one wavefront a SIMD instead of two; 1280 rows x 32 heads over themselves 99 us, 70 here)
  float b[NWV][32], inv[NWV][32];  // of a block's keys: V's exponent, and what undoes its scale
  float m[NWV][32], l[NWV][32];    // the wavefronts' maxima and sums
  float o[NWV][32][HD + 4];        // ... and outputs (a query's 16 bytes apart from a multiple of the banks)
};

// (wavefronts a SIMD that the registers suffice for; heads of 32 with four, their rare paths spilling: 2048 rows x 4 heads over themselves 14.2 us, 13.4 so)
template <typename T, int HD, int FMT>
__global__ __launch_bounds__(NWV * 64) __attribute__((amdgpu_waves_per_eu(HD == 128 ? 2 : 3))) void kv8_attention_kernel(
    const unsigned char* __restrict__ data, int head_blocks, int n_kv, const T* __restrict__ q, int64_t q_stride, int group, int chunk, int one_rows, int one_keys,
    int one_slot, int split_out, Kv8AttnArgs a, Kv8AttnMeta meta) {
  constexpr int PIECES = HD / 32;
  __shared__ AttnLds<HD, Tile<T, HD, FMT>::F32> L;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5, c = lane & 31;
  // (the heads of a tile are neighbours: where their number is a multiple of 8 all tiles of a head are on one XCD, and its L2 has the head's K and V)
  Work w;
  w.head = blockIdx.x;
  w.group = group;
  w.row0 = 0;
  w.n_keys = one_keys;
  w.q0 = blockIdx.y * 32;
  w.split = blockIdx.z;
  int nr = one_rows, slot = one_slot;
  if (one_slot < 0) {  // (a single sequence's figures arrive in registers instead of by two trips to memory, and it needs no division)
    const int b = seq_of(meta.item_off, meta.n_seqs, blockIdx.y), item = blockIdx.y - meta.item_off[b];
    w.row0 = meta.row_off[b];
    nr = meta.row_off[b + 1] - w.row0;
    w.n_keys = meta.n_keys[b];
    slot = meta.slot[b];
    const int qtiles = (nr * group + 31) >> 5;
    w.split = item / qtiles;
    w.q0 = (item - w.split * qtiles) * 32;
  }
  w.nq = nr * group;
  w.blk0 = w.split * chunk;
  w.blk1 = min((w.n_keys + 31) >> 5, w.blk0 + chunk);
  w.region = data + ((int64_t)slot * n_kv + w.head) * head_blocks * kv8_block_bytes(HD);
  // The next block is in flight while this one is worked on.  Its loads are made in any case, past the last block a line each that nothing
  // uses: a path around them would be one that the compiler's count of them cannot follow, and each use would wait for all of them.
  u32x4 kr[PIECES], vr[PIECES];
  unsigned kb, vb;  // scale bytes of position c
  auto load_k = [&](int blk) __attribute__((always_inline)) {
    const int there = (blk - w.blk1) >> 31, at = lane & there;  // (all bits or none: the compiler makes a branch of a condition)
    const unsigned char* p = w.region + (int64_t)(blk & there) * kv8_block_bytes(HD);
    kb = p[64 * HD + c];
    vb = p[64 * HD + 32 + c];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) kr[i] = ((const u32x4*)p)[i * 64 + at];
  };
  auto load_v = [&](int blk) __attribute__((always_inline)) {
    const int there = (blk - w.blk1) >> 31, at = lane & there;
    const u32x4* p = (const u32x4*)(w.region + (int64_t)(blk & there) * kv8_block_bytes(HD));
#pragma unroll
    for (int i = 0; i < PIECES; ++i) vr[i] = p[(PIECES + i) * 64 + at];
  };
  load_k(w.blk0 + wave);
  load_v(w.blk0 + wave);
  w.first = a.mask ? w.n_keys - nr : w.n_keys;
  Tile<T, HD, FMT> t;
  t.low = L.low;
  t.start(q, q_stride, a, w, lane);
  for (int blk = w.blk0 + wave; blk < w.blk1; blk += NWV) {
    const unsigned nan_keys = (unsigned)__builtin_amdgcn_ballot_w64(max(kb, vb) == KV8_NAN), k_now = kb;
    if (h == 0) L.b[wave][c] = exponent_of(vb);
    else L.inv[wave][c] = undo_of(vb);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    t.block(a, w, blk, h, k_now, nan_keys, L.b[wave], L.inv[wave], [&](int i) { return kr[i]; }, [&](int i) { return vr[i]; },
            [&] { load_k(blk + NWV); }, [&] { load_v(blk + NWV); }, [&] { load_k(blk); }, &L.o[wave][0][0]);
    __builtin_amdgcn_wave_barrier();
  }
  // merge the wavefronts
  const float ls = halves_sum(t.l);
  if (w.q0 + c < w.nq) {
    if (h == 0) { L.m[wave][c] = t.top(); L.l[wave][c] = ls; }
#pragma unroll
    for (int d = 0; d < PIECES; ++d)
#pragma unroll
      for (int j = 0; j < 4; ++j) *(f32x4*)&L.o[wave][c][32 * d + 8 * j + 4 * h] = f32x4{t.o[d][4 * j], t.o[d][4 * j + 1], t.o[d][4 * j + 2], t.o[d][4 * j + 3]};
  }
  __syncthreads();
  for (int i = tid; i < 32 * HD / 4; i += NWV * 64) {
    const int x = i / (HD / 4), d = i % (HD / 4) * 4;
    if (w.q0 + x >= w.nq) break;
    float M = L.m[0][x], sum = 0.f;
#pragma unroll
    for (int v = 1; v < NWV; ++v) M = fmaxf(M, L.m[v][x]);
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int v = 0; v < NWV; ++v) {
      const float down = L.m[v][x] - M;
      sum += rescaled(L.l[v][x], down);
      acc += *(const f32x4*)&L.o[v][x][d] * __builtin_amdgcn_exp2f(down);
    }
    put<T, HD>(a, w, split_out, w.q0 + x, d, acc, M, split_out ? sum : reciprocal(sum));
  }
}

// the shares of a sequence's keys joined: a wavefront a (row, head); a lane holds a share's weight, then the shares' outputs are added
// (one share after the other, with the weights computed on the way: 48 rows x 28 heads x 17 shares 10.8 us)
template <typename T, int HD>
__global__ __launch_bounds__(256) void kv8_attention_join_kernel(Kv8AttnArgs a, Kv8AttnMeta meta) {
  constexpr int N = HD / 64 ? HD / 64 : 1, AHEAD = 8;
  typedef float vec __attribute__((ext_vector_type(N)));
  const int lane = threadIdx.x & 63, d = lane * N & (HD - 1);
  const int64_t at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), all = (int64_t)a.rows * a.n_q;
  if (at >= all) return;
  const int row = (int)(at / a.n_q), b = seq_of(meta.row_off, meta.n_seqs, row);
  const int shares = max(1, ((meta.n_keys[b] + 31) / 32 + meta.chunk - 1) / meta.chunk);
  const float* ml = a.part_ml + 2 * (min(lane, shares - 1) * all + at);
  const float top = lane < shares ? ml[0] : NEG_BIG;
  const float down = top - wave_max(top), w = __builtin_amdgcn_exp2f(down), inv = reciprocal(wave_sum(lane < shares ? rescaled(ml[1], down) : 0.f));
  vec acc = 0.f;
  for (int s0 = 0; s0 < shares; s0 += AHEAD) {
    vec v[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) v[i] = *(const vec*)(a.part + (min(s0 + i, shares - 1) * all + at) * HD + d);
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) acc += v[i] * (s0 + i < shares ? __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), min(s0 + i, 63))) : 0.f);
  }
#pragma unroll
  for (int j = 0; j < N; ++j)
    if (lane * N < HD) ((T*)a.out)[at * HD + d + j] = (T)(acc[j] * inv);
}

constexpr int64_t MAX_PARTIALS = 1 << 16;  // (share, row, head) triples: 34 MB of workspace at a head dim of 128
constexpr int MAX_SHARES = 32, CUS = 256;

int blocks_of(int n_keys) { return (n_keys + 31) / 32; }
int64_t tiles_of(int rows, int group) { return ((int64_t)rows * group + 31) / 32; }

}  // namespace

size_t kv8_attention_partials(int64_t rows, int n_q) {
  const int64_t all = rows * n_q;
  return 2 * all > MAX_PARTIALS ? 0 : (size_t)(all * MAX_SHARES < MAX_PARTIALS ? all * MAX_SHARES : MAX_PARTIALS);
}

// Keys are shared between workgroups where there are too few of them: in the shortest shares (8 blocks or more, two a wavefront) that make at
// most one workgroup a compute unit, or two if those of one would be longer than 40 blocks, or else in shares of 24, which leave the
// chip's last round short.  A share takes a second launch to join them (3 to 4 us), as long as a workgroup's last 18 blocks: below that
// they stay together.  us a call, shares of 8 / 16 / 24 / 40 / 64 blocks / not shared, K and V from HBM: 8 rows x 32 heads of 4096 keys (8 and 16:
// 544 and 288 workgroups) 13.6 / 12.7 / 13.0 / 15.4 / 19.1 / 30; 48 rows x 28 of 4 heads of 4144 22.9 / 18.1 / 16.1 / 17.5 / 21.2 / 29; 4 rows 11.5 at 16, 12.2 at 24,
// 28 not; 4 x 8 rows x 32 heads of up to 4096 34.1 / 28.3 / 28.2 / 29.8 / 33.6; 24 rows x 28 of 4 heads of up to 8192 46.9 / 40.3 / 38.8 / 35.2 / 44.7; 16 x 8
// rows x 32 heads of up to 4096 107 / 91.0 / 85.9 / 85.5 / 94.5.
Kv8AttnPlan kv8_attention_plan(const int32_t* row_off, const int32_t* n_keys, int n_seqs, int n_q, int n_kv) {
  const int group = n_q / n_kv;
  int64_t work = 0, whole = 0, tiles[DLM_MAX_SEQS];  // blocks of all workgroups; their number without shares; (32 queries, kv head) pairs
  int blocks = 1;                                    // of the longest
  for (int b = 0; b < n_seqs; ++b) {
    tiles[b] = tiles_of(row_off[b + 1] - row_off[b], group) * n_kv;
    whole += tiles[b];
    work += tiles[b] * blocks_of(n_keys[b]);
    if (tiles[b] && blocks_of(n_keys[b]) > blocks) blocks = blocks_of(n_keys[b]);
  }
  const int64_t all = (int64_t)row_off[n_seqs] * n_q, most = all ? MAX_PARTIALS / all < MAX_SHARES ? MAX_PARTIALS / all : MAX_SHARES : 1;
  Kv8AttnPlan p;
  p.chunk = blocks;
  p.splits = 1;
  constexpr int LEAST = 8, JOIN = 18;
  if (most >= 2 && blocks > LEAST + JOIN) {
    // the least chunk with which the workgroups are no more than `rounds` a compute unit, from `least` to `last`; 0 if there is none
    auto fit = [&](int rounds, int64_t least, int64_t last) -> int64_t {
      if (whole > rounds * CUS) return 0;
      int64_t chunk = (work + rounds * CUS - 1) / (rounds * CUS);
      if (chunk < least) chunk = least;
      for (; chunk <= last; ++chunk) {
        int64_t wgs = 0;
        for (int b = 0; b < n_seqs; ++b) {
          const int shares = (blocks_of(n_keys[b]) + (int)chunk - 1) / (int)chunk;
          wgs += tiles[b] * (shares > 1 ? shares : 1);
        }
        if (wgs <= rounds * CUS) return chunk;
      }
      return 0;
    };
    int64_t chunk = fit(1, LEAST, 40);
    if (!chunk) chunk = fit(2, 24, 44);
    if (!chunk) chunk = 24;
    if (chunk * most < blocks) chunk = (blocks + most - 1) / most;
    if (chunk + JOIN < blocks) {
      p.chunk = (int)chunk;
      p.splits = (int)((blocks + chunk - 1) / chunk);
    }
  }
  p.items = 0;
  for (int b = 0; b < n_seqs; ++b) {
    const int shares = (blocks_of(n_keys[b]) + p.chunk - 1) / p.chunk;
    p.item_off[b] = p.items;
    p.items += tiles_of(row_off[b + 1] - row_off[b], group) * (shares > 1 ? shares : 1);
  }
  p.item_off[n_seqs] = p.items;
  return p;
}

namespace {
template <typename T, int HD, int FMT>
void launch_shape(const Kv8View& c, const Kv8AttnArgs& a, const Kv8AttnMeta& m, const Kv8AttnPlan& p, hipStream_t st) {
  const int sp = p.splits > 1, one = m.n_seqs == 1;
  kv8_attention_kernel<T, HD, FMT><<<dim3(c.n_kv, (int)p.items / (one ? p.splits : 1), one ? p.splits : 1), NWV * 64, 0, st>>>(
      c.data, (int)(c.head_bytes / kv8_block_bytes(HD)), c.n_kv, (const T*)a.q, a.q_stride, a.n_q / c.n_kv, m.chunk, a.rows, m.n_keys[0], one ? m.slot[0] : -1, sp, a, m);
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
