// Product in 8-bit integers for few rows: the weight's bytes are what it costs.
//
// A workgroup of four wavefronts owns up to 64 rows of X and CS subs (16 packed channels each) of W and all of K, which its wavefronts share: each
// multiplies its k-tiles (v_mfma_i32_16x16x64_i8) from registers, three steps of W and X in flight, W non-temporally (one workgroup reads it, once).
// No barrier and no LDS in the loop; at the end the four sums meet in LDS.  Sums of integers are exact, so their order is free.
#include <type_traits>

#include "q8_gemm.h"

namespace {

constexpr int NWV = 4, DEPTH = 3;

template <int MT, int CS, bool GATED, typename TO>
__global__ __launch_bounds__(256) void q8_stream_kernel(const i32x4* __restrict__ wt, const int8_t* __restrict__ x, int64_t x_stride, int M, int K, int subs,
                                                        const float* __restrict__ wscale, const float* __restrict__ x_scale, TO* __restrict__ out, int64_t out_stride, int outputs) {
  extern __shared__ __align__(16) i32x4 red[];  // [NWV][CS * MT][64]
  constexpr int F = CS * MT;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, ml = lane & 15;
  const int KT = (K + 63) >> 6, KTP = q8_ktiles(K), KC = (K + 15) >> 4, sub0 = blockIdx.x * CS, m0 = blockIdx.y * (16 * MT);
  const int per = (KT + NWV - 1) / NWV, t0 = wave * per, t1 = min(KT, t0 + per), steps = t1 - t0;  // this wavefront's k-tiles (possibly none)

  const i32x4* wp[CS];
#pragma unroll
  for (int c = 0; c < CS; ++c) {
    const int s = min(sub0 + c, subs - 1);
    wp[c] = wt + ((int64_t)(s >> 1) * KTP * 2 + (s & 1)) * 64 + lane;
  }
  const int8_t* xp[MT];
#pragma unroll
  for (int j = 0; j < MT; ++j) xp[j] = x + (int64_t)min(m0 + 16 * j + ml, M - 1) * x_stride;

  i32x4 acc[CS][MT], w[DEPTH][CS], v[DEPTH][MT];
#pragma unroll
  for (int c = 0; c < CS; ++c)
#pragma unroll
    for (int j = 0; j < MT; ++j) acc[c][j] = i32x4{0, 0, 0, 0};
  auto load = [&](int slot, int st) __attribute__((always_inline)) {
    const int t = min(t0 + st, t1 - 1), chunk = min(4 * t + g, KC - 1);  // (behind the last chunk of a row the weight is zero)
#pragma unroll
    for (int j = 0; j < MT; ++j) v[slot][j] = *(const i32x4*)(xp[j] + 16 * (int64_t)chunk);
#pragma unroll
    for (int c = 0; c < CS; ++c) w[slot][c] = __builtin_nontemporal_load(wp[c] + (int64_t)t * 128);
  };
  auto step = [&](auto Sc, int st) __attribute__((always_inline)) {
    constexpr int S = decltype(Sc)::value;
    load((S + DEPTH - 1) % DEPTH, st + DEPTH - 1);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int c = 0; c < CS; ++c)
#pragma unroll
      for (int j = 0; j < MT; ++j) acc[c][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[S][c], v[S][j], acc[c][j], 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
  };
  if (steps > 0) {
#pragma unroll
    for (int i = 0; i < DEPTH - 1; ++i) load(i, i);
    int st = 0;
    for (; st + DEPTH <= steps; st += DEPTH) {
      step(std::integral_constant<int, 0>{}, st);
      step(std::integral_constant<int, 1>{}, st + 1);
      step(std::integral_constant<int, 2>{}, st + 2);
    }
    if (st < steps) step(std::integral_constant<int, 0>{}, st);
    if (st + 1 < steps) step(std::integral_constant<int, 1>{}, st + 1);
  }

#pragma unroll
  for (int c = 0; c < CS; ++c)
#pragma unroll
    for (int j = 0; j < MT; ++j) red[(wave * F + c * MT + j) * 64 + lane] = acc[c][j];
  __syncthreads();
  auto sum = [&](int f) {
    return red[f * 64 + lane] + red[(F + f) * 64 + lane] + red[(2 * F + f) * 64 + lane] + red[(3 * F + f) * 64 + lane];
  };
  auto channels = [&](int s) { return *(const f32x4*)(wscale + 16 * s + 4 * g); };
  constexpr int UNITS = GATED ? CS / 2 : CS;  // what is finished together: a sub, or the gate's and the up's
  for (int i = wave; i < UNITS * MT; i += NWV) {
    const int c = i / MT * (GATED ? 2 : 1), j = i % MT, s = sub0 + c, m = m0 + 16 * j + ml;
    if (s >= subs || m >= M) continue;
    const float xs = x_scale[m];
    TO* row = out + (int64_t)m * out_stride;
    if (GATED) {
      const f32x4 gate = scaled(sum(c * MT + j), xs, channels(s)), up = scaled(sum((c + 1) * MT + j), xs, channels(s + 1));
      store4(row, 8 * s + 8 * (g & 1) + 4 * (g >> 1), outputs, gated_unit(gate, up));
    } else {
      store4(row, 32 * (s >> 1) + 16 * (g & 1) + 8 * (s & 1) + 4 * (g >> 1), outputs, scaled(sum(c * MT + j), xs, channels(s)));
    }
  }
}

template <int MT, int CS, bool GATED, typename TO>
void launch_one(const Q8View& w, const Q8GemmArgs& a, hipStream_t st) {
  constexpr int LDS = NWV * CS * MT * 1024;
  static bool configured = false;
  if (!configured) {
    (void)hipFuncSetAttribute((const void*)q8_stream_kernel<MT, CS, GATED, TO>, hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
    configured = true;
  }
  const int subs = 2 * w.units;
  q8_stream_kernel<MT, CS, GATED, TO><<<dim3((subs + CS - 1) / CS, (a.M + 16 * MT - 1) / (16 * MT)), 256, LDS, st>>>(
      (const i32x4*)w.codes, a.x, a.x_stride, a.M, w.k, subs, w.scale, a.x_scale, (TO*)a.out, a.out_stride, w.outputs());
}
template <bool GATED, typename TO>
void launch_rows(const Q8View& w, const Q8GemmArgs& a, hipStream_t st) {
  if (a.M <= 16) launch_one<1, 2, GATED, TO>(w, a, st);
  else if (a.M <= 32) launch_one<2, 2, GATED, TO>(w, a, st);
  else launch_one<4, 2, GATED, TO>(w, a, st);
}

}  // namespace

void launch_q8_stream(const Q8View& w, const Q8GemmArgs& a, hipStream_t st) {
  if (a.out_dtype == DLM_BF16) w.gated ? launch_rows<true, bf16_t>(w, a, st) : launch_rows<false, bf16_t>(w, a, st);
  else w.gated ? launch_rows<true, float>(w, a, st) : launch_rows<false, float>(w, a, st);
}
