// Product in 8-bit integers for few rows: the weight's bytes are what it costs.
//
// A workgroup of NWV wavefronts owns 16 MT rows of X and CS subs (16 packed channels each) of W and all of K, which its wavefronts share: each
// multiplies its k-tiles (v_mfma_i32_16x16x64_i8) from registers, DEPTH steps of W and X in flight or in use.  No barrier and no LDS in the loop; at the end the
// wavefronts' sums meet in LDS.  Sums of integers are exact, so their order is free.
// Bound by W's bytes: 8 x 12288 x 4096 in 9.0 us (5.6 TB/s), 8 x 24576 x 4096, gated, in 16.1 (6.3; a plain non-temporal read of memory reaches 7.1).  With more
// rows, or a long sum for few outputs, bands are faster (24 x 12288 x 4096 10.8 us, 14.9 here; 8 x 512 x 16000 with K split 8.5, 9.8).
#pragma once
#include "q8_gemm.h"

namespace {

template <int MT, int CS, int NWV, int DEPTH>
__global__ __launch_bounds__(64 * NWV) void q8_stream_kernel(const i32x4* __restrict__ wt, const int8_t* __restrict__ x, int64_t x_stride, int M, int K, int subs,
                                                        const float* __restrict__ wscale, const float* __restrict__ x_scale, void* __restrict__ out, int64_t out_stride, int outputs, int form) {
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
    // whole trips of DEPTH steps; the steps left over nested, not skippable one by one (a path around a step's loads is one that the compiler's count
    // of outstanding loads cannot follow: it would wait for all of them)
    auto trip = [&](auto self, auto Ic, int st) __attribute__((always_inline)) {
      constexpr int I = decltype(Ic)::value;
      if constexpr (I < DEPTH) {
        step(Ic, st + I);
        self(self, std::integral_constant<int, I + 1>{}, st);
      }
    };
    auto rest = [&](auto self, auto Ic, int st) __attribute__((always_inline)) {
      constexpr int I = decltype(Ic)::value;
      if constexpr (I < DEPTH - 1) {
        if (st + I < steps) {
          step(Ic, st + I);
          self(self, std::integral_constant<int, I + 1>{}, st);
        }
      }
    };
    int st = 0;
    for (; st + DEPTH <= steps; st += DEPTH) trip(trip, std::integral_constant<int, 0>{}, st);
    rest(rest, std::integral_constant<int, 0>{}, st);
  }

#pragma unroll
  for (int c = 0; c < CS; ++c)
#pragma unroll
    for (int j = 0; j < MT; ++j) red[(wave * F + c * MT + j) * 64 + lane] = acc[c][j];
  __syncthreads();
  auto sum = [&](int f) {
    i32x4 t = red[f * 64 + lane];
#pragma unroll
    for (int i = 1; i < NWV; ++i) t += red[(i * F + f) * 64 + lane];
    return t;
  };
  auto channels = [&](int s) { return *(const f32x4*)(wscale + 16 * s + 4 * g); };
  with_form(form, out, [&](auto gated, auto* to) __attribute__((always_inline)) {
    constexpr bool GATED = decltype(gated)::value;
    if constexpr (!GATED || CS % 2 == 0) {
      constexpr int UNITS = GATED ? CS / 2 : CS;  // what is finished together: a sub, or the gate's and the up's
      for (int i = wave; i < UNITS * MT; i += NWV) {
        const int c = i / MT * (GATED ? 2 : 1), j = i % MT, s = sub0 + c, m = m0 + 16 * j + ml;
        if (s >= subs || m >= M) continue;
        const float xs = x_scale[m];
        auto* row = to + (int64_t)m * out_stride;
        if constexpr (GATED) {
          const f32x4 gate = scaled(sum(c * MT + j), xs, channels(s)), up = scaled(sum((c + 1) * MT + j), xs, channels(s + 1));
          store4(row, 8 * s + 4 * g, outputs, gated_unit(gate, up));
        } else {
          store4(row, 32 * (s >> 1) + 8 * g + 4 * (s & 1), outputs, scaled(sum(c * MT + j), xs, channels(s)));
        }
      }
    }
  });
}

template <int MT, int CS, int NWV, int DEPTH>
void launch_stream(const Q8View& w, const Q8GemmArgs& a, hipStream_t st) {
  constexpr int LDS = NWV * CS * MT * 1024;
  static_assert(LDS <= 160 * 1024, "the sums' meeting");
  auto kernel = q8_stream_kernel<MT, CS, NWV, DEPTH>;
  static bool configured = false;
  if (!configured) {
    (void)hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
    configured = true;
  }
  const int subs = 2 * w.units;
  kernel<<<dim3((subs + CS - 1) / CS, (a.M + 16 * MT - 1) / (16 * MT)), 64 * NWV, LDS, st>>>((const i32x4*)w.codes, a.x, a.x_stride, a.M, w.k, subs, w.scale, a.x_scale,
                                                                                            a.out, a.out_stride, w.outputs(), out_form(w, a));
}

}  // namespace
