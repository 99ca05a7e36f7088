// Product in 8-bit integers for up to some hundred rows: bands of the output, X through LDS, W from memory to registers.
//
// A workgroup of CW wavefronts owns 32 WM rows of X (tokens) x 32 CW packed rows of W, a wavefront one unit of W and all of the rows; it walks K in stages of 128.
// Nobody else in the workgroup uses a wavefront's share of W, so it goes straight to registers, S stages ahead, in the order in which the products take it: a load
// is 1 KiB of consecutive bytes.  X's rows go through LDS, S stages too, as in q8_tile.h.
// One barrier a stage, in front of its last step.
//
// Bound by W's way from memory and X's from the L2s together: 152 x 37888 x 3584 takes 33 to 35 us for 136 MB of W, 27 to 30 when X is a single row.  Against tiles of the same rows with
// W through LDS: 152 x 37888 x 3584 35.2 us there, 152 x 12288 x 4096 19.9 (17.6 here), 90 x 37888 x 3584 32.9 (28), 152 x 4096 x 12288 22.4 (20.1).  Where one row block reads W it is read
// non-temporally, past the memory-side cache, in which the weights of a model do not stay from pass to pass (2 to 3 %); where two do, that costs 7 to 11 %.
// More stages than S do not help (152 x 37888 x 3584 34.6 us with 4 and with 5).
#pragma once
#include "q8_gemm.h"
#include "q8_plan.h"

namespace {

template <int WM, int CW, int S>
struct Q8Band {
  static constexpr int TPB = CW * 64, BM = 32 * WM;
  static constexpr int X_LOADS = BM / 8;                               // copies of 1 KiB (8 rows), a stage
  static constexpr int LPX = (X_LOADS + CW - 1) / CW, LPS = LPX + 4;  // ... of a wavefront (some have surplus ones); with its loads of W
  static constexpr int STAGE = X_LOADS * 1024, LDS_BYTES = S * STAGE;
  static_assert(S >= 3 && LDS_BYTES <= 160 * 1024 && S * LPS <= 63, "band shape");
};

template <int WM, int CW, int S, bool NT>
__global__ __launch_bounds__(CW * 64, CW > 4 ? (CW + 3) / 4 : 2) void q8_band_kernel(const unsigned char* __restrict__ wt, const int8_t* __restrict__ x, int x_stride, int M, int K, int units,
                                                                                     int nblocks, int mblocks, int splits, int split_stages, const float* __restrict__ wscale,
                                                                                     const float* __restrict__ x_scale, void* __restrict__ out, int64_t out_stride, int outputs, int form,
                                                                                     i32x4* __restrict__ parts) {
  typedef Q8Band<WM, CW, S> SH;
  constexpr int BM = SH::BM, LPX = SH::LPX, LPS = SH::LPS, STAGE = SH::STAGE, LOADS = SH::X_LOADS, FM = 2 * WM;
  extern __shared__ __align__(16) unsigned char lds[];

  const Q8At at = tile_of(blockIdx.x, nblocks, mblocks, splits);
  if (at.split < 0) return;  // (the whole workgroup)
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int KTP = (K + 127) >> 7 << 1;                                                                                   // k-tiles of a unit in memory
  const int s0 = at.split * split_stages, nst = min(((K + 63) / 64 + 1) / 2 - s0, split_stages);  // this workgroup's stages s0 .. s0 + nst - 1
  const int u0 = at.cb * CW, m0 = at.rb * BM, mrows = min(BM, M - m0), u = min(u0 + wave, units - 1);

  // Rows past the end are the last one again, chunks past a row's last are that one again (W is zero there): every address is one of the operands'
  const __amdgpu_buffer_rsrc_t wr = __builtin_amdgcn_make_buffer_rsrc((void*)(wt + (int64_t)u * KTP * 2048), 0, KTP * 2048, 0x00020000);
  const __amdgpu_buffer_rsrc_t xr = __builtin_amdgcn_make_buffer_rsrc((void*)(x + (int64_t)m0 * x_stride), 0, (mrows - 1) * x_stride + (K + 15) / 16 * 16, 0x00020000);
  // X's copies: wavefront w moves the ones congruent w mod CW; 8 chunks of 16 bytes of 8 rows each, a chunk's place turned by half its row's number
  auto load_of = [&](int i) { const int f = i * CW + wave; return f < LOADS ? f : LOADS - 2 + (f & 1); };  // (surplus ones repeat one of the last two)
  int off[LPX];
#pragma unroll
  for (int i = 0; i < LPX; ++i) off[i] = min(load_of(i) * 8 + lane / 8, mrows - 1) * x_stride;
  const int my_chunk = ((lane & 7) ^ ((wave & 1) * 4 + lane / 16)) * 16, other_chunk = my_chunk ^ 64;  // (of the copies i CW + wave with i CW even, and odd)
  const int k_last = (K + 15) / 16 * 16 - 16;
  auto copy_x = [&](int s, int buf, int lo, int hi) __attribute__((always_inline)) {
    const int t = s0 + min(s, nst - 1), left = k_last - t * 128, chunk = min(my_chunk, left), chunk2 = min(other_chunk, left);
#pragma unroll
    for (int i = lo; i < hi; ++i) copy_to_lds(xr, lds + buf * STAGE + load_of(i) * 1024, off[i] + ((i * CW) % 2 ? chunk2 : chunk), t * 128);
  };
  auto load_w = [&](i32x4 (&to)[2], int s, int q) __attribute__((always_inline)) {
    const int t = s0 + min(s, nst - 1);
#pragma unroll
    for (int j = 0; j < 2; ++j) to[j] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(wr, lane * 16 + q * 2048 + j * 1024, t * 4096, NT ? 2 : 0));
  };

  i32x4 acc[2][FM], xf[2][FM], wf[S][2][2];
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int i = 0; i < FM; ++i) acc[j][i] = i32x4(0);
  const int row = lane & 15, part = lane >> 4, turn = row >> 1;
  auto read_x = [&](int set, int buf, int q) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < FM; ++i) xf[set][i] = *(const i32x4*)(lds + buf * STAGE + (16 * i + row) * 128 + (((4 * q + part) ^ turn) << 4));
  };

  // Stages 0 .. S - 2 and the first half of S - 1's X go out at once; the rest of it during stage 0, as for every later stage
#pragma unroll
  for (int s = 0; s < S; ++s) {
    copy_x(s, s, 0, s < S - 1 ? LPX : LPX / 2);
#pragma unroll
    for (int q = 0; q < 2; ++q) load_w(wf[s][q], s, q);
    __builtin_amdgcn_sched_barrier(0);
  }
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"((S - 2) * LPS + LPX / 2 + 4) : "memory");  // stage 0 has landed (this wavefront's share)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  read_x(0, 0, 0);
  __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
  // step Q of stage s, which is in LDS buffer and register set R
  auto step = [&](auto Rc, auto Qc, int s) __attribute__((always_inline)) {
    constexpr int R = decltype(Rc)::value, Q = decltype(Qc)::value, LO = Q ? 0 : LPX / 2, HI = Q ? LPX / 2 : LPX;
    if (Q) {
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"((S - 2) * LPS) : "memory");  // stage s + 1 has landed
      __builtin_amdgcn_s_barrier();  // ... for every wavefront, and every wavefront has read the last of stage s
      asm volatile("" ::: "memory");
    }
    __builtin_amdgcn_sched_barrier(0);
    if (Q) copy_x(s + S, R, LO, HI);
    else copy_x(s + S - 1, (R + S - 1) % S, LO, HI);
    read_x(Q ^ 1, Q ? (R + 1) % S : R, Q ^ 1);
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int i = 0; i < FM; ++i) acc[j][i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wf[R][Q][j], xf[Q][i], acc[j][i], 0, 0, 0);
    constexpr int NM = 2 * FM, LI = HI - LO, OPS = 2 * (LI + FM) <= NM ? 1 : LI + FM <= NM ? 2 : 4;
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
#pragma unroll
    for (int i = 0; i < FM; i += OPS) {
      __builtin_amdgcn_sched_group_barrier(0x100, OPS, 0);  // LDS reads
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);    // one product
    }
#pragma unroll
    for (int i = 0; i < LI; i += OPS) {
      __builtin_amdgcn_sched_group_barrier(0x010, OPS, 0);  // copies to LDS
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, NM, 0);
    __builtin_amdgcn_sched_barrier(0);
    load_w(wf[R][Q], s + S, Q);  // where this step's were
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): the reads have had the products' time to complete
  };
  // whole trips of S stages; the stages left over nested, not skippable one by one (a path around a stage's loads is one that the compiler's count of outstanding
  // loads cannot follow: it would wait for all of them)
  auto stages = [&](auto self, auto Rc, int s, int last) __attribute__((always_inline)) {
    constexpr int R = decltype(Rc)::value;
    if constexpr (R < S) {
      if (s < last) {
        step(Rc, std::integral_constant<int, 0>{}, s);
        step(Rc, std::integral_constant<int, 1>{}, s);
        self(self, std::integral_constant<int, R + 1>{}, s + 1, last);
      }
    }
  };
  auto trip = [&](auto self, auto Rc, int s) __attribute__((always_inline)) {
    constexpr int R = decltype(Rc)::value;
    if constexpr (R < S) {
      step(Rc, std::integral_constant<int, 0>{}, s);
      step(Rc, std::integral_constant<int, 1>{}, s);
      self(self, std::integral_constant<int, R + 1>{}, s + 1);
    }
  };
  int s = 0;
  for (; s + S <= nst; s += S) trip(trip, std::integral_constant<int, 0>{}, s);
  stages(stages, std::integral_constant<int, 0>{}, s, nst);
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the surplus copies of the last stages land before the workgroup's LDS is another's

  finish_tile<1, WM>(acc, u0 + wave, m0, lane, at.split, splits, M, units, wscale, x_scale, out, out_stride, outputs, form, parts);
}

template <int WM, int CW, int S, bool NT>
void launch_band(const Q8View& w, const Q8GemmArgs& a, const Q8TilePlan& p, hipStream_t st) {
  typedef Q8Band<WM, CW, S> SH;
  static bool configured = false;  // raise the dynamic LDS limit of this instantiation once
  if (!configured) {
    (void)hipFuncSetAttribute((const void*)q8_band_kernel<WM, CW, S, NT>, hipFuncAttributeMaxDynamicSharedMemorySize, SH::LDS_BYTES);
    configured = true;
  }
  q8_band_kernel<WM, CW, S, NT><<<(p.nblocks * p.mblocks * p.splits + 7) / 8 * 8, SH::TPB, SH::LDS_BYTES, st>>>(
      w.codes, a.x, (int)a.x_stride, a.M, w.k, w.units, p.nblocks, p.mblocks, p.splits, p.stages, w.scale, a.x_scale, a.out, a.out_stride, w.outputs(), out_form(w, a), (i32x4*)a.workspace);
}

}  // namespace
