// Product in 8-bit integers for many rows: tiles of the output, both operands through LDS.
//
// A workgroup of RW x CW wavefronts owns 32 RW WM rows of X (tokens) x 32 CW WN packed rows of W (RW = 2, CW = 4) and walks K in stages of KB k-tiles of
// 64:
//   * W's units lie in memory as the products take them, so a stage of them is copied to LDS as it is; X's rows are 64 KB bytes of each of the tile's
//     rows, in 16-byte chunks whose place in the row is turned by the row's number, so that 16 lanes that read the same chunk of 16 rows
//     meet 16 different banks' groups.  Both by direct-to-LDS loads, S stages of them in flight or in use;
//   * a wavefront multiplies its fragments of a step of 64 k (v_mfma_i32_16x16x64_i8) while it reads the next step's from LDS;
//   * one barrier a stage, in front of its last step: by then every wavefront has the stage's last fragments in registers, and the copies of
//     stage s + S go out over the steps that follow.
//
// 2822 x 12288 x 4096 takes 128 us (2.2 POP/s), 2048 x 37888 x 3584, gated, 247 (2.3).  Bound by a workgroup's own cycles, there being one a compute unit: a tile of
// 256 x 256 takes 2800 for a stage of 128 k, 2048 of which the matrix cores are busy, and 20000 to fill and to finish (4096 x 8192, two tiles a compute unit, 130, 221, 399 and
// 756 thousand with k of 2048, 4096, 8192 and 16384: 50, 59, 66 and 69 % busy).  Power sets their length: codes that are all zero take as many cycles, at 2.26 to 2.33 GHz
// instead of 1.93 to 2.01 (108 us for 128).  With products of 32x32x32 4096 x 8192 x 8192 took 233 us (210 with 16x16x64).  Slower: four
// wavefronts of 128 x 128 (2048 x 32768 x 3584 287 us, 210 here: the accumulators do not leave the fragments enough registers), K begun
// elsewhere by each workgroup, X and W in rings of different depth.
#pragma once
#include "q8_gemm.h"
#include "q8_plan.h"

namespace {

template <int WM, int WN, int KB>
struct Q8Tile {
  static constexpr int RW = 2, CW = 4, NW = RW * CW, TPB = NW * 64, BM = 32 * RW * WM, UN = CW * WN;  // rows of X, units of W
  static constexpr int W_LOADS = UN * KB * 2, X_LOADS = BM * KB / 16;                 // of 1 KiB, a stage
  static constexpr int LPS = (W_LOADS + X_LOADS + NW - 1) / NW;                       // ... of a wavefront (some have surplus ones)
  static constexpr int W_BYTES = W_LOADS * 1024, STAGE = W_BYTES + X_LOADS * 1024;
  static constexpr int S_FIT = 160 * 1024 / STAGE, S_CNT = 63 / LPS + 1, S_ = S_FIT < S_CNT ? S_FIT : S_CNT, S = S_ > 6 ? 6 : S_;
  static constexpr int LDS_BYTES = S * STAGE;
  static_assert(W_LOADS % NW == 0 && X_LOADS % 2 == 0 && S >= 2 && (KB == 1 || KB == 2) && LDS_BYTES <= 160 * 1024, "tile shape");
};

template <int WM, int WN, int KB>
__global__ __launch_bounds__(512, 2) void q8_tile_kernel(const unsigned char* __restrict__ wt, const int8_t* __restrict__ x, int x_stride, int M, int K, int units, int nblocks, int mblocks,
                                                         int splits, int split_stages, const float* __restrict__ wscale, const float* __restrict__ x_scale, void* __restrict__ out,
                                                         int64_t out_stride, int outputs, int form, i32x4* __restrict__ parts) {
  typedef Q8Tile<WM, WN, KB> SH;
  constexpr int CW = SH::CW, NW = SH::NW, BM = SH::BM, UN = SH::UN, LPS = SH::LPS, STAGE = SH::STAGE, S = SH::S, W_LOADS = SH::W_LOADS, LOADS = W_LOADS + SH::X_LOADS;
  extern __shared__ __align__(16) unsigned char lds[];

  const Q8At at = tile_of(blockIdx.x, nblocks, mblocks, splits);
  if (at.split < 0) return;  // (the whole workgroup)
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / CW, wn = wave % CW;
  const int KTP = (K + 127) >> 7 << 1;                                       // k-tiles of a unit in memory
  const int s0 = at.split * split_stages, nst = min(((K + 63) / 64 + KB - 1) / KB - s0, split_stages);  // this workgroup's stages s0 .. s0 + nst - 1
  const int u0 = at.cb * UN, m0 = at.rb * BM, mrows = min(BM, M - m0), nunits = min(UN, units - u0);

  // Direct-to-LDS loads, 1 KiB each: wavefront w moves the ones congruent w mod NW, W's first.  Rows and units past the end are the last one again, chunks
  // past a row's last are that one again (W is zero there): every address is one of the operands'.
  const __amdgpu_buffer_rsrc_t wr = __builtin_amdgcn_make_buffer_rsrc((void*)(wt + (int64_t)u0 * KTP * 2048), 0, nunits * KTP * 2048, 0x00020000);
  const __amdgpu_buffer_rsrc_t xr = __builtin_amdgcn_make_buffer_rsrc((void*)(x + (int64_t)m0 * x_stride), 0, (mrows - 1) * x_stride + (K + 15) / 16 * 16, 0x00020000);
  constexpr int CPR = 4 * KB, RPL = 64 / CPR;  // chunks of a row, rows of a load
  auto load_of = [&](int i) { const int f = i * NW + wave; return f < LOADS ? f : LOADS - 2 + (f & 1); };  // (surplus ones repeat one of the last two)
  int off[LPS];
#pragma unroll
  for (int i = 0; i < LPS; ++i) {
    const int f = load_of(i);
    if (i * NW < W_LOADS) {
      off[i] = min(f / (2 * KB), nunits - 1) * (KTP * 2048) + f % (2 * KB) * 1024 + lane * 16;
    } else {
      off[i] = min((f - W_LOADS) * RPL + lane / CPR, mrows - 1) * x_stride;
    }
  }
  // (a load's rows begin at a multiple of RPL: their numbers mod 16 are a lane's own, or one of two where RPL is 8)
  auto chunk_of = [&](int odd) { const int row = odd * 8 + lane / CPR; return ((lane % CPR) ^ (KB == 2 ? row >> 1 : row >> 2)) * 16; };
  const int my_chunk = chunk_of(RPL == 8 ? wave & 1 : 0), other_chunk = my_chunk ^ 64;  // (of the loads i NW + wave with i NW even, and odd)
  static_assert(W_LOADS % 2 == 0, "X's loads are counted from an even number");
  const int k_last = (K + 15) / 16 * 16 - 16;
  auto issue = [&](int s, int buf, int lo, int hi) __attribute__((always_inline)) {
    const int t = s0 + min(s, nst - 1);
    const int left = k_last - t * (64 * KB), chunk = min(my_chunk, left), chunk2 = min(other_chunk, left);
#pragma unroll
    for (int i = lo; i < hi; ++i) {
      unsigned char* dst = lds + buf * STAGE + load_of(i) * 1024;
      if (i * NW < W_LOADS) copy_to_lds(wr, dst, off[i], t * (KB * 2048));
      else copy_to_lds(xr, dst, off[i] + (RPL == 8 && (i * NW) % 2 ? chunk2 : chunk), t * (64 * KB));
    }
  };

  constexpr int FM = 2 * WM, FN = 2 * WN;  // fragments of 16 rows
  i32x4 acc[FN][FM];
  i32x4 xf[2][FM], wf[2][FN];
#pragma unroll
  for (int j = 0; j < FN; ++j)
#pragma unroll
    for (int i = 0; i < FM; ++i) acc[j][i] = i32x4(0);
  const int row = lane & 15, part = lane >> 4, turn = KB == 2 ? row >> 1 : row >> 2;  // lane -> row of a fragment, which of a k-tile's chunks it has
  auto read_frags = [&](int set, int buf, int q) __attribute__((always_inline)) {
    const unsigned char* st = lds + buf * STAGE;
#pragma unroll
    for (int j = 0; j < FN; ++j) wf[set][j] = *(const i32x4*)(st + ((wn * WN + j / 2) * KB + q) * 2048 + (j & 1) * 1024 + lane * 16);
#pragma unroll
    for (int i = 0; i < FM; ++i) xf[set][i] = *(const i32x4*)(st + SH::W_BYTES + (wm * WM * 32 + 16 * i + row) * (64 * KB) + (((4 * q + part) ^ turn) << 4));
  };
  auto multiply = [&](int set) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int i = 0; i < FM; ++i) acc[j][i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wf[set][j], xf[set][i], acc[j][i], 0, 0, 0);
  };

  // stages 0 .. S - 2 and the first part of S - 1 go out at once; the rest of it during stage 0, as for every later stage
#pragma unroll
  for (int s = 0; s < S - 1; ++s) issue(s, s, 0, LPS);
  issue(S - 1, S - 1, 0, LPS / KB);
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"((S - 2) * LPS + LPS / KB) : "memory");  // stage 0 has landed (this wavefront's share)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  read_frags(0, 0, 0);
  __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
  // step Q of stage s (in LDS buffer buf), whose operands are in register set SET
  auto step = [&](auto Qc, auto SETc, int s, int buf, int nbuf) __attribute__((always_inline)) {
    constexpr int Q = decltype(Qc)::value, SET = decltype(SETc)::value;
    constexpr bool LAST = Q == KB - 1;
    constexpr int LO = LAST ? 0 : LPS * (Q + 1) / KB, HI = LAST ? LPS / KB : LPS * (Q + 2) / KB;
    if (LAST) {
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"((S - 2) * LPS) : "memory");  // stage s + 1 has landed
      __builtin_amdgcn_s_barrier();  // ... for every wavefront, and every wavefront has read the last of stage s
      asm volatile("" ::: "memory");
    }
    __builtin_amdgcn_sched_barrier(0);
    if (LAST) issue(s + S, buf, LO, HI);
    else issue(s + S - 1, buf == 0 ? S - 1 : buf - 1, LO, HI);
    read_frags(SET ^ 1, LAST ? nbuf : buf, LAST ? 0 : Q + 1);
    multiply(SET);
    constexpr int NM = FN * FM, RF = FM + FN, LI = HI - LO;
    constexpr int OPS = 2 * (LI + RF) <= NM ? 1 : LI + RF <= NM ? 2 : 4;
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
#pragma unroll
    for (int i = 0; i < RF; i += OPS) {
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
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): the reads have had the products' time to complete
  };
  typedef std::integral_constant<int, 0> Zero;
  typedef std::integral_constant<int, 1> One;
  auto next = [](int b) { return b + 1 == S ? 0 : b + 1; };
  int buf = 0;
  if constexpr (KB == 2) {
    for (int s = 0; s < nst; ++s, buf = next(buf)) {
      step(Zero{}, Zero{}, s, buf, next(buf));
      step(One{}, One{}, s, buf, next(buf));
    }
  } else {  // two stages a trip, so that each register set has its place
    int s = 0;
    for (; s + 1 < nst; s += 2, buf = next(buf)) {
      step(Zero{}, Zero{}, s, buf, next(buf));
      buf = next(buf);
      step(Zero{}, One{}, s + 1, buf, next(buf));
    }
    if (s < nst) step(Zero{}, Zero{}, s, buf, next(buf));
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the surplus loads of the last stages land before the workgroup's LDS is another's

  finish_tile<WN, WM>(acc, u0 + wn * WN, m0 + wm * WM * 32, lane, at.split, splits, M, units, wscale, x_scale, out, out_stride, outputs, form, parts);
}

template <int WM, int WN, int KB>
void launch_tile(const Q8View& w, const Q8GemmArgs& a, const Q8TilePlan& p, hipStream_t st) {
  typedef Q8Tile<WM, WN, KB> SH;
  static bool configured = false;  // raise the dynamic LDS limit of this instantiation once
  if (!configured) {
    (void)hipFuncSetAttribute((const void*)q8_tile_kernel<WM, WN, KB>, hipFuncAttributeMaxDynamicSharedMemorySize, SH::LDS_BYTES);
    configured = true;
  }
  q8_tile_kernel<WM, WN, KB><<<(p.nblocks * p.mblocks * p.splits + 7) / 8 * 8, SH::TPB, SH::LDS_BYTES, st>>>(
      w.codes, a.x, (int)a.x_stride, a.M, w.k, w.units, p.nblocks, p.mblocks, p.splits, p.stages, w.scale, a.x_scale, a.out, a.out_stride, w.outputs(), out_form(w, a),
      (i32x4*)a.workspace);
}

}  // namespace
