// Linear layers in 8-bit integers: formats, the layout of a packed weight, and what the kernels and the ABI share.
//
// A row of activations, or an output channel of a weight, is held as integers q in [-127, 127] and one fp32 scale s: x = s q.  A
// product of two such matrices is an exact integer sum, y[m][n] = s_m w_n sum_k q[m][k] c[n][k]; |sum| <= K 2^14 stays below 2^31
// for K up to Q8_MAX_K.
//
// Packed weight: units of 32 channels ("packed rows" R = 0 .. 31) by 64 k, 2 KiB each, [unit][k-tile][sub][chunk][16 rows][16 bytes]: packed row
// R = 16 sub + row, k = 64 k-tile + 16 chunk + byte.  A sub is one operand of a 16x16x64 product, lane by lane (row = lane % 16, chunk = lane / 16).  Behind the codes
// lie the scales, [unit][R] fp32.  k-tiles come in pairs; channels and k's past the end are zeros, so that whatever stands behind the last k of a row of
// activations is multiplied by zero.
//
// Which channel packed row R = 16 s + 4 g + c (s = 0, 1; g, c = 0 .. 3) is: the products leave a lane of group g four packed rows of each sub, and these are
// to be neighbours in the output:
//   plain  channel 32 unit + 8 g + 4 s + c
//   gated  s = 0: gate, s = 1: up, of output 16 unit + 4 g + c, so that a lane holds both parts of each of its outputs
#pragma once
#include "common.h"

typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int Q8_MAX_K = 131071;
constexpr int Q8_MAX_N = 1 << 24;
constexpr int Q8_MAX_WIDTH = 1 << 20;  // of rows that are quantised

struct Q8View {
  const unsigned char* codes;
  const float* scale;
  int n, k, units, kt;  // channels, inputs; units of 32 packed rows, k-tiles of 64 (an even number)
  bool gated;
  int outputs() const { return gated ? n / 2 : n; }
};
__host__ __device__ inline int q8_units(int n, int gated) { return gated ? (n / 2 + 15) / 16 : (n + 31) / 32; }
__host__ __device__ constexpr int q8_ktiles(int k) { return (k + 127) / 128 * 2; }
// the channel of packed row R of a unit (n and more: none)
__host__ __device__ inline int q8_channel(int unit, int R, int n, int gated) {
  const int s = R >> 4, g = (R >> 2) & 3, c = R & 3;
  if (!gated) return 32 * unit + 8 * g + 4 * s + c;
  const int o = 16 * unit + 4 * g + c;
  return o >= n / 2 ? n : s == 0 ? o : n / 2 + o;
}

struct Q8RowsArgs {
  const void* x;
  int64_t x_stride;
  int rows, width, dtype;
  const void* residual;  // null: none
  int64_t r_stride;
  void* h;
  int64_t h_stride;
  int h_dtype;
  const void* gain;  // null: rows are quantised as they are
  float eps;
  int8_t* codes;
  int64_t codes_stride;
  float* scale;
};
void launch_q8_rows(const Q8RowsArgs& a, hipStream_t st);
void launch_q8_pack(const int8_t* codes, int64_t stride, const float* scale, const Q8View& w, void* data, hipStream_t st);

struct Q8GemmArgs {
  const int8_t* x;
  int64_t x_stride;
  const float* x_scale;
  int M;
  void* out;
  int64_t out_stride;
  int out_dtype;
  void* workspace;
};
size_t q8_gemm_workspace(int rows, int n, int k, int gated);  // most bytes that a launch of up to that many rows needs
