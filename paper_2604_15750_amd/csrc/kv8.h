// The 8-bit KV cache: its layout, its two formats, and what the kernels that write, read and attend to it share.
//
// A cached vector (K or V of one position and kv head) is held as 8-bit codes and one power-of-two scale 2^E.  The power of two
// makes every step of quantising exact (a vector's codes depend on its values alone, not on the order or precision of any
// arithmetic), costs e4m3 nothing (its steps are relative) and i8 half a bit on average, and takes one byte.
//
// Memory: per (slot, kv head) blocks of 32 positions, each one run of 64 * head_dim + 64 bytes, in the order in which the attention
// feeds the matrix cores:
//   K codes   operand fragments (16 positions x 32 dims, 8 bytes a lane) paired into 1 KiB pieces of 16 bytes a lane
//   V codes   operand fragments (16 dims x 32 positions), paired the same way; a lane's 8 bytes hold positions {4g..4g+3, 16+4g..16+4g+3}:
//             the order in which the first product leaves the keys in a lane's registers
//   scales    for g = 0..3 the bytes of K at positions 4g.., 16+4g.., then of V: what lane group g needs is 16 bytes
// so a wavefront reads a block of 32 positions in HD / 16 loads of 1 KiB and one of 64 bytes, all from one run of memory.
#pragma once
#include "common.h"

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));

__host__ __device__ constexpr int kv8_block_bytes(int hd) { return 64 * hd + 64; }
// byte offsets inside a block (p: position in it)
__host__ __device__ inline int kv8_k_index(int p, int d, int hd) {
  const int f = (p >> 4) * (hd >> 5) + (d >> 5), lane = (p & 15) + 16 * ((d & 31) >> 3);
  return (f >> 1) * 1024 + lane * 16 + (f & 1) * 8 + (d & 7);
}
__host__ __device__ inline int kv8_v_index(int p, int d, int hd) {
  const int f = d >> 4, lane = (d & 15) + 16 * ((p & 15) >> 2);
  return 32 * hd + (f >> 1) * 1024 + lane * 16 + (f & 1) * 8 + (p & 3) + 4 * (p >> 4);
}
__host__ __device__ inline int kv8_scale_index(int p, int is_v, int hd) { return 64 * hd + ((p & 15) >> 2) * 16 + is_v * 8 + (p >> 4) * 4 + (p & 3); }

// Scales: a byte E + 127, E in [-60, 60]; 255 marks a vector that had a NaN or an infinity (its codes are zero, it reads as NaN); 0 is
// a position that was never written (it reads as zero).  The range of E is what lets the attention keep the V scale inside the
// softmax's exponent in 32 bits whatever the scales of the keys are (kv8_attention.hip).
constexpr int KV8_E_MAX = 60;
constexpr unsigned KV8_NAN = 255;

struct Kv8Meta {  // the spans of a write or a read
  int32_t n_seqs;
  int32_t row_off[DLM_MAX_SEQS + 1];
  int32_t start[DLM_MAX_SEQS];       // cached position of a sequence's first row
  int32_t slot[DLM_MAX_SEQS];
  int32_t block_off[DLM_MAX_SEQS + 1];  // blocks of 32 positions the spans touch, all sequences' before this one's
};
struct Kv8View {
  unsigned char* data;
  int64_t head_bytes;  // of one (slot, kv head)
  int n_kv;
};
struct Kv8AttnMeta {
  int32_t n_seqs, chunk;             // chunk: 32-position blocks of a split's share of the keys
  int32_t row_off[DLM_MAX_SEQS + 1];
  int32_t n_keys[DLM_MAX_SEQS];
  int32_t slot[DLM_MAX_SEQS];
  int32_t item_off[DLM_MAX_SEQS + 1];  // (query tiles x splits), all sequences' before this one's
};

// the sequence whose range of off[] holds i: a lane per boundary (a loop over them is a chain of loads); called by whole wavefronts
__device__ inline int seq_of(const int32_t* off, int n_seqs, int i) {
  const int lane = threadIdx.x & 63;
  return __popcll(__ballot(lane < DLM_MAX_SEQS && lane + 1 < n_seqs && i >= off[min(lane, DLM_MAX_SEQS - 1) + 1]));
}

void launch_kv8_write(const Kv8View& c, int format, int hd, const void* k, const void* v, int64_t stride, int dtype, const Kv8Meta& m, hipStream_t st);
void launch_kv8_read(const Kv8View& c, int format, int hd, void* k, void* v, int64_t stride, int dtype, const Kv8Meta& m, hipStream_t st);
struct Kv8AttnPlan {
  int tiles;    // 16-query tiles of a workgroup
  int waves;    // its wavefronts
  int chunk;    // 32-position blocks of a split's share of the keys
  int splits;   // most shares of a sequence (1: the workgroups write the output)
  int64_t items;
};
Kv8AttnPlan kv8_attention_plan(const int32_t* row_off, const int32_t* n_keys, int n_seqs, int n_q, int n_kv, int hd, int dtype);
size_t kv8_attention_partials(int64_t rows, int n_q);  // most (split, row, head) triples a plan for that many rows has
struct Kv8AttnArgs {
  const void* q;
  int64_t q_stride;
  void* out;
  const uint32_t* mask;
  int mask_words, n_q, rows;
  float *part, *part_ml;  // splits > 1: [split][row][n_q] partial outputs and (maximum, sum) pairs
};
void launch_kv8_attention(const Kv8View& c, int format, int hd, int dtype, const Kv8AttnArgs& a, const Kv8AttnMeta& m, const Kv8AttnPlan& p, hipStream_t st);
void launch_qk_norm_rope(const void* x, int64_t x_stride, int rows, int n_q, int n_kv, int hd, int dtype, const void* q_gain, const void* k_gain, float eps,
                         float theta, const int32_t* positions, void* out, int64_t out_stride, hipStream_t st);
