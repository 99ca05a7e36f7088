// The 8-bit KV cache: its layout, its two formats, and what the kernels that write, read and attend to it share.
//
// A cached vector (K or V of one position and kv head) is held as 8-bit codes and one power-of-two scale 2^E.  The power of two
// makes every step of quantising exact (a vector's codes depend on its values alone, not on the order or precision of any
// arithmetic), costs e4m3 nothing (its steps are relative) and i8 half a bit on average, and takes one byte.
//
// Memory: per (slot, kv head) blocks of 32 positions, each one run of 64 * head_dim + 64 bytes, in the order in which the attention
// feeds the matrix cores (32x32x16 products; h = 0, 1: the half of a wavefront):
//   K codes   per 32 dims 1 KiB: 16 bytes a lane, position lane % 32, dims 16h .. 16h + 15
//   V codes   per 32 dims 1 KiB: 16 bytes a lane, dim lane % 32, positions 8j + 4h + i at byte 4j + i (j, i = 0..3): the order in which
//             the first product leaves the keys in a lane's registers
//   scales    32 bytes of K, 32 of V, by position
// so a wavefront reads a block of 32 positions in HD / 16 loads of 1 KiB and two of a byte a lane, all from one run of memory.
#pragma once
#include "common.h"

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));

__host__ __device__ constexpr int kv8_block_bytes(int hd) { return 64 * hd + 64; }
// byte offsets inside a block (p: position in it)
__host__ __device__ inline int kv8_k_index(int p, int d, int) { return (d >> 5) * 1024 + (p + (d & 16) * 2) * 16 + (d & 15); }
__host__ __device__ inline int kv8_v_index(int p, int d, int hd) {
  return 32 * hd + (d >> 5) * 1024 + ((d & 31) + (p & 4) * 8) * 16 + (p >> 3) * 4 + (p & 3);
}
__host__ __device__ inline int kv8_scale_index(int p, int is_v, int hd) { return 64 * hd + 32 * is_v + p; }

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

typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

// eight values of a row as they lie in memory, the bits of their largest magnitude, and the values
template <typename T> struct Eight;
template <> struct Eight<bf16_t> {
  u32x4 w = {0, 0, 0, 0};
  __device__ inline void load(const bf16_t* p) { w = *(const u32x4*)p; }
  __device__ inline unsigned top() const {  // (two at a time)
    u16x2 t = {0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i) t = __builtin_elementwise_max(t, __builtin_bit_cast(u16x2, w[i] & 0x7FFF7FFFu));
    return (unsigned)(t[0] > t[1] ? t[0] : t[1]) << 16;
  }
  __device__ inline float operator[](int i) const { return __uint_as_float(i & 1 ? w[i >> 1] & 0xFFFF0000u : w[i >> 1] << 16); }
};
template <> struct Eight<float> {
  f32x4 a = {0.f, 0.f, 0.f, 0.f}, b = {0.f, 0.f, 0.f, 0.f};
  __device__ inline void load(const float* p) { a = *(const f32x4*)p; b = *(const f32x4*)(p + 4); }
  __device__ inline unsigned top() const {
    unsigned t = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) t = max(t, max(__float_as_uint(a[i]) & 0x7FFFFFFFu, __float_as_uint(b[i]) & 0x7FFFFFFFu));
    return t;
  }
  __device__ inline float operator[](int i) const { return i < 4 ? a[i] : b[i - 4]; }
};

void launch_kv8_write(const Kv8View& c, int format, int hd, const void* k, const void* v, int64_t stride, int dtype, const Kv8Meta& m, hipStream_t st);
void launch_kv8_read(const Kv8View& c, int format, int hd, void* k, void* v, int64_t stride, int dtype, const Kv8Meta& m, hipStream_t st);
struct Kv8AttnPlan {
  int chunk;    // 32-position blocks of a workgroup's share of the keys
  int splits;   // most shares of a sequence (1: the workgroups write the output)
  int64_t items, item_off[DLM_MAX_SEQS + 1];  // (32-query tile, share) pairs: all, and of the sequences before each
};
Kv8AttnPlan kv8_attention_plan(const int32_t* row_off, const int32_t* n_keys, int n_seqs, int n_q, int n_kv);
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
