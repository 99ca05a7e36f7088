// Checks of arguments that the entry points of the 8-bit operators share (kv8_abi.hip, q8_abi.hip).  Host code only.
#pragma once
#include "common.h"

namespace {

inline bool known_dtype(int dtype) { return dtype == DLM_F32 || dtype == DLM_BF16; }
inline int64_t elem_bytes(int dtype) { return dtype == DLM_BF16 ? 2 : 4; }
inline bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }
// rows [rows, width] at `stride` elements of `bytes`: the stride holds a row and keeps 16-byte alignment
inline bool good_stride_bytes(int64_t stride, int64_t width, int64_t bytes) { return stride >= width && stride <= INT64_C(1) << 40 && stride * bytes % 16 == 0; }
inline bool good_stride(int64_t stride, int64_t width, int dtype) { return good_stride_bytes(stride, width, elem_bytes(dtype)); }
typedef __int128 wide;  // (rows x strides do not fit 64 bits)
inline bool overlap(const void* a, wide a_bytes, const void* b, wide b_bytes) {
  return a_bytes && b_bytes && (wide)(uintptr_t)a < (wide)(uintptr_t)b + b_bytes && (wide)(uintptr_t)b < (wide)(uintptr_t)a + a_bytes;
}
// [rows, width] at `stride`: what lies between its first and its last byte
struct Rows {
  const void* p;
  int64_t rows, stride, width;  // bytes
  Rows(const void* at, int64_t n, int64_t stride_elems, int64_t width_elems, int dtype)
      : p(at), rows(n), stride(stride_elems * elem_bytes(dtype)), width(width_elems * elem_bytes(dtype)) {}
  wide span() const { return rows ? (wide)(rows - 1) * stride + width : 0; }
  static Rows of_bytes(const void* at, int64_t n, int64_t stride, int64_t width) {
    Rows r(at, n, 0, 0, DLM_F32);
    r.stride = stride;
    r.width = width;
    return r;
  }
};
// whether two such arrays share a byte: columns of one matrix need not; of different strides: whether their spans do
inline bool overlap(const Rows& a, const Rows& b) {
  if (a.stride != b.stride || a.stride < 1) return overlap(a.p, a.span(), b.p, b.span());
  const Rows &lo = (uintptr_t)a.p <= (uintptr_t)b.p ? a : b, &hi = &lo == &a ? b : a;
  const uintptr_t d = (uintptr_t)hi.p - (uintptr_t)lo.p, n = d / (uintptr_t)a.stride;
  const int64_t r = (int64_t)(d % (uintptr_t)a.stride);
  return hi.rows > 0 && ((n < (uintptr_t)lo.rows && r < lo.width) || (n + 1 < (uintptr_t)lo.rows && a.stride - r < hi.width));
}
constexpr int MAX_GRID = (1 << 24) - 1;  // workgroups of 256 in a dimension of a launch

}  // namespace
