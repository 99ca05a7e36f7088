// C ABI of the 8-bit KV cache and what feeds and reads it: argument validation and packing.  No kernel code here.
#include <cstring>

#include "abi_args.h"
#include "kv8.h"

namespace {

bool known_head(int hd) { return hd == 32 || hd == 64 || hd == 128; }

// bytes of a (slot, kv head), 0 for an unsupported shape
int64_t head_bytes(int n_slots, int max_len, int n_kv, int hd) {
  if (n_slots < 1 || max_len < 1 || max_len > INT32_MAX - 255 || n_kv < 1 || n_kv > 65535 || !known_head(hd)) return 0;
  const int64_t per = ((int64_t)max_len + 31) / 32 * kv8_block_bytes(hd);
  return (INT64_C(1) << 46) / per < (int64_t)n_slots * n_kv ? 0 : per;
}

int check_cache(const char* name, const dlm_kv8_cache* c, Kv8View* view) {
  REQUIRE(c && c->data, DLM_EINVAL, "%s: null cache", name);
  REQUIRE(c->format == DLM_KV8_E4M3 || c->format == DLM_KV8_I8, DLM_EINVAL, "%s: format %d", name, c->format);
  REQUIRE(aligned16(c->data), DLM_EINVAL, "%s: the cache is not 16-byte aligned", name);
  view->head_bytes = head_bytes(c->n_slots, c->max_len, c->n_kv, c->head_dim);
  REQUIRE(view->head_bytes, DLM_ESHAPE, "%s: a cache of %d slots x %d positions x %d heads of %d", name, c->n_slots, c->max_len, c->n_kv, c->head_dim);
  view->data = (unsigned char*)c->data;
  view->n_kv = c->n_kv;
  return DLM_OK;
}

// the packing that all calls share; once: a slot may be given once (a write)
int check_seqs(const char* name, const dlm_kv8_cache* c, const int32_t* row_offsets, const int32_t* slot, int n_seqs, bool once, int32_t* row_off, int32_t* slots) {
  REQUIRE(n_seqs >= 1, DLM_EINVAL, "%s: n_seqs %d < 1", name, n_seqs);
  REQUIRE(n_seqs <= DLM_MAX_SEQS, DLM_ECAPACITY, "%s: n_seqs %d > %d", name, n_seqs, DLM_MAX_SEQS);
  REQUIRE(row_offsets[0] == 0, DLM_EINVAL, "%s: row_offsets[0] != 0", name);
  row_off[0] = 0;
  for (int b = 0; b < n_seqs; ++b) {
    REQUIRE(row_offsets[b + 1] >= row_offsets[b], DLM_EINVAL, "%s: row_offsets decreasing at sequence %d", name, b);
    row_off[b + 1] = row_offsets[b + 1];
    slots[b] = slot ? slot[b] : b;
    REQUIRE(slots[b] >= 0 && slots[b] < c->n_slots, DLM_EINVAL, "%s: slot %d of sequence %d out of range", name, slots[b], b);
    if (once)
      for (int i = 0; i < b; ++i) REQUIRE(slots[i] != slots[b], DLM_EINVAL, "%s: slot %d given twice", name, slots[b]);
  }
  return DLM_OK;
}

int check_spans(const char* name, const dlm_kv8_cache* c, const void* k, const void* v, int64_t row_stride, int dtype, const int32_t* row_offsets,
                const int32_t* start, const int32_t* slot, int n_seqs, bool once, Kv8View* view, Kv8Meta* m) {
  int rc = check_cache(name, c, view);
  if (rc != DLM_OK) return rc;
  REQUIRE(k && v && row_offsets && start, DLM_EINVAL, "%s: null argument", name);
  REQUIRE(known_dtype(dtype), DLM_EINVAL, "%s: dtype %d", name, dtype);
  REQUIRE(aligned16(k) && aligned16(v), DLM_EINVAL, "%s: rows that are not 16-byte aligned", name);
  REQUIRE(good_stride(row_stride, (int64_t)c->n_kv * c->head_dim, dtype), DLM_EINVAL, "%s: row stride %lld of rows of %d x %d", name, (long long)row_stride,
          c->n_kv, c->head_dim);
  memset(m, 0, sizeof *m);
  rc = check_seqs(name, c, row_offsets, slot, n_seqs, once, m->row_off, m->slot);
  if (rc != DLM_OK) return rc;
  m->n_seqs = n_seqs;
  int64_t blocks = 0;
  for (int b = 0; b < n_seqs; ++b) {
    const int64_t n = row_offsets[b + 1] - row_offsets[b];
    REQUIRE(start[b] >= 0, DLM_EINVAL, "%s: negative start of sequence %d", name, b);
    REQUIRE(start[b] + n <= c->max_len, DLM_ECAPACITY, "%s: span end %lld of sequence %d > max_len %d", name, (long long)(start[b] + n), b, c->max_len);
    m->start[b] = start[b];
    if (n) blocks += (start[b] + n - 1) / 32 - start[b] / 32 + 1;
    REQUIRE(blocks * c->n_kv <= MAX_GRID, DLM_ECAPACITY, "%s: too many rows for one launch", name);
    m->block_off[b + 1] = (int32_t)blocks;
  }
  const Rows kr(k, row_offsets[n_seqs], row_stride, (int64_t)c->n_kv * c->head_dim, dtype), vr(v, kr.rows, row_stride, (int64_t)c->n_kv * c->head_dim, dtype);
  const wide cached = (wide)view->head_bytes * c->n_slots * c->n_kv;
  REQUIRE(!overlap(k, kr.span(), c->data, cached) && !overlap(v, vr.span(), c->data, cached), DLM_EINVAL, "%s: rows overlap the cache", name);
  REQUIRE(once || !overlap(kr, vr), DLM_EINVAL, "%s: k overlaps v", name);
  return DLM_OK;
}

}  // namespace

extern "C" int dlm_qk_norm_rope(const void* x, int64_t x_stride, int rows, int n_q, int n_kv, int head_dim, int dtype, const void* q_gain, const void* k_gain,
                                float eps, float theta, const int32_t* positions, void* out, int64_t out_stride, void* stream) {
  REQUIRE(x && out && positions, DLM_EINVAL, "dlm_qk_norm_rope: null argument");
  REQUIRE(known_dtype(dtype), DLM_EINVAL, "dlm_qk_norm_rope: dtype %d", dtype);
  REQUIRE(known_head(head_dim), DLM_ESHAPE, "dlm_qk_norm_rope: head_dim %d not in {32,64,128}", head_dim);
  REQUIRE(rows >= 0 && n_q >= 0 && n_kv >= 0 && (int64_t)n_q + n_kv >= 1 && (int64_t)n_q + n_kv <= 65535, DLM_ESHAPE, "dlm_qk_norm_rope: %d rows of %d + %d heads",
          rows, n_q, n_kv);
  REQUIRE(eps > 0.f && eps < __builtin_inff() && theta > 0.f && theta < __builtin_inff(), DLM_EINVAL, "dlm_qk_norm_rope: eps and theta must be positive and finite");
  const int64_t width = (int64_t)(n_q + n_kv) * head_dim;
  REQUIRE(aligned16(x) && aligned16(out) && aligned16(q_gain) && aligned16(k_gain) && ((uintptr_t)positions & 3) == 0, DLM_EINVAL, "dlm_qk_norm_rope: unaligned pointer");
  REQUIRE(good_stride(x_stride, width, dtype) && good_stride(out_stride, width, dtype), DLM_EINVAL, "dlm_qk_norm_rope: strides %lld and %lld of rows of %lld",
          (long long)x_stride, (long long)out_stride, (long long)width);
  REQUIRE(rows <= 4 * MAX_GRID, DLM_ECAPACITY, "dlm_qk_norm_rope: too many rows for one launch");
  const Rows from(x, rows, x_stride, width, dtype), to(out, rows, out_stride, width, dtype);
  REQUIRE((x == out && x_stride == out_stride) || !overlap(from, to), DLM_EINVAL, "dlm_qk_norm_rope: out overlaps x");
  if (rows == 0) return DLM_OK;
  launch_qk_norm_rope(x, x_stride, rows, n_q, n_kv, head_dim, dtype, q_gain, k_gain, eps, theta, positions, out, out_stride, (hipStream_t)stream);
  DLM_HIP(hipGetLastError());
  return DLM_OK;
}

extern "C" size_t dlm_kv8_bytes(int n_slots, int max_len, int n_kv, int head_dim) {
  return (size_t)head_bytes(n_slots, max_len, n_kv, head_dim) * (size_t)n_slots * (size_t)n_kv;
}

extern "C" int dlm_kv8_write(const dlm_kv8_cache* c, const void* k, const void* v, int64_t row_stride, int dtype, const int32_t* row_offsets, const int32_t* start,
                             const int32_t* slot, int n_seqs, void* stream) {
  Kv8View view;
  Kv8Meta m;
  const int rc = check_spans("dlm_kv8_write", c, k, v, row_stride, dtype, row_offsets, start, slot, n_seqs, true, &view, &m);
  if (rc != DLM_OK) return rc;
  if (m.block_off[n_seqs] == 0) return DLM_OK;
  launch_kv8_write(view, c->format, c->head_dim, k, v, row_stride, dtype, m, (hipStream_t)stream);
  DLM_HIP(hipGetLastError());
  return DLM_OK;
}

extern "C" int dlm_kv8_read(const dlm_kv8_cache* c, void* k, void* v, int64_t row_stride, int dtype, const int32_t* row_offsets, const int32_t* start,
                            const int32_t* slot, int n_seqs, void* stream) {
  Kv8View view;
  Kv8Meta m;
  const int rc = check_spans("dlm_kv8_read", c, k, v, row_stride, dtype, row_offsets, start, slot, n_seqs, false, &view, &m);
  if (rc != DLM_OK) return rc;
  if (m.block_off[n_seqs] == 0) return DLM_OK;
  launch_kv8_read(view, c->format, c->head_dim, k, v, row_stride, dtype, m, (hipStream_t)stream);
  DLM_HIP(hipGetLastError());
  return DLM_OK;
}

extern "C" size_t dlm_kv8_attention_workspace(int rows, int n_q, int head_dim) {
  return rows > 0 && n_q > 0 && known_head(head_dim) ? kv8_attention_partials(rows, n_q) * (size_t)(head_dim + 2) * 4 : 0;
}

extern "C" int dlm_kv8_attention(const dlm_kv8_cache* c, const void* q, int64_t q_stride, void* out, int dtype, int n_q, const int32_t* row_offsets,
                                 const int32_t* n_keys, const int32_t* slot, int n_seqs, const uint32_t* mask, int mask_words, void* workspace,
                                 size_t workspace_bytes, void* stream) {
  Kv8View view;
  Kv8AttnMeta m;
  int rc = check_cache("dlm_kv8_attention", c, &view);
  if (rc != DLM_OK) return rc;
  REQUIRE(q && out && row_offsets && n_keys, DLM_EINVAL, "dlm_kv8_attention: null argument");
  REQUIRE(known_dtype(dtype), DLM_EINVAL, "dlm_kv8_attention: dtype %d", dtype);
  REQUIRE(n_q >= 1 && n_q <= 65535 && n_q % c->n_kv == 0, DLM_ESHAPE, "dlm_kv8_attention: %d query heads over %d", n_q, c->n_kv);
  REQUIRE(aligned16(q) && aligned16(out) && aligned16(workspace) && ((uintptr_t)mask & 3) == 0, DLM_EINVAL, "dlm_kv8_attention: unaligned pointer");
  const int64_t width = (int64_t)n_q * c->head_dim;
  REQUIRE(good_stride(q_stride, width, dtype), DLM_EINVAL, "dlm_kv8_attention: stride %lld of rows of %lld", (long long)q_stride, (long long)width);
  memset(&m, 0, sizeof m);
  rc = check_seqs("dlm_kv8_attention", c, row_offsets, slot, n_seqs, false, m.row_off, m.slot);
  if (rc != DLM_OK) return rc;
  m.n_seqs = n_seqs;
  REQUIRE(!mask || mask_words >= 1, DLM_EINVAL, "dlm_kv8_attention: mask_words %d", mask_words);
  for (int b = 0; b < n_seqs; ++b) {
    const int nr = row_offsets[b + 1] - row_offsets[b];
    REQUIRE(n_keys[b] >= 0 && (!mask || n_keys[b] >= nr), DLM_EINVAL, "dlm_kv8_attention: %d keys of sequence %d with %d rows", n_keys[b], b, nr);
    REQUIRE(n_keys[b] <= c->max_len, DLM_ECAPACITY, "dlm_kv8_attention: %d keys of sequence %d > max_len %d", n_keys[b], b, c->max_len);
    REQUIRE(!mask || ((int64_t)nr + 31) / 32 <= mask_words, DLM_ECAPACITY, "dlm_kv8_attention: mask_words %d for %d rows of sequence %d", mask_words, nr, b);
    m.n_keys[b] = n_keys[b];
  }
  const int rows = row_offsets[n_seqs];
  const Rows from(q, rows, q_stride, width, dtype), to(out, rows, width, width, dtype);
  REQUIRE(!overlap(from, to), DLM_EINVAL, "dlm_kv8_attention: out overlaps q");
  REQUIRE(!overlap(out, to.span(), c->data, (wide)view.head_bytes * c->n_slots * c->n_kv) && !(mask && overlap(out, to.span(), mask, (wide)rows * mask_words * 4)), DLM_EINVAL,
          "dlm_kv8_attention: out overlaps the cache or the mask");
  if (rows == 0) return DLM_OK;
  const Kv8AttnPlan p = kv8_attention_plan(row_offsets, n_keys, n_seqs, n_q, c->n_kv);
  REQUIRE((int64_t)rows * (n_q / c->n_kv) <= INT32_MAX && p.items / (n_seqs == 1 ? p.splits : 1) <= 65535, DLM_ECAPACITY, "dlm_kv8_attention: too many rows for one launch");
  const size_t need = p.splits > 1 ? (size_t)p.splits * rows * n_q * (c->head_dim + 2) * 4 : 0;
  REQUIRE(!need || (workspace && workspace_bytes >= need), DLM_ECAPACITY, "dlm_kv8_attention: workspace of %zu bytes < %zu", workspace ? workspace_bytes : 0, need);
  REQUIRE(!need || !(overlap(workspace, need, q, from.span()) || overlap(workspace, need, out, to.span()) || (mask && overlap(workspace, need, mask, (wide)rows * mask_words * 4)) ||
                     overlap(workspace, need, c->data, (wide)view.head_bytes * c->n_slots * c->n_kv)),
          DLM_EINVAL, "dlm_kv8_attention: the workspace overlaps an array of the call");
  m.chunk = p.chunk;
  for (int b = 0; b <= n_seqs; ++b) m.item_off[b] = (int32_t)p.item_off[b];
  Kv8AttnArgs a{q, q_stride, out, mask, mask_words, n_q, rows, nullptr, nullptr};
  a.part = (float*)workspace;
  a.part_ml = a.part + (size_t)p.splits * rows * n_q * c->head_dim;
  launch_kv8_attention(view, c->format, c->head_dim, dtype, a, m, p, (hipStream_t)stream);
  DLM_HIP(hipGetLastError());
  return DLM_OK;
}
