// C ABI of the linear layers in 8-bit integers: argument validation.  No kernel code here.
#include "abi_args.h"
#include "q8_plan.h"

namespace {

// bytes of a packed weight (its codes, then its scales), 0 for an unsupported shape
int64_t weight_code_bytes(int n, int k, int gated) {
  if (n < 1 || n > Q8_MAX_N || k < 1 || k > Q8_MAX_K || (gated && n % 2)) return 0;
  const int64_t bytes = (int64_t)q8_units(n, gated) * q8_ktiles(k) * 2048;
  return bytes <= INT64_C(1) << 35 ? bytes : 0;  // (16 of them a thread of the packing's launch)
}
int64_t weight_bytes(int n, int k, int gated) {
  const int64_t codes = weight_code_bytes(n, k, gated);
  return codes ? codes + (int64_t)q8_units(n, gated) * 128 : 0;
}
int check_weight(const char* name, const dlm_q8_weight* w, Q8View* view) {
  REQUIRE(w && w->data, DLM_EINVAL, "%s: null weight", name);
  REQUIRE(aligned16(w->data), DLM_EINVAL, "%s: the weight is not 16-byte aligned", name);
  REQUIRE(w->gated == 0 || w->gated == 1, DLM_EINVAL, "%s: gated %d", name, w->gated);
  const int64_t codes = weight_code_bytes(w->n, w->k, w->gated);
  REQUIRE(codes, DLM_ESHAPE, "%s: a weight of %d x %d", name, w->n, w->k);
  *view = Q8View{(const unsigned char*)w->data, (const float*)((const char*)w->data + codes), w->n, w->k, q8_units(w->n, w->gated), q8_ktiles(w->k), w->gated == 1};
  return DLM_OK;
}
// rows of 8-bit codes [rows, k], whose bytes up to a multiple of 16 belong to them
bool good_code_stride(int64_t stride, int64_t k) { return good_stride_bytes(stride, k, 1); }

int check_rows(const char* name, const Q8RowsArgs& a) {
  REQUIRE(a.x && a.codes && a.scale, DLM_EINVAL, "%s: null argument", name);
  REQUIRE(known_dtype(a.dtype), DLM_EINVAL, "%s: dtype %d", name, a.dtype);
  REQUIRE(a.rows >= 0 && a.width >= 1 && a.width <= Q8_MAX_WIDTH, DLM_ESHAPE, "%s: %d rows of %d", name, a.rows, a.width);
  REQUIRE(aligned16(a.x) && aligned16(a.codes) && ((uintptr_t)a.scale & 3) == 0, DLM_EINVAL, "%s: unaligned pointer", name);
  REQUIRE(good_stride(a.x_stride, a.width, a.dtype) && good_code_stride(a.codes_stride, a.width), DLM_EINVAL, "%s: strides %lld and %lld of rows of %d", name,
          (long long)a.x_stride, (long long)a.codes_stride, a.width);
  REQUIRE(a.rows <= MAX_GRID / 4, DLM_ECAPACITY, "%s: too many rows for one launch", name);
  const Rows x(a.x, a.rows, a.x_stride, a.width, a.dtype), codes = Rows::of_bytes(a.codes, a.rows, a.codes_stride, a.width);
  REQUIRE(!overlap(x, codes) && !overlap(a.scale, (wide)a.rows * 4, a.x, x.span()) && !overlap(a.scale, (wide)a.rows * 4, a.codes, codes.span()), DLM_EINVAL,
          "%s: codes or scale overlap an array of the call", name);
  return DLM_OK;
}

}  // namespace

extern "C" int dlm_q8_rows(const void* x, int64_t x_stride, int rows, int width, int dtype, int8_t* codes, int64_t codes_stride, float* scale, void* stream) {
  Q8RowsArgs a{};
  a.x = x; a.x_stride = x_stride; a.rows = rows; a.width = width; a.dtype = dtype;
  a.codes = codes; a.codes_stride = codes_stride; a.scale = scale;
  const int rc = check_rows("dlm_q8_rows", a);
  if (rc != DLM_OK || rows == 0) return rc;
  launch_q8_rows(a, (hipStream_t)stream);
  DLM_HIP(hipGetLastError());
  return DLM_OK;
}

extern "C" int dlm_add_norm_q8(const void* x, int64_t x_stride, int rows, int width, int dtype, const void* residual, int64_t residual_stride, void* h,
                               int64_t h_stride, int h_dtype, const void* gain, float eps, int8_t* codes, int64_t codes_stride, float* scale, void* stream) {
  static const char* name = "dlm_add_norm_q8";
  Q8RowsArgs a{};
  a.x = x; a.x_stride = x_stride; a.rows = rows; a.width = width; a.dtype = dtype;
  a.residual = residual; a.r_stride = residual_stride; a.h = h; a.h_stride = h_stride; a.h_dtype = h_dtype;
  a.gain = gain; a.eps = eps;
  a.codes = codes; a.codes_stride = codes_stride; a.scale = scale;
  const int rc = check_rows(name, a);
  if (rc != DLM_OK) return rc;
  REQUIRE(gain, DLM_EINVAL, "%s: null argument", name);
  REQUIRE(!residual == !h, DLM_EINVAL, "%s: residual and h are given together", name);
  REQUIRE(aligned16(gain) && aligned16(residual) && aligned16(h), DLM_EINVAL, "%s: unaligned pointer", name);
  REQUIRE(eps > 0.f && eps < __builtin_inff(), DLM_EINVAL, "%s: eps must be positive and finite", name);
  const Rows xr(x, rows, x_stride, width, dtype), cr = Rows::of_bytes(codes, rows, codes_stride, width);
  const wide gain_bytes = (wide)width * elem_bytes(dtype), scale_bytes = (wide)rows * 4;
  REQUIRE(!overlap(gain, gain_bytes, codes, cr.span()) && !overlap(gain, gain_bytes, scale, scale_bytes), DLM_EINVAL, "%s: codes or scale overlap the gain", name);
  if (h) {
    REQUIRE(h_dtype == DLM_F32 || (h_dtype == DLM_BF16 && dtype == DLM_BF16), DLM_EINVAL, "%s: h_dtype %d with rows of dtype %d", name, h_dtype, dtype);
    REQUIRE(good_stride(residual_stride, width, h_dtype) && good_stride(h_stride, width, h_dtype), DLM_EINVAL, "%s: strides %lld and %lld of rows of %d", name,
            (long long)residual_stride, (long long)h_stride, width);
    const Rows rr(residual, rows, residual_stride, width, h_dtype), hr(h, rows, h_stride, width, h_dtype);
    REQUIRE((h == residual && h_stride == residual_stride) || !overlap(hr, rr), DLM_EINVAL, "%s: h overlaps the residual", name);
    REQUIRE((h == x && h_stride == x_stride && h_dtype == dtype) || !overlap(hr, xr), DLM_EINVAL, "%s: h overlaps x", name);
    REQUIRE(!overlap(gain, gain_bytes, h, hr.span()), DLM_EINVAL, "%s: h overlaps the gain", name);
    REQUIRE(!overlap(rr, cr) && !overlap(hr, cr) && !overlap(scale, scale_bytes, residual, rr.span()) && !overlap(scale, scale_bytes, h, hr.span()), DLM_EINVAL,
            "%s: codes or scale overlap an array of the call", name);
  }
  if (rows == 0) return DLM_OK;
  launch_q8_rows(a, (hipStream_t)stream);
  DLM_HIP(hipGetLastError());
  return DLM_OK;
}

extern "C" size_t dlm_q8_weight_bytes(int n, int k, int gated) { return (size_t)weight_bytes(n, k, gated); }

extern "C" int dlm_q8_weight_pack(const dlm_q8_weight* w, const int8_t* codes, int64_t codes_stride, const float* scale, void* stream) {
  Q8View view;
  const int rc = check_weight("dlm_q8_weight_pack", w, &view);
  if (rc != DLM_OK) return rc;
  REQUIRE(codes && scale, DLM_EINVAL, "dlm_q8_weight_pack: null argument");
  REQUIRE(aligned16(codes) && ((uintptr_t)scale & 3) == 0, DLM_EINVAL, "dlm_q8_weight_pack: unaligned pointer");
  REQUIRE(good_code_stride(codes_stride, view.k), DLM_EINVAL, "dlm_q8_weight_pack: stride %lld of rows of %d", (long long)codes_stride, view.k);
  const wide bytes = weight_bytes(view.n, view.k, view.gated);
  const Rows from = Rows::of_bytes(codes, view.n, codes_stride, ((int64_t)view.k + 15) / 16 * 16);
  REQUIRE(!overlap(w->data, bytes, codes, from.span()) && !overlap(w->data, bytes, scale, (wide)view.n * 4), DLM_EINVAL, "dlm_q8_weight_pack: the weight overlaps its source");
  launch_q8_pack(codes, codes_stride, scale, view, w->data, (hipStream_t)stream);
  DLM_HIP(hipGetLastError());
  return DLM_OK;
}

extern "C" size_t dlm_q8_gemm_workspace(int rows, int n, int k, int gated) { return rows > 0 && weight_bytes(n, k, gated) ? q8_gemm_workspace(rows, n, k, gated) : 0; }

extern "C" int dlm_q8_gemm(const dlm_q8_weight* w, const int8_t* x, int64_t x_stride, const float* x_scale, int rows, void* out, int64_t out_stride, int out_dtype,
                           void* workspace, size_t workspace_bytes, void* stream) {
  static const char* name = "dlm_q8_gemm";
  Q8View view;
  const int rc = check_weight(name, w, &view);
  if (rc != DLM_OK) return rc;
  REQUIRE(x && x_scale && out, DLM_EINVAL, "%s: null argument", name);
  REQUIRE(known_dtype(out_dtype), DLM_EINVAL, "%s: out_dtype %d", name, out_dtype);
  REQUIRE(rows >= 0, DLM_ESHAPE, "%s: %d rows", name, rows);
  REQUIRE(aligned16(x) && aligned16(out) && aligned16(workspace) && ((uintptr_t)x_scale & 3) == 0, DLM_EINVAL, "%s: unaligned pointer", name);
  const int outputs = view.outputs();
  REQUIRE(good_code_stride(x_stride, view.k) && good_stride(out_stride, outputs, out_dtype), DLM_EINVAL, "%s: strides %lld and %lld of rows of %d and %d", name,
          (long long)x_stride, (long long)out_stride, view.k, outputs);
  REQUIRE(rows <= 1 << 20 && (int64_t)rows * outputs <= INT64_C(1) << 38, DLM_ECAPACITY, "%s: too many rows for one launch", name);
  const Rows xr = Rows::of_bytes(x, rows, x_stride, ((int64_t)view.k + 15) / 16 * 16), to(out, rows, out_stride, outputs, out_dtype);
  const wide bytes = weight_bytes(view.n, view.k, view.gated);
  REQUIRE(!overlap(xr, to) && !overlap(out, to.span(), x_scale, (wide)rows * 4) && !overlap(out, to.span(), w->data, bytes), DLM_EINVAL, "%s: out overlaps an array of the call", name);
  const Q8GemmArgs args{x, x_stride, x_scale, rows, out, out_stride, out_dtype, workspace};
  if (rows == 0) return DLM_OK;
  const Q8Plan plan = q8_plan(rows, view.units, view.k, view.gated, x_stride);
  REQUIRE(plan.streamed || q8_tile_threads(plan.tile) < INT64_C(1) << 32, DLM_ECAPACITY, "%s: too many rows and channels for one launch", name);
  const size_t need = plan.workspace;
  REQUIRE(!need || (workspace && workspace_bytes >= need), DLM_ECAPACITY, "%s: workspace of %zu bytes < %zu", name, workspace ? workspace_bytes : 0, need);
  REQUIRE(!need || !(overlap(workspace, need, x, xr.span()) || overlap(workspace, need, out, to.span()) || overlap(workspace, need, x_scale, (wide)rows * 4) ||
                     overlap(workspace, need, w->data, bytes)),
          DLM_EINVAL, "%s: the workspace overlaps an array of the call", name);
  launch_q8_gemm(view, args, plan, (hipStream_t)stream);
  DLM_HIP(hipGetLastError());
  return DLM_OK;
}

extern "C" int dlm_plan_q8_gemm(int rows, int n, int k, int gated, int32_t plan[6]) {
  REQUIRE(plan, DLM_EINVAL, "dlm_plan_q8_gemm: null plan");
  REQUIRE(gated == 0 || gated == 1, DLM_EINVAL, "dlm_plan_q8_gemm: gated %d", gated);
  REQUIRE(rows >= 1 && rows <= 1 << 20 && weight_bytes(n, k, gated), DLM_ESHAPE, "dlm_plan_q8_gemm: %d rows, a weight of %d x %d", rows, n, k);
  const int units = q8_units(n, gated), tile = rows <= 16 ? 16 : 32;
  const Q8Plan p = q8_plan(rows, units, k, gated, 0);
  if (p.streamed) {
    const int32_t v[6] = {0, tile, 16 * p.stream.subs, 1, (2 * units + p.stream.subs - 1) / p.stream.subs * ((rows + tile - 1) / tile), 0};
    for (int i = 0; i < 6; ++i) plan[i] = v[i];
  } else {
    const int32_t v[6] = {p.tile.tile < Q8_TILE_COUNT ? 1 : 2, p.tile.rows, p.tile.cols, p.tile.splits, p.tile.nblocks * p.tile.mblocks * p.tile.splits, (int32_t)(p.tile.workspace >> 10)};
    for (int i = 0; i < 6; ++i) plan[i] = v[i];
  }
  return DLM_OK;
}
