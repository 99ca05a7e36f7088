// Products in 8-bit integers: the packing of a weight, and the choice of the kernel.
#include "q8_gemm.h"

namespace {

// a thread: the 16 bytes of one (unit, k-tile, sub, chunk, row)
__global__ __launch_bounds__(256) void q8_pack_kernel(const int8_t* __restrict__ codes, int64_t stride, int n, int k, int gated, int kt, i32x4* __restrict__ out, int64_t chunks) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= chunks) return;
  const int row = i & 15, chunk = (i >> 4) & 3, sub = (i >> 6) & 1;
  const int64_t tile = i >> 7;
  const int unit = (int)(tile / kt), k0 = (int)(tile % kt) * 64 + chunk * 16, channel = q8_channel(unit, 16 * sub + row, n, gated);
  union { i32x4 v; int8_t b[16]; } o;
  o.v = i32x4{0, 0, 0, 0};
  if (channel < n && k0 < k) {
    o.v = *(const i32x4*)(codes + channel * stride + k0);
    if (k0 + 16 > k)
#pragma unroll
      for (int j = 0; j < 16; ++j)
        if (k0 + j >= k) o.b[j] = 0;
  }
  out[i] = o.v;
}
__global__ __launch_bounds__(256) void q8_pack_scale_kernel(const float* __restrict__ scale, int n, int gated, int units, float* __restrict__ out) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= units * 32) return;
  const int channel = q8_channel(i >> 5, i & 31, n, gated);
  out[i] = channel < n ? scale[channel] : 0.f;
}

}  // namespace

void launch_q8_pack(const int8_t* codes, int64_t stride, const float* scale, const Q8View& w, void* data, hipStream_t st) {
  const int64_t chunks = (int64_t)w.units * w.kt * 128;
  q8_pack_kernel<<<(unsigned)((chunks + 255) / 256), 256, 0, st>>>(codes, stride, w.n, w.k, w.gated, w.kt, (i32x4*)data, chunks);
  q8_pack_scale_kernel<<<(w.units * 32 + 255) / 256, 256, 0, st>>>(scale, w.n, w.gated, w.units, (float*)w.scale);
}

size_t q8_gemm_workspace(int, int, int, int) { return 0; }

void launch_q8_stream(const Q8View& w, const Q8GemmArgs& a, hipStream_t st);
void launch_q8_gemm(const Q8View& w, const Q8GemmArgs& a, hipStream_t st) { launch_q8_stream(w, a, st); }
