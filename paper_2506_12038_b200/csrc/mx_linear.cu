// The product of two microscaled 4-bit matrices (lcd_mx_linear): y[m][n] = sum over blocks b of 2^(sx + sw) times the sum over the
// block's 32 columns of the elements' products.  Products of elements are multiples of 1/4 up to 36, so a block's sum is exact in
// binary32 in any order; the blocks are added in binary32.
#include <type_traits>

#include "common.h"
#include "device_util.h"
#include "mx.cuh"

namespace lcd {

namespace {

constexpr int kPlainThreads = 128;

// A warp per output; a lane takes every 32nd block of its row pair.
template <typename T>
__global__ void __launch_bounds__(kPlainThreads)
mx_linear_kernel(const uint8_t* __restrict__ wc, int64_t ldwc, const uint8_t* __restrict__ ws, int64_t ldws, int64_t N, int64_t K,
                 const uint8_t* __restrict__ xc, int64_t ldxc, const uint8_t* __restrict__ xs, int64_t ldxs, T* __restrict__ y, int64_t ldy) {
  const int64_t n = (int64_t)blockIdx.x * (kPlainThreads / 32) + threadIdx.x / 32, m = blockIdx.y;
  if (n >= N) return;
  const int64_t blocks = (K + kMxBlock - 1) / kMxBlock;
  float sum = 0.0f;
  for (int64_t b = threadIdx.x & 31; b < blocks; b += 32) {
    const uint4 w = *reinterpret_cast<const uint4*>(wc + n * ldwc + b * 16), x = *reinterpret_cast<const uint4*>(xc + m * ldxc + b * 16);
    const uint32_t wv[4] = {w.x, w.y, w.z, w.w}, xv[4] = {x.x, x.y, x.z, x.w};
    float part = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float a[8], c[8];
      mx_elements8(wv[i], a);
      mx_elements8(xv[i], c);
#pragma unroll
      for (int j = 0; j < 8; ++j) part += a[j] * c[j];
    }
    sum += part * mx_scale_value(ws[n * ldws + b]) * mx_scale_value(xs[m * ldxs + b]);
  }
  for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if ((threadIdx.x & 31) == 0) y[m * ldy + n] = from_f32<T>(sum);
}

template <typename T>
lcd_status launch_typed(const MxProduct& p, cudaStream_t s) {
  for (int64_t m = 0; m < p.M; m += 65535) {
    const int64_t rows = p.M - m < 65535 ? p.M - m : 65535;
    mx_linear_kernel<T><<<dim3((unsigned)((p.N + kPlainThreads / 32 - 1) / (kPlainThreads / 32)), (unsigned)rows), kPlainThreads, 0, s>>>(
        p.w_codes, p.ldwc, p.w_scales, p.ldws, p.N, p.K, p.x_codes + m * p.ldxc, p.ldxc, p.x_scales + m * p.ldxs, p.ldxs,
        static_cast<T*>(p.y) + m * p.ldy, p.ldy);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) { set_cuda_error((int)e); return LCD_ERR_CUDA; }
  }
  return LCD_OK;
}

}  // namespace

lcd_status launch_mx_linear(const MxProduct& p, int32_t*, void* stream) {
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  switch (p.y_type) {
    case LCD_DTYPE_F32: return launch_typed<float>(p, s);
    case LCD_DTYPE_F16: return launch_typed<__half>(p, s);
    default: return launch_typed<__nv_bfloat16>(p, s);
  }
}

}  // namespace lcd
