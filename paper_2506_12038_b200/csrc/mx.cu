// Microscaled 4-bit floating point: quantisation and what the numbers stand for (lcd_mx_quantize, lcd_mx_dequantize).
// Per block of 32 columns: A = max |t|, e = floor(log2 A) - 2, element = round(t * 2^-e).  Scaling by a power of two is exact,
// so the rounding to 4 bits is the only one after t itself and results are the same bit for bit everywhere.
//
// Four lanes share a block and eight consecutive columns are a lane's: one 16-byte load of 16-bit values (two of fp32), the
// block's maximum by two shuffles, four code bytes out, so that loads and stores of a warp are contiguous.
#include <type_traits>

#include "common.h"
#include "device_util.h"
#include "mx.cuh"

namespace lcd {

namespace {

constexpr int kMxThreads = 256;

// VEC: rows of x and the factors start on 16 bytes.  A unit is a lane's eight columns; chunks = CTAs a row.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kMxThreads)
mx_quantize_kernel(const T* __restrict__ x, int64_t K, int64_t ldx, const float* __restrict__ inv, uint8_t* __restrict__ codes,
                   int64_t ldc, uint8_t* __restrict__ scales, int64_t lds, uint32_t units, uint32_t chunks) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // the product of the same call may set itself up
  const int64_t row = blockIdx.x / chunks;
  const uint32_t unit = (blockIdx.x % chunks) * kMxThreads + threadIdx.x;
  float t[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) t[i] = 0.0f;
  const int64_t k0 = (int64_t)unit * 8;
  const T* p = x + row * ldx + k0;
  if (VEC && k0 + 8 <= K) {
    load8(p, t);
    if (inv) {
      float f[8];
      load8(inv + k0, f);
#pragma unroll
      for (int i = 0; i < 8; ++i) t[i] = __fmul_rn(t[i], f[i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (k0 + i < K) t[i] = inv ? __fmul_rn(to_f32(p[i]), inv[k0 + i]) : to_f32(p[i]);
  }
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(t[i]) & 0x7fffffffu);
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
  if (unit >= units) return;
  const uint32_t byte = mx_scale_byte(top);
  uint32_t c = 0;
  if (byte != 255u) {
    const float m = mx_inverse_scale(byte);
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = __fmul_rn(t[i], m);
    c = mx_codes8(t);
  }
  *reinterpret_cast<uint32_t*>(codes + row * ldc + (int64_t)unit * 4) = c;
  if ((unit & 3u) == 0) scales[row * lds + (unit >> 2)] = (uint8_t)byte;
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(kMxThreads)
mx_dequantize_kernel(const uint8_t* __restrict__ codes, int64_t ldc, const uint8_t* __restrict__ scales, int64_t lds, int64_t K,
                     T* __restrict__ out, int64_t ldo, uint32_t units, uint32_t chunks) {
  const int64_t row = blockIdx.x / chunks;
  const uint32_t unit = (blockIdx.x % chunks) * kMxThreads + threadIdx.x;
  if (unit >= units) return;
  float v[8];
  mx_elements8(*reinterpret_cast<const uint32_t*>(codes + row * ldc + (int64_t)unit * 4), v);
  const float s = mx_scale_value(scales[row * lds + (unit >> 2)]);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = __fmul_rn(v[i], s);
  const int64_t k0 = (int64_t)unit * 8;
  T* p = out + row * ldo + k0;
  if (VEC && k0 + 8 <= K) {
    store8(p, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (k0 + i < K) p[i] = from_f32<T>(v[i]);
  }
}

bool on16(const void* p, int64_t ld, int64_t size, int64_t rows) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (rows == 1 || ld * size % 16 == 0);
}

lcd_status launched() {
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) { set_cuda_error((int)e); return LCD_ERR_CUDA; }
  return LCD_OK;
}

template <typename T>
lcd_status quantize_rows(const void* x, int64_t M, int64_t K, int64_t ldx, const float* inv, uint8_t* codes, int64_t ldc,
                         uint8_t* scales, int64_t lds, cudaStream_t s) {
  const uint32_t units = (uint32_t)((K + kMxBlock - 1) / kMxBlock * 4), chunks = (units + kMxThreads - 1) / kMxThreads;
  const bool vec = on16(x, ldx, sizeof(T), M) && (!inv || reinterpret_cast<uintptr_t>(inv) % 16 == 0);
  auto kern = vec ? mx_quantize_kernel<T, true> : mx_quantize_kernel<T, false>;
  kern<<<(unsigned)(M * chunks), kMxThreads, 0, s>>>(static_cast<const T*>(x), K, ldx, inv, codes, ldc, scales, lds, units, chunks);
  return launched();
}

template <typename T>
lcd_status dequantize_rows(const uint8_t* codes, int64_t ldc, const uint8_t* scales, int64_t lds, int64_t M, int64_t K, void* out,
                           int64_t ldo, cudaStream_t s) {
  const uint32_t units = (uint32_t)((K + 7) / 8), chunks = (units + kMxThreads - 1) / kMxThreads;
  auto kern = on16(out, ldo, sizeof(T), M) ? mx_dequantize_kernel<T, true> : mx_dequantize_kernel<T, false>;
  kern<<<(unsigned)(M * chunks), kMxThreads, 0, s>>>(codes, ldc, scales, lds, K, static_cast<T*>(out), ldo, units, chunks);
  return launched();
}

}  // namespace

lcd_status launch_mx_quantize(const void* x, lcd_dtype type, int64_t M, int64_t K, int64_t ldx, const float* inv, uint8_t* codes,
                              int64_t ldc, uint8_t* scales, int64_t lds, void* stream) {
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  switch (type) {
    case LCD_DTYPE_F32: return quantize_rows<float>(x, M, K, ldx, inv, codes, ldc, scales, lds, s);
    case LCD_DTYPE_F16: return quantize_rows<__half>(x, M, K, ldx, inv, codes, ldc, scales, lds, s);
    default: return quantize_rows<__nv_bfloat16>(x, M, K, ldx, inv, codes, ldc, scales, lds, s);
  }
}

lcd_status launch_mx_dequantize(const uint8_t* codes, int64_t ldc, const uint8_t* scales, int64_t lds, int64_t M, int64_t K, void* out,
                                lcd_dtype type, int64_t ldo, void* stream) {
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  switch (type) {
    case LCD_DTYPE_F32: return dequantize_rows<float>(codes, ldc, scales, lds, M, K, out, ldo, s);
    case LCD_DTYPE_F16: return dequantize_rows<__half>(codes, ldc, scales, lds, M, K, out, ldo, s);
    default: return dequantize_rows<__nv_bfloat16>(codes, ldc, scales, lds, M, K, out, ldo, s);
  }
}

}  // namespace lcd
