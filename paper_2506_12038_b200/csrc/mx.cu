// Microscaled 4-bit floating point: quantisation and what the numbers stand for (lcd_mx_quantize, lcd_mx_dequantize).
// Per block of 32 columns: A = max |t|, e = floor(log2 A) - 2, element = round(t * 2^-e).  Scaling by a power of two is exact,
// so the rounding to 4 bits is the only one after t itself and results are the same bit for bit everywhere.
//
// To quantise, four lanes share a block and eight consecutive columns, a unit, are a lane's: one 16-byte load of 16-bit values (two of
// fp32), the block's maximum by two shuffles, four code bytes out.  The other way a unit is 16 bytes of the output, so that a
// warp's store is contiguous (fp32 in units of eight, two stores: 46 us of 11008 x 4096 in place of 35). Of 11008 x 4096 to bf16
// 20.7 us (5.5 TB/s; 20.0 with the hardware's conversion of codes, see mx_values).  What bounds both
// kernels is memory: a thread has its unit of kRowsEach rows in flight at once (one of few rows).  Rows that do not start on 16 bytes go
// through shared memory, element by element and contiguous in memory.
#include <type_traits>

#include "common.h"
#include "device_util.h"
#include "mx.cuh"

namespace lcd {

namespace {

constexpr int kMxThreads = 256;
constexpr int kRowsEach = 4;

// The CTA's threads as (unit, row): blockDim.x units of blockDim.y rows.  A thread has unit blockIdx.y * blockDim.x + threadIdx.x of
// EACH rows, blockDim.y apart.
struct Place {
  uint32_t unit;
  int64_t row0;
};
template <int EACH>
__device__ __forceinline__ Place place() {
  return {blockIdx.y * blockDim.x + threadIdx.x, (int64_t)blockIdx.x * EACH * blockDim.y + threadIdx.y};
}

// VEC: rows of x start on 16 bytes.
template <typename T, bool VEC, int EACH>
__global__ void __launch_bounds__(kMxThreads)
mx_quantize_kernel(const T* x, int64_t M, int64_t K, int64_t ldx, const float* inv, uint8_t* codes, int64_t ldc, uint8_t* scales,
                   int64_t lds, uint32_t units) {
  begin_after_previous();       // (no __restrict__: loads of what the kernel before wrote are coherent ones)
  __shared__ __align__(16) T s_x[VEC ? 1 : EACH * kMxThreads * 8];
  const Place at = place<EACH>();
  const int64_t k0 = (int64_t)at.unit * 8;
  float t[8], f[8];
  const bool whole = VEC && k0 + 8 <= K;
  Raw8<T> raw[EACH];
  if (whole) {
#pragma unroll
    for (int u = 0; u < EACH; ++u) raw[u] = load8(x + min(at.row0 + u * blockDim.y, M - 1) * ldx + k0);
  }
  if (inv) {
    if (k0 + 8 <= K && (reinterpret_cast<uintptr_t>(inv) & 15) == 0) {
      values8(load8(inv + k0), f);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = k0 + i < K ? inv[k0 + i] : 0.0f;
    }
  }
  if (!VEC) {
    const int n = blockDim.x * 8;
    const int64_t from = (int64_t)blockIdx.y * n + threadIdx.x;
#pragma unroll
    for (int u = 0; u < EACH; ++u) {
      const int64_t row = at.row0 + u * blockDim.y;
      T* line = s_x + (u * blockDim.y + threadIdx.y) * n + threadIdx.x;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        line[i * blockDim.x] = row < M && from + i * blockDim.x < K ? x[row * ldx + from + i * blockDim.x] : from_f32<T>(0.0f);
    }
    __syncthreads();
  }
#pragma unroll
  for (int u = 0; u < EACH; ++u) {
    const int64_t row = at.row0 + u * blockDim.y;
    if (whole) {
      values8(raw[u], t);
    } else if (VEC) {
#pragma unroll
      for (int i = 0; i < 8; ++i) t[i] = row < M && k0 + i < K ? to_f32(x[row * ldx + k0 + i]) : 0.0f;
    } else {
      const T* line = s_x + (u * blockDim.y + threadIdx.y) * blockDim.x * 8;
      values8(load8(line + threadIdx.x * 8), t);
    }
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (inv) t[i] = __fmul_rn(t[i], f[i]);
      top = max(top, __float_as_uint(t[i]) & 0x7fffffffu);
    }
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    if (at.unit >= units || row >= M) continue;
    const uint32_t byte = mx_scale_byte(top);
    uint32_t c = 0;
    if (byte != 255u) {
      const float m = mx_inverse_scale(byte);
#pragma unroll
      for (int i = 0; i < 8; ++i) t[i] = __fmul_rn(t[i], m);
      c = mx_codes8(t);
    }
    *reinterpret_cast<uint32_t*>(codes + row * ldc + (int64_t)at.unit * 4) = c;
    if ((at.unit & 3u) == 0) scales[row * lds + (at.unit >> 2)] = (uint8_t)byte;
  }
}

template <typename T, bool VEC, int EACH>
__global__ void __launch_bounds__(kMxThreads)
mx_dequantize_kernel(const uint8_t* codes, int64_t ldc, const uint8_t* scales, int64_t lds, int64_t M, int64_t K, T* out, int64_t ldo,
                     uint32_t units) {
  begin_after_previous();
  constexpr int E = 16 / sizeof(T);
  using Codes = typename std::conditional<E == 8, uint32_t, uint16_t>::type;
  __shared__ T s_out[VEC ? 1 : EACH * kMxThreads * E];
  const Place at = place<EACH>();
  const int64_t k0 = (int64_t)at.unit * E;
  Codes c[EACH];
  uint32_t byte[EACH];
#pragma unroll
  for (int u = 0; u < EACH; ++u) {
    const int64_t row = at.row0 + u * blockDim.y;
    const bool there = row < M && at.unit < units;
    c[u] = there ? *reinterpret_cast<const Codes*>(codes + row * ldc + (int64_t)at.unit * (E / 2)) : Codes(0);
    byte[u] = there ? scales[row * lds + at.unit / (kMxBlock / E)] : 0u;
  }
#pragma unroll
  for (int u = 0; u < EACH; ++u) {
    const int64_t row = at.row0 + u * blockDim.y;
    float v[E];
    mx_values<E>(c[u], byte[u], v);
    T* p = out + row * ldo + k0;
    if (VEC && k0 + E <= K) {
      if (row < M) {
        if constexpr (E == 8) *reinterpret_cast<uint4*>(p) = pack8<T>(v);
        else *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
      }
    } else if (VEC) {
#pragma unroll
      for (int i = 0; i < E; ++i)
        if (row < M && k0 + i < K) p[i] = from_f32<T>(v[i]);
    } else {
      T* line = s_out + (u * blockDim.y + threadIdx.y) * blockDim.x * E;
#pragma unroll
      for (int i = 0; i < E; ++i) line[threadIdx.x * E + i] = from_f32<T>(v[i]);
    }
  }
  if (!VEC) {
    __syncthreads();
    const int n = blockDim.x * E;
    const int64_t from = (int64_t)blockIdx.y * n + threadIdx.x;
#pragma unroll
    for (int u = 0; u < EACH; ++u) {
      const int64_t row = at.row0 + u * blockDim.y;
      const T* line = s_out + (u * blockDim.y + threadIdx.y) * n + threadIdx.x;
#pragma unroll
      for (int i = 0; i < E; ++i)
        if (row < M && from + i * blockDim.x < K) out[row * ldo + from + i * blockDim.x] = line[i * blockDim.x];
    }
  }
}

bool on16(const void* p, int64_t ld, int64_t size, int64_t rows) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (rows == 1 || ld * size % 16 == 0);
}

lcd_status launched(cudaError_t e) {
  if (e != cudaSuccess) { set_cuda_error((int)e); return LCD_ERR_CUDA; }
  return LCD_OK;
}

// CTAs as wide as a row, a warp at least, of as many rows as make up their threads.
struct Shape {
  dim3 grid, block;
  bool each;           // kRowsEach rows a thread
};
Shape shape_of(int64_t rows, uint32_t units, uint32_t threads) {
  uint32_t x = 32;
  while (x < threads && x < units) x *= 2;
  const uint32_t y = threads / x, columns = (units + x - 1) / x;
  const bool each = (rows + y - 1) / y * columns >= 8 * (int64_t)current_sm_count();    // every SM full without
  const int64_t per = each ? (int64_t)y * kRowsEach : y;
  return {dim3((unsigned)((rows + per - 1) / per), columns), dim3(x, y), each};
}

template <typename T>
lcd_status quantize_rows(const void* x, int64_t M, int64_t K, int64_t ldx, const float* inv, uint8_t* codes, int64_t ldc,
                         uint8_t* scales, int64_t lds, cudaStream_t s) {
  const uint32_t units = (uint32_t)((K + kMxBlock - 1) / kMxBlock * 4);
  const bool vec = on16(x, ldx, sizeof(T), M);
  // (2048 x 5120 bf16: 128 threads 7.8 us, 256 8.9; through shared memory, 333 x 5001, 5.1 and 4.2)
  const Shape q = shape_of(M, units, vec ? kMxThreads / 2 : kMxThreads);
  if (q.grid.y > 65535) return LCD_ERR_UNSUPPORTED;
  auto kern = vec ? (q.each ? mx_quantize_kernel<T, true, kRowsEach> : mx_quantize_kernel<T, true, 1>)
                  : (q.each ? mx_quantize_kernel<T, false, kRowsEach> : mx_quantize_kernel<T, false, 1>);
  return launched(launch_overlapping(kern, q.grid, q.block, 0, 1, s, static_cast<const T*>(x), M, K, ldx, inv, codes, ldc, scales, lds, units));
}

template <typename T>
lcd_status dequantize_rows(const uint8_t* codes, int64_t ldc, const uint8_t* scales, int64_t lds, int64_t M, int64_t K, void* out,
                           int64_t ldo, cudaStream_t s) {
  constexpr int E = 16 / sizeof(T);
  const uint32_t units = (uint32_t)((K + E - 1) / E);
  const Shape q = shape_of(M, units, kMxThreads);
  if (q.grid.y > 65535) return LCD_ERR_UNSUPPORTED;
  const bool vec = on16(out, ldo, sizeof(T), M);
  auto kern = vec ? (q.each ? mx_dequantize_kernel<T, true, kRowsEach> : mx_dequantize_kernel<T, true, 1>)
                  : (q.each ? mx_dequantize_kernel<T, false, kRowsEach> : mx_dequantize_kernel<T, false, 1>);
  return launched(launch_overlapping(kern, q.grid, q.block, 0, 1, s, codes, ldc, scales, lds, M, K, static_cast<T*>(out), ldo, units));
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
