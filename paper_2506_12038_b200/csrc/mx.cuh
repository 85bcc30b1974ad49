// The microscaled 4-bit format on the device: one block of 32 columns is a scale 2^(byte - 127) and 32 elements of sign, two
// exponent bits and one mantissa bit.
#ifndef LCD_MX_CUH_
#define LCD_MX_CUH_

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

namespace lcd {

constexpr int kMxBlock = 32;

template <typename T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f32<__half>(__half v) { return __half2float(v); }
template <> __device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// Eight consecutive values as they lie in memory, from an address on 16 bytes.  Apart from their conversion, which waits for them.
template <typename T>
struct Raw8 {
  uint4 w[sizeof(T) == 4 ? 2 : 1];
};
template <typename T>
__device__ __forceinline__ Raw8<T> load8(const T* p) {
  Raw8<T> r;
  r.w[0] = *reinterpret_cast<const uint4*>(p);
  if constexpr (sizeof(T) == 4) r.w[1] = *reinterpret_cast<const uint4*>(p + 4);
  return r;
}
template <typename T>
__device__ __forceinline__ void values8(const Raw8<T>& r, float (&v)[8]) {
  if constexpr (sizeof(T) == 4) {
    const uint4 a = r.w[0], b = r.w[1];
    v[0] = __uint_as_float(a.x); v[1] = __uint_as_float(a.y); v[2] = __uint_as_float(a.z); v[3] = __uint_as_float(a.w);
    v[4] = __uint_as_float(b.x); v[5] = __uint_as_float(b.y); v[6] = __uint_as_float(b.z); v[7] = __uint_as_float(b.w);
  } else {
    const uint32_t w[4] = {r.w[0].x, r.w[0].y, r.w[0].z, r.w[0].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (std::is_same<T, __half>::value) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
        v[2 * i] = f.x; v[2 * i + 1] = f.y;
      } else {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      }
    }
  }
}
// Eight values as one 16-byte word of a 16-bit type.
template <typename T>
__device__ __forceinline__ uint4 pack8(const float (&v)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (std::is_same<T, __half>::value) {
      const __half2 h = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    } else {
      const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&v)[8]) {
  if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
  } else {
    *reinterpret_cast<uint4*>(p) = pack8<T>(v);
  }
}

// A block's scale byte from the bits of its largest magnitude (sign cleared).  Order of the bits is the order of the values, an
// infinity and every NaN above all others, so one integer maximum finds either.  A binary32 number with exponent field f has
// floor(log2) = f - 127, or less than -126 for f = 0, where the byte is 0 either way.
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t top_bits) {
  if (top_bits == 0u) return 127u;
  if (top_bits >= 0x7f800000u) return 255u;
  const uint32_t f = top_bits >> 23;
  return f > 2u ? f - 2u : 0u;
}
// 2^(127 - byte), what a block's values are multiplied by before they are rounded (exact: at most 2^127, at least 2^-125).
__device__ __forceinline__ float mx_inverse_scale(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }
// Eight values as eight codes, the first in the lowest nibble (nearest even, beyond 6: 6).
__device__ __forceinline__ uint32_t mx_codes8(const float (&v)[8]) {
  uint32_t c;
  asm("{\n.reg .b8 b0, b1, b2, b3;\n"
      "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n"
      "cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n"
      "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n"
      "cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n"
      "mov.b32 %0, {b0, b1, b2, b3};\n}"
      : "=r"(c) : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
  return c;
}
// What N codes under one scale byte stand for, the first in the lowest nibble.  A code's exponent and mantissa bits, put where a binary32
// number has them, are its value times 2^-126 (a subnormal number for .5), so that one multiplication does up to scales of 2.  (Not by
// cvt from .b8 parts of the word: where the word was a 16-bit load that way gave zeros from -O1 on, nvcc 12.9.86.)
template <int N>
__device__ __forceinline__ void mx_values(uint32_t c, uint32_t byte, float (&v)[N]) {
  const float s = __uint_as_float((min(byte, 128u) + 126u) << 23);
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = __fmul_rn(__uint_as_float((uint32_t)((int32_t)(c << (28 - 4 * i)) >> 6) & 0x81c00000u), s);
  if (byte > 128u) {
    const float more = __uint_as_float(byte == 255u ? 0x7fc00000u : (byte - 1u) << 23);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = __fmul_rn(v[i], more);
  }
}

}  // namespace lcd
#endif
