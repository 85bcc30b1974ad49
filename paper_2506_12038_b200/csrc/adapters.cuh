// Low-rank adapters beside a shared layer: what the three kernels have in common (adapters_down.cuh: x a^T and dy b, adapters_up.cuh: t b^T
// and dt a, added to what is there, adapters_outer.cu: the adapters' gradients).
//
// All three are bound by the one pass over x, y, dy or dx (a rank of 64 needs 64 FLOP a byte of 16-bit activations), and with few rows by
// latency.  There operands go from memory to registers in the fragment order of mma.sync and nothing is staged: a sum does not care for
// the order of its terms, so a lane takes 16 consecutive bytes of its row for the slots that the instruction gives it, and both operands
// use the same order.  With many rows registers do not hold enough loads to keep memory busy (4096 x 5120 x 13824, rank 64, bf16: 206 us
// a call): those go through shared memory and tcgen05 (adapters_tc.cuh: 79 us).
//
// Arithmetic.  Two 16-bit operands of one type: their products are exact, sums are fp32.  The products with t or dt, which are fp32, whatever
// the result's type (terms may cancel): with bf16 beside them as three bf16 terms (24 bits: exact), else as two tf32 terms (within 2^-23 of
// the value; fp32 beside them likewise in two, the product of the rests, 2^-22, is left out).  On tcgen05 always as kPartsT bf16 terms.
#ifndef LCD_ADAPTERS_CUH_
#define LCD_ADAPTERS_CUH_

#include <type_traits>

#include "common.h"
#include "device_util.h"
#include "mx.cuh"

namespace lcd {

template <typename T> constexpr bool kIs16 = sizeof(T) == 2;

// D (16 x 8) += A (16 x 16) B (16 x 8) of 16-bit values, pairs in a word.
template <typename T>
__device__ __forceinline__ void mma16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if constexpr (std::is_same<T, __half>::value)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// D (16 x 8) += A (16 x 8) B (8 x 8) of tf32 values.
__device__ __forceinline__ void mma_tf32(float (&d)[4], float a0, float a1, float a2, float a3, float b0, float b1) {
  asm volatile("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(__float_as_uint(a0)), "r"(__float_as_uint(a1)), "r"(__float_as_uint(a2)), "r"(__float_as_uint(a3)),
                 "r"(__float_as_uint(b0)), "r"(__float_as_uint(b1)));
}

// v = upper + rest.  The upper part is never rounded up to an infinity (tf32: to the nearest, cut off where that would overflow; bf16: cut off),
// the rest is exact; an infinity has no rest.
__device__ __forceinline__ float nearest_tf32(float v) {
  uint32_t r;
  asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(r) : "f"(v));
  return __uint_as_float(r);
}
__device__ __forceinline__ float upper_tf32(float v) {
  const float r = nearest_tf32(v);
  return fabsf(r) == __uint_as_float(0x7f800000u) ? __uint_as_float(__float_as_uint(v) & 0xffffe000u) : r;
}
__device__ __forceinline__ float upper_bf16(float v) { return __uint_as_float(__float_as_uint(v) & 0xffff0000u); }
__device__ __forceinline__ float rest_of(float v, float upper) { return v == upper ? 0.0f : v - upper; }
// The same rounded to tf32, which the instruction would cut off.
__device__ __forceinline__ float rest_tf32(float v, float upper) { return nearest_tf32(rest_of(v, upper)); }
// Two values as a word of bf16: their upper parts, or rounded.
__device__ __forceinline__ uint32_t pair_upper(float lo, float hi) { return __byte_perm(__float_as_uint(lo), __float_as_uint(hi), 0x7632); }
__device__ __forceinline__ uint32_t pair_rounded(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// N consecutive values of a row as words.
template <typename T, int N>
struct Words {
  static constexpr int kCount = N * (int)sizeof(T) / 4;
  uint32_t w[kCount];
};
// The same at any alignment: the aligned words around them, then shifted (apart, so that several rows' loads are on their way together).
// The row has 16 bytes before them, and kCount words from their first on.
template <typename T, int N>
struct Around {
  static constexpr int kCount = (Words<T, N>::kCount + 3) / 4 * 4 + 4;
  uint32_t w[kCount];
};
template <typename T, int N>
__device__ __forceinline__ void load_around(Around<T, N>& out, const T* p, bool there) {
  const uint4* q = reinterpret_cast<const uint4*>(reinterpret_cast<uintptr_t>(p) & ~(uintptr_t)15);
#pragma unroll
  for (int i = 0; i < Around<T, N>::kCount; i += 4) {
    const uint4 v = there ? q[i / 4] : make_uint4(0u, 0u, 0u, 0u);
    out.w[i] = v.x; out.w[i + 1] = v.y; out.w[i + 2] = v.z; out.w[i + 3] = v.w;
  }
}
template <typename T, int N>
__device__ __forceinline__ void shift_words(Words<T, N>& out, const Around<T, N>& in, const T* p) {
  constexpr int kCount = Words<T, N>::kCount;
  const uint32_t off = (uint32_t)(reinterpret_cast<uintptr_t>(p) & 15u);
  uint32_t w[kCount + 2], u[kCount + 1];
#pragma unroll
  for (int i = 0; i < kCount + 2; ++i) w[i] = off & 8u ? in.w[i + 2] : in.w[i];
#pragma unroll
  for (int i = 0; i < kCount + 1; ++i) u[i] = off & 4u ? w[i + 1] : w[i];
#pragma unroll
  for (int i = 0; i < kCount; ++i) out.w[i] = kIs16<T> ? __byte_perm(u[i], u[i + 1], off & 2u ? 0x5432 : 0x3210) : u[i];
}
// Zeros where `have` ends.  wide: they lie on N * sizeof(T) bytes (16 at most) and are all there or none is.
template <typename T, int N>
__device__ __forceinline__ void load_words(Words<T, N>& out, const T* p, int have, bool wide) {
  constexpr int kCount = Words<T, N>::kCount;
  if (wide) {
    if (have > 0) {
      if constexpr (kCount >= 4) {
#pragma unroll
        for (int i = 0; i < kCount; i += 4) {
          const uint4 v = *reinterpret_cast<const uint4*>(reinterpret_cast<const uint32_t*>(p) + i);
          out.w[i] = v.x; out.w[i + 1] = v.y; out.w[i + 2] = v.z; out.w[i + 3] = v.w;
        }
      } else if constexpr (kCount == 2) {
        const uint2 v = *reinterpret_cast<const uint2*>(p);
        out.w[0] = v.x; out.w[1] = v.y;
      } else {
        out.w[0] = *reinterpret_cast<const uint32_t*>(p);
      }
    } else {
#pragma unroll
      for (int i = 0; i < kCount; ++i) out.w[i] = 0u;
    }
    return;
  }
  if constexpr (kIs16<T>) {
    const uint16_t* q = reinterpret_cast<const uint16_t*>(p);
#pragma unroll
    for (int i = 0; i < N; i += 2) {
      const uint32_t lo = i < have ? q[i] : 0u, hi = i + 1 < have ? q[i + 1] : 0u;
      out.w[i / 2] = lo | hi << 16;
    }
  } else {
    const uint32_t* q = reinterpret_cast<const uint32_t*>(p);
#pragma unroll
    for (int i = 0; i < N; ++i) out.w[i] = i < have ? q[i] : 0u;
  }
}
// Value i of them.
template <typename T, int N>
__device__ __forceinline__ float value_of(const Words<T, N>& v, int i) {
  if constexpr (std::is_same<T, float>::value) {
    return __uint_as_float(v.w[i]);
  } else if constexpr (std::is_same<T, __half>::value) {
    const __half2 h = *reinterpret_cast<const __half2*>(&v.w[i / 2]);
    return i % 2 ? __high2float(h) : __low2float(h);
  } else {
    return __uint_as_float(i % 2 ? v.w[i / 2] & 0xffff0000u : v.w[i / 2] << 16);
  }
}
// Value i of two rows as a word of 16-bit values.
template <typename T, int N>
__device__ __forceinline__ uint32_t pair_of(const Words<T, N>& a, const Words<T, N>& b, int i) {
  return __byte_perm(a.w[i / 2], b.w[i / 2], i % 2 ? 0x7632 : 0x5410);
}

// The bf16 parts of t and dt in the products behind them: 8 bits each.  (Two, 16 bits, left sums of cancelling terms off by 2^-16 of the
// terms.  Times with two and with three, bf16: 4096 x 5120 x 13824, rank 64, 16 adapters 84 and 90 us, the gradient of 4096 x 5120 x 5120,
// rank 32, 4 adapters 82 and 92.)
constexpr int kPartsT = 3;

// The plan of the rows and the adapters, as the kernels see them.
struct AdapterArgs {
  const int32_t *order, *groups, *offsets;
  int rows, G;
  int r;                       // the rank
  long long K;                 // columns of the long side of this launch's adapter matrix
  const void* w;               // adapter matrix: a [G][r][K] or b [G][K][r]
  long long ldw, sw;           // its rows' and adapters' pitch
  const float* scale;          // [G] or null
  int wide_w, wide_x;
};

// A row that the plan names, -1 where it is none.  (Where the plan is read ahead, the check waits until the row is used.)
__device__ __forceinline__ int checked_row(int row, int rows) { return (unsigned)row < (unsigned)rows ? row : -1; }
__device__ __forceinline__ int row_of(const int32_t* order, int at, int rows) { return checked_row(order[at], rows); }

// RT for a rank: 16 * RT is the rank padded.
constexpr int rank_tiles(int64_t r) { return r <= 16 ? 1 : r <= 32 ? 2 : r <= 64 ? 4 : 8; }
constexpr int kMostRank = 128;
// From this many rows on the products run on tcgen05 (adapters_tc.cuh), from twice as many where base and y, or x and the adapters of one
// 16-bit type, do not start on 16 bytes (never the gradients' sums).  Few rows' kernels and many's, us of a call / of the whole gradient, five
// adapters of rank 16:
//   rows                              384            512            768            1024           1536           2048
//   bf16, 4096 to 4096     few    17 /  32       22 /  38       26 /  44       32 /  52       42 /  67       50 /  81
//                          many   24 /  36       24 /  36       28 /  40       28 /  42       30 /  48       34 /  54
//   bf16, 1000 to 1000     few    17 /  24       17 /  24       17 /  26       17 /  26       22 /  38       24 /  40
//                          many   17 /  26       19 /  28       22 /  30       22 /  30       24 /  34       24 /  34
//   fp32, 4096 to 4096     few    26 /  50       32 /  56       38 /  71       46 /  83       60 / 110       73 / 134
//                          many   32 /  46       34 /  48       36 /  56       38 /  60       42 /  71       65 /  99
//   bf16, 4097 to 4099     few    26 /  46       32 /  52       42 /  71       48 /  79       64 / 106       79 / 128
//                          many   50 /  65       52 /  69       61 /  85       60 /  87       64 /  97       75 / 117
//   bf16, 5001 to 5003     few    28 /  48       36 /  58       44 /  77       54 /  87       71 / 118       89 / 146
//                          many   52 /  67       54 /  69       65 /  83       65 /  87       77 / 106       79 / 116
//   fp32, 4097 to 4099     few    38 /  58       46 /  65       54 /  85       67 /  99       89 / 134      110 / 165
//                          many   44 /  60       46 /  63       52 /  75       54 /  81       67 / 103       97 / 142
constexpr int kManyRows = 512;

template <typename F>
lcd_status by_rank(int64_t r, F&& f) {
  switch (rank_tiles(r)) {
    case 1: return f(std::integral_constant<int, 1>{});
    case 2: return f(std::integral_constant<int, 2>{});
    case 4: return f(std::integral_constant<int, 4>{});
    default: return f(std::integral_constant<int, 8>{});
  }
}
template <typename T> struct TypeTag { using type = T; };
template <typename F>
lcd_status by_dtype(lcd_dtype t, F&& f) {
  switch (t) {
    case LCD_DTYPE_F32: return f(TypeTag<float>{});
    case LCD_DTYPE_F16: return f(TypeTag<__half>{});
    default: return f(TypeTag<__nv_bfloat16>{});
  }
}
// Whether pieces of `bytes` bytes of rows with that pitch (elements) and, over several adapters, that distance can be loaded whole.
inline bool on_bytes(const void* p, int64_t pitch, int64_t distance, int64_t size, int64_t bytes) {
  return reinterpret_cast<uintptr_t>(p) % bytes == 0 && pitch * size % bytes == 0 && distance * size % bytes == 0;
}
inline lcd_status adapter_launched(cudaError_t e) {
  if (e != cudaSuccess) { set_cuda_error((int)e); return LCD_ERR_CUDA; }
  return LCD_OK;
}

}  // namespace lcd
#endif
