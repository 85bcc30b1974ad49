// Distillation from a teacher's top logits: loss and gradient (lcd_distill_loss, lcd_distill_grad).  With c = log2(e) / temperature,
// m the row's largest logit and s = sum_v 2^((z_v - m) c), per token
//     log q_v = (z_v - m) / temperature - log s,     loss = w * sum_j p_j (log p_j - log q_idx_j),
//     dz_v = w / temperature * (P * 2^((z_v - m) c) / s - sum_{j: idx_j = v} p_j).
// m and s come of one pass with a running maximum.  They are kept apart, not as one logarithm: with logits near the type's
// lowest value (masked ones) or merely large, the logarithm's rounding would be a large part of z - log s.  Sums are fp32.
#include <cfloat>
#include <type_traits>

#include "common.h"
#include "device_util.h"
#include "mx.cuh"

namespace lcd {

namespace {

constexpr int kDsThreads = 512;
constexpr int kMaxK = 1024;

__device__ __forceinline__ float exp2_fast(float v) {   // 2^-22 relative, results below the normal range are 0
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}

template <typename T> struct Vec { static constexpr int E = 16 / sizeof(T); };

// One 16-byte slot of a row: elements lo .. lo + E - 1, of which those outside [0, V) read as -infinity.
template <typename T, int E>
__device__ __forceinline__ void load_slot(const T* row, int64_t lo, int64_t V, float (&v)[E]) {
  if (lo >= 0 && lo + E <= V) {
    if constexpr (sizeof(T) == 4) {
      const float4 a = *reinterpret_cast<const float4*>(row + lo);
      v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    } else {
      load8(row + lo, v);
    }
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] = lo + i >= 0 && lo + i < V ? to_f32(row[lo + i]) : -INFINITY;
  }
}
template <typename T, int E>
__device__ __forceinline__ void store_slot(T* row, int64_t lo, int64_t V, bool wide, const float (&v)[E]) {
  if (wide && lo >= 0 && lo + E <= V) {
    if constexpr (sizeof(T) == 4) *reinterpret_cast<float4*>(row + lo) = make_float4(v[0], v[1], v[2], v[3]);
    else store8(row + lo, v);
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (lo + i >= 0 && lo + i < V) row[lo + i] = from_f32<T>(v[i]);
  }
}

struct Params {
  const void* z;
  int64_t V, ldz;
  const void* idx;
  int64_t ldi;
  const void* top;
  int64_t ldt;
  int k, idx_bytes, top_type;
  float inv_tau, c;
  const float *lse, *weight;
  float *loss, *stats;
  void* d;
  int64_t ldd;
};

template <int OP>   // 0: sum, 1: maximum; every thread gets the result, the order is fixed
__device__ __forceinline__ float block_reduce(float v, float* s_part) {
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    const float w = __shfl_xor_sync(0xffffffffu, v, o);
    v = OP ? fmaxf(v, w) : v + w;
  }
  __syncthreads();
  if ((threadIdx.x & 31) == 0) s_part[threadIdx.x >> 5] = v;
  __syncthreads();
  v = s_part[0];
  for (int i = 1; i < kDsThreads / 32; ++i) v = OP ? fmaxf(v, s_part[i]) : v + s_part[i];
  return v;
}

// LOSS: m, s and the loss (and the stats) are formed; otherwise they are read.  GRAD: the gradient is written.
template <typename T, bool LOSS, bool GRAD>
__global__ void __launch_bounds__(kDsThreads) distill_kernel(const Params P) {
  constexpr int E = Vec<T>::E, U = 4;
  __shared__ int s_idx[kMaxK];
  __shared__ float s_p[kMaxK], s_z[kMaxK], s_part[kDsThreads / 32];
  const int64_t t = blockIdx.x;
  const int tid = threadIdx.x;
  const T* row = static_cast<const T*>(P.z) + t * P.ldz;
  T* out = GRAD ? static_cast<T*>(P.d) + t * P.ldd : nullptr;
  const int off = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));      // the row's first element in its 16 bytes
  const int64_t slots = (P.V + off + E - 1) / E;
  const bool wide = ((reinterpret_cast<uintptr_t>(row) ^ reinterpret_cast<uintptr_t>(out)) & 15) == 0;
  const float w = P.weight ? P.weight[t] : 1.0f;
  if (w == 0.0f) {
    if (LOSS && tid == 0) {
      P.loss[t] = 0.0f;
      if (P.stats) P.stats[2 * t] = P.stats[2 * t + 1] = NAN;
    }
    if (GRAD) {
      const float zero[E] = {};
      for (int64_t i = tid; i < slots; i += kDsThreads) store_slot<T, E>(out, i * E - off, P.V, wide, zero);
    }
    return;
  }
  // the teacher's entries: index (-1: absent) and p
  float high = -FLT_MAX;
  for (int j = tid; j < P.k; j += kDsThreads) {
    const int64_t i = P.idx_bytes == 4 ? static_cast<const int32_t*>(P.idx)[t * P.ldi + j] : static_cast<const int64_t*>(P.idx)[t * P.ldi + j];
    bool there = i >= 0 && i < P.V;
    const int64_t at = t * P.ldt + j;
    float v = -INFINITY;
    if (there) {
      v = P.inv_tau * (P.top_type == LCD_DTYPE_F32 ? static_cast<const float*>(P.top)[at]
                       : P.top_type == LCD_DTYPE_F16 ? __half2float(static_cast<const __half*>(P.top)[at])
                                                     : __bfloat162float(static_cast<const __nv_bfloat16*>(P.top)[at]));
      there = v != -INFINITY;      // p = 0: as if it were absent
    }
    s_idx[j] = there ? (int)i : -1;
    s_p[j] = v;
    s_z[j] = there ? to_f32(row[i]) : 0.0f;
    high = fmaxf(high, v);
  }
  high = block_reduce<1>(high, s_part);
  float norm;          // log p = (v - high) - norm
  if (P.lse) {
    norm = P.lse[t] - high;
  } else {
    float sum = 0.0f;
    for (int j = tid; j < P.k; j += kDsThreads) sum += s_idx[j] >= 0 ? expf(s_p[j] - high) : 0.0f;
    norm = logf(block_reduce<0>(sum, s_part));
  }
  float m, s;
  if (LOSS) {
    m = -FLT_MAX;
    s = 0.0f;
    for (int64_t i = tid; i < slots; i += U * kDsThreads) {
      float v[U][E];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (i + u * kDsThreads < slots) load_slot<T, E>(row, (i + u * kDsThreads) * E - off, P.V, v[u]);
        else
#pragma unroll
          for (int e = 0; e < E; ++e) v[u][e] = -INFINITY;
      }
      float b = m;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < E; ++e) b = fmaxf(b, v[u][e]);
      s *= exp2_fast((m - b) * P.c);
      m = b;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < E; ++e) s += exp2_fast((v[u][e] - m) * P.c);
    }
    const float all = block_reduce<1>(m, s_part);
    s = block_reduce<0>(s * exp2_fast((m - all) * P.c), s_part);
    m = all;
    if (tid == 0 && P.stats) {
      P.stats[2 * t] = m;
      P.stats[2 * t + 1] = s;
    }
  } else {
    m = P.stats[2 * t];
    s = P.stats[2 * t + 1];
  }
  float part = 0.0f, mass = 0.0f;
  const float log_s = logf(s);
  for (int j = tid; j < P.k; j += kDsThreads) {
    float p = 0.0f;
    if (s_idx[j] >= 0) {
      const float logp = (s_p[j] - high) - norm;
      p = expf(logp);
      if (LOSS && p != 0.0f) part += p * (logp - ((s_z[j] - m) * P.inv_tau - log_s));
    }
    s_p[j] = p;
    mass += p;
  }
  if (LOSS) {
    part = block_reduce<0>(part, s_part);
    if (tid == 0) P.loss[t] = w * part;
  }
  if (GRAD) {
    mass = block_reduce<0>(mass, s_part);     // (its barriers also make every p visible)
    const float wt = w * P.inv_tau, scale = wt * mass / s;
    if (mass == 0.0f) {                       // no entries
      const float zero[E] = {};
      for (int64_t i = tid; i < slots; i += kDsThreads) store_slot<T, E>(out, i * E - off, P.V, wide, zero);
      return;
    }
    for (int64_t i = tid; i < slots; i += kDsThreads) {
      float v[E];
      load_slot<T, E>(row, i * E - off, P.V, v);
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = scale * exp2_fast((v[e] - m) * P.c);
      store_slot<T, E>(out, i * E - off, P.V, wide, v);
    }
    __syncthreads();
    for (int j = tid; j < P.k; j += kDsThreads) {
      const int i = s_idx[j];
      if (i < 0) continue;
      float sum = 0.0f;                       // an index that comes twice: every one of its entries writes the same
      for (int l = 0; l < P.k; ++l) sum += s_idx[l] == i ? s_p[l] : 0.0f;
      out[i] = from_f32<T>(wt * (mass * (exp2_fast((s_z[j] - m) * P.c) / s) - sum));
    }
  }
}

template <typename T>
lcd_status launch_typed(const Params& p, int64_t rows, bool loss, bool grad, cudaStream_t s) {
  auto kern = loss ? (grad ? distill_kernel<T, true, true> : distill_kernel<T, true, false>) : distill_kernel<T, false, true>;
  kern<<<(unsigned)rows, kDsThreads, 0, s>>>(p);
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) { set_cuda_error((int)e); return LCD_ERR_CUDA; }
  return LCD_OK;
}

}  // namespace

lcd_status launch_distill(const Distillation& d, void* stream) {
  Params p = {};
  p.z = d.logits;
  p.V = d.V;
  p.ldz = d.ldz;
  p.idx = d.teacher_idx;
  p.ldi = d.ldi;
  p.top = d.teacher_logits;
  p.ldt = d.ldt;
  p.k = (int)d.k;
  p.idx_bytes = d.idx_bytes;
  p.top_type = (int)d.teacher_type;
  p.inv_tau = 1.0f / d.temperature;
  p.c = (float)(1.4426950408889634 / (double)d.temperature);
  p.lse = d.teacher_lse;
  p.weight = d.weight;
  p.loss = d.loss;
  p.stats = d.stats;
  p.d = d.dlogits;
  p.ldd = d.ldd;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool loss = d.loss != nullptr, grad = d.dlogits != nullptr;
  switch (d.type) {
    case LCD_DTYPE_F32: return launch_typed<float>(p, d.T, loss, grad, s);
    case LCD_DTYPE_F16: return launch_typed<__half>(p, d.T, loss, grad, s);
    default: return launch_typed<__nv_bfloat16>(p, d.T, loss, grad, s);
  }
}

}  // namespace lcd
