// Distillation from a teacher's top logits: loss and gradient (lcd_distill_loss, lcd_distill_grad).  With c = log2(e) / temperature,
// m the row's largest logit and s = sum_v 2^((z_v - m) c), per token
//     log q_v = (z_v - m) / temperature - log s,     loss = w * sum_j p_j (log p_j - log q_idx_j),
//     dz_v = w / temperature * (P * 2^((z_v - m) c) / s - sum_{j: idx_j = v} p_j).
// m and s are kept apart, not as one logarithm: with logits near the type's lowest value (masked ones) or merely large, the
// logarithm's rounding would be a large part of z - log s.  Sums are fp32.
//
// The work is bytes and exponentials: the logits are read once, the gradient is written once, two exponentials a logit (the unit
// for them makes 16 a clock and multiprocessor: 263 us of 4096 x 128000, of which the bytes take 320).  Two forms:
//   distill_stream_kernel  a CTA per row and one after the other, copies running ahead through a ring in shared memory;
//   distill_kernel         few long rows: a cluster per row, whose threads hold it in registers.
// 4096 x 128000 bf16, k = 128, loss and gradient: 452 us alone, 4.6 TB/s of what has to move (5.5 with what is read again); loss of
// 4440 x 32000 61 us, 4.7 TB/s (49 without the exponentials).  What bounds them: neither bytes nor the exponentials' unit, 55 to 67 and
// 58 % busy, but the latencies of a row's beginning and end, which 16 to 24 warps an SM cover in part.
#include <cfloat>
#include <type_traits>

#include "common.h"
#include "device_util.h"
#include "mx.cuh"

namespace lcd {

namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kSlots = 4;             // 16-byte words of a row that a thread holds
constexpr int kMaxK = 1024, kMaxCluster = 8;

__device__ __forceinline__ float exp2_fast(float v) {   // 2^-22 relative, results below the normal range are 0
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}

// A slot is 16 bytes of a row, elements lo .. lo + E - 1; those outside [0, V) read as -infinity and are not written.
template <typename T>
struct Slot {
  static constexpr int E = 16 / sizeof(T);
  static __device__ __forceinline__ uint4 load(const T* row, int64_t lo, int64_t V) {
    if (lo >= 0 && lo + E <= V) return *reinterpret_cast<const uint4*>(row + lo);
    T v[E];
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] = lo + i >= 0 && lo + i < V ? row[lo + i] : from_f32<T>(-INFINITY);
    uint4 w;
    memcpy(&w, v, 16);
    return w;
  }
  static __device__ __forceinline__ void store_all(T* p, const float (&v)[E]) {
    uint4 w;
    if constexpr (sizeof(T) == 4) w = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
    else w = pack8<T>(v);
    *reinterpret_cast<uint4*>(p) = w;
  }
  static __device__ __forceinline__ void store(T* row, int64_t lo, int64_t V, bool wide, const float (&v)[E]) {
    if (wide && lo >= 0 && lo + E <= V) {
      store_all(row + lo, v);
    } else {
#pragma unroll
      for (int i = 0; i < E; ++i)
        if (lo + i >= 0 && lo + i < V) row[lo + i] = from_f32<T>(v[i]);
    }
  }
};

// A maximum and a sum of 2^((v - maximum) c).
struct Pair { float m, s; };
// Two binary32 numbers in a register pair: one instruction adds or multiplies both.
__device__ __forceinline__ uint64_t pair2(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 both(uint64_t p) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(p));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// A 16-byte word as E / 2 pairs.
template <typename T>
__device__ __forceinline__ void pairs_of(const uint4& w, uint64_t (&v)[Slot<T>::E / 2]) {
  const uint32_t x[4] = {w.x, w.y, w.z, w.w};
  if constexpr (sizeof(T) == 4) {
    v[0] = (uint64_t)w.y << 32 | w.x;
    v[1] = (uint64_t)w.w << 32 | w.z;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (std::is_same<T, __half>::value) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&x[i]));
        v[i] = pair2(f.x, f.y);
      } else {
        v[i] = pair2(__uint_as_float(x[i] << 16), __uint_as_float(x[i] & 0xffff0000u));
      }
    }
  }
}
// The largest element of N words, NaN left out.
template <typename T, int N>
__device__ __forceinline__ float largest(const uint4 (&w)[N]) {
  if constexpr (sizeof(T) == 4) {
    float b = -FLT_MAX;
#pragma unroll
    for (int u = 0; u < N; ++u)
      b = fmaxf(b, fmaxf(fmaxf(__uint_as_float(w[u].x), __uint_as_float(w[u].y)), fmaxf(__uint_as_float(w[u].z), __uint_as_float(w[u].w))));
    return b;
  } else {
    using T2 = typename std::conditional<std::is_same<T, __half>::value, __half2, __nv_bfloat162>::type;
    auto as2 = [](const uint32_t& x) { return *reinterpret_cast<const T2*>(&x); };
    T2 b = __hmax2(__hmax2(as2(w[0].x), as2(w[0].y)), __hmax2(as2(w[0].z), as2(w[0].w)));
#pragma unroll
    for (int u = 1; u < N; ++u) b = __hmax2(b, __hmax2(__hmax2(as2(w[u].x), as2(w[u].y)), __hmax2(as2(w[u].z), as2(w[u].w))));
    return fmaxf(to_f32(b.x), to_f32(b.y));
  }
}
template <typename T>
__device__ __forceinline__ uint4 no_logits() {       // a word of -infinity
  const uint32_t x = sizeof(T) == 4 ? 0xff800000u : std::is_same<T, __half>::value ? 0xfc00fc00u : 0xff80ff80u;
  return make_uint4(x, x, x, x);
}
// Adds N words to a pair.
template <typename T, int N>
__device__ __forceinline__ void add_words(const uint4 (&w)[N], float c, Pair& a) {
  const float b = fmaxf(a.m, largest<T, N>(w));
  const uint64_t nb = pair2(-b, -b), cc = pair2(c, c);
  uint64_t s[2] = {pair2(a.s * exp2_fast((a.m - b) * c), 0.0f), 0};
#pragma unroll
  for (int u = 0; u < N; ++u) {
    uint64_t v[Slot<T>::E / 2];
    pairs_of<T>(w[u], v);
#pragma unroll
    for (int i = 0; i < Slot<T>::E / 2; ++i) {
      const float2 x = both(mul2(add2(v[i], nb), cc));
      s[i & 1] = add2(s[i & 1], pair2(exp2_fast(x.x), exp2_fast(x.y)));
    }
  }
  const float2 t = both(add2(s[0], s[1]));
  a.m = b;
  a.s = t.x + t.y;
}
// scale * 2^((z - m) c) of a word's elements.
template <typename T>
__device__ __forceinline__ void shares(const uint4& w, float m, float c, float scale, float (&g)[Slot<T>::E]) {
  uint64_t v[Slot<T>::E / 2];
  pairs_of<T>(w, v);
#pragma unroll
  for (int i = 0; i < Slot<T>::E / 2; ++i) {
    const float2 x = both(mul2(add2(v[i], pair2(-m, -m)), pair2(c, c)));
    const float2 y = both(mul2(pair2(exp2_fast(x.x), exp2_fast(x.y)), pair2(scale, scale)));
    g[2 * i] = y.x;
    g[2 * i + 1] = y.y;
  }
}

struct Params {
  const void* z;
  int64_t V, ldz;
  const void* idx;
  int64_t ldi;
  const void* top;
  int64_t ldt;
  int k, idx_bytes, top_type, parts;     // parts: CTAs a row
  float inv_tau, c;
  const float *lse, *weight;
  float *loss, *stats;
  void* d;
  int64_t ldd;
};

// All lanes get the warp's pair.
__device__ __forceinline__ Pair warp_pair(Pair a, float c) {
  float m = a.m;
#pragma unroll
  for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  float s = a.s * exp2_fast((a.m - m) * c);
#pragma unroll
  for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  return {m, s};
}
// The same of WARPS warps' pairs and numbers (behind a barrier), a power of two.
template <int WARPS>
__device__ __forceinline__ Pair pair_of(const Pair* part, float c) {
  const Pair a = part[threadIdx.x & (WARPS - 1)];
  float m = a.m;
#pragma unroll
  for (int o = WARPS / 2; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  float s = a.s * exp2_fast((a.m - m) * c);
#pragma unroll
  for (int o = WARPS / 2; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  return {m, s};
}
template <int WARPS>
__device__ __forceinline__ float sum_of(const float* part) {
  float s = part[threadIdx.x & (WARPS - 1)];
#pragma unroll
  for (int o = WARPS / 2; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  return s;
}
// The same of any number of warps, in every warp.
__device__ __forceinline__ Pair pair_of_warps(const Pair* part, int warps, float c) {
  const int lane = threadIdx.x & 31;
  return warp_pair(lane < warps ? part[lane] : Pair{-FLT_MAX, 0.0f}, c);
}
template <typename V>
__device__ __forceinline__ V warp_sum(V v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Terms of a row's loss, added before the row's maximum m is known and against a reference of their own: of the entries added (p != 0)
// the one with the largest student's logit r; v is the teacher's there.  part = sum of p ((t - v) - (z - r)) / temperature.  Then
//     loss = sum over shares of part + mass * ((v - r - t_max + m) / temperature - log sum_j exp((t_j - t_max) / temperature) + log s),
// the parentheses with what their roundings lose added at the end: log p and log q are each ten or more times the loss (256 x 32000 at
// temperature 2 with teacher_lse, against 64 bits: 1.8e-7 relative, root mean square; 7.5e-7 with log p and log s summed apart).  The reference
// is of THESE entries, not of other logits, which may all be masked: every z lies at or below r and r at or below m, so that what a
// lane, a warp and the row add, (r' - r) / temperature for the sum's p, is never negative and large parts do not cancel.
struct Share { float r, v, part; };
// Adds an entry to a share whose entries so far have p's sum `mass`.
__device__ __forceinline__ void add_entry(Share& a, float mass, float p, float t, float z, float inv_tau) {
  if (p == 0.0f) return;
  const float r = fmaxf(a.r, z);
  if (mass == 0.0f || r > a.r) {
    if (mass != 0.0f) a.part += mass * (((a.v - t) - (a.r - r)) * inv_tau);
    a.r = r;
    a.v = t;
  }
  a.part += p * (((t - a.v) - (z - a.r)) * inv_tau);
}
// The lanes' shares together, in every lane.  `mass`: the lane's sum of p.
__device__ __forceinline__ Share warp_share(Share a, float mass, float inv_tau) {
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(a.r));       // (five shuffles: 4440 x 32000, k = 128, 62.0 us, 61.2 so)
  const unsigned at = __ballot_sync(0xffffffffu, mass != 0.0f && a.r == r);
  const float v = __shfl_sync(0xffffffffu, a.v, at ? __ffs(at) - 1 : 0);
  if (mass != 0.0f) a.part += mass * (((a.v - v) - (a.r - r)) * inv_tau);
  return {r, v, warp_sum(a.part)};
}
// A sum and what its rounding lost.
__device__ __forceinline__ float two_sum(float a, float b, float& lost) {
  const float s = __fadd_rn(a, b), t = __fsub_rn(s, a);
  lost = __fadd_rn(__fsub_rn(a, __fsub_rn(s, t)), __fsub_rn(b, t));
  return s;
}
// log s = whole * log 2 + rest, rest within [0, log 2] (s >= 1; but for rows without a finite logit, where rest is all of it).
__device__ __forceinline__ void split_log(float s, float& whole, float& rest) {
  const uint32_t bits = __float_as_uint(s);
  const bool fine = s >= 1.0f && s <= FLT_MAX;
  whole = fine ? (float)((int)(bits >> 23) - 127) : 0.0f;
  rest = logf(fine ? __uint_as_float((bits & 0x007fffffu) | 0x3f800000u) : s);
}
// A share's part of the loss.  `all`: m and s of the row; the teacher's normalisation is *lse, or the pair of its logits.
__device__ __forceinline__ float share_loss(float mass, const Share& a, const Pair& all, const Pair& teacher, const float* lse, float inv_tau) {
  constexpr float kLog2Hi = 0.693145751953125f, kLog2Lo = 1.42860682030941723e-6f;       // 16 bits, so that their products are exact; the rest
  float whole, rest, whole_t = 0.0f, rest_t = 0.0f, lost[5];
  split_log(all.s, whole, rest);
  if (!lse) split_log(teacher.s, whole_t, rest_t);
  const float n = whole - whole_t;
  const float t = two_sum(a.v, lse ? 0.0f : -teacher.m, lost[0]), below = two_sum(all.m, -a.r, lost[1]);
  const float both = two_sum(t, below, lost[2]), scaled = both * inv_tau;
  const float logs = two_sum(n * kLog2Hi, lse ? -*lse : 0.0f, lost[3]);
  float sum = two_sum(scaled, logs, lost[4]);
  if (fabsf(sum) <= FLT_MAX) sum += ((lost[3] + lost[4]) + fmaf(lost[0] + (lost[1] + lost[2]), inv_tau, fmaf(both, inv_tau, -scaled))) + n * kLog2Lo;
  sum += rest - rest_t;
  return mass == 0.0f ? 0.0f : a.part + mass * sum;
}
// The teacher's probabilities are exp((t - from) / temperature - norm): differences of its logits, as large ones divided by the temperature
// would not keep them; with teacher_lse from = 0 and norm is that.
struct Teacher { float from, norm; };
__device__ __forceinline__ Teacher teacher_of(const Pair& top, const float* lse) {
  return lse ? Teacher{0.0f, *lse} : Teacher{top.m, logf(top.s)};
}
__device__ __forceinline__ float probability(float t, const Teacher& teacher, float inv_tau) {
  return expf(fmaf(t - teacher.from, inv_tau, -teacher.norm));
}

// What the CTAs of a row tell one another: the pair of their logits, the share of the entries in their slots, and the sum of p over those.
struct alignas(16) Word { float m, s, own, r, v, part, unused[2]; };

// LOSS: m, s and the loss (and the stats) are formed, by a cluster; otherwise they are read.  GRAD: the gradient is written.
// ONCE: the row fits the registers of its CTAs.
template <typename T, bool LOSS, bool GRAD, bool ONCE>
__global__ void __launch_bounds__(kThreads, 2) distill_kernel(const Params P) {
  using S = Slot<T>;
  constexpr int E = S::E;
  __shared__ int s_idx[kMaxK];
  __shared__ float s_t[kMaxK], s_p[kMaxK], s_z[kMaxK];
  __shared__ Pair s_top[kWarps], s_row[kWarps];
  __shared__ float s_mass[kWarps];
  __shared__ Word s_word[kMaxCluster];
  begin_after_previous();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, threads = blockDim.x, warps = threads >> 5;
  const int64_t t = blockIdx.x / P.parts;
  const int rank = blockIdx.x % P.parts;
  const T* row = static_cast<const T*>(P.z) + t * P.ldz;
  T* out = GRAD ? static_cast<T*>(P.d) + t * P.ldd : nullptr;
  const int off = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));      // the row's first element in its 16 bytes
  const int64_t slots = (P.V + off + E - 1) / E;
  const int64_t first = slots * rank / P.parts;                                    // this CTA's slots: first .. first + count - 1
  const int count = (int)(slots * (rank + 1) / P.parts - first);
  const int64_t lo0 = first * E - off;
  const bool wide = ((reinterpret_cast<uintptr_t>(row) ^ reinterpret_cast<uintptr_t>(out)) & 15) == 0;
  const float w = P.weight ? P.weight[t] : 1.0f;
  const float zero[E] = {};
  if (w == 0.0f) {
    if (LOSS && rank == 0 && tid == 0) {
      P.loss[t] = 0.0f;
      if (P.stats) P.stats[2 * t] = P.stats[2 * t + 1] = NAN;
    }
    if (GRAD)
      for (int i = tid; i < count; i += threads) S::store(out, lo0 + (int64_t)i * E, P.V, wide, zero);
    return;
  }
  if (LOSS && P.parts > 1) asm volatile("barrier.cluster.arrive.release;" ::: "memory");   // every CTA of the cluster has begun
  uint4 raw[kSlots];
  auto load = [&](int round) {
#pragma unroll
    for (int u = 0; u < kSlots; ++u) {
      const int i = (round * kSlots + u) * threads + tid;
      raw[u] = i < count ? S::load(row, lo0 + (int64_t)i * E, P.V) : no_logits<T>();
    }
  };
  const int rounds = ONCE ? 1 : (count + kSlots * threads - 1) / (kSlots * threads);
  if (LOSS || ONCE) load(0);

  // the teacher's entries: index (-1: absent or p = 0), t, and z of those in this CTA's slots
  Pair top = {-FLT_MAX, 0.0f};
  for (int j = tid; j < P.k; j += threads) {
    const int64_t i = P.idx_bytes == 4 ? static_cast<const int32_t*>(P.idx)[t * P.ldi + j] : static_cast<const int64_t*>(P.idx)[t * P.ldi + j];
    bool there = i >= 0 && i < P.V;
    const int64_t at = t * P.ldt + j;
    float v = -INFINITY;
    if (there) {
      v = P.top_type == LCD_DTYPE_F32 ? static_cast<const float*>(P.top)[at]
          : P.top_type == LCD_DTYPE_F16 ? __half2float(static_cast<const __half*>(P.top)[at])
                                        : __bfloat162float(static_cast<const __nv_bfloat16*>(P.top)[at]);
      there = v != -INFINITY;
    }
    s_idx[j] = there ? (int)i : -1;
    s_t[j] = v;
    s_z[j] = there && i >= lo0 && i < lo0 + (int64_t)count * E ? to_f32(row[i]) : 0.0f;
    if (there) {
      const float m = fmaxf(top.m, v);
      top.s = top.s * expf((top.m - m) * P.inv_tau) + expf((v - m) * P.inv_tau);
      top.m = m;
    }
  }
  top = warp_pair(top, P.c);
  if (lane == 0) s_top[warp] = top;
  __syncthreads();
  top = pair_of_warps(s_top, warps, P.c);
  const Teacher teacher = teacher_of(top, P.lse ? P.lse + t : nullptr);
  float mass = 0.0f;
  for (int j = tid; j < P.k; j += threads) {
    const float p = s_idx[j] >= 0 ? probability(s_t[j], teacher, P.inv_tau) : 0.0f;
    s_p[j] = p;
    mass += p;
  }
  mass = warp_sum(mass);
  if (lane == 0) s_mass[warp] = mass;

  Pair all;
  if (LOSS) {
    Pair a = {-FLT_MAX, 0.0f};
    for (int r = 0; r < rounds; ++r) {
      if (r) load(r);
      add_words<T, kSlots>(raw, P.c, a);
    }
    a = warp_pair(a, P.c);
    if (lane == 0) s_row[warp] = a;
  }
  __syncthreads();
  mass = warp_sum(lane < warps ? s_mass[lane] : 0.0f);
  if (LOSS) {
    all = pair_of_warps(s_row, warps, P.c);
    float own = 0.0f;
    Share share = {-FLT_MAX, 0.0f, 0.0f};
    if (warp == 0) {
      for (int j = lane; j < P.k; j += 32) {
        const int i = s_idx[j];
        const float p = s_p[j];
        if (i >= 0 && p != 0.0f && i >= lo0 && i < lo0 + (int64_t)count * E) {
          add_entry(share, own, p, s_t[j], s_z[j], P.inv_tau);
          own += p;
        }
      }
      share = warp_share(share, own, P.inv_tau);
      own = warp_sum(own);
    }
    if (P.parts > 1) {
      asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
      if (tid < P.parts) {
        const uint32_t mine = (uint32_t)__cvta_generic_to_shared(&s_word[rank]);
        uint32_t at;
        asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(mine), "r"(tid));
        asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(at), "f"(all.m), "f"(all.s), "f"(own), "f"(share.r) : "memory");
        asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(at + 16), "f"(share.v), "f"(share.part) : "memory");
      }
      asm volatile("barrier.cluster.arrive.release;" ::: "memory");
      asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
      all.m = s_word[0].m;
      for (int i = 1; i < P.parts; ++i) all.m = fmaxf(all.m, s_word[i].m);
      all.s = 0.0f;
      for (int i = 0; i < P.parts; ++i) all.s += s_word[i].s * exp2_fast((s_word[i].m - all.m) * P.c);
    }
    float sum = 0.0f;
    if (rank == 0 && warp == 0) {          // a lane per CTA
      if (P.parts > 1) {
        const Word o = s_word[lane & (kMaxCluster - 1)];
        own = lane < P.parts ? o.own : 0.0f;
        share = {o.r, o.v, o.part};
      }
      const float* lse = P.lse ? P.lse + t : nullptr;
      sum = share_loss(own, share, all, top, lse, P.inv_tau);
      if (P.parts > 1) sum = warp_sum(sum);
    }
    if (rank == 0 && tid == 0) {
      P.loss[t] = mass == 0.0f ? 0.0f : w * sum;
      if (P.stats) {
        P.stats[2 * t] = all.m;
        P.stats[2 * t + 1] = all.s;
      }
    }
  } else {
    all.m = P.stats[2 * t];
    all.s = P.stats[2 * t + 1];
  }
  if (GRAD) {
    const float wt = w * P.inv_tau, scale = wt * mass / all.s;
    for (int r = 0; r < rounds; ++r) {
      if (!ONCE) load(r);
#pragma unroll
      for (int u = 0; u < kSlots; ++u) {
        const int i = (r * kSlots + u) * threads + tid;
        if (i < count) {
          float v[E] = {};
          if (mass != 0.0f) shares<T>(raw[u], all.m, P.c, scale, v);
          S::store(out, lo0 + (int64_t)i * E, P.V, wide, v);
        }
      }
    }
    __syncthreads();
    // the entries, a warp each: an index that comes twice has all of its p, and every one of its entries writes the same
    for (int j = warp; j < P.k; j += warps) {
      const int i = s_idx[j];
      if (i < lo0 || i < 0 || i >= lo0 + (int64_t)count * E || mass == 0.0f) continue;
      float sum = 0.0f;
      for (int l = lane; l < P.k; l += 32) sum += s_idx[l] == i ? s_p[l] : 0.0f;
      sum = warp_sum(sum);
      if (lane == 0) out[i] = from_f32<T>(wt * (mass * (exp2_fast((s_z[j] - all.m) * P.c) / all.s) - sum));
    }
  }
}

// ---------------------------------------------------------------------------------------------------------
// Many rows: a CTA takes one row after the other and its threads copy ahead (cp.async) into a ring in shared memory, each thread
// the words that it reads itself, so that nothing is waited for but one's own copies and memory is busy through the reductions,
// into the next row.  A row's last kDepth chunks stay in the ring between the sum and the gradient, the others are copied twice,
// the second time out of L2, as far as the rows in work fit there.  The teacher's entries of a row are asked for
// while the row before is worked on; the student's logits there when the row has been read, out of L2 (before it is read they are
// single accesses to DRAM: of 4440 x 32000, k = 128, loss 77 us, 62 so), but for the gradient alone, which may take the row's place.
constexpr int kStreamSlots = 4;       // words a thread has of a chunk
template <int THREADS> constexpr int kStreamPerSm = THREADS == 128 ? 6 : 2;
constexpr int kDepth = 4;             // chunks of the ring

__device__ __forceinline__ void copy_wait(int newer) {      // all copies but the `newer` last groups have landed
  if (newer >= kDepth - 1) asm volatile("cp.async.wait_group %0;" ::"n"(kDepth - 1) : "memory");
  else if (newer == 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
  else if (newer == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
  else asm volatile("cp.async.wait_group 0;" ::: "memory");
}

struct Entries {         // of three rows in turn, k each: a row's are read until the last warp has left it
  int* idx;
  float *p, *z;          // p holds t first
};
// write(index, sum of its p, its logit) for every entry, k / warps of them a warp.  An index that comes twice has all of its p, in the
// entries' order, and each of its entries writes the same.  Whether any does is seen by counting what is equal to a warp's
// entries: a lane holds four of 128 and each entry is compared with them (k = 128, 8 warps: 150 instructions a warp; a sum for
// every entry takes 1300).
template <typename Write>
__device__ __forceinline__ void fix_entries(const Entries& n, int k, int warps, Write&& write) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int each = (k + warps - 1) / warps, from = warp * each, to = min(k, from + each);
  int equal = 0, there = 0;
  for (int b = 0; b < k; b += 128) {
    int x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = b + 32 * i + lane < k ? n.idx[b + 32 * i + lane] : -1;
    for (int j = from; j < to; ++j) {
      const int i = n.idx[j];
      if (i < 0) continue;
      there += b == 0;
#pragma unroll
      for (int q = 0; q < 4; ++q) equal += x[q] == i;
    }
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) equal += __shfl_xor_sync(0xffffffffu, equal, o);
  for (int j = from + lane; j < to; j += 32) {
    const int i = n.idx[j];
    if (i < 0) continue;
    float p = n.p[j];
    if (equal > there) {
      p = 0.0f;
      for (int l = 0; l < k; ++l) p += n.idx[l] == i ? n.p[l] : 0.0f;
    }
    write(i, p, n.z[j]);
  }
}

// THREADS a CTA: what a row costs beside its logits is done by every warp, so that few warps are better, but then more rows are in work.
template <typename T, bool LOSS, bool GRAD, int THREADS>
__global__ void __launch_bounds__(THREADS, kStreamPerSm<THREADS>) distill_stream_kernel(const Params P, const int64_t rows) {
  using S = Slot<T>;
  constexpr int kStreamThreads = THREADS, kStreamWarps = THREADS / 32;
  constexpr int kChunkSlots = THREADS * kStreamSlots, kChunkBytes = kChunkSlots * 16;
  constexpr int E = S::E;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ Pair s_top[2][kStreamWarps], s_row[2][kStreamWarps];
  __shared__ float s_mass[2][kStreamWarps];
  __shared__ Share s_share[2][kStreamWarps];
  __shared__ Pair s_teacher[2];
  constexpr int kLossWarp = kStreamWarps - 1;        // has no entries unless there are many (4096 x 1000, k = 64: 19.1 us, by warp 0 20.7)
  begin_after_previous();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  uint4* ring = reinterpret_cast<uint4*>(smem) + tid;
  auto entries = [&](int place) {
    Entries n;
    n.idx = reinterpret_cast<int*>(smem + kDepth * kChunkBytes) + place * 3 * P.k;
    n.p = reinterpret_cast<float*>(n.idx + P.k);
    n.z = n.p + P.k;
    return n;
  };
  const uint8_t* base = static_cast<const uint8_t*>(P.z);
  const int V = (int)P.V;
  struct Row {
    const uint8_t* at;               // the first word: the row begins `off` elements into it
    int off, words, full, chunks, first, wholes;       // words first .. full - 1 and chunks first .. first + wholes - 1 lie inside the row
    __device__ bool whole(int chunk) const { return (unsigned)(chunk - first) < (unsigned)wholes; }
  };
  auto row_of = [&](int64_t t) {
    Row r;
    const uint8_t* p = base + t * P.ldz * (int64_t)sizeof(T);
    const int bytes = (int)(reinterpret_cast<uintptr_t>(p) & 15);
    r.at = p - bytes;
    r.off = bytes / (int)sizeof(T);
    const uint32_t end = (uint32_t)V + (uint32_t)r.off;
    r.words = (int)((end + E - 1) / E);
    r.full = (int)(end / E);
    r.chunks = (int)((end + E * kChunkSlots - 1) / (E * kChunkSlots));
    r.first = r.off > 0;
    r.wholes = max(0, (int)(end / (E * kChunkSlots)) - r.first);
    asm volatile("" : "+r"(r.off), "+r"(r.words), "+r"(r.full), "+r"(r.chunks), "+r"(r.first), "+r"(r.wholes));    // not formed again at each use
    return r;
  };

  // ---- the copies.  With a gradient a row goes through the ring forwards for the sum, and its last kDepth chunks stay there; then
  // backwards for the gradient, those first and the others copied again, the latest of them first, which are the likeliest to be in
  // L2.  So places are taken in one direction by a row's sum and in the other by its gradient and by the next row's sum.  (kDepth
  // is a power of two.)
  // The gradient alone goes backwards too, over rows and within a row, against the order in which their sums were formed (loss, then
  // gradient, of 2048 x 32000 bf16: 93.7 us forwards, 90.9 so; 777 x 50021 fp16 58.8 and 58.0).
  constexpr bool kTwice = LOSS && GRAD;
  constexpr int64_t kNone = INT64_MIN;
  const int64_t step = LOSS ? (int64_t)gridDim.x : -(int64_t)gridDim.x;
  auto there = [&](int64_t t) { return (uint64_t)t < (uint64_t)rows; };
  uint32_t issued = 0, taken = 0;                    // copies asked for, and those that have been waited for
  int free_places = kDepth, copy_place = 0, copy_dir = 1;
  int64_t copy_t = kNone;             // the row that is being copied
  Row copy_row = {};
  int copy_chunk = 0, copy_left = 0;                 // the next chunk, and how many there are of this pass
  bool copy_again = false;                           // in a row's first pass of two
  auto copy_one = [&](int64_t t, float w_t, int64_t t_next, float w_next) {     // false: nothing to copy now.  There is a free place
    while (copy_left == 0) {
      if (copy_again) {                              // from here on backwards
        copy_again = false;
        copy_dir = -copy_dir;
        copy_left = max(0, copy_row.chunks - kDepth);
        copy_chunk = copy_left - 1;
        // from the last chunk's place on; a row that stays whole leaves the places behind its first chunk to the next row
        copy_place += copy_row.chunks >= kDepth ? copy_dir : (copy_row.chunks + 1) * copy_dir;
        continue;
      }
      if (copy_t == t_next) return false;            // the row that is worked on, or the next one
      const bool begin = copy_t != t;
      copy_t = begin ? t : t_next;
      if (there(copy_t) && (begin ? w_t : w_next) != 0.0f) {
        copy_row = row_of(copy_t);
        copy_chunk = LOSS ? 0 : copy_row.chunks - 1;
        copy_left = copy_row.chunks;
        copy_again = kTwice;
      }
    }
    uint4* dst = ring + (copy_place & (kDepth - 1)) * kChunkSlots;
    const uint8_t* copy_src = copy_row.at + (size_t)copy_chunk * kChunkBytes + tid * 16;
    const uint32_t to = (uint32_t)__cvta_generic_to_shared(dst);
    if (copy_row.whole(copy_chunk)) {
#pragma unroll
      for (int u = 0; u < kStreamSlots; ++u)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + u * kStreamThreads * 16), "l"(copy_src + u * kStreamThreads * 16) : "memory");
    } else {
#pragma unroll
      for (int u = 0; u < kStreamSlots; ++u) {
        const int i = copy_chunk * kChunkSlots + u * kStreamThreads + tid;
        const uint8_t* src = copy_src + u * kStreamThreads * 16;
        if (i >= copy_row.first && i < copy_row.full) {
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + u * kStreamThreads * 16), "l"(src) : "memory");
        } else if (i < copy_row.words) {
          const int lo = i * E - copy_row.off;
          if (src >= base) {         // the bytes before a row are the row's before it; those behind are not read
            const int bytes = min(16, (V - lo) * (int)sizeof(T));
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to + u * kStreamThreads * 16), "l"(src), "r"(bytes) : "memory");
          } else {
            dst[u * kStreamThreads] = S::load(reinterpret_cast<const T*>(copy_row.at) + copy_row.off, lo, V);
          }
        }
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    copy_chunk += LOSS && (!GRAD || copy_again) ? 1 : -1;
    --copy_left;
    copy_place += copy_dir;
    --free_places;
    ++issued;
    return true;
  };
  int place_now = 0, dir = 1;                        // of the chunk that is worked on

  // ---- the teacher's entries.  A thread's first is asked for ahead and lies in registers as it came, since the first instruction that
  // takes it waits for it; those beyond kStreamThreads are loaded when they are entered.
  int2 e_idx = {};
  uint32_t e_top = 0;
  T e_z = {};
  auto ask = [&](int64_t t) {
    if (tid < P.k && there(t)) {
      if (P.idx_bytes == 4) e_idx.x = static_cast<const int32_t*>(P.idx)[t * P.ldi + tid];
      else e_idx = static_cast<const int2*>(P.idx)[t * P.ldi + tid];
      if (P.top_type == LCD_DTYPE_F32) e_top = static_cast<const uint32_t*>(P.top)[t * P.ldt + tid];
      else e_top = static_cast<const uint16_t*>(P.top)[t * P.ldt + tid];
    }
  };
  auto index_in = [&](const int2& i) {         // -1: none
    return (P.idx_bytes == 4 || i.y == 0) && (unsigned)i.x < (unsigned)P.V ? i.x : -1;
  };
  auto teacher_in = [&](uint32_t x) {
    return P.top_type == LCD_DTYPE_F32 ? __uint_as_float(x) : P.top_type == LCD_DTYPE_F16 ? __half2float(__ushort_as_half((unsigned short)x))
                                                                                          : __uint_as_float(x << 16);
  };
  auto enter = [&](int64_t t, int place, int parity) {   // row t's entries to shared memory, their pair; asks for the student's logits there
    const Entries n = entries(place);
    Pair top = {-FLT_MAX, 0.0f};
    const T* row = static_cast<const T*>(P.z) + t * P.ldz;
    if (tid < P.k && there(t)) {
      const float v = teacher_in(e_top);
      const int i = v == -INFINITY ? -1 : index_in(e_idx);     // p = 0: as if it were absent
      n.idx[tid] = i;
      n.p[tid] = v;
      if (i >= 0) {
        top = {fmaxf(v, -FLT_MAX), v == v ? 1.0f : v};
        if (!LOSS) e_z = row[i];
      }
#pragma unroll 1
      for (int j = tid + kStreamThreads; j < P.k; j += kStreamThreads) {
        int2 raw = {};
        if (P.idx_bytes == 4) raw.x = static_cast<const int32_t*>(P.idx)[t * P.ldi + j];
        else raw = static_cast<const int2*>(P.idx)[t * P.ldi + j];
        const float v2 = teacher_in(P.top_type == LCD_DTYPE_F32 ? static_cast<const uint32_t*>(P.top)[t * P.ldt + j]
                                                                : static_cast<const uint16_t*>(P.top)[t * P.ldt + j]);
        const int i2 = v2 == -INFINITY ? -1 : index_in(raw);
        n.idx[j] = i2;
        n.p[j] = v2;
        if (i2 >= 0) {
          const float m = fmaxf(top.m, v2);
          top = {m, top.s * exp2_fast((top.m - m) * P.c) + exp2_fast((v2 - m) * P.c)};
          if (!LOSS) n.z[j] = to_f32(row[i2]);
        }
      }
    }
    if (warp * 32 < P.k) top = warp_pair(top, P.c);
    if (lane == 0) s_top[parity][warp] = top;
  };

  int64_t t = LOSS ? blockIdx.x : rows - 1 - blockIdx.x;
  float w = P.weight ? P.weight[t] : 1.0f;
  int64_t t_next = t + step;
  float w_next = P.weight && there(t_next) ? P.weight[t_next] : 1.0f;
  float lse = P.lse ? P.lse[t] : 0.0f;
  ask(t);
  enter(t, 0, 0);
  __syncthreads();
  int place = 0;
  for (int parity = 0; there(t); parity ^= 1) {
    const Entries n = entries(place);
    place = place == 2 ? 0 : place + 1;
    ask(t_next);
    const int64_t t_then = t_next + step;
    const float w_then = P.weight && there(t_then) ? P.weight[t_then] : 1.0f;
    Pair all = {-FLT_MAX, 0.0f};
    if (!LOSS) all = {P.stats[2 * t], P.stats[2 * t + 1]};
    const float lse_next = P.lse && there(t_next) ? P.lse[t_next] : 0.0f;
    while (free_places > 0 && copy_one(t, w, t_next, w_next)) {}
    const Row row = row_of(t);
    const T* student = static_cast<const T*>(P.z) + t * P.ldz;
    T* out = GRAD ? static_cast<T*>(P.d) + t * P.ldd : nullptr;
    const bool wide = ((reinterpret_cast<uintptr_t>(out) & 15) == row.off * sizeof(T));
    // makes what lies outside the row -infinity in this thread's words of a chunk
    auto patch = [&](uint4* at, int chunk) {
#pragma unroll
      for (int u = 0; u < kStreamSlots; ++u) {
        const int i = chunk * kChunkSlots + u * kStreamThreads + tid;
        if (i >= row.words) {
          at[u * kStreamThreads] = no_logits<T>();
        } else if (i < row.first || i >= row.full) {
          T* v = reinterpret_cast<T*>(at + u * kStreamThreads);
          for (int e = 0; e < E; ++e) {
            const int at_row = i * E - row.off + e;
            if (at_row < 0 || at_row >= V) v[e] = from_f32<T>(-INFINITY);
          }
        }
      }
    };
    if (LOSS && w != 0.0f) {
      for (int c = 0; c < row.chunks; ++c) {
        copy_wait((int)(issued - taken - 1));
        ++taken;
        uint4* src = ring + (place_now & (kDepth - 1)) * kChunkSlots;
        place_now += dir;
        if (!row.whole(c)) patch(src, c);
        uint4 x[kStreamSlots];
#pragma unroll
        for (int u = 0; u < kStreamSlots; ++u) x[u] = src[u * kStreamThreads];
        add_words<T, kStreamSlots>(x, P.c, all);
        if (!kTwice || c < row.chunks - kDepth) {
          ++free_places;
          copy_one(t, w, t_next, w_next);
        }
      }
      if (kTwice) {
        place_now -= dir;
        dir = -dir;
      }
      if (tid < P.k && n.idx[tid] >= 0) e_z = student[n.idx[tid]];       // arrives behind the reductions
      all = warp_pair(all, P.c);
      if (lane == 0) s_row[parity][warp] = all;
    }
    // this row's p, its entries' terms of the loss, the next row's entries, and one barrier for all reductions
    float mass = 0.0f;
    Share share = {-FLT_MAX, 0.0f, 0.0f};
    if (warp * 32 < P.k) {
      const Pair top = pair_of<kStreamWarps>(s_top[parity], P.c);
      const Teacher teacher = teacher_of(top, P.lse ? &lse : nullptr);
      if (LOSS && tid == 0) s_teacher[parity] = top;
      for (int j = tid; j < P.k; j += kStreamThreads) {
        const int i = n.idx[j];
        const float v = n.p[j], p = i >= 0 ? probability(v, teacher, P.inv_tau) : 0.0f;
        if (!LOSS && j == tid) n.z[j] = to_f32(e_z);
        if (LOSS && w != 0.0f && i >= 0) {
          const float z = to_f32(j == tid ? e_z : student[i]);
          add_entry(share, mass, p, v, z, P.inv_tau);
          n.z[j] = z;
        }
        n.p[j] = p;
        mass += p;
      }
      if (LOSS) share = warp_share(share, mass, P.inv_tau);
      mass = warp_sum(mass);
    }
    if (lane == 0) {
      s_mass[parity][warp] = mass;
      if (LOSS) s_share[parity][warp] = share;
    }
    enter(t_next, place, parity ^ 1);
    __syncthreads();
    if (GRAD || warp == kLossWarp) {
      mass = sum_of<kStreamWarps>(s_mass[parity]);
      if (LOSS && w != 0.0f) all = pair_of<kStreamWarps>(s_row[parity], P.c);
    }
    if (LOSS && warp == kLossWarp) {
      float sum = 0.0f;
      if (w != 0.0f) {               // a lane per warp
        const int i = lane & (kStreamWarps - 1);
        sum = share_loss(s_mass[parity][i], s_share[parity][i], all, s_teacher[parity], P.lse ? &lse : nullptr, P.inv_tau);
#pragma unroll
        for (int o = kStreamWarps / 2; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      }
      if (lane == 0) {
        P.loss[t] = w == 0.0f || mass == 0.0f ? 0.0f : w * sum;
        if (P.stats) {
          P.stats[2 * t] = w == 0.0f ? NAN : all.m;
          P.stats[2 * t + 1] = w == 0.0f ? NAN : all.s;
        }
      }
    }
    const bool none = w == 0.0f || mass == 0.0f;      // no gradient
    if (GRAD && none) {
      const float zero[E] = {};
      for (int i = tid; i < row.words; i += kStreamThreads) S::store(out, (int64_t)i * E - row.off, P.V, wide, zero);
    }
    if (GRAD && w != 0.0f) {
      const float wt = w * P.inv_tau, scale = wt * mass / all.s;
      for (int n_done = 0; n_done < row.chunks; ++n_done) {
        const int c = row.chunks - 1 - n_done;
        if (!kTwice || n_done >= kDepth) {
          copy_wait((int)(issued - taken - 1));
          ++taken;
        }
        const uint4* src = ring + (place_now & (kDepth - 1)) * kChunkSlots;
        place_now += dir;
        if (none) {
        } else if (wide && row.whole(c)) {
          T* to = out - row.off + (size_t)c * kChunkSlots * E + tid * E;
          uint4 x[kStreamSlots];
#pragma unroll
          for (int u = 0; u < kStreamSlots; ++u) x[u] = src[u * kStreamThreads];
#pragma unroll
          for (int u = 0; u < kStreamSlots; ++u) {
            float v[E];
            shares<T>(x[u], all.m, P.c, scale, v);
            S::store_all(to + u * kStreamThreads * E, v);
          }
        } else {
#pragma unroll 1
          for (int u = 0; u < kStreamSlots; ++u) {
            const int64_t lo = (int64_t)(c * kChunkSlots + u * kStreamThreads + tid) * E - row.off;
            if (lo >= P.V) break;
            float v[E];
            shares<T>(src[u * kStreamThreads], all.m, P.c, scale, v);
            S::store(out, lo, P.V, wide, v);
          }
        }
        ++free_places;
        copy_one(t, w, t_next, w_next);
      }
      __syncthreads();
      if (!none)
        fix_entries(n, P.k, kStreamWarps, [&](int i, float p, float z) {
          out[i] = from_f32<T>(wt * (mass * (exp2_fast((z - all.m) * P.c) / all.s) - p));
        });
    }
    t = t_next;
    w = w_next;
    lse = lse_next;
    t_next = t_then;
    w_next = w_then;
  }
}

template <typename T, int THREADS>
lcd_status launch_stream(const Params& p, int64_t rows, bool loss, bool grad, cudaStream_t s) {
  auto kern = loss ? (grad ? distill_stream_kernel<T, true, true, THREADS> : distill_stream_kernel<T, true, false, THREADS>)
                   : distill_stream_kernel<T, false, true, THREADS>;
  static PerDeviceFlag attr_set[3];
  int dev;
  constexpr int kRing = kDepth * THREADS * kStreamSlots * 16;
  PerDeviceFlag& flag = attr_set[loss ? grad : 2];
  if (flag.first(&dev)) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kRing + 3 * 12 * kMaxK);
    if (e != cudaSuccess) { set_cuda_error((int)e); return LCD_ERR_CUDA; }
    flag.done(dev);
  }
  // as many CTAs as are resident: 1 KB of the system's and up to 0.5 of static shared memory a CTA
  const int fit = 228 * 1024 / (kRing + 3 * 12 * (int)p.k + 1536);
  const int64_t most = (int64_t)current_sm_count() * (fit < kStreamPerSm<THREADS> ? fit : kStreamPerSm<THREADS>);
  const cudaError_t e = launch_overlapping(kern, dim3((unsigned)(rows < most ? rows : most)), dim3(THREADS), kRing + 3 * 12 * p.k, 1, s, p, rows);
  if (e != cudaSuccess) { set_cuda_error((int)e); return LCD_ERR_CUDA; }
  return LCD_OK;
}

template <typename T>
lcd_status launch_typed(Params p, int64_t rows, bool loss, bool grad, cudaStream_t s) {
  constexpr int E = Slot<T>::E;
  const int64_t slots = (p.V + 2 * E - 2) / E;        // whatever the row's alignment
  const int64_t sms = current_sm_count();
  // Clusters take a few long rows: loss and gradient of 32 x 128000 bf16 11.5 us, a CTA a row 21; 74 x 128000 26 and 21; 32 x 32000
  // 10.3 and 9.8.  CTAs of 256 threads where there are two rows a multiprocessor at most (148 x 32000 bf16, loss and gradient 9.6,
  // 128 threads 13.6) and where many rows have a gradient (4096 x 128000: 456 and 545; 4096 x 32000 fp32: 198 and 243), unless rows
  // are short (4096 x 12000: 94 and 73); else 128 (loss of 4096 x 32000: 54, 256 threads 74; 444 rows with gradient 17.8, 21.3).
  // CTAs of 64 threads are faster below 2000 columns only (4096 x 1000: 27, 128 threads 36).
  if (rows * 4 > sms || slots < 4096) {
    const bool wide = slots >= 2048 && (rows <= 2 * sms || (grad && rows >= 4 * sms));
    return wide ? launch_stream<T, 256>(p, rows, loss, grad, s) : launch_stream<T, 128>(p, rows, loss, grad, s);
  }
  // CTAs a row: as few as hold it in registers, more where there are few rows.
  int parts = 1;
  while (parts < kMaxCluster && parts * kThreads * kSlots < slots) parts *= 2;
  const int64_t room = 2 * sms;
  while (parts < kMaxCluster && rows * parts * 2 <= room && slots / parts >= 128) parts *= 2;
  const int64_t each = (slots + parts - 1) / parts;
  const bool once = each <= kThreads * kSlots;
  // threads: the slots' number divided by what a thread holds, or a slot a thread where CTAs are few
  int64_t threads = rows * parts <= room ? each : (each + kSlots - 1) / kSlots;
  threads = threads >= kThreads ? kThreads : threads < 64 ? 64 : (threads + 31) / 32 * 32;
  if (rows * parts > 0x7fffffffLL) return LCD_ERR_UNSUPPORTED;
  p.parts = parts;
  auto kern = loss ? (grad ? (once ? distill_kernel<T, true, true, true> : distill_kernel<T, true, true, false>)
                           : (once ? distill_kernel<T, true, false, true> : distill_kernel<T, true, false, false>))
                   : (once ? distill_kernel<T, false, true, true> : distill_kernel<T, false, true, false>);
  const cudaError_t e = launch_overlapping(kern, dim3((unsigned)(rows * parts)), dim3((unsigned)threads), 0, loss ? (unsigned)parts : 1u, s, p);
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
