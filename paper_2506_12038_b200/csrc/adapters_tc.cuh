// The adapters' products for many rows, on tcgen05 (adapters_up_tc.cuh, adapters_down_tc.cu, adapters_down_parts.cu, adapters_outer_tc.cu): what they have in common.
//
// Operands are tiles of rows of 128 bytes in shared memory, 64 16-bit values a row, with the 128-byte swizzle (a 16-byte piece's number exclusive-or
// the row's in its group of eight).  The same tile serves as a K-major operand (a row is a row of the operand, 16 columns of K are 32 bytes
// further) or as an MN-major one (a row is a column of K: 16 of them are 2048 bytes further), so nothing is transposed: what the sum
// runs over is told to the instruction.  t and dt, and fp32 and fp16 operands that meet them, go in as two or three bf16 parts, in tiles of their own.
#ifndef LCD_ADAPTERS_TC_CUH_
#define LCD_ADAPTERS_TC_CUH_

#include "adapters.cuh"

namespace lcd {

namespace tc {

constexpr unsigned long long kWaitNs = 2000000000ull;

__device__ __forceinline__ unsigned long long timer_ns() {
  unsigned long long t;
  asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
  return t;
}
__device__ __forceinline__ bool elect() {
  uint32_t p;
  asm volatile("{\n.reg .pred P;\nelect.sync _|P, 0xffffffff;\nselp.u32 %0, 1, 0, P;\n}" : "=r"(p));
  return p != 0;
}
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count));
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
               : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
// Bounded: false when another role gave up or after kWaitNs, when the flag is raised for everybody.
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
  if (bar_try(bar, parity)) return true;
  const unsigned long long t0 = timer_ns();
  for (uint32_t it = 1;; ++it) {
    if (bar_try(bar, parity)) return true;
    if ((it & 255u) == 0) {
      if (*abort_flag) return false;
      if (timer_ns() - t0 > kWaitNs) { *abort_flag = 1; return false; }
    }
  }
}
__device__ __forceinline__ void bar_drain(uint32_t bar, uint32_t parity) {
  const unsigned long long t0 = timer_ns();
  for (uint32_t it = 1; !bar_try(bar, parity); ++it)
    if ((it & 255u) == 0 && timer_ns() - t0 > kWaitNs) return;
}
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// A tile's descriptor: 128-byte swizzle, groups of eight rows 1024 bytes apart; MN-major, `block`: bytes from 64 values to the next 64.
__device__ __forceinline__ uint64_t tile_desc(uint32_t addr, uint32_t block) {
  return (uint64_t)((addr & 0x3ffffu) >> 4) | (uint64_t)(block >> 4) << 16 | (uint64_t)(1024u >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
// kind::f16, fp32 sums, 128 x n; both operands bf16 or both fp16; which of them are MN-major.
__host__ __device__ constexpr uint32_t instr_desc(int n, bool bf16, bool a_mn, bool b_mn) {
  return 1u << 4 | (bf16 ? 1u << 7 | 1u << 10 : 0u) | (a_mn ? 1u << 15 : 0u) | (b_mn ? 1u << 16 : 0u) | (uint32_t)(n >> 3) << 17 | 8u << 24;
}
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}"
               ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void mma_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
        "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
      : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_alloc(uint32_t holder, uint32_t columns) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(holder), "r"(columns) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free(uint32_t tmem, uint32_t columns) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(columns) : "memory");
}
__device__ __forceinline__ void before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// 16 bytes from global to shared memory, of which the first `have` (0 to 16) are read and the others zeros.
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, int have) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(have) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void store16(uint32_t dst, uint4 v) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
// Where 16-byte piece `piece` of a tile's row lies.
__device__ __forceinline__ uint32_t piece_at(int row, int piece) { return (uint32_t)(row * 128 + ((piece ^ (row & 7)) << 4)); }

// bf16 parts of eight values, part after part: the first cut off, the last rounded.
template <int PARTS>
__device__ __forceinline__ void parts_of(float (&v)[8], uint4 (&out)[PARTS]) {
#pragma unroll
  for (int p = 0; p < PARTS; ++p) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = p == PARTS - 1 ? pair_rounded(v[2 * i], v[2 * i + 1]) : pair_upper(v[2 * i], v[2 * i + 1]);
    out[p] = make_uint4(w[0], w[1], w[2], w[3]);
    if (p < PARTS - 1) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = rest_of(v[i], upper_bf16(v[i]));
    }
  }
}
// The parts that a type's values take: bf16 is one, fp16 two (11 bits), fp32 three.
template <typename T> constexpr int kParts = std::is_same<T, __nv_bfloat16>::value ? 1 : std::is_same<T, __half>::value ? 2 : 3;

// How many CTAs of a cluster share the stages of a sum, when `tiles` sums of `stages` stages each run on `slots` places at a time: what takes least
// time if starting and joining takes as long as six stages.  With 0, 3, 6, 12 and 30 in place of six, us: x a^T of 20000 rows of 2048, rank 16, bf16
// 71 / 46 / 46 / 38 / 38; gradients of 3000 rows, 2048 x 5000, 55 / 56 / 38 / 38 / 38, of 10000 of 2, 1024 x 4096, rank 64, 178 / 158 / 138 / 138 / 175;
// where the tiles or the cut's eighths fill the SMs (4096 rows and fewer) it makes no difference.
inline unsigned split_of(long long tiles, long long stages, long long slots, unsigned most) {
  unsigned best = 1;
  long long least = 0;
  for (unsigned s = 1; s <= most && s <= stages; ++s) {
    const long long time = (tiles * s + slots - 1) / slots * ((stages + s - 1) / s + 6);
    if (s == 1 || time < least) {
      least = time;
      best = s;
    }
  }
  return best;
}

// The sums over a cluster's CTAs, in their order, of the four values that lie at this shared address in each.
template <int SPLIT>
__device__ __forceinline__ float4 sums_of_ranks(uint32_t at) {
  float4 v[SPLIT];
#pragma unroll
  for (int i = 0; i < SPLIT; ++i) {
    if constexpr (SPLIT == 1) {
      asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[i].x), "=f"(v[i].y), "=f"(v[i].z), "=f"(v[i].w) : "r"(at));
    } else {
      uint32_t there;
      asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(at), "r"(i));
      asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[i].x), "=f"(v[i].y), "=f"(v[i].z), "=f"(v[i].w) : "r"(there));
    }
  }
  float4 sum = v[0];
#pragma unroll
  for (int i = 1; i < SPLIT; ++i) {
    sum.x += v[i].x;
    sum.y += v[i].y;
    sum.z += v[i].z;
    sum.w += v[i].w;
  }
  return sum;
}
// f(std::integral_constant<int, split>) for a split of 1 to 8.
template <typename F>
__device__ __forceinline__ void by_split(uint32_t split, F&& f) {
  switch (split) {
    case 1: f(std::integral_constant<int, 1>{}); break;
    case 2: f(std::integral_constant<int, 2>{}); break;
    case 3: f(std::integral_constant<int, 3>{}); break;
    case 4: f(std::integral_constant<int, 4>{}); break;
    case 5: f(std::integral_constant<int, 5>{}); break;
    case 6: f(std::integral_constant<int, 6>{}); break;
    case 7: f(std::integral_constant<int, 7>{}); break;
    default: f(std::integral_constant<int, 8>{});
  }
}
// Long sums.  An MMA adds to the fp32 sum and cuts off, toward zero, so a sum of n of them is short by up to n 2^-23 of itself.  So the stages
// go to several accumulators in turn, as many as tensor memory has room for, and the products of the parts behind the first to one more, a
// smaller one; they are added when they are read.  Relative error of da, 512 rows of 4096 columns, fp16 with fp32 adapters: 5.3e-6 with one
// accumulator, 2.0e-7 with eight; of x a^T over 8192 columns, fp32: 3.1e-5 and 7.2e-7 (plain fp32 sums 7.1e-7 and 1.6e-6).  Times are the same.
// With three accumulators, ranks above 32: over 8192 columns fp32 1.5e-6 and bf16 0.6e-6 (rank 64) to 1.4e-6 (rank 128; plain fp32 sums 1.6e-6 and
// 1.0e-6), over 32768 6.5e-6 and 2.9e-6 to 6.0e-6 (3.2e-6 and 2.3e-6); da over 32768 rows 1.4e-6 to 1.6e-6 (0.8e-6).
template <int R> constexpr int kSums = R <= 32 ? 7 : 3;
// Sixteen columns of the accumulators of a sum, R columns apart, added up: the first `used` of the kSums, and the one more.
template <int R>
__device__ __forceinline__ void read_sums(uint32_t from, int used, bool more, float (&out)[16]) {
  uint32_t v[16];
  tmem_ld16(from, v);
  tmem_wait_ld();
#pragma unroll
  for (int i = 0; i < 16; ++i) out[i] = __uint_as_float(v[i]);
#pragma unroll 1
  for (int a = 1; a <= kSums<R>; ++a) {
    if (a < kSums<R> ? a >= used : !more) continue;
    tmem_ld16(from + a * R, v);
    tmem_wait_ld();
#pragma unroll
    for (int i = 0; i < 16; ++i) out[i] += __uint_as_float(v[i]);
  }
}
// Sixteen values of a row from an address on 16 bytes, or, wide, on 32.
template <typename Y>
__device__ __forceinline__ void store16_values(Y* p, const float (&v)[16], bool wide) {
  uint32_t w[sizeof(Y) == 4 ? 16 : 8];
  if constexpr (sizeof(Y) == 4) {
#pragma unroll
    for (int i = 0; i < 16; ++i) w[i] = __float_as_uint(v[i]);
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float part[8] = {v[8 * h], v[8 * h + 1], v[8 * h + 2], v[8 * h + 3], v[8 * h + 4], v[8 * h + 5], v[8 * h + 6], v[8 * h + 7]};
      const uint4 q = pack8<Y>(part);
      w[4 * h] = q.x; w[4 * h + 1] = q.y; w[4 * h + 2] = q.z; w[4 * h + 3] = q.w;
    }
  }
#pragma unroll
  for (int i = 0; i < (sizeof(Y) == 4 ? 16 : 8); i += 8) {
    uint32_t* to = reinterpret_cast<uint32_t*>(p) + i;
    if (wide) {
      asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                   ::"l"(to), "r"(w[i]), "r"(w[i + 1]), "r"(w[i + 2]), "r"(w[i + 3]), "r"(w[i + 4]), "r"(w[i + 5]), "r"(w[i + 6]), "r"(w[i + 7]) : "memory");
    } else {
      *reinterpret_cast<uint4*>(to) = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
      *reinterpret_cast<uint4*>(to + 4) = make_uint4(w[i + 4], w[i + 5], w[i + 6], w[i + 7]);
    }
  }
}

// The plan's tiles of 128 places, each of one group, in shared memory: first[g] tiles lie before group g, begins[g] places; group G stands
// for the rows without one.
constexpr int kPlaces = 128;
struct Plan {
  int *first, *begins;
  static constexpr int kBytes = 2 * (kMostGroups + 2) * 4;
  // By one warp.  step: places of a tile.  Offsets that do not ascend (no plan of lcd_group_rows) may make more tiles than there can be: those
  // are left out, so that their number stays within an int.
  __device__ __forceinline__ void make(const AdapterArgs& a, int lane, int step) const {
    const int most = a.rows / step + min(a.G + 1, a.rows);
    int sum = 0;
    for (int g0 = 0; g0 <= a.G; g0 += 32) {
      const int g = g0 + lane;
      int tiles = 0;
      if (g <= a.G) {
        const int begin = min(max(a.offsets[g], 0), a.rows), end = g < a.G ? min(max(a.offsets[g + 1], begin), a.rows) : a.rows;
        tiles = (end - begin + step - 1) / step;
        begins[g] = begin;
      }
      int upto = tiles;
#pragma unroll
      for (int d = 1; d < 32; d *= 2) {
        const int v = __shfl_up_sync(0xffffffffu, upto, d);
        if (lane >= d) upto += v;
      }
      if (g <= a.G) first[g] = min(sum + upto - tiles, most);
      sum = min(sum + __shfl_sync(0xffffffffu, upto, 31), most);
    }
    if (lane == 0) {
      first[a.G + 1] = sum;
      begins[a.G + 1] = a.rows;
    }
  }
  struct Spot { int group, place, count; };
  __device__ __forceinline__ Spot at(int tile, int G, int step) const {
    int low = 0, high = G;                         // the last group that begins at this tile or before
    while (low < high) {
      const int middle = (low + high + 1) / 2;
      if (first[middle] <= tile) low = middle;
      else high = middle - 1;
    }
    const int place = begins[low] + (tile - first[low]) * step;
    return {low, place, min(step, begins[low + 1] - place)};
  }
};

}  // namespace tc

}  // namespace lcd
#endif
