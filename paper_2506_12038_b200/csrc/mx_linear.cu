// The product of two microscaled 4-bit matrices (lcd_mx_linear): y[m][n] = sum over blocks b of 2^(sx + sw) times the sum over the
// block's 32 columns of the elements' products.  The tensor cores take this format as it is: tcgen05.mma kind::mxf4 multiplies
// 128 weight rows by BN tokens over 64 columns, codes from shared memory, scales from tensor memory, sums in fp32.  So there
// is no decoding, and few tokens (weights from HBM) and many (tensor pipe) are one kernel with token tiles of different width.
//
// Roles (11 warps; 15 with tiles of 256 tokens; grouped, of 128 or more):
//   warp 0      TMA producer of codes: stages of 256 columns, 128-byte swizzle
//   warp 10     TMA producer of scales: 512 columns (16 bytes a row) at a time
//   warps 2-5   scales to tensor memory: the unit reads row r's four scale bytes of 128 columns at lane r % 32, column r / 32, in
//               every quarter of the lanes, so each of the four warps stores all rows' words into its own quarter
//   warp 1      owns tensor memory; one elected lane issues the MMAs
//   warps 6-9, 11-    epilogue: tensor memory -> y, coalesced along the weight rows; up to four tokens come as they are, then these warps
//               quantise them into the stages first
// Many tokens take pairs of CTAs (mx_pair_kernel below).
// Products grouped by expert (lcd_mx_linear_grouped) are the same kernel with another list of tiles: the tokens' codes lie sorted by
// expert, a tile is a piece of one expert's tokens, and y's rows are scattered to where the plan says they come from.
// Where tiles are few the columns of a tile are cut among the CTAs of a cluster; their partial sums meet in distributed shared
// memory and are added in the order of the ranks, so results do not depend on timing.
// Every wait is bounded (status word LCD_ERR_TIMEOUT on expiry; then every role leaves its loop, copies and MMAs in flight are
// drained, tensor memory is released).
#include <cuda.h>

#include <cmath>
#include <type_traits>

#include "common.h"
#include "device_util.h"
#include "mx.cuh"

namespace lcd {

namespace {

constexpr int kRows = 128;                      // weight rows of a tile = MMA M
constexpr int kStageK = 256;                    // columns of a stage: 128 bytes of codes a row
constexpr int kAStage = kRows * kStageK / 2;    // 16 KB
constexpr int kScaleSlots = 3;
constexpr int kMostSplit = 8;                  // a cluster's CTAs
constexpr int kOwnTokens = 4;                  // tokens that the kernel quantises itself
constexpr int kMmaWarp = 1, kFirstEpiWarp = 6, kScaleCopyWarp = 10;

constexpr unsigned long long kWaitNs = 2000000000ull;

template <int BN, bool GROUPED = false>
struct Cfg {
  static constexpr int kBStage = BN * kStageK / 2;
  static constexpr int kStages = BN == 32 && GROUPED ? 4 : BN <= 32 ? 5 : BN == 256 ? 4 : BN == 192 ? 5 : BN == 128 ? 6 : 4;
  static constexpr int kScaleBytes = (kRows + BN) * 16;
  static constexpr int kSfbCols = (BN + 127) / 128 * 4;                   // tensor-memory columns of the tokens' scales, per 128 columns
  static constexpr int kSfCols = 4 * (4 + kSfbCols);                     // of a scale slot: 512 columns
  static constexpr int kDBuffers = 2 * BN + 2 * kSfCols <= 512 ? 2 : 1;  // accumulators
  static constexpr int kSfSlots = 2;                                     // (four were no faster)
  static constexpr int kUsed = kDBuffers * BN + kSfSlots * kSfCols;
  static constexpr int kTmemCols = kUsed <= 128 ? 128 : kUsed <= 256 ? 256 : 512;
  static constexpr int kPerSm = BN <= 64 ? 2 : 1;
  // Parts of the columns that are drained by warps of their own: two where there is one accumulator; grouped, where a tile's rows are scattered
  // and its columns often few, always (three of 64 columns with tiles of 192 were slower).
  // Grouped, the tokens of wide tiles come in boxes of 64 rows, as many as the tile has tokens for, and the MMAs are as wide: the loads from
  // L2 bound prompts (a tile of 192 tokens reads 320 rows of codes), and an expert's last tile is often half empty.
  static constexpr int kBox = GROUPED && BN >= 128 ? 64 : BN;
  static constexpr int kEpiParts = (GROUPED && BN >= 128) || kDBuffers == 1 ? 2 : 1, kEpiColumns = BN / kEpiParts;
  // grouped: the token tiles before every expert and where its tokens begin, and for every epilogue warp where its columns go
  static constexpr int kPlanBytes = 8 * (kMostExperts + 1), kPlacesBytes = 4 * BN * 8;
  static constexpr int kSmem = 1024 + kStages * (kAStage + kBStage) + kScaleSlots * kScaleBytes + 256 + (GROUPED ? kPlanBytes + kPlacesBytes : 0);
  static constexpr int kThreads = 32 * (11 + 4 * (kEpiParts - 1));
  // Whatever shares an SM has tensor memory enough, so that no CTA of a cluster waits for columns while another CTA of it holds some:
  // two of the narrow tiles fit, and beside a wide one nothing does (shared memory).
  static_assert(kUsed <= kTmemCols && kTmemCols * kPerSm <= 512, "tensor memory");
  static_assert(kPerSm == 2 || kSmem > 128 * 1024, "one CTA an SM");
  static_assert(kSmem <= 227 * 1024 && kPerSm * (kSmem + 1024) <= 228 * 1024, "shared memory");
  static_assert(BN * 512 <= kStages * (kAStage + kBStage), "partial sums lie in the stages");
};

struct Args {
  void* y;
  long long ldy;
  int y_type, M, N, n_ks, n_ss, n_tiles_m, n_tiles, early;
  int32_t* status;
  const void* x;         // instances that quantise x themselves: its rows, their pitch, the factors and the columns
  long long ldx;
  const float* inv;
  int K, x_wide;
  const int32_t *order, *offsets;    // grouped: the plan of the M rows, and the number of experts
  int G;
};

// A tile's first weight row, first token, number of tokens and, grouped, expert.
struct Spot { int n0, m0, tokens, expert; };

// The tiles in order: along the weight rows, a weight tile's token tiles one after the other; grouped, one expert after the other.
// first: the token tiles before every expert, and of all; begins: where the experts' tokens begin (shared memory).  Tiles are asked for in
// ascending order.
template <int BN, bool GROUPED, int ROWS = kRows>
struct Tiles {
  const Args& P;
  const int *first, *begins;
  int expert = 0;
  __device__ __forceinline__ Spot at(int tile) {
    if constexpr (GROUPED) {
      const int nt = (P.N + ROWS - 1) / ROWS;
      if (expert + 1 < P.G && first[expert + 1] * nt <= tile) {
        int high = P.G - 1;                      // the last expert that begins at this tile or before
        while (expert < high) {
          const int middle = (expert + high + 1) / 2;
          if (first[middle] * nt <= tile) expert = middle;
          else high = middle - 1;
        }
      }
      const int local = tile - first[expert] * nt, mt = max(1, first[expert + 1] - first[expert]);
      const int m0 = begins[expert] + local % mt * BN;
      return {local / mt * ROWS, m0, min(BN, begins[expert + 1] - m0), expert};
    } else {
      const int m0 = tile % P.n_tiles_m * BN;
      return {tile / P.n_tiles_m * ROWS, m0, min(BN, P.M - m0), 0};
    }
  }
};

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
__device__ __forceinline__ void bar_expect_tx(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
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
__device__ __forceinline__ void copy_tile(uint32_t dst, const CUtensorMap* map, int x, int row, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
               ::"r"(dst), "l"(map), "r"(x), "r"(row), "r"(bar) : "memory");
}
__device__ __forceinline__ void copy_tile_of(uint32_t dst, const CUtensorMap* map, int x, int row, int expert, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
               ::"r"(dst), "l"(map), "r"(x), "r"(row), "r"(expert), "r"(bar) : "memory");
}
// Shared-memory matrix descriptor: K-major, 128-byte swizzle, 8-row groups 1024 bytes apart.
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr) {
  return (uint64_t)((addr & 0x3ffffu) >> 4) | (uint64_t)(1024u >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
// Instruction descriptor of kind::mxf4: both operands E2M1 (1), K-major, M = 128, N = n, UE8M0 scales; `pair`: the bytes of a scale
// word that the instruction's two blocks use, 0 and 1 or 2 and 3.
__host__ __device__ constexpr uint32_t instr_desc(int n, int pair) {
  return (uint32_t)(2 * pair) << 4 | 1u << 7 | 1u << 10 | (uint32_t)(n >> 3) << 17 | 1u << 23 | (uint32_t)(kRows >> 4) << 24 |
         (uint32_t)(2 * pair) << 29;
}
__device__ __forceinline__ void mma_mx(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t accumulate) {
  asm volatile(
      "{\n.reg .pred p;\nsetp.ne.b32 p, %6, 0;\n"
      "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n}"
      ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void mma_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* v) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
      ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
      "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]) : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
        "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
      : "r"(taddr) : "memory");
}
// f(y as a pointer to its type): the type is looked at once, not for every output.
template <typename F>
__device__ __forceinline__ void by_type(const Args& P, F&& f) {
  if (P.y_type == LCD_DTYPE_F32) f(static_cast<float*>(P.y));
  else if (P.y_type == LCD_DTYPE_F16) f(static_cast<__half*>(P.y));
  else f(static_cast<__nv_bfloat16*>(P.y));
}

// Scales of 512 columns of `groups` groups of 32 rows, [row][16 bytes] in shared memory, to COLS tensor-memory columns per 128
// columns: word j of row 32 g + lane goes to column j * COLS + g.
template <int GROUPS, int COLS>
__device__ __forceinline__ void scales_to_tmem(const uint8_t* rows, uint32_t taddr, int lane) {
  uint32_t v[4 * COLS];
#pragma unroll
  for (int i = 0; i < 4 * COLS; ++i) v[i] = 0u;
#pragma unroll
  for (int g = 0; g < (GROUPS < 1 ? 1 : GROUPS); ++g) {
    if (GROUPS >= 1 || lane < 16) {             // a tile of 16 tokens fills half a group
      const uint4 w = *reinterpret_cast<const uint4*>(rows + (32 * g + lane) * 16);
      v[g] = w.x;
      v[COLS + g] = w.y;
      v[2 * COLS + g] = w.z;
      v[3 * COLS + g] = w.w;
    }
  }
#pragma unroll
  for (int i = 0; i < 4 * COLS; i += 16) tmem_st16(taddr + i, v + i);
}

// store(first column, 16 columns' sums) for the accumulator's columns begin .. end - 1 of this warp's lanes.  AHEAD: the next columns are on
// their way while these are stored (two CTAs an SM have no registers for it).
template <bool AHEAD, typename Store>
__device__ __forceinline__ void drain_columns(uint32_t from, int begin, int end, Store&& store) {
  uint32_t v[16], w[16];
  if (begin >= end) return;
  if (!AHEAD) {
#pragma unroll 1
    for (int c = begin; c < end; c += 16) {
      tmem_ld16(from + c, v);
      asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
      store(c, v);
    }
    return;
  }
  tmem_ld16(from + begin, v);
#pragma unroll 1
  for (int c = begin;; c += 32) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
    if (c + 16 < end) tmem_ld16(from + c + 16, w);
    store(c, v);
    if (c + 16 >= end) break;
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
    if (c + 32 < end) tmem_ld16(from + c + 32, v);
    store(c + 16, w);
    if (c + 32 >= end) break;
  }
}
// The same to y: this lane's weight row n, tokens m0 + begin .. m0 + end - 1.
template <bool AHEAD>
__device__ __forceinline__ void store_columns(const Args& P, uint32_t from, int begin, int end, int m0, int n) {
  by_type(P, [&](auto* y) {
    using T = std::remove_pointer_t<decltype(y)>;
    T* at = y + (size_t)(m0 + begin) * P.ldy + n;
    const bool inside = n < P.N;
    drain_columns<AHEAD>(from, begin, end, [&](int c, const uint32_t (&v)[16]) {
      // (the address is kept from being formed for all sixteen at once, which takes 32 registers)
      if (!inside) return;
      if (c + 16 <= end) {
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          *at = from_f32<T>(__uint_as_float(v[j]));
          at += P.ldy;
          asm volatile("" : "+l"(at));
        }
      } else {
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          if (c + j < end) *at = from_f32<T>(__uint_as_float(v[j]));
          at += P.ldy;
          asm volatile("" : "+l"(at));
        }
      }
    });
  });
}

// The row of y of a place of the plan, or -1.
__device__ __forceinline__ int planned_row(const Args& P, int place) {
  const int row = place < P.M ? P.order[place] : -1;
  return (unsigned)row < (unsigned)P.M ? row : -1;
}
// store_columns with the tokens' rows from the plan: places[c - begin] is the first element of column c's row in y, or negative.
template <bool AHEAD>
__device__ __forceinline__ void scatter_columns(const Args& P, uint32_t from, int begin, int end, uint32_t places, int n) {
  by_type(P, [&](auto* y) {
    using T = std::remove_pointer_t<decltype(y)>;
    y += n;
    const bool inside = n < P.N;
    drain_columns<AHEAD>(from, begin, end, [&](int c, const uint32_t (&v)[16]) {
#pragma unroll
      for (int half = 0; half < 16; half += 8) {
        // (asked for together: behind a store the compiler would wait for that)
        long long at[8];
#pragma unroll
        for (int j = 0; j < 8; j += 2)
          asm volatile("ld.shared.v2.s64 {%0, %1}, [%2];" : "=l"(at[j]), "=l"(at[j + 1]) : "r"(places + 8 * (c - begin + half + j)));
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (inside && at[j] >= 0) y[at[j]] = from_f32<T>(__uint_as_float(v[half + j]));
      }
    });
  });
}

// Eight columns of a token from k on, zeros beyond K.  `raw` holds them where they lie on 16 bytes inside the row.
template <typename X>
__device__ __forceinline__ void columns8(const Args& P, int m, int k, const Raw8<X>& raw, float (&t)[8]) {
  if (P.x_wide && k + 8 <= P.K) {
    values8(raw, t);
  } else {
    const X* p = static_cast<const X*>(P.x) + m * P.ldx + k;
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = k + i < P.K ? to_f32(p[i]) : 0.0f;
  }
}

// The lists that Tiles takes, by one warp.  The plan was there when the kernel before this one began (P.early).
template <int BN>
__device__ __forceinline__ void make_tiles(const Args& P, int* first, int* begins, int lane) {
      int sum = 0;
      for (int e0 = 0; e0 < P.G; e0 += 32) {
        const int e = e0 + lane;
        int tiles = 0;
        if (e < P.G) {
          const int begin = min(max(P.offsets[e], 0), P.M), end = min(max(P.offsets[e + 1], begin), P.M);
          tiles = (end - begin + BN - 1) / BN;
          begins[e] = begin;
          if (e == P.G - 1) begins[P.G] = end;
        }
        int upto = tiles;
  #pragma unroll
        for (int d = 1; d < 32; d *= 2) {
          const int v = __shfl_up_sync(0xffffffffu, upto, d);
          if (lane >= d) upto += v;
        }
        if (e < P.G) first[e] = sum + upto - tiles;
        sum += __shfl_sync(0xffffffffu, upto, 31);
      }
      if (lane == 0) first[P.G] = sum;
}

// Rows of y without an expert become zeros, CTAs in turn.
__device__ __forceinline__ void zero_rows(const Args& P, int thread, int threads) {
  by_type(P, [&](auto* y) {
    using T = std::remove_pointer_t<decltype(y)>;
    for (long long i = (long long)max(P.offsets[P.G], 0) + blockIdx.x; i < P.M; i += gridDim.x) {
      const int r = planned_row(P, (int)i);
      if (r < 0) continue;
      for (int n = thread; n < P.N; n += threads) y[(size_t)r * P.ldy + n] = from_f32<T>(0.0f);
    }
  });
}

// X: the type of x where the kernel quantises its tokens itself (few tokens), void where codes and scales come ready.  Then the
// epilogue warps, which wait for the sums, take the stages in turn: a CTA needs its own columns of x only and blocks are complete in
// them, so it can be done in every CTA, and a launch is saved (times: mx_linear_quantizes); from eight tokens on it takes longer than the
// weights' copies (8 x 4096 x 4096 8.4 us, 6.9 with two launches).
template <int BN, typename X, bool GROUPED>
__global__ void __launch_bounds__(Cfg<BN, GROUPED>::kThreads, Cfg<BN, GROUPED>::kPerSm)
mx_linear_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x,
                 const __grid_constant__ CUtensorMap map_ws, const __grid_constant__ CUtensorMap map_xs, const Args P) {
  using C = Cfg<BN, GROUPED>;
  extern __shared__ uint8_t smem_raw[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t raw_addr = (uint32_t)__cvta_generic_to_shared(smem_raw);
  const uint32_t base = (raw_addr + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (base - raw_addr);
  constexpr uint32_t kScaleAt = C::kStages * (kAStage + C::kBStage), kBarAt = kScaleAt + kScaleSlots * C::kScaleBytes;
  const uint32_t a_base = base, b_base = base + C::kStages * kAStage, s_base = base + kScaleAt, bars = base + kBarAt;
  auto full = [&](int s) { return bars + 8u * s; };
  auto empty = [&](int s) { return bars + 8u * (C::kStages + s); };
  auto sc_full = [&](int s) { return bars + 8u * (2 * C::kStages + s); };
  auto sc_empty = [&](int s) { return bars + 8u * (2 * C::kStages + kScaleSlots + s); };
  constexpr int kB0 = 2 * C::kStages + 2 * kScaleSlots, kB1 = kB0 + 2 * C::kSfSlots;
  auto ts_full = [&](int b) { return bars + 8u * (kB0 + b); };
  auto ts_empty = [&](int b) { return bars + 8u * (kB0 + C::kSfSlots + b); };
  auto d_full = [&](int b) { return bars + 8u * (kB1 + b); };
  auto d_empty = [&](int b) { return bars + 8u * (kB1 + 2 + b); };
  const uint32_t drain = bars + 8u * (kB1 + 4);
  static_assert(8 * (kB1 + 5) + 8 <= 256, "barriers");
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(gen + kBarAt + 8 * (kB1 + 5));
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_holder + 1);

  uint32_t rank, split;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(split));
  const int ss0 = (int)((long long)P.n_ss * rank / split), ss1 = (int)((long long)P.n_ss * (rank + 1) / split);   // this CTA's columns
  const int ks0 = 2 * ss0, ks1 = min(P.n_ks, 2 * ss1);
  const int tile0 = blockIdx.x / split, tile_step = gridDim.x / split;
  constexpr bool kReady = std::is_same<X, void>::value;
  static_assert(kReady || !GROUPED, "grouped tokens' codes come ready");
  long long* places = reinterpret_cast<long long*>(gen + kBarAt + 256);          // grouped
  int* first = reinterpret_cast<int*>(gen + kBarAt + 256 + C::kPlacesBytes);
  int* begins = first + kMostExperts + 1;

  if (threadIdx.x == 0) {
    for (int s = 0; s < C::kStages; ++s) {
      bar_init(full(s), kReady ? 1 : 2);            // the copies' thread, and the warp that quantises
      bar_init(empty(s), 1);
    }
    for (int s = 0; s < kScaleSlots; ++s) {
      bar_init(sc_full(s), kReady ? 1 : 3);         // the copies' thread, and a warp for either half
      bar_init(sc_empty(s), 4);
    }
    for (int b = 0; b < C::kSfSlots; ++b) {
      bar_init(ts_full(b), 4);
      bar_init(ts_empty(b), 1);
    }
    for (int b = 0; b < 2; ++b) {
      bar_init(d_full(b), 1);
      bar_init(d_empty(b), 4 * C::kEpiParts);
    }
    bar_init(drain, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                 ::"r"((uint32_t)__cvta_generic_to_shared(tmem_holder)), "r"((uint32_t)C::kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (GROUPED && warp == 2) make_tiles<BN>(P, first, begins, lane);
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const int n_tiles = GROUPED ? min(P.n_tiles, first[P.G] * ((P.N + kRows - 1) / kRows)) : P.n_tiles;
  Tiles<BN, GROUPED> tiles{P, first, begins};
  const uint32_t tmem = *tmem_holder;
  const uint32_t sf_tmem = tmem + C::kDBuffers * BN;
  // The kernel before may run on for long: no other role starts the time of a wait before it has ended.  (The copying threads wait for it
  // behind their first copies, warps that quantise where they begin to: here, 1 x 1024 x 4096 took 4.2 us in place of 4.0.)
  if (warp != 0 && warp != kScaleCopyWarp && (kReady || warp < kFirstEpiWarp)) wait_for_previous();

  if (warp == 0 || warp == kScaleCopyWarp) {
    // ---------------------------------------------------------------- TMA producers.  With P.early the kernel before this one wrote x's
    // codes and nothing else that is read here, and itself began when all before it was done: the weights' first copies do not wait.
    // What this thread does a stage is on the critical path of narrow tiles: 16 x 11008 x 4096 8.4 us with a division by the ring's length,
    // 7.9 without, 7.5 with a loop of its own for either kind of copies.
    auto produce = [&](auto of_codes) {
      constexpr bool codes = decltype(of_codes)::value;
      constexpr int slots = codes ? C::kStages : kScaleSlots;
      const int from = codes ? ks0 : ss0, to = codes ? ks1 : ss1;
      auto bytes_of = [&](const Spot& q) {
        if (!codes) return (uint32_t)(kReady ? C::kScaleBytes : kRows * 16);
        return (uint32_t)(kAStage + (!kReady ? 0 : C::kBox < BN ? (q.tokens + C::kBox - 1) / C::kBox * (C::kBox * kStageK / 2) : C::kBStage));
      };
      auto full_of = [&](int s) { return codes ? full(s) : sc_full(s); };
      auto copy_w = [&](int s, int k, const Spot& q) {
        if (GROUPED) copy_tile_of(codes ? a_base + s * kAStage : s_base + s * C::kScaleBytes, codes ? &map_w : &map_ws, k * (codes ? kStageK / 2 : 16), q.n0, q.expert, full_of(s));
        else if (codes) copy_tile(a_base + s * kAStage, &map_w, k * (kStageK / 2), q.n0, full(s));
        else copy_tile(s_base + s * C::kScaleBytes, &map_ws, k * 16, q.n0, sc_full(s));
      };
      auto copy_x = [&](int s, int k, const Spot& q) {
        if (!codes) copy_tile(s_base + s * C::kScaleBytes + kRows * 16, &map_xs, k * 16, q.m0, sc_full(s));
        else if (C::kBox == BN) copy_tile(b_base + s * C::kBStage, &map_x, k * (kStageK / 2), q.m0, full(s));
        else
          for (int r = 0; r < q.tokens; r += C::kBox) copy_tile(b_base + s * C::kBStage + r * (kStageK / 2), &map_x, k * (kStageK / 2), q.m0 + r, full(s));
      };
      const int ahead = P.early && tile0 < n_tiles ? min(slots, to - from) : 0;
      if (ahead > 0) {
        const Spot q = tiles.at(tile0);
        const uint32_t bytes = bytes_of(q);
        for (int i = 0; i < ahead; ++i) {
          bar_expect_tx(full_of(i), bytes);
          copy_w(i, from + i, q);
        }
      }
      begin_after_previous();
      int it = 0, s = 0;
      uint32_t round = 1;          // the parity of a stage's barrier
      bool ok = true;
      for (int tile = tile0; tile < n_tiles && ok; tile += tile_step) {
        const Spot q = tiles.at(tile);
        const uint32_t bytes = bytes_of(q);
        for (int k = from; k < to; ++k, ++it) {
          if (it >= ahead) {
            ok = bar_wait(codes ? empty(s) : sc_empty(s), round, abort_flag);
            if (!ok) break;
            bar_expect_tx(full_of(s), bytes);
            copy_w(s, k, q);
          }
          if (kReady) copy_x(s, k, q);
          if (++s == slots) {
            s = 0;
            round ^= 1u;
          }
        }
      }
      // nothing this thread issued may be in flight when the CTA exits
      const int back = min(it, slots);
      for (int i = 1; i <= back; ++i) bar_drain(full_of((it - i) % slots), ((it - i) / slots) & 1u);
    };
    if (elect()) {
      if (warp == 0) produce(std::true_type{});
      else produce(std::false_type{});
    }
    __syncwarp();
  } else if (warp == kMmaWarp) {
    if (elect()) {
      uint32_t idesc[2] = {instr_desc(BN, 0), instr_desc(BN, 1)};
      const uint64_t a_desc0 = smem_desc(a_base), b_desc0 = smem_desc(b_base);
      uint32_t it = 0, sit = 0, tl = 0;
      bool ok = true;
      for (int tile = tile0; tile < n_tiles && ok; tile += tile_step, ++tl) {
        if (C::kBox < BN) {
          const int width = (tiles.at(tile).tokens + C::kBox - 1) / C::kBox * C::kBox;
          idesc[0] = instr_desc(width, 0);
          idesc[1] = instr_desc(width, 1);
        }
        const uint32_t buf = tl % C::kDBuffers;
        ok = bar_wait(d_empty(buf), ((tl / C::kDBuffers) & 1u) ^ 1u, abort_flag);
        if (!ok) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint32_t d = tmem + buf * BN;
        for (int ss = ss0; ss < ss1 && ok; ++ss, ++sit) {
          const uint32_t sb = sit % C::kSfSlots;
          ok = bar_wait(ts_full(sb), (sit / C::kSfSlots) & 1u, abort_flag);
          if (!ok) break;
          const uint32_t sfa = sf_tmem + sb * C::kSfCols, sfb = sfa + 16;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (2 * ss + h >= P.n_ks) break;
            const uint32_t slot = it % C::kStages;
            ok = bar_wait(full(slot), (it / C::kStages) & 1u, abort_flag);
            if (!ok) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint64_t ad = a_desc0 + (uint64_t)(slot * kAStage >> 4), bd = b_desc0 + (uint64_t)(slot * C::kBStage >> 4);
#pragma unroll
            for (int i = 0; i < 4; ++i)
              mma_mx(d, ad + 2 * i, bd + 2 * i, idesc[i & 1], sfa + (2 * h + i / 2) * 4, sfb + (2 * h + i / 2) * C::kSfbCols,
                     (uint32_t)(ss != ss0 || h != 0 || i != 0));
            mma_commit(empty(slot));
            ++it;
          }
          mma_commit(ts_empty(sb));
        }
        if (ok) mma_commit(d_full(buf));
      }
      // every MMA must have finished before tensor memory is released
      mma_commit(drain);
      bar_drain(drain, 0);
    }
    __syncwarp();
  } else if (warp < kFirstEpiWarp) {
    // ---------------------------------------------------------------- scales to tensor memory
    const uint32_t quarter = (uint32_t)(32 * (warp & 3)) << 16;
    uint32_t sit = 0;
    bool ok = true;
    for (int tile = tile0; tile < n_tiles && ok; tile += tile_step)
      for (int ss = ss0; ss < ss1; ++ss, ++sit) {
        const uint32_t slot = sit % kScaleSlots, sb = sit % C::kSfSlots;
        ok = __all_sync(0xffffffffu, bar_wait(sc_full(slot), (sit / kScaleSlots) & 1u, abort_flag) &&
                                         bar_wait(ts_empty(sb), ((sit / C::kSfSlots) & 1u) ^ 1u, abort_flag));
        if (!ok) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint8_t* rows = gen + kScaleAt + slot * C::kScaleBytes;
        const uint32_t at = sf_tmem + sb * C::kSfCols + quarter;
        scales_to_tmem<4, 4>(rows, at, lane);
        scales_to_tmem<BN / 32, C::kSfbCols>(rows + kRows * 16, at + 16, lane);
        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncwarp();
        if (lane == 0) {
          bar_arrive(sc_empty(slot));
          bar_arrive(ts_full(sb));
        }
        __syncwarp();
      }
  } else {
    // ---------------------------------------------------------------- epilogue
    const int quad = warp & 3;
    const uint32_t quarter = (uint32_t)(32 * quad) << 16;
    uint32_t tl = 0;
    bool ok = true;
    // grouped: the next tile, and the rows of y that this warp's columns of it go to, asked for while this one is drained
    Spot next = {};
    int next_row[(C::kEpiColumns + 31) / 32];
    auto look = [&](int tile) {
      if (tile >= n_tiles) return;
      next = tiles.at(tile);
      const int begin = (warp > kScaleCopyWarp ? (warp - kScaleCopyWarp + 3) / 4 : 0) * C::kEpiColumns;
#pragma unroll
      for (int i = 0; i < C::kEpiColumns; i += 32) {
        const int c = begin + i + lane;
        next_row[i / 32] = i + lane < C::kEpiColumns && c < next.tokens && next.m0 + c < P.M ? P.order[next.m0 + c] : -1;
      }
    };
    if constexpr (GROUPED) look(tile0);
    for (int tile = tile0; tile < n_tiles && ok; tile += tile_step, ++tl) {
      if constexpr (!kReady) {
        if (tl == 0) begin_after_previous();
        // Stage i of the CTA's belongs to warp i % 4: a lane has eight columns, four lanes a block, of one token after the other.  The
        // next stage's columns and factors are asked for when this one's have been taken.
        const int m0 = tile % P.n_tiles_m * BN, tokens = min(kOwnTokens, P.M - m0), stages = 2 * (ss1 - ss0);
        Raw8<X> raw[kOwnTokens];
        float f[8];
        auto load = [&](int i) {
          const int k = (ks0 + i) * kStageK + lane * 8;
          if (P.inv) {
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = k + e < P.K ? P.inv[k + e] : 0.0f;
          }
          if (P.x_wide && k + 8 <= P.K) {
#pragma unroll
            for (int j = 0; j < kOwnTokens; ++j) raw[j] = load8(static_cast<const X*>(P.x) + min(m0 + j, P.M - 1) * P.ldx + k);
          }
        };
        load(warp - kFirstEpiWarp);
        for (int i = warp - kFirstEpiWarp; i < stages; i += 4) {
          const int k = (ks0 + i) * kStageK + lane * 8;
          const uint32_t it = tl * (ks1 - ks0) + i, sit = tl * (ss1 - ss0) + i / 2, slot = it % C::kStages, ss = sit % kScaleSlots;
          const bool there = ks0 + i < ks1;           // (the last 256 columns of 512 may be beyond the row)
          uint32_t c[kOwnTokens], byte[kOwnTokens];
#pragma unroll
          for (int j = 0; j < kOwnTokens; ++j) {
            if (j >= tokens || !there) break;
            float t[8];
            columns8<X>(P, m0 + j, k, raw[j], t);
            uint32_t top = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              if (P.inv) t[e] = __fmul_rn(t[e], f[e]);
              top = max(top, __float_as_uint(t[e]) & 0x7fffffffu);
            }
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
            byte[j] = mx_scale_byte(top);
            c[j] = 0;
            if (byte[j] != 255u) {
              const float s = mx_inverse_scale(byte[j]);
#pragma unroll
              for (int e = 0; e < 8; ++e) t[e] = __fmul_rn(t[e], s);
              c[j] = mx_codes8(t);
            }
          }
          load(i + 4);
          ok = __all_sync(0xffffffffu, (!there || bar_wait(empty(slot), ((it / C::kStages) & 1u) ^ 1u, abort_flag)) &&
                                           bar_wait(sc_empty(ss), ((sit / kScaleSlots) & 1u) ^ 1u, abort_flag));
          if (!ok) break;
          // 128-byte swizzle: the 16-byte piece's number in the row, exclusive-or the row in its group of eight
          uint8_t* codes = gen + C::kStages * kAStage + slot * C::kBStage + (lane & 3) * 4;
          uint8_t* bytes = gen + kScaleAt + ss * C::kScaleBytes + kRows * 16 + (i & 1) * 8 + lane / 4;
#pragma unroll
          for (int j = 0; j < kOwnTokens; ++j) {
            if (j >= tokens || !there) break;
            *reinterpret_cast<uint32_t*>(codes + j * 128 + ((lane / 4) ^ j) * 16) = c[j];
            if ((lane & 3) == 0) bytes[j * 16] = (uint8_t)byte[j];
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) {
            if (there) bar_arrive(full(slot));
            bar_arrive(sc_full(ss));
          }
          __syncwarp();
        }
        if (!ok) break;
      }
      const uint32_t buf = tl % C::kDBuffers;
      const Spot q = GROUPED ? next : tiles.at(tile);
      const int n = q.n0 + 32 * quad + lane, m0 = q.m0, tokens = q.tokens;
      const int part = warp > kScaleCopyWarp ? (warp - kScaleCopyWarp + 3) / 4 : 0, begin = part * C::kEpiColumns;
      const int end = min(tokens, begin + C::kEpiColumns);
      long long* mine = places + (4 * part + quad) * C::kEpiColumns;
      if constexpr (GROUPED) {
        __syncwarp();
#pragma unroll
        for (int i = 0; i < C::kEpiColumns; i += 32) {
          if (i + lane < C::kEpiColumns) {
            const int row = next_row[i / 32];
            mine[i + lane] = (unsigned)row < (unsigned)P.M ? row * P.ldy : -1;
          }
        }
        __syncwarp();
        look(tile + tile_step);
      }
      ok = __all_sync(0xffffffffu, bar_wait(d_full(buf), (tl / C::kDBuffers) & 1u, abort_flag));
      if (!ok) break;
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      const uint32_t from = tmem + quarter + buf * BN;
      if (split > 1) {            // every copy into the stages has landed and been read: they hold the partial sums
        float* part = reinterpret_cast<float*>(gen) + 32 * quad + lane;
        drain_columns<(BN > 64)>(from, begin, end, [&](int c, const uint32_t (&v)[16]) {
#pragma unroll
          for (int j = 0; j < 16; ++j) part[(c + j) * kRows] = __uint_as_float(v[j]);
        });
      } else if constexpr (GROUPED) {
        scatter_columns<(BN > 64)>(P, from, begin, end, (uint32_t)__cvta_generic_to_shared(mine), n);
      } else {
        store_columns<(BN > 64)>(P, from, begin, end, m0, n);
      }
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      if (lane == 0) bar_arrive(d_empty(buf));
      __syncwarp();
    }
    if constexpr (GROUPED) zero_rows(P, (warp > kScaleCopyWarp ? warp - 1 : warp) * 32 + lane - 32 * kFirstEpiWarp, 128 * C::kEpiParts);
  }
  if (split > 1) {
    // Token t of the tile is added up by rank t % split, a warp for 32 rows; the loads from all ranks are on their way together.
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
    const Spot q = !GROUPED || tile0 < n_tiles ? Tiles<BN, GROUPED>{P, first, begins}.at(tile0) : Spot{0, 0, 0, 0};
    const int n0 = q.n0, m0 = q.m0, tokens = q.tokens;
    constexpr int kBatch = BN == 16 ? 1 : 4;           // groups of 32 rows that a warp adds at a time
    for (int item = warp;; item += C::kThreads / 32) {
      const int t = rank + split * (item * kBatch / 4), row = item * kBatch % 4 * 32 + lane;
      if (t >= tokens) break;
      float v[kMostSplit][kBatch];
#pragma unroll
      for (int r = 0; r < kMostSplit; ++r) {
#pragma unroll
        for (int j = 0; j < kBatch; ++j) v[r][j] = 0.0f;
        if (r < (int)split) {
          uint32_t at;
          asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(base + (uint32_t)(t * kRows + row) * 4u), "r"(r));
#pragma unroll
          for (int j = 0; j < kBatch; ++j) asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v[r][j]) : "r"(at + 128 * j) : "memory");
        }
      }
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
#pragma unroll
        for (int r = 1; r < kMostSplit; ++r) v[0][j] += v[r][j];
      }
      by_type(P, [&](auto* y) {
        using T = std::remove_pointer_t<decltype(y)>;
        const int y_row = GROUPED ? planned_row(P, m0 + t) : m0 + t;
        T* to = y + (size_t)max(y_row, 0) * P.ldy + n0 + row;
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
          if (n0 + row + 32 * j < P.N && (!GROUPED || y_row >= 0)) to[32 * j] = from_f32<T>(v[0][j]);
      });
    }
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (warp == kMmaWarp) {
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)C::kTmemCols) : "memory");
  }
  if (threadIdx.x == 0 && *abort_flag && P.status) *P.status = LCD_ERR_TIMEOUT;
}

// ---------------------------------------------------------------------------------------------------------
// Many tokens: a pair of CTAs shares a tile of 256 weight rows x BN tokens (cta_group::2).  Each brings its own 128 rows of the weights
// and half of the tokens into its shared memory; the instruction reads both halves of the tokens for either CTA's rows.  So a CTA
// writes and reads 16 KB + BN / 2 rows a stage where it alone would need BN rows: shared memory's bandwidth, what bounds
// the kernel above, is enough (256 tokens: 128 bytes a clock).  Roles as above; the MMAs are issued by the pair's first CTA, and the
// copies of both CTAs' codes complete on its barriers.  The tokens' scales are needed by both and lie in both CTAs' tensor memory.
template <int BN, bool GROUPED = false>
struct PairCfg {
  static constexpr int kBStage = BN / 2 * kStageK / 2;
  static constexpr int kStages = 6;
  static constexpr int kScaleBytes = (kRows + BN) * 16;
  static constexpr int kSfCols = Cfg<BN>::kSfCols, kSfbCols = Cfg<BN>::kSfbCols, kSfSlots = BN == 256 ? 5 : 2;
  static constexpr int kDBuffers = 2 * BN + kSfSlots * kSfCols <= 512 ? 2 : 1;
  static constexpr int kEpiHalves = 2;
  static constexpr int kThreads = 32 * 15;
  static constexpr int kBox = GROUPED ? 32 : BN / 2;              // grouped: rows of a CTA's half that are copied together, see Cfg
  static constexpr int kPlanBytes = 8 * (kMostExperts + 1), kPlacesBytes = 4 * BN * 8;
  static constexpr int kSmem = 1024 + kStages * (kAStage + kBStage) + kScaleSlots * kScaleBytes + 512 + (GROUPED ? kPlanBytes + kPlacesBytes : 0);
  static_assert(kDBuffers * BN + kSfSlots * kSfCols <= 512 && kSmem <= 227 * 1024 && kSmem > 128 * 1024, "one CTA an SM");
};

__device__ __forceinline__ bool bar_try_cluster(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
               : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
// bar_wait for barriers that the other CTA arrives at.
__device__ __forceinline__ bool bar_wait_cluster(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
  if (bar_try_cluster(bar, parity)) return true;
  const unsigned long long t0 = timer_ns();
  for (uint32_t it = 1;; ++it) {
    if (bar_try_cluster(bar, parity)) return true;
    if ((it & 255u) == 0) {
      if (*abort_flag) return false;
      if (timer_ns() - t0 > kWaitNs) { *abort_flag = 1; return false; }
    }
  }
}
// An address of this CTA's shared memory, in the pair's CTA of that rank.
__device__ __forceinline__ uint32_t in_cta(uint32_t addr, uint32_t rank) {
  uint32_t a;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(addr), "r"(rank));
  return a;
}
// Arrives at the first CTA's barrier of the pair.  What it tells of is tensor memory that has been written or read, which the tcgen05 fences
// on both sides order around any signal; no other memory is handed over, so the signal itself is relaxed (with release at
// cluster scope the call of 2048 x 13824 x 5120 takes 87 us, 67 so).
__device__ __forceinline__ void bar_arrive_first(uint32_t bar) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(in_cta(bar, 0)) : "memory");
}
// A tile into this CTA's shared memory that completes on a barrier of either CTA (an address in the cluster's window).
__device__ __forceinline__ void copy_tile_pair(uint32_t dst, const CUtensorMap* map, int x, int row, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3}], [%4];"
               ::"r"(dst), "l"(map), "r"(x), "r"(row), "r"(bar) : "memory");
}
__device__ __forceinline__ void mma_mx_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t accumulate) {
  asm volatile(
      "{\n.reg .pred p;\nsetp.ne.b32 p, %6, 0;\n"
      "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n}"
      ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory");
}
// At both CTAs' barriers, once the MMAs so far have finished.
__device__ __forceinline__ void mma_commit_pair(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3) : "memory");
}

__device__ __forceinline__ void copy_tile_pair_of(uint32_t dst, const CUtensorMap* map, int x, int row, int expert, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3, %4}], [%5];"
               ::"r"(dst), "l"(map), "r"(x), "r"(row), "r"(expert), "r"(bar) : "memory");
}

template <int BN, bool GROUPED>
__global__ void __launch_bounds__(PairCfg<BN, GROUPED>::kThreads, 1)
mx_pair_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x,
               const __grid_constant__ CUtensorMap map_ws, const __grid_constant__ CUtensorMap map_xs, const Args P) {
  using C = PairCfg<BN, GROUPED>;
  extern __shared__ uint8_t smem_raw[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t raw_addr = (uint32_t)__cvta_generic_to_shared(smem_raw);
  const uint32_t base = (raw_addr + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (base - raw_addr);
  constexpr uint32_t kScaleAt = C::kStages * (kAStage + C::kBStage), kBarAt = kScaleAt + kScaleSlots * C::kScaleBytes;
  const uint32_t a_base = base, b_base = base + C::kStages * kAStage, s_base = base + kScaleAt, bars = base + kBarAt;
  auto full = [&](int s) { return bars + 8u * s; };
  auto empty = [&](int s) { return bars + 8u * (C::kStages + s); };
  auto sc_full = [&](int s) { return bars + 8u * (2 * C::kStages + s); };
  auto sc_empty = [&](int s) { return bars + 8u * (2 * C::kStages + kScaleSlots + s); };
  constexpr int kB0 = 2 * C::kStages + 2 * kScaleSlots, kB1 = kB0 + 2 * C::kSfSlots;
  auto ts_full = [&](int b) { return bars + 8u * (kB0 + b); };
  auto ts_empty = [&](int b) { return bars + 8u * (kB0 + C::kSfSlots + b); };
  auto d_full = [&](int b) { return bars + 8u * (kB1 + b); };
  auto d_empty = [&](int b) { return bars + 8u * (kB1 + 2 + b); };
  const uint32_t drain = bars + 8u * (kB1 + 4);
  static_assert(8 * (kB1 + 5) + 24 <= 512, "barriers");
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(gen + kBarAt + 8 * (kB1 + 5));
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_holder + 1);
  // stages that this CTA has asked for copies of; the other CTA's flag and number, which it sends at its end
  volatile int *asked = abort_flag + 1, *other_abort = abort_flag + 2, *other_asked = abort_flag + 3;
  long long* places = reinterpret_cast<long long*>(gen + kBarAt + 512);              // grouped
  int* first_tiles = reinterpret_cast<int*>(gen + kBarAt + 512 + C::kPlacesBytes);
  int* begins = first_tiles + kMostExperts + 1;
  // Tokens of a tile that a CTA brings, and so the bytes of a stage: grouped, as many boxes as the tile has tokens for.
  auto half_of = [](const Spot& q) { return GROUPED ? (q.tokens + 2 * C::kBox - 1) / (2 * C::kBox) * C::kBox : BN / 2; };
  auto stage_bytes = [&](const Spot& q) { return (uint32_t)(kAStage + half_of(q) * (kStageK / 2)); };
  uint32_t rank;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  const bool first = rank == 0;
  const int tile0 = blockIdx.x / 2, tile_step = gridDim.x / 2;

  if (threadIdx.x == 0) {
    for (int s = 0; s < C::kStages; ++s) {
      bar_init(full(s), 1);                          // the first CTA's take both CTAs' copies, the other's are not used
      bar_init(empty(s), 1);
    }
    for (int s = 0; s < kScaleSlots; ++s) {
      bar_init(sc_full(s), 1);
      bar_init(sc_empty(s), 4);
    }
    for (int b = 0; b < C::kSfSlots; ++b) {
      bar_init(ts_full(b), 8);                       // both CTAs' warps
      bar_init(ts_empty(b), 1);
    }
    for (int b = 0; b < 2; ++b) {
      bar_init(d_full(b), 1);
      bar_init(d_empty(b), 2 * 4 * C::kEpiHalves);
    }
    bar_init(drain, 1);
    *abort_flag = 0;
    *asked = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (GROUPED && warp == 2) make_tiles<BN>(P, first_tiles, begins, lane);
  if (warp == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;"
                 ::"r"((uint32_t)__cvta_generic_to_shared(tmem_holder)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("barrier.cluster.arrive.release;" ::: "memory");      // both CTAs' barriers and tensor memory are there
  asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = *tmem_holder;
  const uint32_t sf_tmem = tmem + C::kDBuffers * BN;
  const int n_tiles = GROUPED ? min(P.n_tiles, first_tiles[P.G] * ((P.N + 2 * kRows - 1) / (2 * kRows))) : P.n_tiles;
  Tiles<BN, GROUPED, 2 * kRows> tiles{P, first_tiles, begins};
  if (warp != 0 && warp != kScaleCopyWarp) wait_for_previous();      // as above

  if (warp == 0 || warp == kScaleCopyWarp) {
    auto produce = [&](auto of_codes) {
      constexpr bool codes = decltype(of_codes)::value;
      constexpr int slots = codes ? C::kStages : kScaleSlots;
      const int to = codes ? P.n_ks : P.n_ss;
      // Codes: the first CTA's thread announces the bytes of both CTAs' copies (those of the other may have landed by then; its arrival is
      // what the phase waits for).  The other is never a phase ahead: it waits for the MMAs that read what it overwrites.
      const uint32_t full_first = in_cta(full(0), 0);
      auto announce = [&](int s, uint32_t bytes) {
        if (!codes) bar_expect_tx(sc_full(s), C::kScaleBytes);
        else if (first) bar_expect_tx(full(s), 2 * bytes);
      };
      auto copy_w = [&](int s, int k, const Spot& q) {
        const int row = q.n0 + (int)rank * kRows;
        if (GROUPED && codes) copy_tile_pair_of(a_base + s * kAStage, &map_w, k * (kStageK / 2), row, q.expert, full_first + 8u * s);
        else if (GROUPED) copy_tile_of(s_base + s * C::kScaleBytes, &map_ws, k * 16, row, q.expert, sc_full(s));
        else if (codes) copy_tile_pair(a_base + s * kAStage, &map_w, k * (kStageK / 2), row, full_first + 8u * s);
        else copy_tile(s_base + s * C::kScaleBytes, &map_ws, k * 16, row, sc_full(s));
      };
      auto copy_x = [&](int s, int k, const Spot& q, int half) {
        const int row = q.m0 + (int)rank * half;
        if (!codes) copy_tile(s_base + s * C::kScaleBytes + kRows * 16, &map_xs, k * 16, q.m0, sc_full(s));
        else
          for (int r = 0; r < half; r += C::kBox)
            copy_tile_pair(b_base + s * C::kBStage + r * (kStageK / 2), &map_x, k * (kStageK / 2), row + r, full_first + 8u * s);
      };
      const int ahead = P.early && tile0 < n_tiles ? min(slots, to) : 0;
      if (ahead > 0) {
        const Spot q = tiles.at(tile0);
        for (int i = 0; i < ahead; ++i) {
          announce(i, stage_bytes(q));
          copy_w(i, i, q);
        }
      }
      begin_after_previous();
      int it = 0, s = 0;
      uint32_t round = 1;          // the parity of a stage's barrier
      bool ok = true;
      for (int tile = tile0; tile < n_tiles && ok; tile += tile_step) {
        const Spot q = tiles.at(tile);
        const int half = half_of(q);
        for (int k = 0; k < to; ++k, ++it) {
          if (it >= ahead) {
            ok = codes ? bar_wait_cluster(empty(s), round, abort_flag) : bar_wait(sc_empty(s), round, abort_flag);
            if (!ok) break;
            announce(s, stage_bytes(q));
            copy_w(s, k, q);
          }
          copy_x(s, k, q, half);
          if (++s == slots) {
            s = 0;
            round ^= 1u;
          }
        }
      }
      // Nothing that this thread issued may be in flight when the CTA exits.  Codes have landed where every MMA has run; if not, see
      // the end.
      if (codes) {
        *asked = it;
      } else {
        const int back = min(it, slots);
        for (int i = 1; i <= back; ++i) bar_drain(sc_full((it - i) % slots), ((it - i) / slots) & 1u);
      }
    };
    if (elect()) {
      if (warp == 0) produce(std::true_type{});
      else produce(std::false_type{});
    }
    __syncwarp();
  } else if (warp == kMmaWarp) {
    if (first && elect()) {
      constexpr uint32_t kM = (uint32_t)(2 * kRows >> 4) << 24 ^ (uint32_t)(kRows >> 4) << 24;     // M = 256 in place of 128
      uint32_t idesc[2] = {instr_desc(BN, 0) ^ kM, instr_desc(BN, 1) ^ kM};
      const uint64_t a_desc0 = smem_desc(a_base), b_desc0 = smem_desc(b_base);
      uint32_t it = 0, sit = 0, tl = 0;
      bool ok = true;
      for (int tile = tile0; tile < n_tiles && ok; tile += tile_step, ++tl) {
        if (GROUPED) {
          const int width = 2 * half_of(tiles.at(tile));
          idesc[0] = instr_desc(width, 0) ^ kM;
          idesc[1] = instr_desc(width, 1) ^ kM;
        }
        const uint32_t buf = tl % C::kDBuffers;
        ok = bar_wait_cluster(d_empty(buf), ((tl / C::kDBuffers) & 1u) ^ 1u, abort_flag);
        if (!ok) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint32_t d = tmem + buf * BN;
        for (int ss = 0; ss < P.n_ss && ok; ++ss, ++sit) {
          const uint32_t sb = sit % C::kSfSlots;
          ok = bar_wait_cluster(ts_full(sb), (sit / C::kSfSlots) & 1u, abort_flag);
          if (!ok) break;
          const uint32_t sfa = sf_tmem + sb * C::kSfCols, sfb = sfa + 16;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (2 * ss + h >= P.n_ks) break;
            const uint32_t slot = it % C::kStages;
            ok = bar_wait_cluster(full(slot), (it / C::kStages) & 1u, abort_flag);
            if (!ok) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint64_t ad = a_desc0 + (uint64_t)(slot * kAStage >> 4), bd = b_desc0 + (uint64_t)(slot * C::kBStage >> 4);
#pragma unroll
            for (int i = 0; i < 4; ++i)
              mma_mx_pair(d, ad + 2 * i, bd + 2 * i, idesc[i & 1], sfa + (2 * h + i / 2) * 4, sfb + (2 * h + i / 2) * C::kSfbCols,
                          (uint32_t)(ss != 0 || h != 0 || i != 0));
            mma_commit_pair(empty(slot));
            ++it;
          }
          mma_commit_pair(ts_empty(sb));
        }
        if (ok) mma_commit_pair(d_full(buf));
      }
      // every MMA must have finished before tensor memory is released, the other CTA's too
      mma_commit_pair(drain);
      bar_drain(drain, 0);
    }
    __syncwarp();
  } else if (warp < kFirstEpiWarp) {
    const uint32_t quarter = (uint32_t)(32 * (warp & 3)) << 16;
    uint32_t sit = 0;
    bool ok = true;
    for (int tile = tile0; tile < n_tiles && ok; tile += tile_step)
      for (int ss = 0; ss < P.n_ss; ++ss, ++sit) {
        const uint32_t slot = sit % kScaleSlots, sb = sit % C::kSfSlots;
        ok = __all_sync(0xffffffffu, bar_wait(sc_full(slot), (sit / kScaleSlots) & 1u, abort_flag) &&
                                         bar_wait_cluster(ts_empty(sb), ((sit / C::kSfSlots) & 1u) ^ 1u, abort_flag));
        if (!ok) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint8_t* rows = gen + kScaleAt + slot * C::kScaleBytes;
        const uint32_t at = sf_tmem + sb * C::kSfCols + quarter;
        scales_to_tmem<4, 4>(rows, at, lane);
        scales_to_tmem<BN / 32, C::kSfbCols>(rows + kRows * 16, at + 16, lane);
        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncwarp();
        if (lane == 0) {
          bar_arrive(sc_empty(slot));
          bar_arrive_first(ts_full(sb));
        }
        __syncwarp();
      }
  } else {
    const int quad = warp & 3;
    const uint32_t quarter = (uint32_t)(32 * quad) << 16;
    const int part = warp > kScaleCopyWarp;
    long long* mine = places + (4 * part + quad) * (BN / 2);
    uint32_t tl = 0;
    bool ok = true;
    // grouped: as above
    Spot next = {};
    int next_row[BN / 64];
    auto look = [&](int tile) {
      if (tile >= n_tiles) return;
      next = tiles.at(tile);
      const int half = half_of(next);
#pragma unroll
      for (int i = 0; i < BN / 2; i += 32) {
        const int c = part * half + i + lane;
        next_row[i / 32] = i + lane < half && c < next.tokens && next.m0 + c < P.M ? P.order[next.m0 + c] : -1;
      }
    };
    if constexpr (GROUPED) look(tile0);
    for (int tile = tile0; tile < n_tiles && ok; tile += tile_step, ++tl) {
      const uint32_t buf = tl % C::kDBuffers;
      const Spot q = GROUPED ? next : tiles.at(tile);
      const int n = q.n0 + (int)rank * kRows + 32 * quad + lane, m0 = q.m0, tokens = q.tokens, begin = part ? half_of(q) : 0;
      if constexpr (GROUPED) {
        __syncwarp();
#pragma unroll
        for (int i = 0; i < BN / 2; i += 32) mine[i + lane] = (unsigned)next_row[i / 32] < (unsigned)P.M ? next_row[i / 32] * P.ldy : -1;
        __syncwarp();
        look(tile + tile_step);
      }
      ok = __all_sync(0xffffffffu, bar_wait_cluster(d_full(buf), (tl / C::kDBuffers) & 1u, abort_flag));
      if (!ok) break;
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      const int end = part ? tokens : min(tokens, half_of(q));
      if constexpr (GROUPED) scatter_columns<true>(P, tmem + quarter + buf * BN, begin, end, (uint32_t)__cvta_generic_to_shared(mine), n);
      else store_columns<true>(P, tmem + quarter + buf * BN, begin, end, m0, n);
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      if (lane == 0) bar_arrive_first(d_empty(buf));
      __syncwarp();
    }
    if constexpr (GROUPED) zero_rows(P, (warp > kScaleCopyWarp ? warp - 1 : warp) * 32 + lane - 32 * kFirstEpiWarp, 256);
  }
  // neither CTA leaves while the other may still read its shared memory or arrive at its barriers
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (!first && warp == kMmaWarp && elect()) bar_drain(drain, 0);      // the last of the signals that the first CTA's MMAs send here
  if (threadIdx.x == 0) {
    const uint32_t to = (uint32_t)__cvta_generic_to_shared(const_cast<int*>(other_abort));
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(in_cta(to, rank ^ 1u)), "r"(*abort_flag) : "memory");
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(in_cta(to + 4, rank ^ 1u)), "r"(*asked) : "memory");
  }
  asm volatile("barrier.cluster.arrive.release;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
  if (*abort_flag || *other_abort) {          // in both CTAs or in neither
    if (first && threadIdx.x == 0) {
      // Stages that one CTA alone has asked for: the other's part is announced, or taken back, so that their barriers complete when the
      // copies have landed.
      const int own = *asked, other = *other_asked, most = max(own, other);
      for (int i = min(own, other); i < most; ++i) {
        const uint32_t bar = full(i % C::kStages);
        Tiles<BN, GROUPED, 2 * kRows> again{P, first_tiles, begins};
        const uint32_t bytes = stage_bytes(again.at(tile0 + i / P.n_ks * tile_step));
        if (other > own) bar_expect_tx(bar, bytes);
        else asm volatile("mbarrier.complete_tx.relaxed.cluster.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
      }
      for (int i = max(0, most - C::kStages); i < most; ++i) bar_drain(full(i % C::kStages), (i / C::kStages) & 1u);
    }
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
  }
  if (warp == kMmaWarp) {
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
  if (threadIdx.x == 0 && *abort_flag && P.status) *P.status = LCD_ERR_TIMEOUT;
}

bool encode_rows(CUtensorMap* map, const uint8_t* p, int64_t bytes, int64_t rows, int64_t ld, int box_bytes, int box_rows, bool swizzled) {
  const EncodeTiledFn encode = encode_tiled();
  const cuuint64_t dims[2] = {(cuuint64_t)bytes, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld};
  const cuuint32_t box[2] = {(cuuint32_t)box_bytes, (cuuint32_t)box_rows}, one[2] = {1, 1};
  return encode && encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<uint8_t*>(p), dims, strides, box, one,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, swizzled ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE,
                          CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// How a product is cut: the width of the token tiles, whether a pair of CTAs shares one, or how many share its columns.
struct Plan { int width, split; bool pair; };

// Estimated in microseconds: a stage (upper values of what products timed alone on B200 show), an epilogue that only the widest tile
// cannot overlap with the next one's columns, for a shared tile the cluster's barrier and 1 us a 64 tokens to add up.  Pairs to bf16:
// 4096 x 8192 x 8192 97 us with 256 tokens, 100 with 192, single CTAs 107; 2048 x 13824 x 5120 58, 60 and 63; 1024 x 8192 x 8192
// 27.9, 30.9 and 30.1.  To fp32: 2048 x 5120 x 13824 57 with pairs and 192 tokens, single CTAs 62; 333 x 5003 x 5001 13.8 with pairs,
// single CTAs of 128 tokens 13.1, of 192 16; 512 x 5120 x 5120 10.8 with pairs and 192 tokens, single CTAs of 192 10.5, of 256 12.8,
// of 128 14.2.  8 x 4096 x 4096 5.5 / 5.2 / 4.4 with 1 / 2 / 4 CTAs a tile, 16 x 4096 x 11008 12.9 / 10.3 / 8.5; eight a tile are more
// than one an SM there and slower.
Plan plan(int64_t M, int64_t N, int64_t n_ks) {
  static constexpr struct { int width; double stage, epilogue; bool pair; } kWidths[] = {
      {16, 0.33, 0.1, false}, {32, 0.33, 0.2, false}, {64, 0.34, 0.4, false}, {128, 0.31, 0.4, false},
      {192, 0.39, 0.2, false}, {256, 0.35, 2.9, false}, {192, 0.33, 0.1, true}, {256, 0.31, 2.6, true}};
  const int64_t sms = current_sm_count(), n_ss = (n_ks + 1) / 2;
  Plan best = {256, 1, false};
  double least = 1e300;
  for (const auto& w : kWidths) {
    if (M > w.width && w.width < 128) continue;           // few tokens: one tile of them
    const int64_t rows = w.pair ? 2 * kRows : kRows, tiles = (M + w.width - 1) / w.width * ((N + rows - 1) / rows);
    const int64_t at_once = w.pair ? sms / 2 : sms, waves = (tiles + at_once - 1) / at_once;
    for (int s = 1; s <= (w.pair ? 1 : kMostSplit) && s <= n_ss && (s == 1 || tiles * s <= sms); ++s) {
      if (s > 4 && (w.width >= 128 || tiles * s > sms / 2)) break;      // clusters of more than four do not fill the GPU
      const double time = waves * (2 * w.stage * ((n_ss + s - 1) / s) + w.epilogue) + (w.pair ? 1.0 : 0.0) +
                          (s > 1 ? 2.0 + (M < w.width ? M : w.width) / (64.0 * s) : 0.0);
      if (time < least) {
        least = time;
        best = {w.width, s, w.pair};
      }
    }
    if (M <= w.width && w.width < 128) break;
  }
  return best;
}

// The width and the cut of a product grouped by expert.  How many rows an expert has is not known here; from the mean m over the experts
// that can occur, taken for exponentially distributed, an expert has 1 / (1 - exp(-w / m)) tiles of w tokens.  Times of a stage and of a
// tile's end in microseconds, from whole calls on B200 one behind the other over the same buffers, so that weights of less than L2's size come
// from there (with others every time the 71 of the first, 128 wide, is 82; widths 16 / 32 / 64 / 128 / 192 / 256 / pairs of 192 / of 256):
//     2048 tokens x 4 of 32 experts, 4096 x 2048: 158 / 102 / 79 / 71 / 72 / 90 / 72 / 89 us; 4096 x 8192: - / - / 268 / 232 / 221 / 245 / 218 / 230
//     4096 x 2 of 8, 14336 x 4096: - / - / 446 / 320 / 289 / 363 / 272 / 358;   512 x 4 of 32, 4096 x 2048: 53 / 40 / 36 / 38 / 46 / 54 / 45 / 52
//     48 x 2 of 8, 11008 x 4096: 37 / 38 / 39 / 41 / 46 / 56;   200 x 4 of 32, 4096 x 2048: 34 / 31 / 33 / 35 / 41 / 46
Plan plan_grouped(int64_t rows, int64_t G, int64_t N, int64_t n_ks) {
  static constexpr struct { int width; double stage, end; bool pair; } kWidths[] = {
      {16, 0.15, 0.1, false}, {32, 0.18, 0.1, false}, {64, 0.24, 0.2, false}, {128, 0.36, 0.4, false},
      {192, 0.43, 1.1, false}, {256, 0.54, 2.7, false}, {192, 0.42, 1.2, true}, {256, 0.49, 3.1, true}};
  const double experts = (double)(G < rows ? G : rows), mean = (double)rows / experts, sms = current_sm_count();
  const int64_t n_ss = (n_ks + 1) / 2;
  Plan best = {256, 1, false};
  double least = 1e300;
  for (const auto& w : kWidths) {
    const int64_t n_tiles_n = w.pair ? (N + 2 * kRows - 1) / (2 * kRows) : (N + kRows - 1) / kRows;
    const double tiles = experts * n_tiles_n / (1.0 - exp(-w.width / mean)), at_once = w.pair ? sms / 2 : sms;
    const int64_t bound = (rows / w.width + (int64_t)experts) * n_tiles_n;
    for (int s = 1; s <= (w.pair ? 1 : kMostSplit) && s <= n_ss && (s == 1 || bound * s <= (int64_t)sms); s *= 2) {
      if (s > 4 && (w.width >= 128 || bound * s > (int64_t)sms / 2)) break;
      const double waves = tiles < at_once ? 1.0 : tiles / at_once;
      const double time = waves * (2 * w.stage * ((n_ss + s - 1) / s) + w.end) + (s > 1 ? 2.0 + fmin(mean, w.width) / (64.0 * s) : 0.0);
      if (time < least) {
        least = time;
        best = {w.width, s, w.pair};
      }
    }
  }
  return best;
}

template <int BN, typename X = void>
lcd_status launch_width(const MxProduct& p, int split, bool early, int32_t* status, cudaStream_t s) {
  using C = Cfg<BN>;
  auto kern = mx_linear_kernel<BN, X, false>;
  static PerDeviceFlag attr_set;
  int dev;
  if (attr_set.first(&dev)) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem);
    if (e != cudaSuccess) { set_cuda_error((int)e); return LCD_ERR_CUDA; }
    attr_set.done(dev);
  }
  const int64_t blocks = (p.K + kMxBlock - 1) / kMxBlock;
  const int64_t n_tiles_m = (p.M + BN - 1) / BN, tiles = n_tiles_m * ((p.N + kRows - 1) / kRows);
  if (tiles > 0x7fffffff) return LCD_ERR_UNSUPPORTED;
  CUtensorMap w, x, ws, xs;
  bool encoded = encode_rows(&w, p.w_codes, blocks * 16, p.N, p.ldwc, kStageK / 2, kRows, true) &&
                 encode_rows(&ws, p.w_scales, blocks, p.N, p.ldws, 16, kRows, false);
  if (std::is_same<X, void>::value) {
    encoded = encoded && encode_rows(&x, p.x_codes, blocks * 16, p.M, p.ldxc, kStageK / 2, BN, true) &&
              encode_rows(&xs, p.x_scales, blocks, p.M, p.ldxs, 16, BN, false);
  } else {
    x = w;               // not used
    xs = ws;
  }
  if (!encoded) {
    set_cuda_error((int)cudaErrorInvalidValue);
    return LCD_ERR_CUDA;
  }
  Args a = {};
  a.x = p.x;
  a.ldx = p.ldx;
  a.inv = p.inv_smooth;
  a.K = (int)p.K;
  a.x_wide = p.x && reinterpret_cast<uintptr_t>(p.x) % 16 == 0 && (p.M == 1 || p.ldx * (p.x_type == LCD_DTYPE_F32 ? 4 : 2) % 16 == 0);
  a.y = p.y;
  a.ldy = p.ldy;
  a.y_type = (int)p.y_type;
  a.M = (int)p.M;
  a.N = (int)p.N;
  a.n_ks = (int)((blocks * kMxBlock + kStageK - 1) / kStageK);
  a.n_ss = (a.n_ks + 1) / 2;
  a.n_tiles_m = (int)n_tiles_m;
  a.n_tiles = (int)tiles;
  a.early = early;
  a.status = status;
  const int64_t room = (int64_t)current_sm_count() * C::kPerSm;
  const unsigned grid = (unsigned)(split > 1 ? tiles * split : tiles < room ? tiles : room);
  const cudaError_t e = launch_overlapping(kern, dim3(grid), dim3(C::kThreads), C::kSmem, (unsigned)split, s, w, x, ws, xs, a);
  if (e != cudaSuccess) { set_cuda_error((int)e); return LCD_ERR_CUDA; }
  return LCD_OK;
}

// The matrices of all experts: the third coordinate is the expert.
bool encode_experts(CUtensorMap* map, const uint8_t* p, int64_t bytes, int64_t rows, int64_t ld, int64_t experts, int64_t distance, int box_bytes,
                    bool swizzled) {
  const EncodeTiledFn encode = encode_tiled();
  const cuuint64_t dims[3] = {(cuuint64_t)bytes, (cuuint64_t)rows, (cuuint64_t)experts}, strides[2] = {(cuuint64_t)ld, (cuuint64_t)distance};
  const cuuint32_t box[3] = {(cuuint32_t)box_bytes, (cuuint32_t)kRows, 1}, one[3] = {1, 1, 1};
  return encode && encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<uint8_t*>(p), dims, strides, box, one,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, swizzled ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE,
                          CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int BN>
lcd_status launch_pair(const MxProduct& p, bool early, int32_t* status, cudaStream_t s) {
  using C = PairCfg<BN>;
  auto kern = mx_pair_kernel<BN, false>;
  static PerDeviceFlag attr_set;
  int dev;
  if (attr_set.first(&dev)) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem);
    if (e != cudaSuccess) { set_cuda_error((int)e); return LCD_ERR_CUDA; }
    attr_set.done(dev);
  }
  const int64_t blocks = (p.K + kMxBlock - 1) / kMxBlock;
  const int64_t n_tiles_m = (p.M + BN - 1) / BN, tiles = n_tiles_m * ((p.N + 2 * kRows - 1) / (2 * kRows));
  if (tiles > 0x7fffffff) return LCD_ERR_UNSUPPORTED;
  CUtensorMap w, x, ws, xs;
  if (!encode_rows(&w, p.w_codes, blocks * 16, p.N, p.ldwc, kStageK / 2, kRows, true) ||
      !encode_rows(&ws, p.w_scales, blocks, p.N, p.ldws, 16, kRows, false) ||
      !encode_rows(&x, p.x_codes, blocks * 16, p.M, p.ldxc, kStageK / 2, BN / 2, true) ||
      !encode_rows(&xs, p.x_scales, blocks, p.M, p.ldxs, 16, BN, false)) {
    set_cuda_error((int)cudaErrorInvalidValue);
    return LCD_ERR_CUDA;
  }
  Args a = {};
  a.y = p.y;
  a.ldy = p.ldy;
  a.y_type = (int)p.y_type;
  a.M = (int)p.M;
  a.N = (int)p.N;
  a.n_ks = (int)((blocks * kMxBlock + kStageK - 1) / kStageK);
  a.n_ss = (a.n_ks + 1) / 2;
  a.n_tiles_m = (int)n_tiles_m;
  a.n_tiles = (int)tiles;
  a.early = early;
  a.status = status;
  const int64_t pairs = current_sm_count() / 2;
  const cudaError_t e = launch_overlapping(kern, dim3((unsigned)(2 * (tiles < pairs ? tiles : pairs))), dim3(C::kThreads), C::kSmem, 2u, s, w, x, ws, xs, a);
  if (e != cudaSuccess) { set_cuda_error((int)e); return LCD_ERR_CUDA; }
  return LCD_OK;
}

template <int BN, bool PAIR>
lcd_status launch_grouped(const MxGrouped& p, int split, int32_t* status, cudaStream_t s) {
  using C = std::conditional_t<PAIR, PairCfg<BN, true>, Cfg<BN, true>>;
  auto kern = [] {
    if constexpr (PAIR) return mx_pair_kernel<BN, true>;
    else return mx_linear_kernel<BN, void, true>;
  }();
  static PerDeviceFlag attr_set;
  int dev;
  if (attr_set.first(&dev)) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem);
    if (e != cudaSuccess) { set_cuda_error((int)e); return LCD_ERR_CUDA; }
    attr_set.done(dev);
  }
  const int64_t blocks = (p.K + kMxBlock - 1) / kMxBlock, rows = PAIR ? 2 * kRows : kRows, n_tiles_n = (p.N + rows - 1) / rows;
  // at most: every expert's last tile may hold one token
  const int64_t tiles = (p.rows.count / BN + (p.G < p.rows.count ? p.G : p.rows.count)) * n_tiles_n;
  if (tiles * split > 0x7fffffff) return LCD_ERR_UNSUPPORTED;
  CUtensorMap w, x, ws, xs;
  if (!encode_experts(&w, p.w_codes, blocks * 16, p.N, p.ldwc, p.G, p.dwc, kStageK / 2, true) ||
      !encode_experts(&ws, p.w_scales, blocks, p.N, p.ldws, p.G, p.dws, 16, false) ||
      !encode_rows(&x, p.x_codes, blocks * 16, p.rows.count, p.ldxc, kStageK / 2, C::kBox, true) ||
      !encode_rows(&xs, p.x_scales, blocks, p.rows.count, p.ldxs, 16, BN, false)) {
    set_cuda_error((int)cudaErrorInvalidValue);
    return LCD_ERR_CUDA;
  }
  Args a = {};
  a.y = p.y;
  a.ldy = p.ldy;
  a.y_type = (int)p.y_type;
  a.M = (int)p.rows.count;
  a.N = (int)p.N;
  a.n_ks = (int)((blocks * kMxBlock + kStageK - 1) / kStageK);
  a.n_ss = (a.n_ks + 1) / 2;
  a.n_tiles = (int)tiles;
  a.early = 1;
  a.status = status;
  a.order = p.rows.order;
  a.offsets = p.rows.offsets;
  a.G = (int)p.G;
  int64_t room = 0;
  if constexpr (PAIR) room = current_sm_count() / 2;
  else room = (int64_t)current_sm_count() * C::kPerSm;
  const int64_t at_once = split > 1 || tiles < room ? tiles : room;
  const cudaError_t e = launch_overlapping(kern, dim3((unsigned)(at_once * (PAIR ? 2 : split))), dim3(C::kThreads), C::kSmem,
                                           PAIR ? 2u : (unsigned)split, s, w, x, ws, xs, a);
  if (e != cudaSuccess) { set_cuda_error((int)e); return LCD_ERR_CUDA; }
  return LCD_OK;
}

}  // namespace

// Device time, one launch and two, us (N x K: 1 / 2 / 3 / 4 tokens):
//     1024 x 4096    4.1 4.9 / 4.3 4.9 / 4.7 5.0 / 4.8 5.2         11008 x 4096   6.6 7.6 / 7.8 7.6 / 8.1 7.8 / 8.7 7.6
//     4096 x 4096    4.8 6.2 / 5.0 5.7 / 5.5 6.4 / 5.5 5.9         11008 x 8192   13.8 13.3 / 15.7 13.3 / 17.4 13.3 / 18.2 13.1
//     4096 x 8192    5.7 6.9 / 6.2 7.1 / 6.7 7.1 / 7.0 7.0         28672 x 4096   12.9 16.2 / 13.3 14.8 / 14.2 17.5 / 14.2 14.9
//     4096 x 14336   8.7 9.3 / 9.0 9.0 / 9.9 9.1 / 10.4 9.0        28672 x 8192   21.7 23.8 / 23.1 24.1 / 24.4 24.0 / 25.4 24.4
//     4096 x 28672   15.1 15.4 / 16.5 15.4 / 17.7 15.4 / 18.4 15.4
// One launch gains up to M * K of about 28672 where a tile's columns are cut or two CTAs share an SM, and on the host (5.4 us a call, 8.1);
// with one CTA an SM and columns uncut (N of 9500 to 19000) only up to 8192.  The border goes by M and K alone, as the workspace does.
bool mx_linear_quantizes(int64_t M, int64_t K) { return M <= kOwnTokens && M * K <= 28672; }

lcd_status launch_mx_linear(const MxProduct& p, bool x_just_written, int32_t* status_word, void* stream) {
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const Plan w = plan(p.M, p.N, ((p.K + kMxBlock - 1) / kMxBlock * kMxBlock + kStageK - 1) / kStageK);
  if (p.x) {
    switch (p.x_type) {
      case LCD_DTYPE_F32: return launch_width<16, float>(p, w.split, false, status_word, s);
      case LCD_DTYPE_F16: return launch_width<16, __half>(p, w.split, false, status_word, s);
      default: return launch_width<16, __nv_bfloat16>(p, w.split, false, status_word, s);
    }
  }
  if (w.pair) return w.width == 192 ? launch_pair<192>(p, x_just_written, status_word, s) : launch_pair<256>(p, x_just_written, status_word, s);
  switch (w.width) {
    case 16: return launch_width<16>(p, w.split, x_just_written, status_word, s);
    case 32: return launch_width<32>(p, w.split, x_just_written, status_word, s);
    case 64: return launch_width<64>(p, w.split, x_just_written, status_word, s);
    case 128: return launch_width<128>(p, w.split, x_just_written, status_word, s);
    case 192: return launch_width<192>(p, w.split, x_just_written, status_word, s);
    default: return launch_width<256>(p, w.split, x_just_written, status_word, s);
  }
}

MxGroupedShape mx_grouped_shape(int64_t count, int64_t G, int64_t N, int64_t K) {
  const Plan w = plan_grouped(count, G, N, ((K + kMxBlock - 1) / kMxBlock * kMxBlock + kStageK - 1) / kStageK);
  return {w.width, w.split, w.pair};
}

lcd_status launch_mx_grouped(const MxGrouped& p, int32_t* status_word, void* stream) {
  if (p.G > kMostExperts) return LCD_ERR_UNSUPPORTED;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const MxGroupedShape w = mx_grouped_shape(p.rows.count, p.G, p.N, p.K);
  if (w.pair) return w.width == 192 ? launch_grouped<192, true>(p, 1, status_word, s) : launch_grouped<256, true>(p, 1, status_word, s);
  switch (w.width) {
    case 16: return launch_grouped<16, false>(p, w.split, status_word, s);
    case 32: return launch_grouped<32, false>(p, w.split, status_word, s);
    case 64: return launch_grouped<64, false>(p, w.split, status_word, s);
    case 128: return launch_grouped<128, false>(p, w.split, status_word, s);
    case 192: return launch_grouped<192, false>(p, w.split, status_word, s);
    default: return launch_grouped<256, false>(p, w.split, status_word, s);
  }
}

}  // namespace lcd
