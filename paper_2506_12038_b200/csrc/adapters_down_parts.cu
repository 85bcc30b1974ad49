// adapters_down_tc.cu's products where x and the adapters are not of one 16-bit type: both go through registers and into shared memory as bf16
// parts (bf16 is one, fp16 two, fp32 three; products of parts that together are beyond the third are left out: 2^-22 of a term).
//
// Tiles, clusters and the joining of their sums as there.  Roles (9 warps): two groups of four warps take the stages in turn and have the next
// one's values on their way while they split this one's; the first group reads the sums; the last warp issues the MMAs.
#include "adapters_down.cuh"
#include "adapters_launch.h"
#include "adapters_tc.cuh"

namespace lcd {

namespace {

using namespace tc;

constexpr int kThreads = 9 * 32, kMmaWarp = 8;

template <typename X, typename W, int R, bool TRANSPOSED>
struct Shape {
  static constexpr int kPartsX = kParts<X>, kPartsW = kParts<W>;
  static constexpr int kX = 128 * 128, kW = TRANSPOSED ? (R + 63) / 64 * 64 * 128 : R * 128, kStage = kPartsX * kX + kPartsW * kW;
  static constexpr int kStages = 4 * kStage <= 200 * 1024 ? 4 : 2;                // whoever fills a place has filled it the time before
  static constexpr int kPitch = R + 4;                                            // of the sums, fp32
  static constexpr int kSmem = 1024 + kStages * kStage + Plan::kBytes + 128;
  static constexpr int kTmem = (kSums<R> + 1) * R;
  static_assert(kSmem > 114 * 1024 || kTmem <= 256, "tensor memory of CTAs that share an SM");
  static_assert(128 * kPitch * 4 <= kStages * kStage && kSmem <= 227 * 1024, "sums lie in the stages");
};

template <typename X, typename W, int R, bool TRANSPOSED>
__global__ void __launch_bounds__(kThreads, 1) adapters_down_parts_kernel(const DownArgs P) {
  using S = Shape<X, W, R, TRANSPOSED>;
  extern __shared__ uint8_t smem_raw[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t raw_addr = (uint32_t)__cvta_generic_to_shared(smem_raw);
  const uint32_t base = (raw_addr + 1023u) & ~1023u, at_plan = base + S::kStages * S::kStage, bars = at_plan + Plan::kBytes;
  uint8_t* gen = smem_raw - raw_addr;
  const Plan plan = {reinterpret_cast<int*>(gen + at_plan), reinterpret_cast<int*>(gen + at_plan) + kMostGroups + 2};
  auto full = [&](int s) { return bars + 8u * s; };
  auto empty = [&](int s) { return bars + 8u * (S::kStages + s); };
  const uint32_t d_full = bars + 8u * 2 * S::kStages;
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(gen + d_full + 8u);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(gen + d_full + 12u);
  uint32_t rank, split;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(split));
  wait_for_previous();
  if (threadIdx.x == 0) {
    for (int s = 0; s < S::kStages; ++s) {
      bar_init(full(s), 128);
      bar_init(empty(s), 1);
    }
    bar_init(d_full, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async();
  }
  if (warp == kMmaWarp) tmem_alloc((uint32_t)__cvta_generic_to_shared(tmem_holder), S::kTmem);
  if (warp == 0) plan.make(P.a, lane, kPlaces);
  before_sync();
  __syncthreads();
  after_sync();
  let_next_begin();          // not before this CTA has its tensor memory: the next kernel's may take some and then wait for this one
  const uint32_t tmem = *tmem_holder;
  const int tile = blockIdx.x / split, G = P.a.G;
  const Plan::Spot q = tile < plan.first[G + 1] ? plan.at(tile, G, kPlaces) : Plan::Spot{G, 0, 0};
  const bool real = q.group < G;                         // the same in all CTAs of the cluster
  const int stages = (int)((P.a.K + 63) / 64);
  const int k0 = (int)((long long)stages * rank / split), n = real ? (int)((long long)stages * (rank + 1) / split) - k0 : 0;
  bool ok = true;

  if (warp == kMmaWarp) {
    if (elect()) {
      constexpr uint32_t idesc = instr_desc(R, true, false, TRANSPOSED);
      for (int it = 0; it < n && ok; ++it) {
        const int s = it % S::kStages;
        ok = bar_wait(full(s), (it / S::kStages) & 1u, abort_flag);
        if (!ok) break;
        after_sync();
        const uint64_t xd = tile_desc(base + s * S::kStage, 0), wd = tile_desc(base + s * S::kStage + S::kPartsX * S::kX, TRANSPOSED ? 64 * 128 : 0);
#pragma unroll
        for (int px = 0; px < S::kPartsX; ++px)
#pragma unroll
          for (int pw = 0; pw < S::kPartsW; ++pw) {
            if (px + pw >= 3) continue;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const bool main = px + pw == 0;
              mma(tmem + (main ? it % kSums<R> : kSums<R>) * R, xd + ((px * S::kX + 32 * i) >> 4), wd + ((pw * S::kW + (TRANSPOSED ? 2048 : 32) * i) >> 4), idesc,
                  (uint32_t)(main ? it >= kSums<R> || i > 0 : it > 0 || i > 0 || px + 3 * pw != (S::kPartsW > 1 ? 3 : 1)));
            }
          }
        mma_commit(empty(s));
      }
      mma_commit(d_full);
      bar_drain(d_full, 0);            // every MMA has finished before this CTA leaves, whatever the others wait for
    }
    __syncwarp();
  } else {
    // A row's eight pieces belong to eight neighbouring threads, 16 rows to a pass.
    const int thread = threadIdx.x % 128, piece = thread & 7, mine = warp / 4;
    int row[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int at = thread / 8 + 16 * i;
      row[i] = at < q.count ? row_of(P.a.order, q.place + at, P.a.rows) : -1;
    }
    const W* w = static_cast<const W*>(P.a.w) + (real ? q.group : 0) * P.a.sw;
    constexpr int kRowsW = TRANSPOSED ? (R + 63) / 64 * 64 : R, kPieces = TRANSPOSED && R < 64 ? R / 8 : 8, kEachW = kRowsW * kPieces / 128 < 1 ? 1 : kRowsW * kPieces / 128;
    Words<X, 8> in[8];
    Words<W, 8> in_w[kEachW];
    auto load = [&](int it) {
      const long long k = (long long)(k0 + it) * 64, c = k + piece * 8;
      const int have = it < n ? (int)max(0ll, min(8ll, P.a.K - c)) : 0;
      constexpr int kSide = 16 / (int)sizeof(X);
      if (!P.a.wide_x && have >= 8 && c >= kSide && c + 8 + kSide <= P.a.K) {
#pragma unroll
        for (int i0 = 0; i0 < 8; i0 += 4) {
          Around<X, 8> around[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) load_around(around[i], static_cast<const X*>(P.x) + max(row[i0 + i], 0) * P.ldx + c, row[i0 + i] >= 0);
#pragma unroll
          for (int i = 0; i < 4; ++i) shift_words(in[i0 + i], around[i], static_cast<const X*>(P.x) + max(row[i0 + i], 0) * P.ldx + c);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          load_words(in[i], static_cast<const X*>(P.x) + max(row[i], 0) * P.ldx + c, row[i] >= 0 ? have : 0, P.a.wide_x && (have <= 0 || have >= 8));
      }
#pragma unroll
      for (int i = 0; i < kEachW; ++i) {
        const int u = thread + 128 * i, p = u % kPieces, at = u / kPieces % (TRANSPOSED ? 64 : R), block = TRANSPOSED ? u / kPieces / 64 : 0;
        const long long at_row = TRANSPOSED ? k + at : at, at_col = TRANSPOSED ? block * 64 + p * 8 : k + p * 8;
        const int there = u < kRowsW * kPieces && it < n && at_row < (TRANSPOSED ? P.a.K : P.a.r) ? (int)max(0ll, min(8ll, (TRANSPOSED ? P.a.r : P.a.K) - at_col)) : 0;
        load_words(in_w[i], w + at_row * P.a.ldw + at_col, there, P.a.wide_w && (there <= 0 || there >= 8));
      }
    };
    load(mine);
    for (int it = mine; it < n && ok; it += 2) {
      const int s = it % S::kStages;
      ok = bar_wait(empty(s), ((it / S::kStages) & 1u) ^ 1u, abort_flag);
      if (!ok) break;
      const uint32_t to_x = base + s * S::kStage, to_w = to_x + S::kPartsX * S::kX;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = value_of(in[i], e);
        uint4 parts[S::kPartsX];
        parts_of<S::kPartsX>(v, parts);
#pragma unroll
        for (int p = 0; p < S::kPartsX; ++p) store16(to_x + p * S::kX + piece_at(thread / 8 + 16 * i, piece), parts[p]);
      }
#pragma unroll
      for (int i = 0; i < kEachW; ++i) {
        const int u = thread + 128 * i, pc = u % kPieces, at = u / kPieces % (TRANSPOSED ? 64 : R), block = TRANSPOSED ? u / kPieces / 64 : 0;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = value_of(in_w[i], e);
        uint4 parts[S::kPartsW];
        parts_of<S::kPartsW>(v, parts);
        if (u < kRowsW * kPieces) {
#pragma unroll
          for (int p = 0; p < S::kPartsW; ++p) store16(to_w + p * S::kW + block * 64 * 128 + piece_at(at, pc), parts[p]);
        }
      }
      fence_async();
      bar_arrive(full(s));
      load(it + 2);
    }
    ok = __all_sync(0xffffffffu, ok && bar_wait(d_full, 0, abort_flag));
    after_sync();
    // the stages are done with: they hold the sums
    if (mine == 0) {
      float* sum = reinterpret_cast<float*>(gen + base) + thread * S::kPitch;
#pragma unroll
      for (int c = 0; c < R; c += 16) {
        float v[16] = {};
        if (n > 0) read_sums<R>(tmem + ((uint32_t)(32 * warp) << 16) + c, n, true, v);
#pragma unroll
        for (int i = 0; i < 16; i += 4) *reinterpret_cast<float4*>(sum + c + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
      }
    }
    before_sync();
  }
  if (split > 1) {
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
  } else {
    __syncthreads();
  }
  const float factor = P.a.scale && real ? P.a.scale[q.group] : 1.0f;
  by_split(split, [&](auto ranks) {
    constexpr int kRanks = decltype(ranks)::value;
    for (int e = rank * kThreads + threadIdx.x; e < q.count * (R / 4); e += kRanks * kThreads) {
      const int at = e / (R / 4), r = e % (R / 4) * 4;
      float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      if (real) sum = sums_of_ranks<kRanks>(base + (at * S::kPitch + r) * 4);
      const float v[4] = {r < P.a.r ? sum.x * factor : 0.0f, r + 1 < P.a.r ? sum.y * factor : 0.0f, r + 2 < P.a.r ? sum.z * factor : 0.0f,
                          r + 3 < P.a.r ? sum.w * factor : 0.0f};
      store_t4(P, R, q.place + at, r, v);
      if (P.t_rows) {
        const int row = row_of(P.a.order, q.place + at, P.a.rows);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (row >= 0 && r + i < P.a.r) P.t_rows[row * P.ldt_rows + r + i] = v[i];
      }
    }
  });
  if (split > 1) {
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
  }
  before_sync();
  __syncthreads();
  if (warp == kMmaWarp) {
    after_sync();
    tmem_free(tmem, S::kTmem);
  }
  if (threadIdx.x == 0 && *abort_flag && P.status) *P.status = LCD_ERR_TIMEOUT;
}

template <typename X, typename W, int R, bool TRANSPOSED>
lcd_status launch_shape(const DownArgs& P, cudaStream_t s) {
  using S = Shape<X, W, R, TRANSPOSED>;
  auto kern = adapters_down_parts_kernel<X, W, R, TRANSPOSED>;
  static PerDeviceFlag attr_set;
  int dev;
  if (attr_set.first(&dev)) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem);
    if (e != cudaSuccess) { set_cuda_error((int)e); return LCD_ERR_CUDA; }
    attr_set.done(dev);
  }
  // as in adapters_down_tc.cu
  const long long tiles = P.a.rows / kPlaces + (P.a.G + 1 < P.a.rows ? P.a.G + 1 : P.a.rows), likely = P.a.rows / kPlaces + (P.a.G + 1) / 2;
  const unsigned split = split_of(likely, (P.a.K + 63) / 64, current_sm_count(), kDownSplit);
  return adapter_launched(launch_overlapping(kern, dim3((unsigned)(tiles * split)), dim3(kThreads), S::kSmem, split, s, P));
}

template <typename X, typename W>
lcd_status launch_types(DownArgs P, bool backward, cudaStream_t s) {
  P.a.wide_x = on_bytes(P.x, P.ldx, 0, sizeof(X), 16);
  P.a.wide_w = on_bytes(P.a.w, P.a.ldw, P.a.sw, sizeof(W), 16);
  return by_rank(P.a.r, [&](auto rt) {
    constexpr int R = 16 * decltype(rt)::value;
    return backward ? launch_shape<X, W, R, true>(P, s) : launch_shape<X, W, R, false>(P, s);
  });
}

}  // namespace

bool adapters_down_parts_takes(const DownArgs& P, lcd_dtype x_type, lcd_dtype w_type) {
  return (x_type == LCD_DTYPE_F32 || w_type == LCD_DTYPE_F32) && P.a.rows >= kManyRows;
}

lcd_status launch_adapters_down_parts(const DownArgs& P, lcd_dtype x_type, lcd_dtype w_type, bool backward, cudaStream_t s) {
  if (x_type == LCD_DTYPE_F16) return launch_types<__half, float>(P, backward, s);
  if (x_type == LCD_DTYPE_BF16) return launch_types<__nv_bfloat16, float>(P, backward, s);
  if (w_type == LCD_DTYPE_F16) return launch_types<float, __half>(P, backward, s);
  if (w_type == LCD_DTYPE_BF16) return launch_types<float, __nv_bfloat16>(P, backward, s);
  return launch_types<float, float>(P, backward, s);
}

}  // namespace lcd
