// adapters_down.cuh's products for many rows: x a^T and dy b, where x and the adapters have one 16-bit type.
//
// A tile is 128 rows of one adapter by the whole rank; a cluster's CTAs share its columns and add their sums up in distributed shared
// memory, in the order of the ranks.  Rows of x follow the plan through 16-byte cp.async copies, 64 columns a stage; what bounds it is that
// one pass over x (4096 x 5120, rank 64, bf16: 22 us with cold caches, 6.5 of them the bytes; a CTA's 15 us are 2 until its first copy, 5 of
// copies, 3 until all of a cluster's sums are there and 3.5 to add and store them).
// Rows that do not start on 16 bytes go through registers.
// Roles (5 warps): warps 0-3 copy, then read the sums from tensor memory; warp 4 owns tensor memory, one elected lane issues the MMAs.
// TRANSPOSED: the adapter matrix is b [K][r], the MN-major operand as it lies.
#include "adapters_down.cuh"
#include "adapters_launch.h"
#include "adapters_tc.cuh"

namespace lcd {

namespace {

using namespace tc;

constexpr int kThreads = 5 * 32, kCopyThreads = 128;

template <int R, bool TRANSPOSED>
struct Shape {
  static constexpr int kX = 128 * 128, kW = TRANSPOSED ? (R + 63) / 64 * 64 * 128 : R * 128, kStage = kX + kW;
  static constexpr int kStages = R == 128 ? 5 : 4;                                // (two CTAs an SM but at rank 128)
  static constexpr int kPitch = R + 4;                                            // of the sums, fp32
  static constexpr int kSmem = 1024 + kStages * kStage + Plan::kBytes + 128;
  static constexpr int kTmem = (kSums<R> + 1) * R;
  static_assert(128 * kPitch * 4 <= kStages * kStage && kSmem <= 227 * 1024, "sums lie in the stages");
};

// COPIED: rows of x and of the adapter matrix start on 16 bytes.
template <typename X, int R, bool TRANSPOSED, bool COPIED>
__global__ void __launch_bounds__(kThreads, 1) adapters_down_tc_kernel(const DownArgs P) {
  using S = Shape<R, TRANSPOSED>;
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
      bar_init(full(s), kCopyThreads);
      bar_init(empty(s), 1);
    }
    bar_init(d_full, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async();
  }
  if (warp == 4) tmem_alloc((uint32_t)__cvta_generic_to_shared(tmem_holder), S::kTmem);
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
  const int k0 = (int)((long long)stages * rank / split), k1 = real ? (int)((long long)stages * (rank + 1) / split) : k0;
  bool ok = true;

  if (warp == 4) {
    if (elect()) {
      constexpr uint32_t idesc = instr_desc(R, std::is_same<X, __nv_bfloat16>::value, false, TRANSPOSED);
      for (int k = k0; k < k1 && ok; ++k) {
        const int it = k - k0, s = it % S::kStages;
        ok = bar_wait(full(s), (it / S::kStages) & 1u, abort_flag);
        if (!ok) break;
        after_sync();
        const uint64_t xd = tile_desc(base + s * S::kStage, 0), wd = tile_desc(base + s * S::kStage + S::kX, TRANSPOSED ? 64 * 128 : 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) mma(tmem + it % kSums<R> * R, xd + 2 * i, wd + (TRANSPOSED ? 128 * i : 2 * i), idesc, (uint32_t)(it >= kSums<R> || i != 0));
        mma_commit(empty(s));
      }
      mma_commit(d_full);
      bar_drain(d_full, 0);            // every MMA has finished before this CTA leaves, whatever the others wait for
    }
    __syncwarp();
  } else {
    // A row's eight pieces belong to eight neighbouring threads, 16 rows to a pass.
    const int thread = threadIdx.x, piece = thread & 7;
    const X* x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int at = thread / 8 + 16 * i, row = at < q.count ? row_of(P.a.order, q.place + at, P.a.rows) : -1;
      x[i] = row >= 0 ? static_cast<const X*>(P.x) + row * P.ldx : nullptr;
    }
    const X* w = static_cast<const X*>(P.a.w) + (real ? q.group : 0) * P.a.sw;
    auto arrive = [&](int it) {
      fence_async();
      bar_arrive(full(it % S::kStages));
    };
    constexpr int kBehind = S::kStages - 1;               // stages on their way before the first of them is handed over
    // Rows that do not start on 16 bytes: through registers, a stage at a time.
    for (int k = k0; k < k1 && ok && !COPIED; ++k) {
      const int it = k - k0, s = it % S::kStages;
      const long long c = (long long)k * 64 + piece * 8;
      const int have = (int)max(0ll, min(8ll, P.a.K - c));
      const bool within = c >= 8 && c + 16 <= P.a.K;
      const uint32_t to_x = base + s * S::kStage, to_w = to_x + S::kX;
      bool free = false;
#pragma unroll
      for (int i0 = 0; i0 < 8; i0 += 4) {
        Words<X, 8> in[4];
        if (within && !P.a.wide_x) {
          Around<X, 8> around[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) load_around(around[i], x[i0 + i] ? x[i0 + i] + c : static_cast<const X*>(P.x), x[i0 + i] != nullptr);
#pragma unroll
          for (int i = 0; i < 4; ++i) shift_words(in[i], around[i], x[i0 + i] + c);
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) load_words(in[i], x[i0 + i] + c, x[i0 + i] ? have : 0, P.a.wide_x && (have <= 0 || have >= 8));
        }
        if (!free) ok = bar_wait(empty(s), ((it / S::kStages) & 1u) ^ 1u, abort_flag);
        free = true;
        if (!ok) break;
#pragma unroll
        for (int i = 0; i < 4; ++i) store16(to_x + piece_at(thread / 8 + 16 * (i0 + i), piece), make_uint4(in[i].w[0], in[i].w[1], in[i].w[2], in[i].w[3]));
      }
      if (!ok) break;
      constexpr int kRowsW = TRANSPOSED ? (R + 63) / 64 * 64 : R, kPieces = TRANSPOSED && R < 64 ? R / 8 : 8;
#pragma unroll 4
      for (int u = thread; u < kRowsW * kPieces; u += kCopyThreads) {
        const int p = u % kPieces, row = u / kPieces % (TRANSPOSED ? 64 : R), block = TRANSPOSED ? u / kPieces / 64 : 0;
        const long long at_row = TRANSPOSED ? (long long)k * 64 + row : row, at = TRANSPOSED ? block * 64 + p * 8 : (long long)k * 64 + p * 8;
        const long long rows = TRANSPOSED ? P.a.K : P.a.r, columns = TRANSPOSED ? P.a.r : P.a.K;
        const int there = at_row < rows ? (int)max(0ll, min(8ll, columns - at)) : 0;
        const X* from = w + at_row * P.a.ldw + at;
        Words<X, 8> in;
        if (!P.a.wide_w && there == 8 && at >= 8 && at + 16 <= columns) {
          Around<X, 8> around;
          load_around(around, from, true);
          shift_words(in, around, from);
        } else {
          load_words(in, from, there, P.a.wide_w && (there <= 0 || there >= 8));
        }
        store16(to_w + block * 64 * 128 + piece_at(row, p), make_uint4(in.w[0], in.w[1], in.w[2], in.w[3]));
      }
      arrive(it);
    }
    for (int k = k0; k < k1 && ok && COPIED; ++k) {
      const int it = k - k0, s = it % S::kStages;
      ok = bar_wait(empty(s), ((it / S::kStages) & 1u) ^ 1u, abort_flag);
      if (!ok) break;
      const long long c = (long long)k * 64 + piece * 8;
      const int have = (int)max(0ll, min(8ll, P.a.K - c)) * 2;
      const uint32_t to_x = base + s * S::kStage, to_w = to_x + S::kX;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int there = x[i] ? have : 0;
        copy16(to_x + piece_at(thread / 8 + 16 * i, piece), there ? static_cast<const void*>(x[i] + c) : P.x, there);
      }
      if (TRANSPOSED) {
        constexpr int kPieces = R / 8 < 8 ? R / 8 : 8;     // of a row of 64 ranks
#pragma unroll
        for (int u = thread; u < (R + 63) / 64 * 64 * kPieces; u += kCopyThreads) {
          const int p = u % kPieces, row = u / kPieces % 64, block = u / kPieces / 64;
          const long long n = (long long)k * 64 + row;
          const int r = block * 64 + p * 8, there = n < P.a.K ? max(0, min(8, P.a.r - r)) * 2 : 0;
          copy16(to_w + block * 64 * 128 + piece_at(row, p), there ? static_cast<const void*>(w + n * P.a.ldw + r) : P.a.w, there);
        }
      } else {
#pragma unroll
        for (int i = 0; i < R / 16; ++i) {
          const int r = thread / 8 + 16 * i, there = r < P.a.r ? have : 0;
          copy16(to_w + piece_at(r, piece), there ? static_cast<const void*>(w + r * P.a.ldw + c) : P.a.w, there);
        }
      }
      copies_commit();
      if (it >= kBehind) {
        copies_wait<kBehind>();
        arrive(it - kBehind);
      }
    }
    copies_wait<0>();
    if (ok && COPIED)
      for (int it = max(0, k1 - k0 - kBehind); it < k1 - k0; ++it) arrive(it);
    ok = __all_sync(0xffffffffu, ok && bar_wait(d_full, 0, abort_flag));
    after_sync();
    // the stages are done with: they hold the sums
    float* sum = reinterpret_cast<float*>(gen + base) + thread * S::kPitch;
#pragma unroll
    for (int c = 0; c < R; c += 16) {
      float v[16] = {};
      if (k1 > k0) read_sums<R>(tmem + ((uint32_t)(32 * warp) << 16) + c, k1 - k0, false, v);
#pragma unroll
      for (int i = 0; i < 16; i += 4) *reinterpret_cast<float4*>(sum + c + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
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
  if (warp == 4) {
    after_sync();
    tmem_free(tmem, S::kTmem);
  }
  if (threadIdx.x == 0 && *abort_flag && P.status) *P.status = LCD_ERR_TIMEOUT;
}

template <typename X, int R, bool TRANSPOSED, bool COPIED>
lcd_status launch_shape(const DownArgs& P, cudaStream_t s) {
  using S = Shape<R, TRANSPOSED>;
  auto kern = adapters_down_tc_kernel<X, R, TRANSPOSED, COPIED>;
  static PerDeviceFlag attr_set;
  int dev;
  if (attr_set.first(&dev)) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem);
    if (e != cudaSuccess) { set_cuda_error((int)e); return LCD_ERR_CUDA; }
    attr_set.done(dev);
  }
  // at most that many tiles; those that hold rows are about half of the groups fewer
  const long long tiles = P.a.rows / kPlaces + (P.a.G + 1 < P.a.rows ? P.a.G + 1 : P.a.rows), likely = P.a.rows / kPlaces + (P.a.G + 1) / 2;
  const unsigned split = split_of(likely, (P.a.K + 63) / 64, (long long)current_sm_count() * (228 * 1024 / (S::kSmem + 1024)), kDownSplit);
  return adapter_launched(launch_overlapping(kern, dim3((unsigned)(tiles * split)), dim3(kThreads), S::kSmem, split, s, P));
}

template <typename X>
lcd_status launch_type(DownArgs P, bool backward, cudaStream_t s) {
  P.a.wide_x = on_bytes(P.x, P.ldx, 0, sizeof(X), 16);
  P.a.wide_w = on_bytes(P.a.w, P.a.ldw, P.a.sw, sizeof(X), 16);
  const bool copied = P.a.wide_x && P.a.wide_w;
  return by_rank(P.a.r, [&](auto rt) {
    constexpr int R = 16 * decltype(rt)::value;
    if (copied) return backward ? launch_shape<X, R, true, true>(P, s) : launch_shape<X, R, false, true>(P, s);
    return backward ? launch_shape<X, R, true, false>(P, s) : launch_shape<X, R, false, false>(P, s);
  });
}

}  // namespace

bool adapters_down_tc_takes(const DownArgs& P, lcd_dtype x_type, lcd_dtype w_type) {
  return x_type == w_type && x_type != LCD_DTYPE_F32 &&
         P.a.rows >= (on_bytes(P.x, P.ldx, 0, 2, 16) && on_bytes(P.a.w, P.a.ldw, P.a.sw, 2, 16) ? kManyRows : 2 * kManyRows);
}

lcd_status launch_adapters_down_tc(const DownArgs& P, lcd_dtype type, bool backward, cudaStream_t s) {
  return type == LCD_DTYPE_F16 ? launch_type<__half>(P, backward, s) : launch_type<__nv_bfloat16>(P, backward, s);
}

}  // namespace lcd
