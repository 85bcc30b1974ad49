// adapters_outer.cu's gradients for many rows: da = sum over an adapter's rows of dt^T x, db = s sum of dy^T t.
//
// A tile is 128 columns of z (x or dy) by the whole rank of one adapter; the sum runs over its rows, 64 a stage, so both operands are
// MN-major as they lie.  Rows of z follow the plan through 16-byte copies (bf16 as it is where rows start on 16 bytes; else, and fp16 and fp32, through
// registers, in one to three bf16 parts), those of t or dt are split into parts on their way.  A cluster's CTAs share an adapter's rows where there are few tiles and
// add their sums up in distributed shared memory, in the order of the ranks.  Reading z bounds it.
// Roles (8 to 13 warps): warps 0-3 bring z, then read the sums from tensor memory; the last one owns tensor memory, one elected lane issues
// the MMAs; those between bring t or dt, one of them (two at ranks above 32) for every stage's place, so that its loads have the time of
// all stages.
#include "adapters_launch.h"
#include "adapters_tc.cuh"

namespace lcd {

namespace {

using namespace tc;

constexpr int kStageRows = 64, kOuterSplit = 8;

template <typename Z, typename O, int R>
struct Shape {
  static constexpr int kParts_u = kPartsFor<Z, O>, kParts_z = kParts<Z> < kParts_u ? kParts<Z> : kParts_u;
  static constexpr int kZPart = 2 * kStageRows * 128, kUPart = (R + 63) / 64 * kStageRows * 128;
  static constexpr int kStage = kParts_z * kZPart + kParts_u * kUPart;
  // two CTAs an SM where they have three stages each
  static constexpr int kStages = 4 * kStage <= 110 * 1024 ? 4 : 3 * kStage <= 110 * 1024 ? 3 : 4 * kStage <= 220 * 1024 ? 4 : 3;
  // Warps that bring a stage of t.  A stage's place belongs to the same ones every time: a wait for a parity passes two phases early, so whoever
  // fills a place has to have filled it the time before.
  static constexpr int kPer = R == 64 ? 2 : 1;
  static constexpr int kMmaWarp = 4 + kStages * kPer, kThreads = 32 * (kMmaWarp + 1);
  static constexpr int kPitch = R + 4;                                            // of the sums, fp32
  static constexpr int kSmem = 1024 + kStages * kStage + 128;
  static constexpr int kTmem = R < 32 ? 32 : R;
  static constexpr int kPerSm = 2 * (kSmem + 1024) <= 228 * 1024 ? 2 : 1;
  static_assert(128 * kPitch * 4 <= kStages * kStage && kSmem <= 227 * 1024, "sums lie in the stages");
};

template <typename Z, typename O, int R>
__global__ void __launch_bounds__(Shape<Z, O, R>::kThreads, Shape<Z, O, R>::kPerSm) adapters_outer_tc_kernel(const __grid_constant__ OuterArgs P) {
  using S = Shape<Z, O, R>;
  constexpr bool kCopied = S::kParts_z == 1;
  extern __shared__ uint8_t smem_raw[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t raw_addr = (uint32_t)__cvta_generic_to_shared(smem_raw);
  const uint32_t base = (raw_addr + 1023u) & ~1023u, bars = base + S::kStages * S::kStage;
  uint8_t* gen = smem_raw - raw_addr;
  auto full = [&](int s) { return bars + 8u * s; };
  auto empty = [&](int s) { return bars + 8u * (S::kStages + s); };
  const uint32_t d_full = bars + 8u * 2 * S::kStages;
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(gen + d_full + 8u);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(gen + d_full + 12u);
  uint32_t rank, split;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(split));
  begin_after_previous();
  const int group = blockIdx.y;
  long long slab = blockIdx.x / split;
  const int side = slab >= P.slabs[0];
  if (side) slab -= P.slabs[0];
  const OuterSide& E = P.side[side];
  const long long col0 = slab * 128;
  const int from = max(0, min(P.rows, P.offsets[group])), to = max(from, min(P.rows, P.offsets[group + 1]));
  O* out = static_cast<O*>(E.out);
  auto place_of = [&](int r, int c) {
    return E.by_column ? ((long long)group * E.columns + col0 + c) * P.r + r : ((long long)group * P.r + r) * E.columns + col0 + c;
  };
  if (to == from) {                                  // in all CTAs of the cluster: zeros
    for (int e = rank * S::kThreads + threadIdx.x; e < 128 * R; e += split * S::kThreads) {
      const int r = E.by_column ? e % R : e / 128, c = E.by_column ? e / R : e % 128;
      if (r < P.r && col0 + c < E.columns) out[place_of(r, c)] = from_f32<O>(0.0f);
    }
    return;
  }
  if (threadIdx.x == 0) {
    for (int s = 0; s < S::kStages; ++s) {
      bar_init(full(s), 128 + 32 * S::kPer);
      bar_init(empty(s), 1);
    }
    bar_init(d_full, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async();
  }
  if (warp == S::kMmaWarp) tmem_alloc((uint32_t)__cvta_generic_to_shared(tmem_holder), S::kTmem);
  before_sync();
  __syncthreads();
  after_sync();
  const uint32_t tmem = *tmem_holder;
  const int stages = (to - from + kStageRows - 1) / kStageRows;
  const int k0 = (int)((long long)stages * rank / split), n = (int)((long long)stages * (rank + 1) / split) - k0;
  bool ok = true;

  if (warp == S::kMmaWarp) {
    if (elect()) {
      constexpr uint32_t idesc = instr_desc(R, true, true, true);
      uint32_t more = 0;
      for (int it = 0; it < n && ok; ++it) {
        const int s = it % S::kStages;
        ok = bar_wait(full(s), (it / S::kStages) & 1u, abort_flag);
        if (!ok) break;
        after_sync();
        const uint64_t zd = tile_desc(base + s * S::kStage, kStageRows * 128), ud = tile_desc(base + s * S::kStage + S::kParts_z * S::kZPart, kStageRows * 128);
#pragma unroll
        for (int pz = 0; pz < S::kParts_z; ++pz)
#pragma unroll
          for (int pu = 0; pu < S::kParts_u; ++pu) {
            if (pz + pu >= S::kParts_u) continue;        // smaller than what the parts leave out
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              mma(tmem, zd + ((pz * S::kZPart + 2048 * i) >> 4), ud + ((pu * S::kUPart + 2048 * i) >> 4), idesc, more);
              more = 1;
            }
          }
        mma_commit(empty(s));
      }
      mma_commit(d_full);
      bar_drain(d_full, 0);            // every MMA has finished before this CTA leaves, whatever the others wait for
    }
    __syncwarp();
  } else if (warp < 4) {
    // A row's sixteen pieces belong to sixteen neighbouring threads, eight rows to a pass.
    const int thread = threadIdx.x, piece = thread & 15;
    const long long c = col0 + piece * 8;
    const int have = (int)max(0ll, min(8ll, E.columns - c));
    const uint32_t at_piece = (uint32_t)(piece / 8 * kStageRows * 128);
    const Z* z = static_cast<const Z*>(E.z) + c;
    const bool inside = have >= 8 && c >= 16 / (int)sizeof(Z) && c + 8 + 16 / (int)sizeof(Z) <= E.columns;
    auto row_at = [&](int it, int i) {
      const int place = from + (k0 + it) * kStageRows + thread / 16 + 8 * i;
      return place < to ? P.order[place] : -1;
    };
    int row[8], then[8];                                // of this stage and the next
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      row[i] = checked_row(row_at(0, i), P.rows);
      then[i] = 1 < n ? row_at(1, i) : -1;
    }
    auto next_rows = [&](int it) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        row[i] = checked_row(then[i], P.rows);
        then[i] = it + 2 < n ? row_at(it + 2, i) : -1;
      }
    };
    if (kCopied && E.wide_z) {
      constexpr int kBehind = S::kStages - 1;
      for (int it = 0; it < n && ok; ++it) {
        const int s = it % S::kStages;
        ok = bar_wait(empty(s), ((it / S::kStages) & 1u) ^ 1u, abort_flag);
        if (!ok) break;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int there = row[i] >= 0 ? have * 2 : 0;
          copy16(base + s * S::kStage + at_piece + piece_at(thread / 16 + 8 * i, piece % 8), there ? static_cast<const void*>(z + row[i] * E.ldz) : E.z, there);
        }
        copies_commit();
        next_rows(it);
        if (it >= kBehind) {
          copies_wait<kBehind>();
          fence_async();
          bar_arrive(full((it - kBehind) % S::kStages));
        }
      }
      copies_wait<0>();
      if (ok) {
        fence_async();
        for (int it = max(0, n - kBehind); it < n; ++it) bar_arrive(full(it % S::kStages));
      }
    } else {
      Words<Z, 8> in[8];
      auto load = [&] {
        if (!E.wide_z && inside) {
#pragma unroll
          for (int i0 = 0; i0 < 8; i0 += 4) {
            Around<Z, 8> around[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) load_around(around[i], z + max(row[i0 + i], 0) * E.ldz, row[i0 + i] >= 0);
#pragma unroll
            for (int i = 0; i < 4; ++i) shift_words(in[i0 + i], around[i], z + max(row[i0 + i], 0) * E.ldz);
          }
          return;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) load_words(in[i], z + (row[i] >= 0 ? row[i] * E.ldz : 0), row[i] >= 0 ? have : 0, E.wide_z && (have <= 0 || have >= 8));
      };
      load();
      for (int it = 0; it < n && ok; ++it) {
        const int s = it % S::kStages;
        next_rows(it);
        ok = bar_wait(empty(s), ((it / S::kStages) & 1u) ^ 1u, abort_flag);
        if (!ok) break;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          float v[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = value_of(in[i], e);
          uint4 parts[S::kParts_z];
          parts_of<S::kParts_z>(v, parts);
#pragma unroll
          for (int p = 0; p < S::kParts_z; ++p) store16(base + s * S::kStage + p * S::kZPart + at_piece + piece_at(thread / 16 + 8 * i, piece % 8), parts[p]);
        }
        fence_async();
        bar_arrive(full(s));
        if (it + 1 < n) load();
      }
    }
    ok = __all_sync(0xffffffffu, ok && bar_wait(d_full, 0, abort_flag));
    after_sync();
    float* sum = reinterpret_cast<float*>(gen + base) + thread * S::kPitch;      // the stages are done with
#pragma unroll
    for (int c2 = 0; c2 < R; c2 += 16) {
      uint32_t v[16];
      if (n > 0) {
        tmem_ld16(tmem + ((uint32_t)(32 * warp) << 16) + c2, v);
        tmem_wait_ld();
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = 0u;
      }
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        *reinterpret_cast<float4*>(sum + c2 + i) = make_float4(__uint_as_float(v[i]), __uint_as_float(v[i + 1]), __uint_as_float(v[i + 2]), __uint_as_float(v[i + 3]));
    }
    before_sync();
  } else {
    // t or dt: pieces of eight ranks
    const int mine = (warp - 4) / S::kPer, first = (warp - 4) % S::kPer * 32 + lane;
    constexpr int kUnits = R / 8, kEach = kStageRows * kUnits / (32 * S::kPer);
    Words<float, 8> in[kEach];
    int row[kEach];
    auto find = [&](int it) {
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int place = from + (k0 + it) * kStageRows + (first + 32 * S::kPer * i) / kUnits;
        row[i] = it < n && place < to ? (E.u_by_place ? place : P.order[place]) : -1;
      }
    };
    auto load = [&] {
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int at = checked_row(row[i], P.rows), unit = (first + 32 * S::kPer * i) % kUnits, have = at >= 0 ? max(0, min(8, P.r - unit * 8)) : 0;
        load_words(in[i], E.u + (long long)max(at, 0) * E.ldu + unit * 8, have, E.wide_u && (have <= 0 || have >= 8));
      }
    };
    find(mine);
    load();
    find(mine + S::kStages);
    for (int it = mine; it < n && ok; it += S::kStages) {
      const int s = mine;
      ok = __all_sync(0xffffffffu, bar_wait(empty(s), ((it / S::kStages) & 1u) ^ 1u, abort_flag));
      if (!ok) break;
      const uint32_t to_u = base + s * S::kStage + S::kParts_z * S::kZPart;
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int u = first + 32 * S::kPer * i, unit = u % kUnits, at = u / kUnits;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = value_of(in[i], e);
        uint4 parts[S::kParts_u];
        parts_of<S::kParts_u>(v, parts);
#pragma unroll
        for (int p = 0; p < S::kParts_u; ++p) store16(to_u + p * S::kUPart + unit / 8 * kStageRows * 128 + piece_at(at, unit % 8), parts[p]);
      }
      fence_async();
      bar_arrive(full(s));
      load();
      find(it + 2 * S::kStages);
    }
  }
  if (split > 1) {
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
  } else {
    __syncthreads();
  }
  const float factor = E.scale ? E.scale[group] : 1.0f;
  by_split(split, [&](auto ranks) {
    constexpr int kRanks = decltype(ranks)::value;
#pragma unroll 2
    for (int e = rank * S::kThreads + threadIdx.x; e < 128 * R / 4; e += kRanks * S::kThreads) {
      // four ranks of a column; consecutive threads: consecutive places of the output
      const int r = E.by_column ? e % (R / 4) * 4 : e / 128 * 4, c = E.by_column ? e / (R / 4) : e % 128;
      if (r >= P.r || col0 + c >= E.columns) continue;
      const float4 sum = sums_of_ranks<kRanks>(base + (c * S::kPitch + r) * 4);
      const float v[4] = {sum.x * factor, sum.y * factor, sum.z * factor, sum.w * factor};
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (r + i < P.r) out[place_of(r + i, c)] = from_f32<O>(v[i]);
    }
  });
  if (split > 1) {
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
  }
  before_sync();
  __syncthreads();
  if (warp == S::kMmaWarp) {
    after_sync();
    tmem_free(tmem, S::kTmem);
  }
  if (threadIdx.x == 0 && *abort_flag && P.status) *P.status = LCD_ERR_TIMEOUT;
}

template <typename Z, typename O, int R>
lcd_status launch_shape(OuterArgs P, cudaStream_t s) {
  using S = Shape<Z, O, R>;
  auto kern = adapters_outer_tc_kernel<Z, O, R>;
  static PerDeviceFlag attr_set;
  int dev;
  if (attr_set.first(&dev)) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem);
    if (e != cudaSuccess) { set_cuda_error((int)e); return LCD_ERR_CUDA; }
    attr_set.done(dev);
  }
  long long slabs = 0;
  for (int i = 0; i < 2; ++i) {
    P.slabs[i] = i < P.sides ? (P.side[i].columns + 127) / 128 : 0;
    slabs += P.slabs[i];
    P.side[i].wide_z = on_bytes(P.side[i].z, P.side[i].ldz, 0, sizeof(Z), 16);
    P.side[i].wide_u = on_bytes(P.side[i].u, P.side[i].ldu, 0, 4, 16);
  }
  const long long stages = P.rows / (P.G < P.rows ? P.G : P.rows) / kStageRows + 1;
  const unsigned split = split_of(slabs * P.G, stages, (long long)current_sm_count() * S::kPerSm, kOuterSplit);
  return adapter_launched(launch_overlapping(kern, dim3((unsigned)(slabs * split), (unsigned)P.G), dim3(S::kThreads), S::kSmem, split, s, P));
}

}  // namespace

bool adapters_outer_tc_takes(const OuterArgs& P, lcd_dtype z_type) {
  long long slabs = 0;
  for (int i = 0; i < P.sides; ++i) {
    slabs += (P.side[i].columns + 127) / 128;
  }
  return P.rows >= kManyRows && P.r <= 64 && slabs <= 0x7fffffff / kOuterSplit;
}

lcd_status launch_adapters_outer_tc(const OuterArgs& P, lcd_dtype z_type, cudaStream_t s) {
  return by_dtype(z_type, [&](auto z) {
    return by_dtype((lcd_dtype)P.out_type, [&](auto o) {
      using Z = typename decltype(z)::type;
      using O = typename decltype(o)::type;
      switch (rank_tiles(P.r)) {
        case 1: return launch_shape<Z, O, 16>(P, s);
        case 2: return launch_shape<Z, O, 32>(P, s);
        default: return launch_shape<Z, O, 64>(P, s);
      }
    });
  });
}

}  // namespace lcd
