// adapters_outer.cu's gradients for many rows: da = sum over an adapter's rows of dt^T x, db = s sum of dy^T t.
//
// A sum is 128 columns of z (x or dy) by the whole rank of one adapter; it runs over the adapter's rows, 64 a stage, so both operands are
// MN-major as they lie.  Rows of z follow the plan through 16-byte copies (bf16 as it is where rows start on 16 bytes; else, and fp16 and
// fp32, through registers, in one to three bf16 parts), those of t or dt are split into parts on their way.  One CTA an SM takes every
// gridDim.x-th sum; while one is read from tensor memory and stored, the next one's stages come in (a CTA for each sum spent more time on
// beginning and ending than on an adapter's 256 rows: 148 us at 4096 x 5120 x 13824, rank 64, 16 adapters, two parts of u).  Where there are few sums a
// cluster's CTAs share one's rows and add up in distributed shared memory, in the order of the ranks.  Reading z bounds it.
// Roles: kZWarps warps bring z and kUWarps t or dt, in groups that take stages in turn (finding a stage's rows and addresses takes longer than
// its bytes), one owns tensor memory and an elected lane issues the MMAs, four store.
// Rank 128 has one sum in tensor memory, which the next waits for: 4096 x 4096 x 4096, bf16, 97 us for one adapter and 128 for 16
// (adapters_outer.cu 286 and 445 with two parts of u); fp32, 4096 rows, 206 and 255 (417 and 646).
#include "adapters_launch.h"
#include "adapters_tc.cuh"

namespace lcd {

namespace {

using namespace tc;

constexpr int kStageRows = 64, kOuterSplit = 8;

template <typename Z, int R>
struct Shape {
  static constexpr int kParts_u = kPartsT, kParts_z = kParts<Z>;
  static constexpr int kZPart = 2 * kStageRows * 128, kUPart = (R + 63) / 64 * kStageRows * 128;
  static constexpr int kStage = kParts_z * kZPart + kParts_u * kUPart;
  static constexpr int kStages = 6 * kStage <= 200 * 1024 ? 6 : 4 * kStage <= 200 * 1024 ? 4 : 2;
  // Groups that take stages in turn.  A stage's place belongs to the same ones every time: a wait for a parity passes two phases early, so
  // whoever fills a place has to have filled it the time before.  (Four places: two groups for u 71 us at 4096 x 5120 x 5120, rank 32, bf16, four
  // 64; rank 64 103 and 94.)
  static constexpr int kZGroups = R == 128 ? 1 : 2, kUGroups = kStages == 6 ? 3 : kStages, kUWarpsEach = R <= 32 ? 1 : R / 32;
  static constexpr int kZWarps = 4 * kZGroups, kUWarps = kUGroups * kUWarpsEach;
  static constexpr int kMmaWarp = kZWarps + kUWarps, kFirstEpiWarp = kMmaWarp + 1, kThreads = 32 * (kFirstEpiWarp + 4);
  static constexpr int kPitch = R + 4;                                            // of a cluster's sums, fp32
  static constexpr int kSmem = 1024 + kStages * kStage + 4 * (kMostGroups + 1) + 256;
  static constexpr int kBuffers = R == 128 ? 1 : 2;                                // sums in tensor memory: one is read while the next is made
  static constexpr int kTmem = kBuffers * (kSums<R> + 1) * R;
  static_assert(kStages % kZGroups == 0 && kStages % kUGroups == 0 && 128 * kPitch * 4 <= kStages * kStage && kSmem <= 227 * 1024, "shapes");
  static_assert(kSmem > 114 * 1024 && kTmem <= 512, "one CTA an SM");
};

// The stages that a role walks through: sum after sum, this CTA's share of each.
struct Walk {
  const OuterArgs& P;
  const int* offsets;
  int slabs, step, rank, split;
  long long sums;
  long long sum;
  int it = 0, n = 0, from = 0, to = 0, group = 0, side = 0;      // stage of the sum, stages, its first place, the places' end
  long long col0 = 0;
  __device__ __forceinline__ void look() {
    if (sum >= sums) return;
    group = (int)(sum / slabs);
    long long slab = sum % slabs;
    side = slab >= P.slabs[0];
    if (side) slab -= P.slabs[0];
    col0 = slab * 128;
    const int begin = offsets[group];
    to = offsets[group + 1];
    const int stages = (to - begin + kStageRows - 1) / kStageRows, k0 = (int)((long long)stages * rank / split);
    n = max(0, (int)((long long)stages * (rank + 1) / split) - k0);
    from = begin + k0 * kStageRows;
  }
  // To the stage `by` further on; false behind the last.
  __device__ __forceinline__ bool advance(int by) {
    it += by;
    while (sum < sums && it >= n) {
      it -= n;
      n = 0;
      sum += step;
      look();
    }
    return sum < sums;
  }
};

template <typename Z, typename O, int R>
__global__ void __launch_bounds__(Shape<Z, R>::kThreads, 1) adapters_outer_tc_kernel(const __grid_constant__ OuterArgs P) {
  using S = Shape<Z, R>;
  constexpr bool kCopied = S::kParts_z == 1;
  extern __shared__ uint8_t smem_raw[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t raw_addr = (uint32_t)__cvta_generic_to_shared(smem_raw);
  const uint32_t base = (raw_addr + 1023u) & ~1023u, at_offsets = base + S::kStages * S::kStage, bars = (at_offsets + 4 * (kMostGroups + 1) + 7u) & ~7u;
  uint8_t* gen = smem_raw - raw_addr;
  int* offsets = reinterpret_cast<int*>(gen + at_offsets);
  auto full = [&](int s) { return bars + 8u * s; };
  auto empty = [&](int s) { return bars + 8u * (S::kStages + s); };
  auto d_full = [&](int b) { return bars + 8u * (2 * S::kStages + b); };
  auto d_empty = [&](int b) { return bars + 8u * (2 * S::kStages + 2 + b); };
  const uint32_t drain = bars + 8u * (2 * S::kStages + 4);
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(gen + drain + 8u);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(gen + drain + 12u);
  uint32_t rank, split;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(split));
  wait_for_previous();
  for (int g = threadIdx.x; g <= P.G; g += blockDim.x) offsets[g] = max(0, min(P.rows, P.offsets[g]));
  if (threadIdx.x == 0) {
    for (int s = 0; s < S::kStages; ++s) {
      bar_init(full(s), 128 + 32 * S::kUWarpsEach);
      bar_init(empty(s), 1);
    }
    for (int b = 0; b < 2; ++b) {
      bar_init(d_full(b), 1);
      bar_init(d_empty(b), 4);
    }
    bar_init(drain, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async();
  }
  if (warp == S::kMmaWarp) tmem_alloc((uint32_t)__cvta_generic_to_shared(tmem_holder), S::kTmem);
  before_sync();
  __syncthreads();
  after_sync();
  let_next_begin();          // not before this CTA has its tensor memory: the next kernel's may take some and then wait for this one
  const uint32_t tmem = *tmem_holder;
  const int slabs = (int)(P.slabs[0] + P.slabs[1]);
  Walk w{P, offsets, slabs, (int)(gridDim.x / split), (int)rank, (int)split, (long long)slabs * P.G, (long long)(blockIdx.x / split)};
  w.look();
  bool ok = true;

  if (warp == S::kMmaWarp) {
    if (elect()) {
      constexpr uint32_t idesc = instr_desc(R, true, true, true);
      uint32_t stage = 0, tl = 0;
      for (; w.sum < w.sums && ok; w.sum += w.step, w.n = 0, w.look()) {
        if (w.n <= 0) continue;
        const uint32_t b = tl % S::kBuffers;
        ok = bar_wait(d_empty(b), ((tl / S::kBuffers) & 1u) ^ 1u, abort_flag);
        for (int it = 0; it < w.n && ok; ++it, ++stage) {
          const uint32_t s = stage % S::kStages;
          ok = bar_wait(full(s), (stage / S::kStages) & 1u, abort_flag);
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
                const bool main = pz + pu == 0;             // the others begin with pz = 0, pu = 1
                mma(tmem + ((kSums<R> + 1) * b + (main ? it % kSums<R> : kSums<R>)) * R, zd + ((pz * S::kZPart + 2048 * i) >> 4), ud + ((pu * S::kUPart + 2048 * i) >> 4), idesc,
                    (uint32_t)(main ? it >= kSums<R> || i > 0 : it > 0 || i > 0 || pz > 0 || pu > 1));
              }
            }
          mma_commit(empty(s));
        }
        if (!ok) break;
        mma_commit(d_full(b));
        ++tl;
      }
      mma_commit(drain);
      bar_drain(drain, 0);             // every MMA has finished before this CTA leaves, whatever the others wait for
    }
    __syncwarp();
  } else if (warp < S::kZWarps) {
    // A row's sixteen pieces belong to sixteen neighbouring threads, eight rows to a pass.
    const int thread = threadIdx.x % 128, piece = thread & 15, mine = warp / 4;
    const uint32_t at_piece = (uint32_t)(piece / 8 * kStageRows * 128);
    int row[8];                                       // the next stage's, as the plan has them: looked at when they are used
    auto find = [&](const Walk& v, bool there) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int place = v.from + v.it * kStageRows + thread / 16 + 8 * i;
        row[i] = there && place < v.to ? P.order[place] : -1;
      }
    };
    bool there = w.advance(mine);
    find(w, there);
    uint32_t stage = mine;
    auto columns = [&](const OuterSide& E, long long c) { return (int)max(0ll, min(8ll, E.columns - c)); };
    if (kCopied && P.side[0].wide_z && P.side[1].wide_z) {
      constexpr int kBehind = S::kStages / S::kZGroups - 1;         // of this group's stages, on their way before the first is handed over
      uint32_t own = 0;
      for (; there && ok; stage += S::kZGroups, ++own) {
        const int s = stage % S::kStages;
        const OuterSide& E = P.side[w.side];
        const long long c = w.col0 + piece * 8;
        const int have = columns(E, c) * 2;
        const Z* z = static_cast<const Z*>(E.z) + c;
        ok = bar_wait(empty(s), ((stage / S::kStages) & 1u) ^ 1u, abort_flag);
        if (!ok) break;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int r = checked_row(row[i], P.rows), bytes = r >= 0 ? have : 0;
          copy16(base + s * S::kStage + at_piece + piece_at(thread / 16 + 8 * i, piece % 8), bytes ? static_cast<const void*>(z + r * E.ldz) : E.z, bytes);
        }
        copies_commit();
        there = w.advance(S::kZGroups);
        find(w, there);
        if (own >= kBehind) {
          copies_wait<kBehind>();
          fence_async();
          bar_arrive(full((stage - kBehind * S::kZGroups) % S::kStages));
        }
      }
      copies_wait<0>();
      if (ok) {
        fence_async();
        for (uint32_t i = min(own, (uint32_t)kBehind); i > 0; --i) bar_arrive(full((stage - i * S::kZGroups) % S::kStages));
      }
    } else {
      Words<Z, 8> in[8];
      auto load = [&](const Walk& v, bool valid) {
        const OuterSide& E = P.side[v.side];
        const long long c = v.col0 + piece * 8;
        const int have = valid ? columns(E, c) : 0;
        const Z* z = static_cast<const Z*>(E.z) + c;
        if (!E.wide_z && have >= 8 && c >= 16 / (int)sizeof(Z) && c + 8 + 16 / (int)sizeof(Z) <= E.columns) {
#pragma unroll
          for (int i0 = 0; i0 < 8; i0 += 4) {
            Around<Z, 8> around[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) load_around(around[i], z + max(checked_row(row[i0 + i], P.rows), 0) * E.ldz, checked_row(row[i0 + i], P.rows) >= 0);
#pragma unroll
            for (int i = 0; i < 4; ++i) shift_words(in[i0 + i], around[i], z + max(checked_row(row[i0 + i], P.rows), 0) * E.ldz);
          }
          return;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int r = checked_row(row[i], P.rows);
          load_words(in[i], z + max(r, 0) * E.ldz, r >= 0 ? have : 0, E.wide_z && (have <= 0 || have >= 8));
        }
      };
      load(w, there);
      for (; there && ok; stage += S::kZGroups) {
        const int s = stage % S::kStages;
        there = w.advance(S::kZGroups);
        find(w, there);
        ok = bar_wait(empty(s), ((stage / S::kStages) & 1u) ^ 1u, abort_flag);
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
        load(w, there);
      }
    }
  } else if (warp < S::kMmaWarp) {
    // t or dt: pieces of eight ranks
    const int mine = (warp - S::kZWarps) / S::kUWarpsEach, first = (warp - S::kZWarps) % S::kUWarpsEach * 32 + lane;
    constexpr int kUnits = R / 8, kEach = kStageRows * kUnits / (32 * S::kUWarpsEach);
    Words<float, 8> in[kEach];
    int row[kEach];
    auto find = [&](const Walk& v, bool there) {
      const bool by_place = P.side[v.side].u_by_place;
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int place = v.from + v.it * kStageRows + (first + 32 * S::kUWarpsEach * i) / kUnits;
        row[i] = there && place < v.to ? (by_place ? place : P.order[place]) : -1;
      }
    };
    auto load = [&](const OuterSide& E) {
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int at = checked_row(row[i], P.rows), unit = (first + 32 * S::kUWarpsEach * i) % kUnits, have = at >= 0 ? max(0, min(8, P.r - unit * 8)) : 0;
        load_words(in[i], E.u + (long long)max(at, 0) * E.ldu + unit * 8, have, E.wide_u && (have <= 0 || have >= 8));
      }
    };
    // the stage whose values wait in registers, and the one after it, whose rows are asked for
    uint32_t stage = mine;
    bool there = w.advance(mine);
    find(w, there);
    load(P.side[w.side]);
    bool then = there && w.advance(S::kUGroups);
    find(w, then);
    for (; there && ok; stage += S::kUGroups) {
      const int s = stage % S::kStages;
      ok = __all_sync(0xffffffffu, bar_wait(empty(s), ((stage / S::kStages) & 1u) ^ 1u, abort_flag));
      if (!ok) break;
      const uint32_t to_u = base + s * S::kStage + S::kParts_z * S::kZPart;
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int u = first + 32 * S::kUWarpsEach * i, unit = u % kUnits, at = u / kUnits;
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
      there = then;
      load(P.side[w.side]);
      then = there && w.advance(S::kUGroups);
      find(w, then);
    }
  } else {
    // ------------------------------------------------------------------------------------------ the sums
    const int quad = warp & 3, mine = 32 * quad + lane;
    uint32_t tl = 0;
    for (; w.sum < w.sums && ok; w.sum += w.step, w.n = 0, w.look()) {
      const OuterSide& E = P.side[w.side];
      const uint32_t b = tl % S::kBuffers;
      const bool some = w.n > 0;
      if (some) ok = __all_sync(0xffffffffu, bar_wait(d_full(b), (tl / S::kBuffers) & 1u, abort_flag));
      if (!ok) break;
      after_sync();
      const float factor = E.scale ? E.scale[w.group] : 1.0f;
      O* out = static_cast<O*>(E.out);
      const long long c = w.col0 + mine;
      const bool inside = c < E.columns;
      float* sum = reinterpret_cast<float*>(gen + base) + mine * S::kPitch;       // a cluster's: it has one sum, whose stages are done with
#pragma unroll
      for (int r0 = 0; r0 < R; r0 += 16) {
        float v[16] = {};
        if (some) read_sums<R>(tmem + ((uint32_t)(32 * quad) << 16) + (kSums<R> + 1) * b * R + r0, w.n, true, v);
        if (split > 1) {
#pragma unroll
          for (int i = 0; i < 16; i += 4)
            *reinterpret_cast<float4*>(sum + r0 + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
        } else if (inside) {
          // (a group without rows has zeros whatever its factor is)
          O* to = out + (E.by_column ? ((long long)w.group * E.columns + c) * P.r + r0 : ((long long)w.group * P.r + r0) * E.columns + c);
          const long long pitch = E.by_column ? 1 : E.columns;
          float x[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) x[i] = some ? v[i] * factor : 0.0f;
          if (E.wide_out && r0 + 16 <= P.r) {
            store16_values(to, x, false);
          } else {
#pragma unroll
            for (int i = 0; i < 16; ++i)
              if (r0 + i < P.r) to[i * pitch] = from_f32<O>(x[i]);
          }
        }
      }
      before_sync();
      __syncwarp();
      if (some) {
        if (lane == 0) bar_arrive(d_empty(b));
        ++tl;
      }
    }
  }
  if (split > 1) {
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
    Walk v{P, offsets, slabs, 1, 0, 1, (long long)slabs * P.G, (long long)(blockIdx.x / split)};
    v.look();
    if (v.sum < v.sums) {
      const OuterSide& E = P.side[v.side];
      const bool some = v.n > 0;
      const float factor = E.scale ? E.scale[v.group] : 1.0f;
      O* out = static_cast<O*>(E.out);
      by_split(split, [&](auto ranks) {
        constexpr int kRanks = decltype(ranks)::value;
        for (int e = rank * S::kThreads + threadIdx.x; e < 128 * R / 4; e += kRanks * S::kThreads) {
          // four ranks of a column; consecutive threads: consecutive places of the output
          const int r = E.by_column ? e % (R / 4) * 4 : e / 128 * 4, c = E.by_column ? e / (R / 4) : e % 128;
          if (r >= P.r || v.col0 + c >= E.columns) continue;
          const float4 sum = sums_of_ranks<kRanks>(base + (c * S::kPitch + r) * 4);
          const float x[4] = {sum.x * factor, sum.y * factor, sum.z * factor, sum.w * factor};
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (r + i < P.r)
              out[E.by_column ? ((long long)v.group * E.columns + v.col0 + c) * P.r + r + i : ((long long)v.group * P.r + r + i) * E.columns + v.col0 + c] =
                  from_f32<O>(some ? x[i] : 0.0f);
        }
      });
    }
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
  using S = Shape<Z, R>;
  auto kern = adapters_outer_tc_kernel<Z, O, R>;
  static PerDeviceFlag attr_set;
  int dev;
  if (attr_set.first(&dev)) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem);
    if (e != cudaSuccess) { set_cuda_error((int)e); return LCD_ERR_CUDA; }
    attr_set.done(dev);
  }
  for (int i = 0; i < 2; ++i) {
    if (i >= P.sides) P.side[i] = P.side[0];
    P.slabs[i] = i < P.sides ? (P.side[i].columns + 127) / 128 : 0;
    P.side[i].wide_z = on_bytes(P.side[i].z, P.side[i].ldz, 0, sizeof(Z), 16);
    P.side[i].wide_u = on_bytes(P.side[i].u, P.side[i].ldu, 0, 4, 16);
    P.side[i].wide_out = P.side[i].by_column && on_bytes(P.side[i].out, P.r, 0, sizeof(O), 16);
  }
  const long long sums = (P.slabs[0] + P.slabs[1]) * P.G, sms = current_sm_count();
  const long long stages = P.rows / (P.G < P.rows ? P.G : P.rows) / kStageRows + 1;
  const unsigned split = sums < sms ? split_of(sums, stages, sms, kOuterSplit) : 1;
  const long long ctas = split > 1 || sums < sms ? sums * split : sms;
  return adapter_launched(launch_overlapping(kern, dim3((unsigned)ctas), dim3(S::kThreads), S::kSmem, split, s, P));
}

}  // namespace

bool adapters_outer_tc_takes(const OuterArgs& P) {
  long long slabs = 0;
  for (int i = 0; i < P.sides; ++i) slabs += (P.side[i].columns + 127) / 128;
  return P.rows >= kManyRows && slabs <= 0x7fffffff / kOuterSplit;
}

lcd_status launch_adapters_outer_tc(const OuterArgs& P, lcd_dtype z_type, cudaStream_t s) {
  return by_dtype(z_type, [&](auto z) {
    return by_dtype((lcd_dtype)P.out_type, [&](auto o) {
      using Z = typename decltype(z)::type;
      using O = typename decltype(o)::type;
      switch (rank_tiles(P.r)) {
        case 1: return launch_shape<Z, O, 16>(P, s);
        case 2: return launch_shape<Z, O, 32>(P, s);
        case 4: return launch_shape<Z, O, 64>(P, s);
        default: return launch_shape<Z, O, 128>(P, s);
      }
    });
  });
}

}  // namespace lcd
