// adapters_up.cuh's products for many rows: y = base + s t b^T, dx = base + dt a.
//
// A tile is 128 rows of one adapter by NC columns.  Rows of base follow the plan through 16-byte cp.async copies, whole rows side by side (one bulk
// copy a row takes a thread some 120 clocks, 128 of them three times as long as their bytes need); the product, t's parts times the adapter
// matrix's, waits in tensor memory meanwhile.  A CTA has consecutive tiles of the list (columns, rows), so that the adapter's part stays
// in shared memory from tile to tile.
//
// Roles (17 warps): warps 0-3 copy base in; warp 4 owns tensor memory, one elected lane issues the MMAs; warps 5-8 bring the parts of t and, where it
// changes, those of the adapter matrix; warps 9-16 add: a thread has a row and half of the columns, reads the base's from
// shared memory (rows 16 bytes longer than their columns: no bank conflicts) and stores 32 bytes at a time, whole sectors.
// Two tiles are in flight: while one is added up, the next one's base comes in.
// 4096 x 13824, rank 64, bf16: 56 us, 4.0 TB/s (55 with two parts of t; then 79 with t split here in place of where it is made, 61 with the matrix through registers).  A tile
// takes 3.5 us: copies of base 3.5, adding and storing 2.5, both behind one another's memory traffic.
#ifndef LCD_ADAPTERS_UP_TC_CUH_
#define LCD_ADAPTERS_UP_TC_CUH_

#include "adapters_launch.h"
#include "adapters_tc.cuh"

namespace lcd {

namespace {

using namespace tc;

constexpr int kMmaWarp = 4, kFirstLoadWarp = 5, kFirstEpiWarp = 9, kThreads = 17 * 32;
constexpr int kMostSmem = 227 * 1024;

template <typename W, typename Y, int R, bool TRANSPOSED>
struct Shape {
  static constexpr int kParts_t = kPartsT, kParts_w = kParts<W>, kSteps = R / 16;
  // t: [128 rows][parts][R], in blocks of 64 columns
  static constexpr int kT = (kParts_t * R + 63) / 64 * 128 * 128;
  static constexpr int w_bytes(int nc) { return TRANSPOSED ? nc / 64 * kParts_w * R * 128 : (kParts_w * R + 63) / 64 * nc * 128; }
  static constexpr int pitch(int nc) { return nc * (int)sizeof(Y) + 16; }
  static constexpr int smem(int nc) { return 1024 + kT + w_bytes(nc) + 2 * 128 * pitch(nc) + Plan::kBytes + 256; }
  static constexpr int kNC = sizeof(Y) == 2 && smem(256) <= kMostSmem ? 256 : smem(128) <= kMostSmem ? 128 : 64;
  static constexpr int kSmem = smem(kNC), kPitch = pitch(kNC), kW = w_bytes(kNC), kTmem = 2 * kNC;
  // whatever shares an SM has tensor memory enough
  static constexpr int kPerSm = 228 * 1024 / (kSmem + 1024);
  static_assert(kSmem <= kMostSmem && kPerSm * kTmem <= 512, "shared and tensor memory");
};

// WIDE: rows of base and y start on 16 bytes and end on them.
template <typename W, typename Y, int R, bool TRANSPOSED, bool WIDE>
__global__ void __launch_bounds__(kThreads, 1) adapters_up_tc_kernel(const UpArgs P) {
  using S = Shape<W, Y, R, TRANSPOSED>;
  constexpr int NC = S::kNC;
  extern __shared__ uint8_t smem_raw[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t raw_addr = (uint32_t)__cvta_generic_to_shared(smem_raw);
  const uint32_t at_t = (raw_addr + 1023u) & ~1023u, at_w = at_t + S::kT, at_y = at_w + S::kW, at_plan = at_y + 2 * 128 * S::kPitch;
  const uint32_t bars = at_plan + Plan::kBytes;
  uint8_t* gen = smem_raw - raw_addr;                       // gen + a shared address
  const Plan plan = {reinterpret_cast<int*>(gen + at_plan), reinterpret_cast<int*>(gen + at_plan) + kMostGroups + 2};
  auto y_full = [&](int b) { return bars + 8u * b; };
  auto y_empty = [&](int b) { return bars + 16u + 8u * b; };
  auto d_full = [&](int b) { return bars + 32u + 8u * b; };
  auto d_empty = [&](int b) { return bars + 48u + 8u * b; };
  const uint32_t t_full = bars + 64u, t_empty = bars + 72u, drain = bars + 80u;
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(gen + bars + 88u);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(gen + bars + 92u);
  if (!P.early) wait_for_previous();
  if (threadIdx.x == 0) {
    for (int b = 0; b < 2; ++b) {
      bar_init(y_full(b), 128);
      bar_init(y_empty(b), 8);
      bar_init(d_full(b), 1);
      bar_init(d_empty(b), 8);
    }
    bar_init(t_full, 128);
    bar_init(t_empty, 1);
    bar_init(drain, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async();
  }
  if (warp == kMmaWarp) tmem_alloc((uint32_t)__cvta_generic_to_shared(tmem_holder), S::kTmem);
  if (warp == 0) plan.make(P.a, lane, kPlaces);
  before_sync();
  __syncthreads();
  after_sync();
  const uint32_t tmem = *tmem_holder;
  const int G = P.a.G, row_tiles = plan.first[P.in_place ? G : G + 1];
  const long long tiles = (long long)row_tiles * ((P.a.K + NC - 1) / NC);
  const int tile0 = (int)(tiles * blockIdx.x / gridDim.x), tile1 = (int)(tiles * (blockIdx.x + 1) / gridDim.x);
  auto columns_of = [&](long long c0) { return (int)min((long long)NC, P.a.K - c0); };

  if (warp < kMmaWarp) {
    // ------------------------------------------------------------------------------------------ rows of base
    if (P.base) {
      constexpr int kPieces = NC * (int)sizeof(Y) / 16, kRowsEach = 32 / kPieces;     // 16-byte pieces of a row; rows of a warp's copy
      const int piece = lane % kPieces;
      bool ok = true;
      uint32_t it = 0;
      int next = -1;                             // lane l: row l of the warp's 32 of the next tile
      auto look = [&](int tile) {
        if (tile >= tile1) return;
        const Plan::Spot q = plan.at(tile % row_tiles, G, kPlaces);
        next = 32 * warp + lane < q.count ? P.a.order[q.place + 32 * warp + lane] : -1;
      };
      look(tile0);
      for (int tile = tile0; tile < tile1 && ok; ++tile, ++it) {
        const long long c0 = (long long)(tile / row_tiles) * NC;
        const uint32_t b = it & 1u;
        const int row = checked_row(next, P.a.rows);
        const bool inside = piece * 16 < columns_of(c0) * (int)sizeof(Y);
        const Y* from = static_cast<const Y*>(P.base) + c0 + piece * (16 / (int)sizeof(Y));
        look(tile + 1);
        // Both buffers are on their way, the next waits for the epilogue: its time does not start before the kernel before this one has ended.
        if (it == 2) begin_after_previous();
        ok = __all_sync(0xffffffffu, bar_wait(y_empty(b), ((it >> 1) & 1u) ^ 1u, abort_flag));
        if (!ok) break;
        const uint32_t to = at_y + (b * 128 + 32 * warp + lane / kPieces) * S::kPitch + piece * 16;
        if (!WIDE) {                             // rows that do not start on 16 bytes: through registers
          constexpr int kOwn = 16 / (int)sizeof(Y);
          const long long c = c0 + piece * kOwn;
          const int have = (int)max(0ll, min((long long)kOwn, P.a.K - c));
          const bool within = c >= kOwn && c + 2 * kOwn <= P.a.K;
          constexpr int kBatch = 32 / kRowsEach < 8 ? 32 / kRowsEach : 8;
#pragma unroll 1
          for (int i0 = 0; i0 < 32; i0 += kBatch * kRowsEach) {
            Words<Y, kOwn> in[kBatch];
            int r[kBatch];
#pragma unroll
            for (int i = 0; i < kBatch; ++i) r[i] = __shfl_sync(0xffffffffu, row, i0 + i * kRowsEach + lane / kPieces);
            if (within && !P.wide_base) {
              Around<Y, kOwn> around[kBatch];
#pragma unroll
              for (int i = 0; i < kBatch; ++i) load_around(around[i], from + max(r[i], 0) * P.ldbase, r[i] >= 0);
#pragma unroll
              for (int i = 0; i < kBatch; ++i) shift_words(in[i], around[i], from + max(r[i], 0) * P.ldbase);
            } else {
#pragma unroll
              for (int i = 0; i < kBatch; ++i) load_words(in[i], from + max(r[i], 0) * P.ldbase, r[i] >= 0 ? have : 0, P.wide_base && (have <= 0 || have >= kOwn));
            }
#pragma unroll
            for (int i = 0; i < kBatch; ++i) store16(to + (i0 + i * kRowsEach) * S::kPitch, make_uint4(in[i].w[0], in[i].w[1], in[i].w[2], in[i].w[3]));
          }
          bar_arrive(y_full(b));
          continue;
        }
#pragma unroll 8
        for (int i = 0; i < 32; i += kRowsEach) {
          const int r = __shfl_sync(0xffffffffu, row, i + lane / kPieces);
          if (r >= 0 && inside) copy16(to + i * S::kPitch, from + r * P.ldbase, 16);
        }
        asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(y_full(b)) : "memory");
      }
      asm volatile("cp.async.wait_all;" ::: "memory");
    }
    begin_after_previous();
  } else if (warp == kMmaWarp) {
    // ------------------------------------------------------------------------------------------ MMAs
    begin_after_previous();
    if (elect()) {
      constexpr uint32_t idesc = instr_desc(NC, true, false, TRANSPOSED);
      const uint64_t t_desc = tile_desc(at_t, 0), w_desc = tile_desc(at_w, TRANSPOSED ? S::kParts_w * R * 128 : 0);
      uint32_t it = 0;
      bool ok = true;
      for (int tile = tile0; tile < tile1 && ok; ++tile) {
        if (plan.at(tile % row_tiles, G, kPlaces).group >= G) continue;
        const uint32_t b = it & 1u;
        ok = bar_wait(d_empty(b), ((it >> 1) & 1u) ^ 1u, abort_flag) && bar_wait(t_full, it & 1u, abort_flag);
        if (!ok) break;
        after_sync();
        uint32_t more = 0;
#pragma unroll
        for (int pt = 0; pt < S::kParts_t; ++pt)
#pragma unroll
          for (int pw = 0; pw < S::kParts_w; ++pw) {
            if (pt + pw >= S::kParts_t) continue;         // smaller than what the parts leave out
#pragma unroll
            for (int k = 0; k < S::kSteps; ++k) {
              const int kt = pt * S::kSteps + k, kw = pw * S::kSteps + k;
              const uint32_t w_off = TRANSPOSED ? kw * 2048 : kw / 4 * NC * 128 + kw % 4 * 32;
              mma(tmem + b * NC, t_desc + ((kt / 4 * 128 * 128 + kt % 4 * 32) >> 4), w_desc + (w_off >> 4), idesc, more);
              more = 1;
            }
          }
        mma_commit(t_empty);
        mma_commit(d_full(b));
        ++it;
      }
      mma_commit(drain);
      bar_drain(drain, 0);
    }
    __syncwarp();
  } else if (warp < kFirstEpiWarp) {
    // ------------------------------------------------------------------------------------------ t and the adapter matrix, in parts
    const int thread = threadIdx.x - 32 * kFirstLoadWarp;
    bool waited = false, ok = true;
    uint32_t it = 0;
    int group = -1;
    long long columns = -1;
    Plan::Spot q = {};
    auto find = [&](int tile) {                  // the next tile of an adapter, or tile1
      for (; tile < tile1; ++tile) {
        q = plan.at(tile % row_tiles, G, kPlaces);
        if (q.group < G) break;
      }
      return tile;
    };
    for (int tile = find(tile0); tile < tile1 && ok;) {
      const long long c0 = (long long)(tile / row_tiles) * NC;
      ok = __all_sync(0xffffffffu, bar_wait(t_empty, (it & 1u) ^ 1u, abort_flag));
      if (!ok) break;
      if (q.group != group || c0 != columns) {
        group = q.group;
        columns = c0;
        const W* w = static_cast<const W*>(P.a.w) + group * P.a.sw;
        constexpr int kRowsW = TRANSPOSED ? R : NC, kUnits = TRANSPOSED ? NC / 8 : R / 8, kEachW = kRowsW * kUnits / 128, kMostBatch = sizeof(W) == 2 ? 8 : 4,
                      kBatch = kEachW < kMostBatch ? kEachW : kMostBatch;
        const bool copied = S::kParts_w == 1 && P.a.wide_w;          // as it lies, all pieces on their way together
        if (copied) {
#pragma unroll 8
          for (int u = thread; u < kRowsW * kUnits; u += 128) {
            const int row = u / kUnits, unit = u % kUnits;
            const long long at_row = TRANSPOSED ? row : c0 + row, at_col = TRANSPOSED ? c0 + unit * 8 : unit * 8;
            const long long rows = TRANSPOSED ? P.a.r : P.a.K, cols = TRANSPOSED ? P.a.K : P.a.r;
            const int have = at_row < rows ? (int)max(0ll, min(8ll, cols - at_col)) * 2 : 0;
            const uint32_t to = TRANSPOSED ? unit / 8 * (S::kParts_w * R * 128) + piece_at(row, unit % 8) : unit / 8 * (NC * 128) + piece_at(row, unit % 8);
            copy16(at_w + to, have ? static_cast<const void*>(w + at_row * P.a.ldw + at_col) : P.a.w, have);
          }
        }
#pragma unroll 1
        for (int u0 = copied ? kRowsW * kUnits : thread; u0 < kRowsW * kUnits; u0 += 128 * kBatch) {
          Words<W, 8> in[kBatch];
#pragma unroll
          for (int i = 0; i < kBatch; ++i) {
            const int row = (u0 + 128 * i) / kUnits, unit = (u0 + 128 * i) % kUnits;
            const long long at_row = TRANSPOSED ? row : c0 + row, at_col = TRANSPOSED ? c0 + unit * 8 : unit * 8;
            const long long rows = TRANSPOSED ? P.a.r : P.a.K, cols = TRANSPOSED ? P.a.K : P.a.r;
            const int have = at_row < rows ? (int)max(0ll, min(8ll, cols - at_col)) : 0;
            load_words(in[i], w + at_row * P.a.ldw + at_col, have, P.a.wide_w && (have <= 0 || have >= 8));
          }
#pragma unroll
          for (int i = 0; i < kBatch; ++i) {
            const int row = (u0 + 128 * i) / kUnits, unit = (u0 + 128 * i) % kUnits;
            uint4 out[S::kParts_w];
            if constexpr (S::kParts_w == 1) {
              out[0] = make_uint4(in[i].w[0], in[i].w[1], in[i].w[2], in[i].w[3]);
            } else {
              float v[8];
#pragma unroll
              for (int e = 0; e < 8; ++e) v[e] = value_of(in[i], e);
              parts_of<S::kParts_w>(v, out);
            }
#pragma unroll
            for (int p = 0; p < S::kParts_w; ++p) {
              if (TRANSPOSED) {
                store16(at_w + unit / 8 * (S::kParts_w * R * 128) + piece_at(p * R + row, unit % 8), out[p]);
              } else {
                const int k = p * S::kSteps + unit / 2;
                store16(at_w + k / 4 * (NC * 128) + piece_at(row, k % 4 * 2 + unit % 2), out[p]);
              }
            }
          }
        }
      }
      if (!waited) {
        begin_after_previous();
        waited = true;
      }
      constexpr int kUnits = S::kParts_t * (R / 8);               // pieces of eight ranks of a row
      const __nv_bfloat16* t = static_cast<const __nv_bfloat16*>(P.t_parts) + (long long)q.place * (S::kParts_t * R);
#pragma unroll 8
      for (int u = thread; u < 128 * kUnits; u += 128) {
        const int row = u / kUnits, unit = u % kUnits;
        // part after part, steps of 16 ranks four to a block
        copy16(at_t + unit / 8 * (128 * 128) + piece_at(row, unit % 8), row < q.count ? t + (long long)u * 8 : P.t_parts, row < q.count ? 16 : 0);
      }
      asm volatile("cp.async.wait_all;" ::: "memory");
      fence_async();
      bar_arrive(t_full);
      ++it;
      tile = find(tile + 1);
    }
    if (!waited) begin_after_previous();
  } else {
    // ------------------------------------------------------------------------------------------ sums, and rows of y
    begin_after_previous();
    const int quad = warp & 3, half = (warp - kFirstEpiWarp) / 4, mine = 32 * quad + lane;
    constexpr int kHalf = NC / 2;
    bool ok = true;
    uint32_t it = 0, dt = 0;
    // of the next tile: asked for while this one is added up
    Plan::Spot q = {};
    int row = -1;
    float factor = 1.0f;
    auto look = [&](int tile) {
      if (tile >= tile1) return;
      q = plan.at(tile % row_tiles, G, kPlaces);
      row = mine < q.count ? P.a.order[q.place + mine] : -1;
      factor = P.a.scale && q.group < G ? P.a.scale[q.group] : 1.0f;
    };
    look(tile0);
    for (int tile = tile0; tile < tile1 && ok; ++tile, ++it) {
      const long long c0 = (long long)(tile / row_tiles) * NC + half * kHalf;
      const int columns = (int)min((long long)kHalf, P.a.K - c0), to_row = checked_row(row, P.a.rows);
      const float s = factor;
      const bool real = q.group < G;
      const uint32_t b = it & 1u, db = dt & 1u;
      look(tile + 1);
      // (without base the buffers are this warp's own)
      if (P.base) ok = __all_sync(0xffffffffu, bar_wait(y_full(b), (it >> 1) & 1u, abort_flag));
      if (ok && real) ok = __all_sync(0xffffffffu, bar_wait(d_full(db), (dt >> 1) & 1u, abort_flag));
      if (!ok) break;
      after_sync();
      Y* own = reinterpret_cast<Y*>(gen + at_y + (b * 128 + mine) * S::kPitch) + half * kHalf;
      Y* y = static_cast<Y*>(P.y) + max(to_row, 0) * P.ldy + c0;
      const uint32_t from = tmem + ((uint32_t)(32 * quad) << 16) + db * NC + half * kHalf;
      uint32_t d[2][16];
      if (real) tmem_ld16(from, d[0]);
#pragma unroll
      for (int c = 0; c < kHalf; c += 16) {
        float v[16];
        if (P.base) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float part[8];
            values8(load8(own + c + 8 * h), part);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[8 * h + i] = part[i];
          }
        } else {
#pragma unroll
          for (int i = 0; i < 16; ++i) v[i] = 0.0f;
        }
        if (real) {
          tmem_wait_ld();
          if (c + 16 < kHalf) tmem_ld16(from + c + 16, d[(c / 16 + 1) & 1]);
#pragma unroll
          for (int i = 0; i < 16; ++i) v[i] = __fmaf_rn(s, __uint_as_float(d[(c / 16) & 1][i]), v[i]);
        }
        if (!WIDE) {                                          // the sums go where the base was
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const float part[8] = {v[8 * h], v[8 * h + 1], v[8 * h + 2], v[8 * h + 3], v[8 * h + 4], v[8 * h + 5], v[8 * h + 6], v[8 * h + 7]};
            store8(own + c + 8 * h, part);
          }
          continue;
        }
        if (to_row < 0 || c >= columns) continue;
        if (c + 16 <= columns) {
          store16_values(y + c, v, P.wide_y > 16);
        } else {                                              // the row ends after four, eight or twelve
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (c + i < columns) y[c + i] = from_f32<Y>(v[i]);
        }
      }
      if (!WIDE) {                                            // rows that do not start on 16 bytes: value by value, neighbours side by side
        __syncwarp();
        const Y* rows = reinterpret_cast<const Y*>(gen + at_y + (b * 128 + 32 * quad) * S::kPitch) + half * kHalf;
#pragma unroll 4
        for (int i = 0; i < 32; ++i) {
          const int r = __shfl_sync(0xffffffffu, to_row, i);
          if (r < 0) continue;
          Y* to = static_cast<Y*>(P.y) + r * P.ldy + c0;
          const Y* from_row = rows + i * (S::kPitch / (int)sizeof(Y));
#pragma unroll
          for (int c = lane; c < kHalf; c += 32)
            if (c < columns) to[c] = from_row[c];
        }
      }
      before_sync();
      __syncwarp();
      if (lane == 0) {
        bar_arrive(y_empty(b));
        if (real) bar_arrive(d_empty(db));
      }
      if (real) ++dt;
    }
  }
  before_sync();
  __syncthreads();
  if (warp == kMmaWarp) {
    after_sync();
    tmem_free(tmem, S::kTmem);
  }
  if (threadIdx.x == 0 && *abort_flag && P.status) *P.status = LCD_ERR_TIMEOUT;
}

template <typename W, typename Y, int R, bool TRANSPOSED, bool WIDE>
lcd_status launch_shape(const UpArgs& P, cudaStream_t s) {
  using S = Shape<W, Y, R, TRANSPOSED>;
  auto kern = adapters_up_tc_kernel<W, Y, R, TRANSPOSED, WIDE>;
  static PerDeviceFlag attr_set;
  int dev;
  if (attr_set.first(&dev)) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem);
    if (e != cudaSuccess) { set_cuda_error((int)e); return LCD_ERR_CUDA; }
    attr_set.done(dev);
  }
  const long long most = ((long long)P.a.rows / kPlaces + (P.a.G + 1 < P.a.rows ? P.a.G + 1 : P.a.rows)) * ((P.a.K + S::kNC - 1) / S::kNC);
  const long long room = (long long)current_sm_count() * S::kPerSm;
  return adapter_launched(launch_overlapping(kern, dim3((unsigned)(most < room ? most : room)), dim3(kThreads), S::kSmem, 1, s, P));
}

template <typename W, typename Y, bool TRANSPOSED>
lcd_status launch_up_tc_types(UpArgs P, cudaStream_t s) {
  P.a.wide_w = on_bytes(P.a.w, P.a.ldw, P.a.sw, sizeof(W), 16);
  P.wide_base = on_bytes(P.base, P.ldbase, P.a.K, sizeof(Y), 16);
  P.wide_y = on_bytes(P.y, P.ldy, P.a.K, sizeof(Y), 16) ? on_bytes(P.y, P.ldy, 0, sizeof(Y), 32) ? 32 : 16 : 0;
  P.in_place = P.base == P.y && P.ldbase == P.ldy;
  const bool wide = P.wide_base && P.wide_y;
  return by_rank(P.a.r, [&](auto rt) {
    constexpr int R = 16 * decltype(rt)::value;
    if constexpr (R <= 64 || (std::is_same<W, __nv_bfloat16>::value && sizeof(Y) == 2))
      return wide ? launch_shape<W, Y, R, TRANSPOSED, true>(P, s) : launch_shape<W, Y, R, TRANSPOSED, false>(P, s);
    return (lcd_status)LCD_ERR_UNSUPPORTED;
  });
}

}  // namespace

template <typename W>
lcd_status launch_up_tc_weights(const UpArgs& P, lcd_dtype y_type, bool transposed, cudaStream_t s) {
  return by_dtype(y_type, [&](auto y) {
    using Y = typename decltype(y)::type;
    return transposed ? launch_up_tc_types<W, Y, true>(P, s) : launch_up_tc_types<W, Y, false>(P, s);
  });
}

}  // namespace lcd
#endif
